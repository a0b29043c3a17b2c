"""Float products with factors down to the smallest subnormal number, and with infinities beside such factors.

Tolerance.  A sum of n products in any order is off by at most (n + 4) 2^-24 of the products' magnitudes.  Taken in three bfloat16 parts a number is
off by less than 2^-131 (bfloat16 ends at 2^-133; up to three parts are cut there or are that number in place of a zero), a product a b so by less than
2^-131 (|a| + |b|), and by less than 2^-21 + 2^-30 of itself by what is left out.  Sums and results round to 2^-149 where they are subnormal themselves,
six times per product at most."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

E, LEFT_OUT, SMALL, LAST = 2.0 ** -24, 2.0 ** -21 + 2.0 ** -30, 2.0 ** -131, 2.0 ** -149
ROWS, COLS, REDUCED = 2040, 2041, 601      # 256 tiles of 128 x 128: taken in parts, without ranges


def _u():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from tests import feed_forward_util
    return feed_forward_util


def _product(u, kind, a, b, lend):
    """a b^T (rows of a, rows of b, the reduction along both) by one of the three passes; a and b float tensors"""
    import torch
    ig, h = u.ig, u.handle()
    (m, n), (k, _) = a.shape, b.shape
    out = torch.full((m, k), float("nan"), device="cuda")
    desc = lambda t: ig.TensorDescriptor().set(ig.IGC_DATA_FLOAT, t.shape[0], t.shape[1], 1, 1, (t.stride(0), 1, 1, 1))
    parts = sum(-(-r // 16) * -(-n // 32) * 3 * 1024 for r in (m, k))

    def workspace(size):
        assert parts <= size < parts + 4 * m * k, "not taken in parts"
        return u.Workspace(size if lend else 0)

    if kind == "forward":
        w = u.filter_desc("f32", k, n)
        ws = workspace(ig.get_linear_forward_workspace_size(h, desc(a), w, desc(out)))
        ig.check(ig.linear_forward(h, 1.0, desc(a), a.data_ptr(), w, b.data_ptr(), ws.buf.data_ptr(), ws.size, 0, -1, 0.0, None, 0, desc(out), 0, out.data_ptr()))
    elif kind == "data":
        f, w = b.t().contiguous(), u.filter_desc("f32", n, k)
        ws = workspace(ig.get_linear_backward_data_workspace_size(h, w, desc(a), desc(out)))
        ig.check(ig.linear_backward_data(h, 1.0, w, f.data_ptr(), desc(a), a.data_ptr(), ws.buf.data_ptr(), ws.size, -1, None, 0, 0.0, None, 0, desc(out),
                                         out.data_ptr()))
    else:
        dy, x, w = a.t().contiguous(), b.t().contiguous(), u.filter_desc("f32", m, k)
        ws = workspace(ig.get_linear_backward_filter_workspace_size(h, desc(x), desc(dy), w))
        ig.check(ig.linear_backward_filter(h, 1.0, desc(x), x.data_ptr(), desc(dy), dy.data_ptr(), ws.buf.data_ptr(), ws.size, 0.0, w, out.data_ptr()))
    ws.check()
    return out


def _numbers(rows, cols, lowest, highest, seed):
    """Significands in [1, 2), exponents spread evenly, subnormal numbers among them, a tenth zeros; the values that float holds"""
    rng = np.random.default_rng(seed)
    v = np.ldexp(rng.uniform(1, 2, (rows, cols)), rng.integers(lowest, highest, (rows, cols))) * rng.choice([-1.0, 1.0], (rows, cols))
    v[rng.random((rows, cols)) < 0.1] = 0.0
    return v.astype(np.float32)


@pytest.mark.parametrize("lend", [True, False], ids=["workspace", "alone"])
@pytest.mark.parametrize("kind", ["forward", "data", "filter"])
@pytest.mark.parametrize("exponents", [((-149, -95), (-10, 10)), ((-140, -100), (60, 100)), ((-149, 20), (-149, 20)), ((-125, -109), (-30, 0))], ids=str)
def test_small_numbers(exponents, kind, lend):
    import torch
    u = _u()
    a, b = (torch.from_numpy(_numbers(r, REDUCED, *e, seed)).cuda() for seed, (r, e) in enumerate(zip((ROWS, COLS), exponents)))
    got = _product(u, kind, a, b, lend).double()
    A, B = a.double(), b.double()
    want, size = A @ B.t(), A.abs() @ B.abs().t()
    tol = ((REDUCED + 4) * E + LEFT_OUT) * size + SMALL * (A.abs().sum(1)[:, None] + B.abs().sum(1)[None, :]) + (6 * REDUCED + 2) * LAST
    assert bool(torch.isfinite(got).all())
    off = ((got - want).abs() / tol).max()
    assert float(off) <= 1, float(off)


@pytest.mark.parametrize("lend", [True, False], ids=["workspace", "alone"])
@pytest.mark.parametrize("kind", ["forward", "data", "filter"])
def test_infinities_beside_small_numbers(kind, lend):
    """An infinity times anything but zero is an infinity, the smallest subnormal number included; times zero it is undefined."""
    import torch
    u = _u()
    a, b = (torch.from_numpy(_numbers(r, REDUCED, -20, 20, 7 + r)).cuda() for r in (ROWS, COLS))
    powers = [2.0 ** -e for e in (60, 99, 100, 101, 109, 118, 126, 127, 133, 134, 140, 149)]
    small = torch.tensor(powers + [1.7 * 2.0 ** -101, 1.9 * 2.0 ** -120, 0.0], dtype=torch.float32, device="cuda")
    for i in range(15):
        b[i * 130, 5], a[i * 130 + 1, 600] = small[i] * (-1.0) ** i, small[i]
    a[3, 5], b[4, 600] = float("inf"), float("-inf")
    a[3][a[3] == 0], b[4][b[4] == 0] = 1.0, 1.0
    got = _product(u, kind, a, b, lend)
    A, B = a.double(), b.double()
    for row, at in ((got[3], B[:, 5]), (got[:, 4], -A[:, 600])):
        other = torch.ones_like(row, dtype=torch.bool)
        other[4 if row.shape[0] == COLS else 3] = False      # (where the two infinities' rows meet)
        want = torch.where(at == 0, float("nan"), torch.sign(at) * float("inf")).float()
        assert bool(((row == want) | (torch.isnan(row) & torch.isnan(want)))[other].all())
    rest = torch.ones(ROWS, dtype=torch.bool), torch.ones(COLS, dtype=torch.bool)
    rest[0][3], rest[1][4] = False, False
    assert bool(torch.isfinite(got[rest[0]][:, rest[1]]).all())
