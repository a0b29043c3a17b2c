"""The feed-forward functions with every kind of workspace between none and what the query reports: the plan then gives up ranges, copies, the bias
gradient's sums, one by one.  Behind the bytes that are lent lies a guard band.

Tolerance: as in test_gpu_feed_forward: a sum of n products in any order is off by at most (n + 4) 2^-24 of their magnitudes, in three parts by 2^-21 +
2^-30 more; the result rounds by half a step of its type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests import test_gpu_feed_forward as plain

SHAPES = [(3, 2000, 130), (40, 1001, 300), (515, 259, 261), (2000, 72, 65), (700, 600, 640)]
SHARES = [0.01, 0.1, 0.3, 0.5, 0.7, 0.9]


def sizes(size):
    return sorted({0, 1, 16, *(int(size * s) for s in SHARES), max(0, size - 16), max(0, size - 1), size})


class Lent:
    """`size` bytes, `shift` behind a 16-byte boundary, full of NaN, guard bytes behind them"""

    def __init__(self, size, shift=0):
        import torch
        self.size, self.shift = size, shift
        self.buf = torch.full((shift + size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        self.buf[shift + size:] = 0x5A
        self.buf[:shift] = 0x5A
        self.ptr = self.buf.data_ptr() + shift

    def check(self):
        import torch
        torch.cuda.synchronize()
        assert bool((self.buf[self.shift + self.size:] == 0x5A).all()) and bool((self.buf[:self.shift] == 0x5A).all()), "store outside the workspace"


@pytest.mark.parametrize("pad,lead", [(0, 0), (1, 1), (2, 2)])
@pytest.mark.parametrize("types", plain.LINEAR_TYPES, ids="-".join)
@pytest.mark.parametrize("kind", ["forward", "data", "filter"])
def test_products(kind, types, pad, lead):
    u = plain._u()
    ig, h = u.ig, u.handle()
    dtype, out = types
    half = 1.01 * u.HALF_STEP[out]
    for M, C, K in SHAPES:
        print(kind, types, M, C, K, pad, lead, flush=True)
        _, x, w, dy = plain.linear_case(types, M, C, K)
        X, DY = u.Rows(x, dtype, pad, lead), u.Rows(dy, dtype, pad, lead)
        W = u.vector(w, dtype)
        if kind == "forward":
            Y, F = u.Rows((M, K), out, pad, lead), u.filter_desc(dtype, K, C)
            size = ig.get_linear_forward_workspace_size(h, X.desc, F, Y.desc)
            want, tol = x @ w.T, plain.sum_error(C, np.abs(x) @ np.abs(w).T, dtype)
        elif kind == "data":
            Y, F = u.Rows((M, C), out, pad, lead), u.filter_desc(dtype, K, C)
            size = ig.get_linear_backward_data_workspace_size(h, F, DY.desc, Y.desc)
            want, tol = dy @ w, plain.sum_error(K, np.abs(dy) @ np.abs(w), dtype)
        else:
            Y, F, DB = u.Rows((K, C), out), u.filter_desc(out, K, C), u.vector(np.zeros(K))
            size = ig.get_linear_backward_filter_workspace_size(h, X.desc, DY.desc, F)
            want, tol = dy.T @ x, plain.sum_error(M, np.abs(dy).T @ np.abs(x), dtype)
        for n in [(s, 0) for s in sizes(size)] + [(size, 8)]:
            Y.view.fill_(float("nan"))
            ws = Lent(*n)
            if kind == "forward":
                ig.check(ig.linear_forward(h, 1.0, X.desc, X.ptr, F, W.data_ptr(), ws.ptr, ws.size, 0, -1, 0.0, None, 0, Y.desc, 0, Y.ptr))
            elif kind == "data":
                ig.check(ig.linear_backward_data(h, 1.0, F, W.data_ptr(), DY.desc, DY.ptr, ws.ptr, ws.size, -1, None, 0, 0.0, None, 0, Y.desc, Y.ptr))
            else:
                DB.fill_(float("nan"))
                ig.check(ig.linear_backward_filter(h, 1.0, X.desc, X.ptr, DY.desc, DY.ptr, ws.ptr, ws.size, 0.0, F, Y.ptr, DB.data_ptr()))
            ws.check()
            u.close(Y.numpy(), want, tol + half * np.abs(want) + 1e-30, "%s with %s of %d bytes" % (kind, n, size))
            if kind == "filter":
                u.close(DB.double().cpu().numpy(), dy.sum(0), (M + 8) * 2.0 ** -24 * np.abs(dy).sum(0) + 1e-30, "dbias with %s of %d bytes" % (n, size))


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16"), ("f64", "f64")], ids="-".join)
@pytest.mark.parametrize("M,C", [(300, 5), (701, 264), (65, 1001), (40, 16500)])
def test_layer_norm_gradient(M, C, types):
    """Sums over rows of whole numbers: exact with any workspace."""
    u = plain._u()
    ig, h = u.ig, u.handle()
    rng = np.random.default_rng(M)
    x, dy = rng.integers(-2, 3, (M, C)).astype(float), rng.integers(-1, 2, (M, C)).astype(float)
    wide = "f64" if types[0] == "f64" else "f32"
    mean, inv = u.vector(rng.integers(-1, 2, M).astype(float), wide), u.vector(rng.integers(1, 3, M).astype(float), wide)
    X, DY, DX = u.Rows(x, types[0]), u.Rows(dy, types[1]), u.Rows((M, C), types[0])
    hh = (x - mean.double().cpu().numpy()[:, None]) * inv.double().cpu().numpy()[:, None]
    size = ig.get_layer_norm_backward_workspace_size(h, X.desc, DY.desc, DX.desc)
    for n in [(s, 0) for s in sizes(size)] + [(size, 4)]:
        ds, db = u.vector(np.full(C, np.nan), wide), u.vector(np.full(C, np.nan), wide)
        ws = Lent(*n)
        ig.check(ig.layer_norm_backward(h, 1.0, X.desc, X.ptr, DY.desc, DY.ptr, 0, mean.data_ptr(), inv.data_ptr(), ws.ptr, ws.size, 0.0, None, 0, DX.desc,
                                        DX.ptr, 0.0, ds.data_ptr(), db.data_ptr()))
        ws.check()
        assert np.array_equal(ds.double().cpu().numpy(), (dy * hh).sum(0)) and np.array_equal(db.double().cpu().numpy(), dy.sum(0)), n
