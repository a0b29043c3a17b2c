"""Products with filters in four bits on the tiles that long prompts and wide filters take, named by the profiler: against the numbers that random codes and scales stand for,
in 64 bits.

Tolerances as for the small products (e = 2^-24): a product x q is exact, its sums have at most C (float x: 3 C) + 2 groups + 20 (ranges: 16 more) roundings of no more than the sum of
the magnitudes; the activation has slopes of at most 1.13 and is off by 4e-7 (1 + |z|) (bfloat16) or 4 e (1 + |z|); then half a step of the result's type."""
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _t():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from tests import feed_forward_util as u
    from tests import kernel_names
    return torch, u, u.ig, kernel_names


def product(M, C, K, group, types, layout, units=256, residual=True, want_kernel="", ranges=None, copies=None):
    torch, u, ig, kn = _t()
    print("four-bit product", M, C, K, group, types, layout, units, flush=True)
    g = torch.Generator(device="cuda").manual_seed(M * 7 + C * 3 + K)
    xt, yt = types
    code = torch.randint(0, 16, (K, C), generator=g, device="cuda", dtype=torch.uint8)
    blocks = -(-C // 128)
    full = torch.zeros(K, blocks * 128, dtype=torch.uint8, device="cuda")
    full[:, :C] = code
    v = full.view(K, blocks, 4, 4, 4, 2).permute(0, 1, 3, 2, 4, 5)       # word 4 g + i: features 32 i + 8 g ...
    codes = (v[..., 0] | v[..., 1] << 4).reshape(K, blocks * 64).contiguous()
    groups = -(-C // group)
    scales = ((0.5 + torch.rand(groups, K, generator=g, device="cuda")) / C ** 0.5).to(torch.bfloat16)
    table = torch.tensor(VALUES + tuple(-q for q in VALUES), dtype=torch.float64, device="cuda")
    w = table[code.long()] * scales.double().t().repeat_interleave(group, 1)[:, :C]
    X, Y, R = u.Rows((M, C), xt, *layout), u.Rows((M, K), yt, *layout, fill=float("nan")), u.Rows((M, K), yt, *layout)
    X.view.copy_(torch.randn(M, C, generator=g, device="cuda") + 0.3)
    R.view.copy_(torch.randn(M, K, generator=g, device="cuda"))
    b = torch.randn(K, generator=g, device="cuda")
    h = u.handle()
    ig.set_compute_units(h, units)
    fd = u.filter_desc("bf16", K, C)
    size = ig.get_linear4_forward_workspace_size(h, X.desc, fd, group, Y.desc)
    space = u.Workspace(size)
    call = lambda: ig.check(ig.linear4_forward(h, 1.0, X.desc, X.ptr, fd, group, codes.data_ptr(), scales.data_ptr(), space.buf.data_ptr(), size, b.data_ptr(),
                                               ig.IGC_ACTIVATION_SILU, 0.5 if residual else 0.0, R.desc if residual else None, R.ptr if residual else 0, Y.desc, Y.ptr))
    _, names = kn.launched(call)
    assert any(want_kernel in n for n in names), names
    assert ranges is None or any("linear4_finish_kernel" in n for n in names) == ranges, names
    assert copies is None or any("lay_out_kernel" in n for n in names) == copies, names
    space.check()
    first = Y.view.clone()
    call()
    torch.cuda.synchronize()
    assert torch.equal(first, Y.view)                 # bit by bit
    x = X.view.double()
    z = x @ w.t() + b.double()
    y = z / (1 + torch.exp(-z))
    want = y + (0.5 * R.view.double() if residual else 0.0)
    n = (3 if xt == "f32" else 1) * C + 2 * groups + 36
    tol = n * E * (x.abs() @ w.abs().t()) + 4 * E * (z.abs() + b.double().abs())
    tol = 1.13 * tol + (4 * E if yt == "f32" else 4e-7) * (1 + z.abs()) + 4 * E * (y.abs() + (0.5 * R.view.double().abs() if residual else 0.0))
    tol = tol + u.HALF_STEP[yt] * (want.abs() + tol)
    far = ~((Y.view.double() - want).abs() <= tol)
    assert not bool(far.any()), (int(far.sum()), far.nonzero()[0].tolist(), float((Y.view.double() - want).abs().max()))
    Y.numpy()                                         # (guards)


HALF = [("bf16", "bf16"), ("bf16", "f32")]
WIDE = "linear4_wide_kernel<igc::Tile4Config<256, 256"


@pytest.mark.parametrize("types", HALF, ids="-".join)
@pytest.mark.parametrize("group", [64, 128])
def test_tiles_of_256_by_256(group, types):
    """As long prompts have them, and with the planning for eight compute units at smaller sizes: tokens and rows one off the tile, an odd number of steps, features off eight, odd rows of
    scales, one step."""
    product(2047, 1000, 8190, group, types, (8, 8), want_kernel=WIDE, copies=False)
    for i, (M, C, K) in enumerate([(1025, 449, 2047), (1023, 1001, 2305), (511, 192, 2046), (512, 64, 2048), (1024, 520, 2047), (509, 130, 2043), (1025, 2049, 2047)]):
        product(M, C, K, group, types, [(0, 0), (1, 1), (8, 8), (2, 2)][i % 4], units=8, residual=i % 2 == 0, want_kernel=WIDE)


@pytest.mark.parametrize("types", HALF, ids="-".join)
def test_tiles_of_128_by_256_in_ranges(types):
    for group in (32, 64, 128):
        product(70, 3008, 33070, group, types, (8, 8), want_kernel="Tile4Config<128, 256", ranges=True, copies=False)
        product(8193, 7895, 129, group, types, (1, 1), want_kernel="Tile4Config<128, 256", ranges=True, copies=True)


@pytest.mark.parametrize("types", HALF, ids="-".join)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_tiles_of_128_by_128(group, types):
    product(1023, 1001, 8193, group, types, (3, 1), want_kernel="Tile4Config<128, 128", copies=True)
    product(1029, 840, 2222, group, types, (0, 0), want_kernel="Tile4Config<128, 128", copies=False)
    product(300, 1001, 515, group, types, (2, 2), units=8, want_kernel="Tile4Config<128, 128")
    product(129, 192, 3329, group, types, (8, 8), units=8, residual=False)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_tiles_of_parts(group):
    """Float tokens in three parts: 64 x 256, alone and in ranges; tokens and rows one off the tile, odd widths, one step."""
    t = ("f32", "f32")
    product(1025, 1000, 8190, group, t, (8, 8), want_kernel="Tile4Config<64, 256", ranges=False)
    product(129, 2029, 5619, group, t, (1, 1), want_kernel="Tile4Config<64, 256", ranges=True)
    for i, (M, C, K) in enumerate([(513, 840, 1111), (300, 1001, 515), (255, 64, 2047), (257, 192, 2305), (191, 33, 4001)]):
        product(M, C, K, group, t, [(0, 0), (3, 1), (8, 8)][i % 3], units=8, residual=i % 2 == 0, want_kernel="Tile4Config<64, 256")
