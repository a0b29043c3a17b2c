"""Filters in four bits on the GPU: codes and scales exactly, products against the numbers they stand for, in 64 bits.

Tolerances: e = 2^-24.  A product x q is exact (float x in three parts, each product exact); its sums over a group, the scales' products and the sum over the groups
and wavefronts are at most C (float x: 3 C) + 2 groups + 20 roundings of no more than the sum of the magnitudes.  What follows has slopes of at most 1.13; the
activations are off by 4e-7 (1 + |z|) (results in bfloat16) or 4 e (1 + |z|); then half a step of the result's type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import feed_forward_oracle as fo
from oracle import four_bits_oracle as qo

E = 2.0 ** -24
GROUPS = (32, 64, 128)
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


def _u():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from tests import feed_forward_util
    return feed_forward_util


def held(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(_u().DTYPES[dtype]).double().numpy()


def on_gpu(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def stored(w, dtype, group):
    """Codes and scales by the library, guards behind both."""
    import torch
    u, ig = _u(), _u().ig
    K, C = w.shape
    fd = u.filter_desc(dtype, K, C)
    cb, sb = ig.get_filter4_size(fd, group)
    codes, scales = (torch.full((b + 64,), 0xA5, dtype=torch.uint8, device="cuda") for b in (cb, sb))
    W = on_gpu(w, u.DTYPES[dtype])
    ig.check(ig.quantize_filter4(u.handle(), fd, W.data_ptr(), group, codes.data_ptr(), scales.data_ptr()))
    torch.cuda.synchronize()
    assert bool((codes[cb:] == 0xA5).all()) and bool((scales[sb:] == 0xA5).all())
    return codes[:cb], scales[:sb]


FILTERS = [(1, 1), (3, 7), (16, 32), (5, 33), (70, 64), (64, 128), (65, 129), (17, 200), (130, 255), (33, 1001), (257, 512)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", GROUPS)
def test_into_four_bits_and_back(group, dtype):
    import torch
    u, ig = _u(), _u().ig
    for K, C in FILTERS:
        print("four bits", dtype, group, K, C, flush=True)
        rng = np.random.default_rng(K * 1000 + C)
        w = rng.standard_normal((K, C)) * np.exp(2 * rng.standard_normal((K, 1)))
        w[rng.random((K, C)) < 0.05] = 0.0
        if K > 2:
            w[1] = 0.0                                     # a row of zeros
            w[2] = np.round(w[2] * 4 / np.abs(w[2]).max()) / 4 * 6   # numbers on the borders
        w = held(w, dtype)
        codes, scales = stored(w, dtype, group)
        wc, ws = qo.quantize(w, group)
        gs = scales.view(torch.bfloat16).double().cpu().numpy().reshape(ws.shape)
        assert np.array_equal(gs, ws)
        assert np.array_equal(codes.cpu().numpy().reshape(K, -1), qo.pack(wc))
        want = qo.values(wc, ws, group)
        for back in ("f32", "bf16"):
            out = torch.full((K * C + 32,), 777.0, dtype=u.DTYPES[back], device="cuda")
            ig.check(ig.dequantize_filter4(u.handle(), group, codes.data_ptr(), scales.data_ptr(), u.filter_desc(back, K, C), out.data_ptr()))
            assert np.array_equal(out[:K * C].double().cpu().numpy().reshape(K, C), held(want, back))
            assert bool((out[K * C:] == 777.0).all())


def test_sizes_of_numbers():
    """From the smallest floats to the largest; an infinity or NaN marks its own group."""
    import torch
    u = _u()
    rng = np.random.default_rng(3)
    w = held(rng.standard_normal((40, 256)) * 10.0 ** rng.uniform(-36, 37, (40, 1)), "f32")
    w[0] = held(np.full(256, 2.0 ** -140), "f32")
    codes, scales = stored(w, "f32", 64)
    wc, ws = qo.quantize(w, 64)
    assert np.array_equal(scales.view(torch.bfloat16).double().cpu().numpy().reshape(ws.shape), ws)
    assert np.array_equal(codes.cpu().numpy().reshape(40, -1), qo.pack(wc))
    w[7, 70], w[9, 5] = np.inf, np.nan
    codes, scales = stored(w, "f32", 64)
    s = scales.view(torch.bfloat16).double().cpu().numpy().reshape(4, 40)
    bad = np.zeros((4, 40), bool)
    bad[1, 7] = bad[0, 9] = True
    assert np.array_equal(np.isnan(s), bad) and np.array_equal(s[~bad], ws[~bad])


def product(M, C, K, group, types, layout=(0, 0), act=None, residual=False, bias=True, alpha=1.0, beta=1.0, room=None, check=True, rng=None):
    u, ig = _u(), _u().ig
    xt, yt = types
    rng = rng or np.random.default_rng(M * 7 + C * 3 + K)
    wc, ws = qo.quantize(held(rng.standard_normal((K, C)) / np.sqrt(C), "bf16"), group)
    w = qo.values(wc, ws, group)
    x = held(rng.standard_normal((M, C)) + 0.3, xt)
    X = u.Rows(x, xt, *layout)
    Y = u.Rows((M, K), yt, *layout, fill=float("nan"))
    r = held(rng.standard_normal((M, K)), yt) if residual else None
    R = u.Rows(r, yt, *layout) if residual else None
    b = held(rng.standard_normal(K), "f32") if bias else None
    fd, h = u.filter_desc("bf16", K, C), u.handle()
    import torch
    codes, scales = on_gpu(qo.pack(wc)), on_gpu(ws, torch.bfloat16)
    size = ig.get_linear4_forward_workspace_size(h, X.desc, fd, group, Y.desc)
    ws_ = u.Workspace(size if room is None else min(size, room))
    code = {None: -1, "relu": ig.IGC_ACTIVATION_RELU, "gelu": ig.IGC_ACTIVATION_GELU, "silu": ig.IGC_ACTIVATION_SILU, "tanh": ig.IGC_ACTIVATION_TANH,
            "sigmoid": ig.IGC_ACTIVATION_SIGMOID}[act]
    bt = u.vector(b) if bias else None
    ig.check(ig.linear4_forward(h, alpha, X.desc, X.ptr, fd, group, codes.data_ptr(), scales.data_ptr(), ws_.buf.data_ptr() if ws_.size else 0, ws_.size, u.ptr(bt), code,
                                beta if residual else 0.0, u.desc(R), u.ptr(R), Y.desc, Y.ptr), "igcLinear4Forward")
    ws_.check()
    z = alpha * (x @ w.T) + (b if bias else 0.0)
    y = fo.activation(code, z)
    want = y + (beta * r if residual else 0.0)
    n = (3 if xt == "f32" else 1) * C + 2 * len(ws) + 20
    tol = n * E * abs(alpha) * (np.abs(x) @ np.abs(w).T) + 4 * E * (np.abs(z) + (np.abs(b) if bias else 0.0))
    tol = 1.13 * tol + (4 * E if yt == "f32" else 4e-7) * (1 + np.abs(z)) * (act is not None) + 4 * E * (np.abs(y) + (np.abs(beta * r) if residual else 0.0))
    got = Y.numpy()
    if check:
        u.close(got, want, tol + u.HALF_STEP[yt] * (np.abs(want) + tol) + 1e-37, "y of %s" % ((M, C, K, group, types, layout, act, residual),))
    return got


SHAPES = [(1, 1, 1), (1, 64, 64), (2, 33, 5), (3, 128, 17), (7, 200, 70), (16, 256, 64), (17, 1001, 33), (1, 4096, 130), (33, 640, 257), (40, 96, 1000), (64, 129, 48),
          (65, 512, 80), (130, 333, 190), (300, 160, 520)]


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("group", GROUPS)
def test_products(group, types):
    for i, (M, C, K) in enumerate(SHAPES):
        print("four-bit product", group, types, M, C, K, flush=True)
        layout = [(0, 0), (3, 1), (8, 8), (1, 0)][i % 4]
        product(M, C, K, group, types, layout, [None, "gelu", "relu", "silu", "tanh", "sigmoid"][i % 6], residual=i % 2 == 1, bias=i % 3 != 2,
                alpha=1.0 if i % 5 else -0.75, beta=1.0 if i % 4 else 2.5)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_wide_and_long(types):
    """Enough rows of W for the wider pieces, and more tokens than a piece."""
    for M, C, K, group in ((1, 384, 16400, 32), (5, 130, 20000, 64), (20, 384, 9000, 128), (50, 64, 8200, 64), (100, 260, 9000, 32),
                           (700, 512, 2050, 128), (1029, 200, 1111, 64)):
        print("four-bit product", types, M, C, K, group, flush=True)
        product(M, C, K, group, types, (8, 8) if M % 2 else (1, 1), "gelu", residual=True)


def test_rows_of_x_keep_to_themselves():
    """What is infinite or undefined in a row of x stays in that row of y; what lies behind a row is not read."""
    import torch
    u, ig = _u(), _u().ig
    for types in TYPES:
        for M, C, K in ((5, 200, 40), (70, 200, 300), (600, 200, 300)):
            rng = np.random.default_rng(4)
            wc, ws = qo.quantize(held(rng.standard_normal((K, C)), "bf16"), 32)
            x = held(rng.standard_normal((M, C)), types[0])
            X = u.Rows(x, types[0], 3, 1)
            X.buf.fill_(float("nan"))
            X.view.copy_(torch.from_numpy(x))
            X.view[1, 3] = float("inf")
            X.view[3, 199] = float("nan")
            Y = u.Rows((M, K), types[1], 3, 1, fill=0.0)
            codes, scales, h, fd = on_gpu(qo.pack(wc)), on_gpu(ws, torch.bfloat16), u.handle(), u.filter_desc("bf16", K, C)
            size = ig.get_linear4_forward_workspace_size(h, X.desc, fd, 32, Y.desc)
            space = u.Workspace(size)
            ig.check(ig.linear4_forward(h, 1.0, X.desc, X.ptr, fd, 32, codes.data_ptr(), scales.data_ptr(), space.buf.data_ptr(), size, 0, -1, 0.0, None, 0, Y.desc, Y.ptr))
            got = Y.numpy()
            assert not np.isfinite(got[1]).any() and np.isnan(got[3]).all()
            rest = [m for m in range(M) if m not in (1, 3)]
            w = qo.values(wc, ws, 32)
            assert np.isfinite(got[rest]).all() and np.abs(got[rest] - x[rest] @ w.T).max() < 0.02 * np.abs(w).sum(1).max()


def test_residual_in_place_and_workspaces():
    """y over r itself; the same results to rounding whatever the room lent."""
    import torch
    u, ig = _u(), _u().ig
    rng = np.random.default_rng(6)
    M, C, K, group = 90, 300, 200, 64
    for types in TYPES:
        wc, ws = qo.quantize(held(rng.standard_normal((K, C)) / 17, "bf16"), group)
        w = qo.values(wc, ws, group)
        x, r = held(rng.standard_normal((M, C)), types[0]), held(rng.standard_normal((M, K)), types[1])
        X, Y = u.Rows(x, types[0], 1, 1), u.Rows(r, types[1], 2, 0)
        codes, scales, h, fd = on_gpu(qo.pack(wc)), on_gpu(ws, torch.bfloat16), u.handle(), u.filter_desc("f32", K, C)
        ig.check(ig.linear4_forward(h, 1.0, X.desc, X.ptr, fd, group, codes.data_ptr(), scales.data_ptr(), 0, 0, 0, -1, 1.0, Y.desc, Y.ptr, Y.desc, Y.ptr))
        want = x @ w.T + r
        u.close(Y.numpy(), want, 1e-4 + u.HALF_STEP[types[1]] * np.abs(want) * 1.01, "in place")
    for room in (0, 16, 5000, 1 << 20):
        product(700, 520, 600, 32, ("f32", "f32"), (1, 1), None, room=room)
        product(700, 520, 600, 32, ("bf16", "bf16"), (1, 1), None, room=room)


def test_repeats_in_a_graph_and_on_another_stream():
    import torch
    u, ig = _u(), _u().ig
    rng = np.random.default_rng(8)
    for M in (1, 300):
        C, K, group = 1000, 500, 128
        wc, ws = qo.quantize(held(rng.standard_normal((K, C)), "bf16"), group)
        codes, scales, fd = on_gpu(qo.pack(wc)), on_gpu(ws, torch.bfloat16), u.filter_desc("bf16", K, C)
        x = torch.randn(M, C, device="cuda").to(torch.bfloat16)
        xd, yd = (ig.TensorDescriptor().set(ig.IGC_DATA_BFLOAT16, M, n, 1, 1, (n, 1, 1, 1)) for n in (C, K))
        size = ig.get_linear4_forward_workspace_size(u.handle(), xd, fd, group, yd)

        def call(y, space, stream):
            h = ig.Handle()
            h.set_stream(stream.cuda_stream)
            ig.check(ig.linear4_forward(h, 1.0, xd, x.data_ptr(), fd, group, codes.data_ptr(), scales.data_ptr(), space.data_ptr(), size, 0, ig.IGC_ACTIVATION_GELU, 0.0, None, 0,
                                        yd, y.data_ptr()))

        y, z, e = (torch.zeros(M, K, dtype=torch.bfloat16, device="cuda") for _ in range(3))
        a, b = (torch.empty(max(size, 16), dtype=torch.uint8, device="cuda") for _ in range(2))
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            call(y, a, torch.cuda.current_stream())
        for i in range(4):
            x.copy_(torch.randn(M, C, device="cuda"))
            graph.replay()
            call(e, b, torch.cuda.current_stream())
            torch.cuda.synchronize()
            assert torch.equal(y, e), i
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        call(z, b, other)
        other.synchronize()
        assert torch.equal(y, z)


def test_codes_beyond_32_bits():
    """A filter of 4.6 GB in four bits, whose last rows lie behind 2^32 bytes, and of 18 GB as bfloat16: codes, numbers, and products with one token to many."""
    import torch
    u, ig = _u(), _u().ig
    K, C, group, some = 140001, 65536 + 40, 128, 24
    rng = np.random.default_rng(21)
    rows = np.concatenate([np.arange(some), np.arange(K - some, K)])
    w = held(rng.standard_normal((2 * some, C)), "bf16")
    W = torch.zeros(K, C, dtype=torch.bfloat16, device="cuda")
    W[torch.from_numpy(rows).cuda()] = on_gpu(w, torch.bfloat16)
    fd, h = u.filter_desc("bf16", K, C), u.handle()
    cb, sb = ig.get_filter4_size(fd, group)
    assert cb > 2 ** 32
    codes, scales = (torch.full((b,), 0xA5, dtype=torch.uint8, device="cuda") for b in (cb, sb))
    ig.check(ig.quantize_filter4(h, fd, W.data_ptr(), group, codes.data_ptr(), scales.data_ptr()))
    wc, ws = qo.quantize(w, group)
    at = torch.from_numpy(rows).cuda()
    assert np.array_equal(codes.view(K, -1)[at].cpu().numpy(), qo.pack(wc))
    assert np.array_equal(scales.view(torch.bfloat16).view(-1, K)[:, at].double().cpu().numpy(), ws)
    assert not bool(codes.view(K, -1)[some:K - some].any())
    W.fill_(7.0)
    ig.check(ig.dequantize_filter4(h, group, codes.data_ptr(), scales.data_ptr(), fd, W.data_ptr()))
    values = qo.values(wc, ws, group)
    assert np.array_equal(W[at].double().cpu().numpy(), held(values, "bf16")) and not bool(W[some:K - some].any())
    del W
    for M in (1, 20, 300):
        print("far codes", M, flush=True)
        x = held(rng.standard_normal((M, C)), "bf16")
        X = on_gpu(x, torch.bfloat16)
        Y = torch.full((M, K), float("nan"), device="cuda")
        xd, yd = ig.TensorDescriptor().set(ig.IGC_DATA_BFLOAT16, M, C, 1, 1, (C, 1, 1, 1)), ig.TensorDescriptor().set(ig.IGC_DATA_FLOAT, M, K, 1, 1, (K, 1, 1, 1))
        space = u.Workspace(ig.get_linear4_forward_workspace_size(h, xd, fd, group, yd))
        ig.check(ig.linear4_forward(h, 1.0, xd, X.data_ptr(), fd, group, codes.data_ptr(), scales.data_ptr(), space.buf.data_ptr(), space.size, 0, -1, 0.0, None, 0, yd,
                                    Y.data_ptr()))
        space.check()
        want = x @ values.T
        tol = (C + 2 * len(ws) + 20) * E * (np.abs(x) @ np.abs(values).T)
        u.close(Y[:, at].double().cpu().numpy(), want, tol + E * (np.abs(want) + tol), "y of far codes, %d tokens" % M)
        assert not bool(Y[:, some:K - some].any())
    del codes, scales, Y, X
    torch.cuda.empty_cache()


def test_rows_beyond_32_bits():
    """Rows of x and y 2^25 elements apart: the last ones lie behind 2^32 bytes."""
    import torch
    u, ig = _u(), _u().ig
    C, K, group, apart = 200, 90, 64, 2 ** 25
    for types in TYPES:
        for M in (70, 130):
            print("far rows", types, M, flush=True)
            rng = np.random.default_rng(M)
            wc, ws = qo.quantize(held(rng.standard_normal((K, C)) / 14, "bf16"), group)
            w = qo.values(wc, ws, group)
            x = held(rng.standard_normal((M, C)), types[0])
            X = torch.empty(M * apart, dtype=u.DTYPES[types[0]], device="cuda").view(M, apart)
            X[:, :C] = on_gpu(x, u.DTYPES[types[0]])
            Y = torch.empty(M * apart, dtype=u.DTYPES[types[1]], device="cuda").view(M, apart)
            Y[:, :K + 8] = float("nan")
            data = {"f32": ig.IGC_DATA_FLOAT, "bf16": ig.IGC_DATA_BFLOAT16}
            xd, yd = ig.TensorDescriptor().set(data[types[0]], M, C, 1, 1, (apart, 1, 1, 1)), ig.TensorDescriptor().set(data[types[1]], M, K, 1, 1, (apart, 1, 1, 1))
            codes, scales, h, fd = on_gpu(qo.pack(wc)), on_gpu(ws, torch.bfloat16), u.handle(), u.filter_desc("bf16", K, C)
            space = u.Workspace(ig.get_linear4_forward_workspace_size(h, xd, fd, group, yd))
            ig.check(ig.linear4_forward(h, 1.0, xd, X.data_ptr(), fd, group, codes.data_ptr(), scales.data_ptr(), space.buf.data_ptr(), space.size, 0, -1, 0.0, None, 0, yd,
                                        Y.data_ptr()))
            want = x @ w.T
            tol = ((3 if types[0] == "f32" else 1) * C + 2 * len(ws) + 20) * E * (np.abs(x) @ np.abs(w).T)
            u.close(Y[:, :K].double().cpu().numpy(), want, tol + u.HALF_STEP[types[1]] * (np.abs(want) + tol), "y of far rows %s" % ((types, M),))
            assert bool(Y[:, K:K + 8].isnan().all())
            del X, Y
            torch.cuda.empty_cache()


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_ranges_of_the_reduction(types):
    """Few rows of W and long ones: ranges of blocks, which end anywhere in the rows, added in a second launch."""
    for M, C, K, group in ((3, 16000, 100, 32), (16, 9001, 65, 128), (20, 5001, 333, 64), (17, 4096, 40, 32), (33, 3000, 700, 128), (64, 4096, 600, 64), (100, 8000, 130, 32),
                           (129, 2500, 257, 64), (257, 3000, 260, 128), (500, 1500, 130, 32)):
        for layout in ((0, 0), (1, 1)):
            print("four-bit product in ranges", types, M, C, K, group, layout, flush=True)
            product(M, C, K, group, types, layout, "silu", residual=True)


def test_off_words():
    """x of even rows and scales that begin 2 bytes behind a word."""
    import torch
    u, ig = _u(), _u().ig
    for M, C, K, group in ((20, 4096, 300, 32), (64, 512, 200, 64), (700, 520, 602, 128)):
        rng = np.random.default_rng(M)
        wc, ws = qo.quantize(held(rng.standard_normal((K, C)) / 20, "bf16"), group)
        w, x = qo.values(wc, ws, group), held(rng.standard_normal((M, C)), "bf16")
        X, Y, h, fd = u.Rows(x, "bf16", 8, 1), u.Rows((M, K), "f32", 0, 0, fill=float("nan")), u.handle(), u.filter_desc("bf16", K, C)
        codes, scales = on_gpu(qo.pack(wc)), torch.zeros(ws.size + 1, dtype=torch.bfloat16, device="cuda")
        scales[1:] = on_gpu(ws.reshape(-1), torch.bfloat16)
        space = u.Workspace(ig.get_linear4_forward_workspace_size(h, X.desc, fd, group, Y.desc))
        ig.check(ig.linear4_forward(h, 1.0, X.desc, X.ptr, fd, group, codes.data_ptr(), scales[1:].data_ptr(), space.buf.data_ptr(), space.size, 0, -1, 0.0, None, 0, Y.desc, Y.ptr))
        space.check()
        want = x @ w.T
        tol = (C + 2 * len(ws) + 20) * E * (np.abs(x) @ np.abs(w).T)
        u.close(Y.numpy(), want, tol + E * (np.abs(want) + tol), "y off words %s" % ((M, C, K, group),))
