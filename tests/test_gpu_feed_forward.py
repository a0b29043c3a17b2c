"""Layer norm and the matrix products with their epilogues on the GPU, element by element against the formulas in 64 bits.

Tolerances.  u: half a step of the result's type; e = 2^-24 (2^-53 for double).  A sum of n products in any order is off by at
most (n + 4) e times the sum of the products' magnitudes; float products taken in three parts (8 bits of the
significand each, m < 2^-7 and l < 2^-15 of the number) leave out m l + l m + l l, less than 2^-21 + 2^-30 of a product.  What
follows the sum has slopes of at most 1.13 (GELU), 1.1 (SiLU) or 1; the activations computed for bfloat16 results are off by up
to 4e-7 (1 + |z|) (the polynomial's 1.5e-7, the exponential, the reciprocal), those for float results by 4e (1 + |z|)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import feed_forward_oracle as fo

EPS = 1e-5
# (layout: elements between the rows, elements in front of the first)
LAYOUTS = [(0, 0), (3, 1), (8, 8), (1, 0)]


def _u():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from tests import feed_forward_util
    return feed_forward_util


def rounded(a, dtype):
    """float64 values that the type holds"""
    import torch
    u = _u()
    return torch.from_numpy(np.ascontiguousarray(a)).to(u.DTYPES[dtype]).double().numpy()


def normal(rng, *shape):
    return rng.standard_normal(shape)


def eps_of(dtype):
    return 2.0 ** -53 if dtype == "f64" else 2.0 ** -24


# ---- layer norm -------------------------------------------------------------------------------------------------------
NORM_TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f64", "f64")]
NORM_SHAPES = [(1, 1), (3, 2), (5, 33), (2, 64), (7, 255), (4, 512), (3, 777), (66, 1000), (5, 1001), (3, 1024), (2, 2049), (3, 4096), (2, 8200), (1, 16384),
               (2, 16391), (1, 40000)]


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("types", NORM_TYPES, ids="-".join)
def test_layer_norm_forward(types, layout):
    u, ig = _u(), _u().ig
    dtype, out = types
    wide, e, half = ("f64" if dtype == "f64" else "f32"), eps_of(dtype), _u().HALF_STEP[out]
    h = u.handle()
    for M, C in NORM_SHAPES:
        rng = np.random.default_rng(M * 100003 + C)
        x = rounded(normal(rng, M, C) * 2 + 3 * normal(rng, M, 1), dtype)
        scale, shift = rounded(1 + 0.3 * normal(rng, C), wide), rounded(0.2 * normal(rng, C), wide)
        old = rounded(normal(rng, M, C), out)
        for given, alpha, beta in ((True, 1.0, 0.0), (False, 1.0, 0.0), (True, 0.75, -1.5)):
            print("layer norm", types, layout, M, C, given, beta, flush=True)
            X, Y = u.Rows(x, dtype, *layout), (u.Rows(old, out, *layout) if beta else u.Rows((M, C), out, *layout, fill=float("nan")))
            S, B = (u.vector(scale, wide), u.vector(shift, wide)) if given else (None, None)
            mean, inv = (u.vector(np.full(M, np.nan), wide) for _ in range(2))
            ig.check(ig.layer_norm_forward(h, alpha, X.desc, X.ptr, u.ptr(S), u.ptr(B), EPS, beta, Y.desc, Y.ptr, mean.data_ptr(), inv.data_ptr()))
            wy, wm, ws = fo.layer_norm(x, scale if given else None, shift if given else None, EPS)
            # a sum of C elements: (C + 4) e of the magnitudes' sum; the deviation's average of squares the same relative to itself
            em = (C + 4) * e * np.abs(x).mean(1)
            d = np.abs(x - wm[:, None])
            es = ws * (2 * (C + 8) * e + ws * ws * 2 * em * d.mean(1) + ws * ws * em * em)
            u.close(mean.double().cpu().numpy(), wm, em + 1e-300, "mean")
            u.close(inv.double().cpu().numpy(), ws, es + 4 * e * ws, "1/deviation")
            sc = np.abs(scale) if given else 1.0
            tol = (em[:, None] * ws[:, None] + d * (es[:, None] + 6 * e * ws[:, None])) * sc + 4 * e * (np.abs(wy) + (np.abs(shift) if given else 0) + np.abs(beta * old))
            want = alpha * wy + (beta * old if beta else 0)
            u.close(Y.numpy(), want, abs(alpha) * tol + 4 * e * np.abs(beta * old) + half * np.abs(want) * 1.01 + 1e-30, "y")


def test_layer_norm_in_place_and_rows_without_spread():
    u, ig = _u(), _u().ig
    import torch
    h = u.handle()
    rng = np.random.default_rng(5)
    for C in (64, 1000, 5000):
        x = rounded(normal(rng, 6, C), "f32")
        x[1], x[2], x[3] = 0.0, 2.5, 1e4 + rounded(normal(rng, C), "f32")
        x = rounded(x, "f32")
        X = u.Rows(x, "f32")
        ig.check(ig.layer_norm_forward(h, 1.0, X.desc, X.ptr, 0, 0, EPS, 0.0, X.desc, X.ptr))
        want, m, s = fo.layer_norm(x, None, None, EPS)
        em = (C + 4) * 2.0 ** -24 * np.abs(x).mean(1)
        d = np.abs(x - m[:, None])
        es = s * (2 * (C + 8) * 2.0 ** -24 + s * s * 2 * em * d.mean(1) + s * s * em * em)
        u.close(X.numpy(), want, em[:, None] * s[:, None] + d * (es + 6 * 2.0 ** -24 * s)[:, None] + 1e-6 * np.abs(want) + 1e-30, "in place")
        # infinities and NaN stay in their rows
        y = x.copy()
        y[0, 3], y[4, C - 1] = np.inf, np.nan
        Y, O = u.Rows(y, "f32"), u.Rows((6, C), "f32", fill=0.0)
        ig.check(ig.layer_norm_forward(h, 1.0, Y.desc, Y.ptr, 0, 0, EPS, 0.0, O.desc, O.ptr))
        got = O.view.cpu().numpy()
        assert np.isnan(got[0, 3]) and np.isnan(got[4]).all() and np.isfinite(got[[1, 2, 3, 5]]).all()


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("types", NORM_TYPES, ids="-".join)
def test_layer_norm_backward(types, layout):
    u, ig = _u(), _u().ig
    dtype, out = types
    wide, e = ("f64" if dtype == "f64" else "f32"), eps_of(dtype)
    h = u.handle()
    for M, C in NORM_SHAPES + [(700, 40), (1500, 264), (333, 2056)]:
        rng = np.random.default_rng(M * 7919 + C)
        x = rounded(normal(rng, M, C) * 2 + normal(rng, M, 1), dtype)
        dy = rounded(normal(rng, M, C), out)
        scale = rounded(1 + 0.3 * normal(rng, C), wide)
        r = rounded(normal(rng, M, C), dtype)
        _, mean, inv = fo.layer_norm(x, None, None, EPS)
        mean, inv = rounded(mean, wide), rounded(inv, wide)
        old = rounded(normal(rng, 2, C), wide)
        for given, beta, pb, lend in ((True, 1.0, 0.0, True), (False, 0.0, 0.5, False), (True, -0.5, 2.0, True)):
            print("layer norm backward", types, layout, M, C, given, beta, lend, flush=True)
            alpha = 1.0 if beta == 1.0 else 1.25
            X, DY = u.Rows(x, dtype, *layout), u.Rows(dy, out, *layout)
            R = u.Rows(r, dtype, *layout) if beta else None
            DX = R if beta == -0.5 else u.Rows((M, C), dtype, *layout, fill=float("nan"))       # (once into r itself)
            S, m, s = u.vector(scale, wide) if given else None, u.vector(mean, wide), u.vector(inv, wide)
            ds, db = (u.vector(old[i] if pb else np.full(C, np.nan), wide) for i in range(2))
            size = ig.get_layer_norm_backward_workspace_size(h, X.desc, DY.desc, DX.desc) if lend else 0
            ws = u.Workspace(size)
            ig.check(ig.layer_norm_backward(h, alpha, X.desc, X.ptr, DY.desc, DY.ptr, u.ptr(S), m.data_ptr(), s.data_ptr(), ws.buf.data_ptr(), size,
                                            beta, u.desc(R), u.ptr(R), DX.desc, DX.ptr, pb, ds.data_ptr(), db.data_ptr()))
            ws.check()
            wdx, wds, wdb = fo.layer_norm_backward(x, dy, scale if given else None, mean, inv)
            hh = np.abs(x - mean[:, None]) * inv[:, None] + np.abs(mean * inv)[:, None] * 2.0
            q = np.abs(dy * scale) if given else np.abs(dy)
            tol = inv[:, None] * ((C + 8) * e * (q.mean(1) + 0 * q.T).T + (C + 16) * e * hh * (q * hh).mean(1)[:, None] + 8 * e * q)
            want = alpha * wdx + (beta * r if beta else 0)
            half = u.HALF_STEP[dtype]
            u.close(DX.numpy(), want, abs(alpha) * tol + 4 * e * np.abs(beta * r) + half * np.abs(want) * 1.01 + 1e-30, "dx")
            for got, w, o, mag in ((ds, wds, old[0], (np.abs(dy) * hh).sum(0)), (db, wdb, old[1], np.abs(dy).sum(0))):
                want = alpha * w + (pb * o if pb else 0)
                u.close(got.double().cpu().numpy(), want, (M + 8) * e * (alpha * mag + np.abs(pb * o)) + 1e-30, "dscale or dshift")
            if beta != -0.5:   # dscale and dshift left out: the same dx
                DX2 = u.Rows((M, C), dtype, *layout, fill=float("nan"))
                ig.check(ig.layer_norm_backward(h, alpha, X.desc, X.ptr, DY.desc, DY.ptr, u.ptr(S), m.data_ptr(), s.data_ptr(), 0, 0, beta, u.desc(R),
                                                u.ptr(R), DX2.desc, DX2.ptr, pb, 0, 0))
                u.close(DX2.numpy(), DX.numpy(), 2 * abs(alpha) * tol + half * 2.02 * np.abs(DX.numpy()) + 1e-30, "dx alone")


def test_layer_norm_gradient_against_differences():
    """dx, dscale and dshift of sum(dy * y) in double against central differences of the forward pass on the GPU."""
    u, ig = _u(), _u().ig
    rng = np.random.default_rng(11)
    M, C, step = 3, 37, 1e-5
    x, dy, scale, shift = normal(rng, M, C), normal(rng, M, C), 1 + 0.3 * normal(rng, C), normal(rng, C)
    h = u.handle()

    def loss(x, scale, shift):
        X, Y, S, B = u.Rows(x, "f64"), u.Rows((M, C), "f64"), u.vector(scale, "f64"), u.vector(shift, "f64")
        ig.check(ig.layer_norm_forward(h, 1.0, X.desc, X.ptr, S.data_ptr(), B.data_ptr(), EPS, 0.0, Y.desc, Y.ptr))
        return float((Y.numpy() * dy).sum())

    X, DY, Y, DX = u.Rows(x, "f64"), u.Rows(dy, "f64"), u.Rows((M, C), "f64"), u.Rows((M, C), "f64")
    S, B = u.vector(scale, "f64"), u.vector(shift, "f64")
    mean, inv, ds, db = (u.vector(np.zeros(n), "f64") for n in (M, M, C, C))
    ig.check(ig.layer_norm_forward(h, 1.0, X.desc, X.ptr, S.data_ptr(), B.data_ptr(), EPS, 0.0, Y.desc, Y.ptr, mean.data_ptr(), inv.data_ptr()))
    ig.check(ig.layer_norm_backward(h, 1.0, X.desc, X.ptr, DY.desc, DY.ptr, S.data_ptr(), mean.data_ptr(), inv.data_ptr(), 0, 0, 0.0, None, 0, DX.desc,
                                    DX.ptr, 0.0, ds.data_ptr(), db.data_ptr()))
    dx = DX.numpy()
    for i, c in ((0, 0), (1, 17), (2, 36)):
        d = np.zeros_like(x)
        d[i, c] = step
        assert abs((loss(x + d, scale, shift) - loss(x - d, scale, shift)) / (2 * step) - dx[i, c]) < 1e-7
        v = d[i]
        assert abs((loss(x, scale + v, shift) - loss(x, scale - v, shift)) / (2 * step) - ds[c].item()) < 1e-7
        assert abs((loss(x, scale, shift + v) - loss(x, scale, shift - v)) / (2 * step) - db[c].item()) < 1e-7


# ---- products ---------------------------------------------------------------------------------------------------------
LINEAR_TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]
# rows, features in, features out
LINEAR_SHAPES = [(1, 1, 1), (1, 64, 64), (3, 65, 70), (8, 256, 192), (17, 130, 33), (31, 8, 520), (64, 64, 64), (65, 72, 136), (100, 257, 129), (128, 192, 128),
                 (130, 40, 24), (200, 136, 264), (257, 320, 255), (300, 64, 512), (520, 328, 264)]


def act_error(out, z):
    return (4e-7 if out == "bf16" else 4 * 2.0 ** -24) * (1 + np.abs(z))


def linear_case(types, M, C, K):
    dtype, out = types
    rng = np.random.default_rng(M * 1000003 + C * 1009 + K)
    x, w, dy = rounded(normal(rng, M, C), dtype), rounded(normal(rng, K, C) / np.sqrt(C), dtype), rounded(normal(rng, M, K), dtype)
    return rng, x, w, dy


def sum_error(n, magnitude, dtype):
    return ((n + 4) * 2.0 ** -24 + (2.0 ** -21 + 2.0 ** -30 if dtype == "f32" else 0)) * magnitude


@pytest.mark.parametrize("lend", [True, False], ids=["workspace", "alone"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("types", LINEAR_TYPES, ids="-".join)
def test_linear_forward(types, layout, lend):
    u, ig = _u(), _u().ig
    dtype, out = types
    h, half = u.handle(), u.HALF_STEP[out]
    acts = list(fo.ACTIVATIONS)
    for i, (M, C, K) in enumerate(LINEAR_SHAPES):
        rng, x, w, _ = linear_case(types, M, C, K)
        bias, r = rounded(normal(rng, K), "f32"), rounded(normal(rng, M, K), out)
        W, WD = u.vector(w, dtype), u.filter_desc(dtype, K, C)
        X = u.Rows(x, dtype, *layout)
        for j, (alpha, beta, has_bias, keep) in enumerate(((1.0, 0.0, True, False), (1.0, 1.0, True, True), (-0.5, 0.5, False, True))):
            act = fo.ACTIVATIONS[acts[(i + 2 * j) % len(acts)]]
            print("linear", types, layout, M, C, K, act, alpha, beta, flush=True)
            R = u.Rows(r, out, *layout) if beta else None
            Y = R if beta == 0.5 else u.Rows((M, K), out, *layout, fill=float("nan"))           # (once into r itself)
            Z = u.Rows((M, K), out, *layout, fill=float("nan")) if keep else None
            B = u.vector(bias) if has_bias else None
            size = ig.get_linear_forward_workspace_size(h, X.desc, WD, Y.desc) if lend else 0
            ws = u.Workspace(size)
            ig.check(ig.linear_forward(h, alpha, X.desc, X.ptr, WD, W.data_ptr(), ws.buf.data_ptr() if lend else 0, size, u.ptr(B), act, beta, u.desc(R),
                                       u.ptr(R), Y.desc, u.ptr(Z), Y.ptr))
            ws.check()
            wy, wz = fo.linear(x, w, bias if has_bias else None, act, r if beta else None, alpha, beta)
            ez = abs(alpha) * sum_error(C, np.abs(x) @ np.abs(w).T, dtype) + 2 * 2.0 ** -24 * np.abs(wz)
            u.close(Y.numpy(), wy, 1.13 * ez + act_error(out, wz) + 2 * 2.0 ** -24 * np.abs(beta * r) + 1.01 * half * np.abs(wy) + 1e-30, "y")
            if keep:
                u.close(Z.numpy(), wz, ez + 1.01 * half * np.abs(wz) + 1e-30, "z")


@pytest.mark.parametrize("lend", [True, False], ids=["workspace", "alone"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("types", LINEAR_TYPES, ids="-".join)
def test_linear_backward_data(types, layout, lend):
    u, ig = _u(), _u().ig
    dtype, out = types
    h, half = u.handle(), u.HALF_STEP[out]
    acts = list(fo.ACTIVATIONS)
    for i, (M, C, K) in enumerate(LINEAR_SHAPES):
        rng, _, w, dy = linear_case(types, M, C, K)
        z, r = rounded(1.5 * normal(rng, M, C), out), rounded(normal(rng, M, C), out)
        W, WD = u.vector(w, dtype), u.filter_desc(dtype, K, C)
        DY, Z = u.Rows(dy, dtype, *layout), u.Rows(z, out, *layout)
        for j, (alpha, beta) in enumerate(((1.0, 0.0), (1.0, 1.0), (-0.5, 0.5))):
            act = fo.ACTIVATIONS[acts[(i + 2 * j) % len(acts)]]
            print("linear backward data", types, layout, M, C, K, act, alpha, beta, flush=True)
            R = u.Rows(r, out, *layout) if beta else None
            DX = R if beta == 0.5 else u.Rows((M, C), out, *layout, fill=float("nan"))
            size = ig.get_linear_backward_data_workspace_size(h, WD, DY.desc, DX.desc) if lend else 0
            ws = u.Workspace(size)
            ig.check(ig.linear_backward_data(h, alpha, WD, W.data_ptr(), DY.desc, DY.ptr, ws.buf.data_ptr() if lend else 0, size, act,
                                             u.desc(Z) if act != -1 else None, Z.ptr if act != -1 else 0, beta, u.desc(R), u.ptr(R), DX.desc, DX.ptr))
            ws.check()
            want = fo.linear_backward_data(dy, w, act, z, r if beta else None, alpha, beta)
            g = np.abs(alpha * (dy @ w))
            tol = 1.13 * abs(alpha) * sum_error(K, np.abs(dy) @ np.abs(w), dtype) + g * act_error(out, z) + 4 * 2.0 ** -24 * (g + np.abs(beta * r))
            u.close(DX.numpy(), want, tol + 1.01 * half * np.abs(want) + 1e-30, "dx")


@pytest.mark.parametrize("lend", [True, False], ids=["workspace", "alone"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("types", LINEAR_TYPES, ids="-".join)
def test_linear_backward_filter(types, layout, lend):
    u, ig = _u(), _u().ig
    dtype, out = types
    h, half = u.handle(), u.HALF_STEP[out]
    for M, C, K in LINEAR_SHAPES + [(2000, 64, 72), (1111, 65, 33), (1, 600, 520), (4000, 8, 300)]:
        rng, x, _, dy = linear_case(types, M, C, K)
        old, oldb = rounded(normal(rng, K, C), out), rounded(normal(rng, K), "f32")
        X, DY = u.Rows(x, dtype, *layout), u.Rows(dy, dtype, *layout)
        for alpha, beta, with_bias in ((1.0, 0.0, True), (0.5, -1.0, True), (1.0, 1.0, False)):
            print("linear backward filter", types, layout, M, C, K, alpha, beta, flush=True)
            DW = u.Rows(old, out) if beta else u.Rows((K, C), out, fill=float("nan"))
            DB = u.vector(oldb if beta else np.full(K, np.nan)) if with_bias else None
            WD = u.filter_desc(out, K, C)
            size = ig.get_linear_backward_filter_workspace_size(h, X.desc, DY.desc, WD) if lend else 0
            ws = u.Workspace(size)
            ig.check(ig.linear_backward_filter(h, alpha, X.desc, X.ptr, DY.desc, DY.ptr, ws.buf.data_ptr() if lend else 0, size, beta, WD, DW.ptr, u.ptr(DB)))
            ws.check()
            ww, wb = fo.linear_backward_filter(dy, x, alpha, beta, old if beta else None, oldb if beta else None)
            tol = abs(alpha) * sum_error(M, np.abs(dy).T @ np.abs(x), dtype) + 4 * 2.0 ** -24 * np.abs(beta * old)
            u.close(DW.numpy(), ww, tol + 1.01 * half * np.abs(ww) + 1e-30, "dw")
            if with_bias:
                u.close(DB.double().cpu().numpy(), wb, (M + 8) * 2.0 ** -24 * (np.abs(dy).sum(0) + np.abs(beta * oldb)) + 1e-30, "dbias")


# sizes at which the large tiles, the ranges of the reduction and the kernels for few tokens run, none a multiple of theirs
LARGE_SHAPES = [(4000, 4104, 4040), (1023, 2050, 1000), (3, 9000, 520), (40, 5000, 300), (600, 776, 640), (1, 640, 9003)]


@pytest.mark.parametrize("pad", [0, 1, 8])
@pytest.mark.parametrize("types", LINEAR_TYPES, ids="-".join)
def test_large_products(types, pad):
    """Forward with residual and kept z, backward data through SiLU, backward filter with the bias, against products in 64 bits on the GPU."""
    import torch
    u, ig = _u(), _u().ig
    dtype, out = types
    h, half = u.handle(), u.HALF_STEP[out]
    e = 2.0 ** -24

    def matrix(rows, cols, t, fill=None):
        wide = torch.full((rows, cols + pad), u.GUARD, dtype=u.DTYPES[t], device="cuda")
        view = wide[:, :cols]
        view.copy_(torch.randn(rows, cols, device="cuda", generator=g)) if fill is None else view.fill_(fill)
        return wide, view, ig.TensorDescriptor().set(u.DATA[t], rows, cols, 1, 1, (cols + pad, 1, 1, 1))

    def near(got, want, tol, what):
        bad = ~((got.double() - want).abs() <= tol + 1e-30)
        assert not bool(bad.any()), (what, int(bad.sum()), float(((got.double() - want).abs() / (tol + 1e-30)).max()))

    def product_error(n, a, b, scale=1.0):
        return scale * ((n + 4) * e + (2.0 ** -21 + 2.0 ** -30 if dtype == "f32" else 0)) * (a.abs() @ b.abs())

    for M, C, K in LARGE_SHAPES:
        g = torch.Generator(device="cuda").manual_seed(M + C + K)
        print("large", types, pad, M, C, K, flush=True)
        _, x, xd = matrix(M, C, dtype)
        _, dy, dyd = matrix(M, K, dtype)
        w, wd = torch.randn(K, C, device="cuda", generator=g).to(u.DTYPES[dtype]), u.filter_desc(dtype, K, C)
        bias = torch.randn(K, device="cuda", generator=g)
        X, W, DY = x.double(), w.double(), dy.double()
        # forward
        _, r, rd = matrix(M, K, out)
        yw, y, yd = matrix(M, K, out, float("nan"))
        zw, z, _ = matrix(M, K, out, float("nan"))
        ws = u.Workspace(ig.get_linear_forward_workspace_size(h, xd, wd, yd))
        ig.check(ig.linear_forward(h, 0.5, xd, x.data_ptr(), wd, w.data_ptr(), ws.buf.data_ptr(), ws.size, bias.data_ptr(), ig.IGC_ACTIVATION_GELU, 2.0, rd,
                                   r.data_ptr(), yd, z.data_ptr(), y.data_ptr()))
        ws.check()
        wz = 0.5 * (X @ W.t()) + bias.double()
        ez = product_error(C, X, W.t(), 0.5) + 3 * e * wz.abs()
        wy = 0.5 * wz * torch.special.erfc(-wz / 2 ** 0.5) + 2 * r.double()
        near(z, wz, ez + 1.01 * half * wz.abs(), "z")
        near(y, wy, 1.13 * ez + (4e-7 if out == "bf16" else 4 * e) * (1 + wz.abs()) + 4 * e * r.double().abs() + 1.01 * half * wy.abs(), "y")
        assert pad == 0 or (bool((yw[:, K:] == u.GUARD).all()) and bool((zw[:, K:] == u.GUARD).all()))
        # backward data
        _, zi, zid = matrix(M, C, out)
        dw_, dx, dxd = matrix(M, C, out, float("nan"))
        ws = u.Workspace(ig.get_linear_backward_data_workspace_size(h, wd, dyd, dxd))
        ig.check(ig.linear_backward_data(h, 1.0, wd, w.data_ptr(), dyd, dy.data_ptr(), ws.buf.data_ptr(), ws.size, ig.IGC_ACTIVATION_SILU, zid, zi.data_ptr(), 0.0,
                                         None, 0, dxd, dx.data_ptr()))
        ws.check()
        G, Z = DY @ W, zi.double()
        s = torch.sigmoid(Z)
        want = G * (s + Z * s * (1 - s))
        near(dx, want, 1.1 * product_error(K, DY, W) + G.abs() * ((4e-7 if out == "bf16" else 4 * e) * (1 + Z.abs()) + 4 * e) + 1.01 * half * want.abs(), "dx")
        assert pad == 0 or bool((dw_[:, C:] == u.GUARD).all())
        # backward filter
        dw, db, dwd = torch.full((K, C), float("nan"), dtype=u.DTYPES[out], device="cuda"), torch.full((K,), float("nan"), device="cuda"), u.filter_desc(out, K, C)
        ws = u.Workspace(ig.get_linear_backward_filter_workspace_size(h, xd, dyd, dwd))
        ig.check(ig.linear_backward_filter(h, 1.0, xd, x.data_ptr(), dyd, dy.data_ptr(), ws.buf.data_ptr(), ws.size, 0.0, dwd, dw.data_ptr(), db.data_ptr()))
        ws.check()
        want = DY.t() @ X
        near(dw, want, product_error(M, DY.t(), X) + 1.01 * half * want.abs(), "dw")
        near(db, DY.sum(0), (M + 8) * e * DY.abs().sum(0), "dbias")


@pytest.mark.parametrize("lend", [True, False], ids=["workspace", "alone"])
@pytest.mark.parametrize("types", LINEAR_TYPES, ids="-".join)
def test_products_with_infinities_and_nan(types, lend):
    """An infinite factor makes its row of results infinite (of the other factor's sign) or, against an infinity of the other sign or a
    zero, undefined, as a sum of products is; every other row stays as it was.  Large and small finite numbers keep their products."""
    u, ig = _u(), _u().ig
    dtype, out = types
    h = u.handle()
    M, C, K = 40, 100, 72
    rng, x, w, _ = linear_case(types, M, C, K)
    x[3, 7], x[5, 9], x[8, 11], x[9, 99] = np.inf, -np.inf, np.nan, 3.0e38
    x[20] *= 2.0 ** -90
    x[11, 4], x[11, 60] = np.inf, -np.inf
    w[6, 7], w[7, 9] = 0.0, 2.0 ** -60
    w[:, 99] = np.sign(w[:, 99]) * 0.25
    w[30, 7] = 1.0
    x, w = rounded(x, dtype), rounded(w, dtype)
    X, W, WD, Y = u.Rows(x, dtype), u.vector(w, dtype), u.filter_desc(dtype, K, C), u.Rows((M, K), out)
    size = ig.get_linear_forward_workspace_size(h, X.desc, WD, Y.desc) if lend else 0
    ws = u.Workspace(size)
    ig.check(ig.linear_forward(h, 1.0, X.desc, X.ptr, WD, W.data_ptr(), ws.buf.data_ptr() if lend else 0, size, 0, -1, 0.0, None, 0, Y.desc, 0, Y.ptr))
    got = Y.view.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = (x[:, None, :] * w[None, :, :]).sum(2)
        scale = (np.abs(x)[:, None, :] * np.abs(w)[None, :, :]).sum(2)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.isinf(got), np.isinf(want)) and np.array_equal(got[np.isinf(got)], want[np.isinf(want)])
    fin = np.isfinite(want)
    tol = sum_error(C, scale[fin], dtype) + 1.01 * u.HALF_STEP[out] * np.abs(want[fin])
    assert np.all(np.abs(got[fin] - want[fin]) <= tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_activations_far_out(dtype):
    """f and f' where exponentials overflow and vanish: limits, no NaN; infinities of z too."""
    u, ig = _u(), _u().ig
    h = u.handle()
    z = np.array([[-np.inf, -3e38, -1e4, -200.0, -30.0, -9.0, -1e-6, 0.0, 1e-6, 9.0, 30.0, 200.0, 1e4, 3e38, np.inf, 0.5]])
    z = rounded(z, dtype)
    one, wd = u.vector(np.ones((1, 1)), dtype), u.filter_desc(dtype, 1, 1)
    for act in (fo.SIGMOID, fo.RELU, fo.TANH, fo.GELU, fo.SILU):
        X, Y = u.Rows(z.T, dtype), u.Rows((16, 1), dtype)
        ig.check(ig.linear_forward(h, 1.0, X.desc, X.ptr, wd, one.data_ptr(), 0, 0, 0, act, 0.0, None, 0, Y.desc, 0, Y.ptr))
        got = Y.view.double().cpu().numpy()[:, 0]
        v = np.clip(z[0], -1e5, 1e5)
        with np.errstate(over="ignore", invalid="ignore"):
            want = fo.activation(act, v)
            want = np.where(v <= -1e4, {fo.TANH: -1.0}.get(act, 0.0), np.where(v >= 1e4, 1.0 if act in (fo.SIGMOID, fo.TANH) else z[0], want))
            assert np.array_equal(np.isinf(got), np.isinf(want)) and not np.isnan(got).any(), act
            fin = np.isfinite(want)
            assert np.all(np.abs(got - want)[fin] <= (act_error(dtype, np.clip(v, -1, 1)) + 1.02 * u.HALF_STEP[dtype] * np.abs(want) * 4)[fin]), act
            DY, Z, DX = u.Rows(np.ones((16, 1)), dtype), u.Rows(z.T, dtype), u.Rows((16, 1), dtype)
            ig.check(ig.linear_backward_data(h, 1.0, wd, one.data_ptr(), DY.desc, DY.ptr, 0, 0, act, Z.desc, Z.ptr, 0.0, None, 0, DX.desc, DX.ptr))
            got = DX.view.double().cpu().numpy()[:, 0]
            want = np.where(np.abs(v) >= 1e4, ((v > 0) & (act in (fo.RELU, fo.GELU, fo.SILU))).astype(float), fo.activation_slope(act, np.clip(v, -300, 300)))
            assert np.all(np.abs(got - want) <= 2e-6 + 1.02 * u.HALF_STEP[dtype] * np.abs(want)), act
