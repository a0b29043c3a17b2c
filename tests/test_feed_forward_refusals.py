"""What the feed-forward functions refuse, and their workspace queries: host logic, no GPU call."""
import ctypes

import pytest

import paper_1410_0759_amd as ig

F, B, D = ig.IGC_DATA_FLOAT, ig.IGC_DATA_BFLOAT16, ig.IGC_DATA_DOUBLE
OK, BAD, UNSUPPORTED, UNSET = (ig.IGC_STATUS_SUCCESS, ig.IGC_STATUS_BAD_PARAM, ig.IGC_STATUS_NOT_SUPPORTED, ig.IGC_STATUS_NOT_INITIALIZED)
P = 1 << 20          # a pointer that is never followed


def rows(dt, M, C, stride=None):
    return ig.TensorDescriptor().set(dt, M, C, 1, 1, (stride or C, 1, 1, 1))


def filt(dt, K, C, r=1):
    return ig.FilterDescriptor().set(dt, K, C, r, 1)


def status(call):
    try:
        call()
        return OK
    except ig.IgcError as e:
        return e.status


def norm(h=None, x=None, y=None, xp=P, yp=P, scale=P, shift=P, mean=P, inv=P, eps=1e-5):
    return ig.layer_norm_forward(h or ig.Handle(), 1.0, x or rows(F, 4, 8), xp, scale, shift, eps, 0.0, y or rows(F, 4, 8), yp, mean, inv)


def test_layer_norm_forward_refuses():
    assert norm(xp=0) == BAD and norm(yp=0) == BAD
    assert norm(xp=P + 2) == BAD and norm(yp=P + 1) == BAD and norm(scale=P + 2) == BAD and norm(mean=P + 2) == BAD
    assert norm(eps=-1.0) == BAD and norm(eps=float("nan")) == BAD and norm(eps=float("inf")) == BAD
    assert norm(y=rows(F, 5, 8)) == BAD and norm(y=rows(F, 4, 9)) == BAD
    assert norm(y=rows(F, 4, 8, 7)) == BAD                                            # rows of y overlap
    assert norm(x=rows(D, 4, 8)) == UNSUPPORTED and norm(y=rows(D, 4, 8)) == UNSUPPORTED
    nchw = ig.TensorDescriptor().set(F, 2, 8, 3, 3, (72, 9, 3, 1))
    nhwc = ig.TensorDescriptor().set(F, 2, 8, 3, 3, (72, 1, 24, 8))
    assert norm(x=nchw, y=nhwc) == UNSUPPORTED and norm(x=nhwc, y=nchw) == UNSUPPORTED
    gap = ig.TensorDescriptor().set(F, 2, 8, 3, 3, (100, 1, 24, 8))                   # positions not evenly spaced
    assert norm(x=gap, y=nhwc) == UNSUPPORTED
    unset = ig.TensorDescriptor()
    unset.dtype = F
    assert norm(x=unset) == UNSET
    one = ctypes.c_float(1.0)
    assert ig.lib().igcLayerNormForward(None, ctypes.byref(one), None, None, None, None, 0.0, None, None, None, None, None) == BAD


def test_layer_norm_backward_refuses():
    h = ig.Handle()
    d = rows(F, 40, 8)

    def call(x=d, dy=d, r=d, dx=d, beta=1.0, **ptrs):
        p = dict(x=P, dy=P, scale=P, mean=P, inv=P, r=P, dx=P, dscale=P, dshift=P)
        p.update({k[:-1] if k.endswith("_") else k: v for k, v in ptrs.items()})
        return ig.layer_norm_backward(h, 1.0, x, p["x"], dy, p["dy"], p["scale"], p["mean"], p["inv"], 0, 0, beta, r, p["r"], dx, p["dx"], 0.0,
                                      p["dscale"], p["dshift"])

    for name in ("x_", "dy_", "mean_", "inv_", "dx_", "r_"):
        assert call(**{name: 0}) == BAD, name
    for name in ("x_", "dy_", "scale_", "mean_", "inv_", "dx_", "r_", "dscale_", "dshift_"):
        assert call(**{name: P + 2}) == BAD, name
    assert call(r=None) == BAD and call(r=rows(F, 40, 9)) == BAD and call(r=rows(B, 40, 8)) == UNSUPPORTED
    assert call(dy=rows(F, 41, 8)) == BAD and call(dx=rows(F, 40, 8, 7)) == BAD
    assert call(dx=rows(B, 40, 8)) == UNSUPPORTED and call(dy=rows(D, 40, 8)) == UNSUPPORTED
    size = lambda a, b, c: status(lambda: ig.get_layer_norm_backward_workspace_size(h, a, b, c))
    assert size(d, d, d) == OK and size(d, rows(F, 40, 9), d) == BAD and size(d, d, rows(B, 40, 8)) == UNSUPPORTED


def test_linear_forward_refuses():
    h = ig.Handle()
    x, w, y = rows(B, 6, 16), filt(B, 24, 16), rows(B, 6, 24)

    def call(x=x, w=w, y=y, r=y, beta=1.0, act=ig.IGC_ACTIVATION_GELU, **ptrs):
        p = dict(x=P, w=P, bias=P, r=P, z=P, y=P)
        p.update({k[:-1] if k.endswith("_") else k: v for k, v in ptrs.items()})
        return ig.linear_forward(h, 1.0, x, p["x"], w, p["w"], 0, 0, p["bias"], act, beta, r, p["r"], y, p["z"], p["y"])

    for name in ("x_", "w_", "y_", "r_"):
        assert call(**{name: 0}) == BAD, name
        assert call(**{name: P + 1}) == BAD, name
    assert call(z=P + 1) == BAD and call(bias=P + 2) == BAD
    assert call(act=5) == BAD and call(act=-2) == BAD
    assert call(x=rows(B, 6, 17)) == BAD and call(w=filt(B, 25, 16)) == BAD and call(w=filt(B, 24, 16, 3)) == BAD and call(y=rows(B, 7, 24)) == BAD
    assert call(y=rows(B, 6, 24, 23)) == BAD and call(r=None) == BAD and call(r=rows(B, 6, 25)) == BAD
    assert call(x=rows(F, 6, 16)) == UNSUPPORTED and call(r=rows(F, 6, 24)) == UNSUPPORTED and call(y=rows(D, 6, 24), r=None, beta=0.0) == UNSUPPORTED
    fx, fw = rows(F, 6, 16), filt(F, 24, 16)
    assert call(x=fx, w=fw, y=rows(B, 6, 24)) == UNSUPPORTED
    assert call(x=rows(D, 6, 16), w=filt(D, 24, 16), y=rows(D, 6, 24), r=None, beta=0.0) == UNSUPPORTED
    size = lambda a, b, c: status(lambda: ig.get_linear_forward_workspace_size(h, a, b, c))
    assert size(x, w, y) == OK and size(x, w, rows(B, 6, 25)) == BAD and size(fx, fw, rows(B, 6, 24)) == UNSUPPORTED


def test_linear_backward_data_refuses():
    h = ig.Handle()
    dy, w, dx = rows(B, 6, 24), filt(B, 24, 16), rows(B, 6, 16)

    def call(dy=dy, w=w, dx=dx, z=dx, r=dx, beta=1.0, act=ig.IGC_ACTIVATION_RELU, **ptrs):
        p = dict(w=P, dy=P, z=P, r=P, dx=P)
        p.update({k[:-1] if k.endswith("_") else k: v for k, v in ptrs.items()})
        return ig.linear_backward_data(h, 1.0, w, p["w"], dy, p["dy"], 0, 0, act, z, p["z"], beta, r, p["r"], dx, p["dx"])

    for name in ("w_", "dy_", "z_", "r_", "dx_"):
        assert call(**{name: 0}) == BAD, name
        assert call(**{name: P + 1}) == BAD, name
    assert call(act=9) == BAD and call(z=None) == BAD and call(r=None) == BAD
    assert call(z=rows(B, 6, 17)) == BAD and call(dy=rows(B, 6, 16)) == BAD and call(dx=rows(B, 6, 16, 15)) == BAD
    assert call(z=rows(F, 6, 16)) == UNSUPPORTED and call(dy=rows(F, 6, 24)) == UNSUPPORTED
    size = lambda a, b, c: status(lambda: ig.get_linear_backward_data_workspace_size(h, a, b, c))
    assert size(w, dy, dx) == OK and size(w, dx, dy) == BAD


def test_linear_backward_filter_refuses():
    h = ig.Handle()
    x, dy, dw = rows(B, 6, 16), rows(B, 6, 24), filt(F, 24, 16)

    def call(x=x, dy=dy, dw=dw, **ptrs):
        p = dict(x=P, dy=P, dw=P, dbias=P)
        p.update({k[:-1] if k.endswith("_") else k: v for k, v in ptrs.items()})
        return ig.linear_backward_filter(h, 1.0, x, p["x"], dy, p["dy"], 0, 0, 0.0, dw, p["dw"], p["dbias"])

    for name in ("x_", "dy_", "dw_"):
        assert call(**{name: 0}) == BAD, name
        assert call(**{name: P + 1}) == BAD, name
    assert call(dbias=P + 2) == BAD
    assert call(x=rows(B, 7, 16)) == BAD and call(dw=filt(F, 16, 24)) == BAD and call(dw=filt(F, 24, 16, 3)) == BAD
    assert call(dy=rows(F, 6, 24)) == UNSUPPORTED and call(dw=filt(D, 24, 16)) == UNSUPPORTED
    size = lambda a, b, c: status(lambda: ig.get_linear_backward_filter_workspace_size(h, a, b, c))
    assert size(x, dy, dw) == OK and size(dy, x, dw) == BAD


def test_the_elementwise_functions_keep_their_three_activations():
    h, d = ig.Handle(), ig.TensorDescriptor().set(F, 1, 4, 1, 1, (4, 1, 1, 1))
    for mode in (ig.IGC_ACTIVATION_GELU, ig.IGC_ACTIVATION_SILU):
        assert ig.activation_forward(h, mode, 1.0, d, P, 0.0, d, P) == BAD


@pytest.mark.parametrize("M,C,K", [(1, 1, 1), (3, 1001, 64), (8, 4096, 16384), (5000, 1000, 1200)])
def test_workspace_queries_answer(M, C, K):
    h = ig.Handle()
    for dt, out in ((B, B), (B, F), (F, F)):
        x, y, w, dw = rows(dt, M, C), rows(out, M, K), filt(dt, K, C), filt(out, K, C)
        dy, dx = rows(dt, M, K), rows(out, M, C)
        assert ig.get_linear_forward_workspace_size(h, x, w, y) >= 0
        assert ig.get_linear_backward_data_workspace_size(h, w, dy, dx) >= 0
        assert ig.get_linear_backward_filter_workspace_size(h, x, dy, dw) >= 0
