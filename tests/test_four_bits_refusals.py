"""What the functions on four-bit filters refuse, and their size queries: host logic, no GPU call."""
import ctypes

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


def test_sizes():
    assert ig.get_filter4_size(filt(B, 5, 1), 32) == (5 * 64, 5 * 2)
    assert ig.get_filter4_size(filt(F, 7, 129), 64) == (7 * 128, 3 * 7 * 2)
    assert ig.get_filter4_size(filt(B, 16384, 4096), 128) == (16384 * 2048, 32 * 16384 * 2)
    assert ig.get_filter4_size(filt(B, 1 << 20, 1 << 16), 32) == (1 << 35, 1 << 32)          # past 32 bits
    for w, group, want in ((filt(B, 5, 8), 16, UNSUPPORTED), (filt(B, 5, 8), 0, UNSUPPORTED), (filt(D, 5, 8), 32, UNSUPPORTED), (filt(B, 5, 8, 3), 32, BAD),
                           (ig.FilterDescriptor(), 32, UNSET)):
        assert status(lambda: ig.get_filter4_size(w, group)) == want
    out = ctypes.c_size_t()
    assert ig.lib().igcGetFilter4Size(filt(B, 5, 8).ptr, 32, None, ctypes.byref(out)) == BAD
    assert ig.lib().igcGetFilter4Size(None, 32, ctypes.byref(out), ctypes.byref(out)) == BAD


def test_storing_refuses():
    h = ig.Handle()
    for call in (lambda w=filt(F, 5, 8), wp=P, group=32, codes=P, scales=P: ig.quantize_filter4(h, w, wp, group, codes, scales),
                 lambda w=filt(F, 5, 8), wp=P, group=32, codes=P, scales=P: ig.dequantize_filter4(h, group, codes, scales, w, wp)):
        assert call(wp=0) == BAD and call(codes=0) == BAD and call(scales=0) == BAD
        assert call(wp=P + 2) == BAD and call(codes=P + 8) == BAD and call(scales=P + 1) == BAD and call(w=filt(B, 5, 8), wp=P + 1) == BAD
        assert call(group=48) == UNSUPPORTED and call(w=filt(D, 5, 8)) == UNSUPPORTED and call(w=filt(F, 5, 8, 3)) == BAD and call(w=ig.FilterDescriptor()) == UNSET


def test_product_refuses():
    h = ig.Handle()

    def call(x=rows(B, 4, 64), w=filt(B, 8, 64), y=rows(B, 4, 8), r=rows(B, 4, 8), group=32, beta=1.0, act=-1, **ptrs):
        p = dict(x=P, codes=P, scales=P, bias=P, r=P, y=P)
        p.update({k[:-1]: v for k, v in ptrs.items()})
        return ig.linear4_forward(h, 1.0, x, p["x"], w, group, p["codes"], p["scales"], 0, 0, p["bias"], act, beta, r, p["r"], y, p["y"])

    for name in ("x", "codes", "scales", "y", "r"):
        assert call(**{name + "_": 0}) == BAD, name
    assert call(x_=P + 1) == BAD and call(y_=P + 1) == BAD and call(r_=P + 1) == BAD and call(codes_=P + 8) == BAD and call(scales_=P + 1) == BAD and call(bias_=P + 2) == BAD
    assert call(act=5) == BAD and call(act=-2) == BAD
    assert call(x=rows(B, 4, 63)) == BAD and call(x=rows(B, 5, 64)) == BAD and call(y=rows(B, 4, 9)) == BAD and call(y=rows(B, 4, 8, 7)) == BAD
    assert call(r=rows(B, 4, 9)) == BAD and call(r=rows(B, 5, 8)) == BAD and call(r=None) == BAD and call(r=rows(F, 4, 8)) == UNSUPPORTED
    assert call(group=256) == UNSUPPORTED and call(w=filt(D, 8, 64)) == UNSUPPORTED and call(x=rows(D, 4, 64)) == UNSUPPORTED
    assert call(x=rows(F, 4, 64)) == UNSUPPORTED                        # float rows with bfloat16 results
    nchw = ig.TensorDescriptor().set(B, 2, 64, 3, 3, (576, 9, 3, 1))
    nhwc = ig.TensorDescriptor().set(B, 2, 8, 3, 3, (72, 1, 24, 8))
    assert call(x=nchw, y=nhwc, beta=0.0) == UNSUPPORTED
    assert call(w=ig.FilterDescriptor()) == UNSET
    assert status(lambda: ig.get_linear4_forward_workspace_size(h, rows(B, 4, 63), filt(B, 8, 64), 32, rows(B, 4, 8))) == BAD
    assert status(lambda: ig.get_linear4_forward_workspace_size(h, rows(F, 4, 64), filt(B, 8, 64), 32, rows(B, 4, 8))) == UNSUPPORTED
    assert ig.get_linear4_forward_workspace_size(h, rows(F, 4, 64), filt(F, 8, 64), 32, rows(F, 4, 8)) >= 0


def test_workspace_holds_copies_of_what_lies_off_words():
    """bfloat16 rows may begin at any 2 bytes: a prompt's room holds their copy whatever the descriptor says."""
    h = ig.Handle()
    for M, C, K in ((2048, 4096, 8192), (700, 520, 602), (64, 4096, 16384)):
        assert ig.get_linear4_forward_workspace_size(h, rows(B, M, C), filt(B, K, C), 64, rows(B, M, K)) >= 2 * M * C
