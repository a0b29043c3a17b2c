"""What the cross entropy over a vocabulary refuses, and its workspace queries: host logic, no GPU call."""
import paper_1410_0759_amd as ig

F, B, D = ig.IGC_DATA_FLOAT, ig.IGC_DATA_BFLOAT16, ig.IGC_DATA_DOUBLE
OK, BAD, UNSUPPORTED, UNSET = (ig.IGC_STATUS_SUCCESS, ig.IGC_STATUS_BAD_PARAM, ig.IGC_STATUS_NOT_SUPPORTED, ig.IGC_STATUS_NOT_INITIALIZED)
P = 1 << 20          # a pointer that is never followed
h = None


def handle():
    global h
    h = h or ig.Handle()
    return h


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


def forward(x=rows(B, 4, 64), w=filt(B, 100, 64), room=None, **ptrs):
    p = dict(x=P, w=P, bias=P, targets=P, ws=P, loss=P, log_sum=P)
    p.update({k[:-1]: v for k, v in ptrs.items()})
    if room is None:
        room = 0
    return ig.linear_cross_entropy_forward(handle(), x, p["x"], w, p["w"], p["bias"], p["targets"], p["ws"], room, p["loss"], p["log_sum"])


def backward(x=rows(B, 4, 64), w=filt(B, 100, 64), dxd=rows(B, 4, 64), dwd=filt(B, 100, 64), room=0, **ptrs):
    p = dict(x=P, w=P, bias=P, targets=P, log_sum=P, dloss=P, ws=P, dx=P, dw=P, dbias=P)
    p.update({k[:-1]: v for k, v in ptrs.items()})
    return ig.linear_cross_entropy_backward(handle(), 1.0, x, p["x"], w, p["w"], p["bias"], p["targets"], p["log_sum"], p["dloss"], p["ws"], room, 0.0, dxd, p["dx"], 0.0, dwd,
                                            p["dw"], p["dbias"])


def test_forward_refuses():
    for name in ("x", "w", "targets", "ws", "loss"):
        assert forward(**{name + "_": 0}, room=1 << 40) == BAD, name
    for name, by in (("x", 1), ("w", 1), ("bias", 2), ("targets", 2), ("ws", 8), ("loss", 2), ("log_sum", 1)):
        assert forward(**{name + "_": P + by}, room=1 << 40) == BAD, name
    assert forward(x=rows(B, 4, 63)) == BAD and forward(w=filt(B, 100, 64, 3)) == BAD and forward(w=filt(F, 100, 64)) == UNSUPPORTED
    assert forward(x=rows(D, 4, 64), w=filt(D, 100, 64)) == UNSUPPORTED and forward(w=ig.FilterDescriptor()) == UNSET
    need = ig.get_linear_cross_entropy_forward_workspace_size(handle(), rows(B, 4, 64), filt(B, 100, 64))
    assert need > 0 and forward(room=need - 1) == BAD
    nchw = ig.TensorDescriptor().set(B, 2, 64, 3, 3, (576, 9, 3, 1))
    assert forward(x=nchw) == UNSUPPORTED


def test_backward_refuses():
    for name in ("x", "w", "targets", "log_sum", "ws"):
        assert backward(**{name + "_": 0}, room=1 << 40) == BAD, name
    assert backward(dx_=0, dw_=0, dbias_=0, room=1 << 40) == BAD
    for name, by in (("x", 1), ("w", 1), ("bias", 2), ("targets", 2), ("log_sum", 2), ("dloss", 1), ("ws", 8), ("dx", 1), ("dw", 1), ("dbias", 2)):
        assert backward(**{name + "_": P + by}, room=1 << 40) == BAD, name
    assert backward(dxd=rows(B, 5, 64)) == BAD and backward(dxd=rows(B, 4, 63)) == BAD and backward(dxd=rows(B, 4, 64, 60)) == BAD and backward(dxd=None) == BAD
    assert backward(dwd=filt(B, 99, 64)) == BAD and backward(dwd=filt(B, 100, 63)) == BAD and backward(dwd=filt(B, 100, 64, 3)) == BAD and backward(dwd=None) == BAD
    assert backward(dxd=rows(D, 4, 64)) == UNSUPPORTED and backward(dwd=filt(D, 100, 64)) == UNSUPPORTED
    assert backward(x=rows(F, 4, 64), w=filt(F, 100, 64), dwd=filt(F, 100, 64)) == UNSUPPORTED          # float rows, bfloat16 gradient
    assert backward(dxd=ig.TensorDescriptor()) == UNSET
    need = ig.get_linear_cross_entropy_backward_workspace_size(handle(), rows(B, 4, 64), filt(B, 100, 64), rows(B, 4, 64), filt(B, 100, 64))
    assert backward(room=need - 1) == BAD


def test_workspaces():
    """Bounded by pieces of the vocabulary, whatever its size; not by every logit."""
    size = lambda M, V, C=4096, t=B: ig.get_linear_cross_entropy_forward_workspace_size(handle(), rows(t, M, C), filt(t, V, C))
    assert size(8192, 131072) < 1 << 30 < 8192 * 131072 * 4
    back = lambda M, V, C=4096, t=B: ig.get_linear_cross_entropy_backward_workspace_size(handle(), rows(t, M, C), filt(t, V, C), rows(t, M, C), filt(t, V, C))
    assert back(8192, 131072) < 1 << 30
    assert back(1, 1 << 26, 8) < 1 << 30 and size(1, 1 << 26, 8) < 1 << 30
    whole = back(64, 1000)
    assert ig.get_linear_cross_entropy_backward_workspace_size(handle(), rows(B, 64, 4096), filt(B, 1000, 4096), None, None) <= whole
    assert status(lambda: ig.get_linear_cross_entropy_forward_workspace_size(handle(), rows(B, 4, 63), filt(B, 100, 64))) == BAD
    assert status(lambda: ig.get_linear_cross_entropy_backward_workspace_size(handle(), rows(B, 4, 64), filt(B, 100, 64), rows(B, 4, 64), filt(B, 10, 64))) == BAD
