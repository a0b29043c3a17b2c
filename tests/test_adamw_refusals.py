"""What the optimiser's step refuses: host logic, no GPU call."""
import ctypes

import paper_1410_0759_amd as ig

F, B, D = ig.IGC_DATA_FLOAT, ig.IGC_DATA_BFLOAT16, ig.IGC_DATA_DOUBLE
BAD, UNSUPPORTED = ig.IGC_STATUS_BAD_PARAM, ig.IGC_STATUS_NOT_SUPPORTED
P = 1 << 20          # a pointer that is never followed


def step(parameters=None, **fields):
    """A list of one tensor, refused before anything is launched, or (count 0) nothing to do."""
    t = (ig.AdamWTensor * 1)()
    base = dict(param=P, grad=P, copy=0, m=P, v=P, m_scale=P, v_scale=P, count=10, weight_decay=0.1, param_type=F, grad_type=F, state_bits=32)
    for k, v in {**base, **fields}.items():
        setattr(t[0], k, v)
    return ig.adamw_step(ig.Handle(), parameters or params(), t)


def params(**more):
    return ig.AdamWParameters(**{**dict(learning_rate=1e-3, beta1=0.9, beta2=0.99, epsilon=1e-8, gradient_scale=1.0, step=1), **more})


def test_numbers():
    nan, inf = float("nan"), float("inf")
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=nan), dict(beta2=1.0), dict(beta2=-1.0), dict(beta2=nan), dict(epsilon=0.0), dict(epsilon=-1.0),
                dict(epsilon=nan), dict(epsilon=inf), dict(epsilon=1e-60), dict(epsilon=1e-39), dict(step=0), dict(step=-3), dict(learning_rate=nan), dict(learning_rate=inf),
                dict(gradient_scale=nan), dict(gradient_scale=inf), dict(device_step=P + 2), dict(device_learning_rate=P + 1), dict(device_gradient_scale=P + 2)):
        assert step(params(**bad), count=0) == BAD, bad
    assert step(params(), count=0) == 0
    # what the device holds instead is not asked of the host
    assert step(params(step=0, device_step=P), count=0) == 0
    assert step(params(learning_rate=nan, device_learning_rate=P), count=0) == 0


def test_tensors():
    for bad in (dict(param=0), dict(grad=0), dict(m=0), dict(v=0), dict(param=P + 2), dict(grad=P + 1), dict(m=P + 2), dict(v=P + 2), dict(copy=P + 1), dict(count=-1),
                dict(weight_decay=float("nan")), dict(param=P + 1, param_type=B), dict(grad=P + 1, grad_type=B), dict(copy=P, param_type=B),
                dict(state_bits=8, m_scale=0), dict(state_bits=8, v_scale=0), dict(state_bits=8, m_scale=P + 2)):
        assert step(**bad) == BAD, bad
    for bad in (dict(param_type=D), dict(grad_type=D), dict(state_bits=16), dict(state_bits=4), dict(count=(1 << 40) + 1)):
        assert step(**bad) == UNSUPPORTED, bad
    # a tensor without elements needs no pointers, but its types are looked at
    assert step(count=0, param=0, grad=0, m=0, v=0) == 0
    assert step(count=0, state_bits=5) == UNSUPPORTED
    # one bad tensor and none is taken (the first has pointers that nothing may follow)
    t = (ig.AdamWTensor * 2)()
    assert ig.adamw_step(ig.Handle(), params(), t) == UNSUPPORTED


def test_arguments():
    q, t = params(), (ig.AdamWTensor * 1)()
    L = ig.lib()
    assert L.igcAdamWStep(None, ctypes.byref(q), 1, t) == BAD
    h = ig.Handle()
    assert L.igcAdamWStep(h.ptr, None, 1, t) == BAD
    assert L.igcAdamWStep(h.ptr, ctypes.byref(q), -1, t) == BAD
    assert L.igcAdamWStep(h.ptr, ctypes.byref(q), 1, None) == BAD
    assert L.igcAdamWStep(h.ptr, ctypes.byref(q), 0, None) == 0
    try:
        ig.AdamWParameters(rate=1.0)
        raise AssertionError("an unknown name was taken")
    except TypeError:
        pass
    try:
        t[0].gradient = P
        raise AssertionError("an unknown name was taken")
    except AttributeError:
        pass


def test_numbers_beyond_floats():
    for bad in (dict(learning_rate=1e39), dict(gradient_scale=-1e39), dict(epsilon=1e39)):
        assert step(params(**bad), count=0) == BAD, bad
    assert step(weight_decay=1e39) == BAD
