"""Rows as far apart as a descriptor allows, 2^32 - 16 bytes: offsets within a matrix pass 32 bits.  Tolerances as in test_gpu_feed_forward.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import feed_forward_oracle as fo
from tests import test_gpu_feed_forward as plain

E = 2.0 ** -24
APART = (1 << 31) - 8


@pytest.fixture(scope="module")
def buffer():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch.empty(3 * APART * 2, dtype=torch.uint8, device="cuda")


def far(ig, buffer, values, dtype, stride):
    """The rows in the buffer, `stride` elements apart, and their descriptor"""
    import torch
    u = plain._u()
    flat = buffer[:buffer.numel() // 8 * 8].view(u.DTYPES[dtype])
    rows, cols = values.shape
    m = torch.as_strided(flat, (rows, cols), (stride, 1))
    m.copy_(torch.from_numpy(np.ascontiguousarray(values)).cuda())
    return m, ig.TensorDescriptor().set(u.DATA[dtype], rows, cols, 1, 1, (stride, 1, 1, 1))


@pytest.mark.parametrize("C", [64, 100, 101])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products(dtype, C, buffer):
    u = plain._u()
    ig, h = u.ig, u.handle()
    M, K = (3, 40) if dtype == "bf16" else (2, 40)
    stride = APART if dtype == "bf16" else APART + 7
    rng = np.random.default_rng(C)
    x, w, dy = (plain.rounded(plain.normal(rng, *s), dtype) for s in ((M, C), (K, C), (M, K)))
    X, xd = far(ig, buffer, x, dtype, stride)
    part = 2.0 ** -21 + 2.0 ** -30
    half = u.HALF_STEP[dtype]
    W, DY = u.Rows(w, dtype), u.Rows(dy, dtype)
    Y = u.Rows((M, K), dtype, fill=float("nan"))
    WD = u.filter_desc(dtype, K, C)
    size = ig.get_linear_forward_workspace_size(h, xd, WD, Y.desc)
    for lend in (size, 0):
        print("forward", dtype, C, lend, flush=True)
        ws = u.Workspace(size)
        ig.check(ig.linear_forward(h, 1.0, xd, X.data_ptr(), WD, W.ptr, ws.buf.data_ptr(), lend, 0, ig.IGC_ACTIVATION_IDENTITY, 0.0, None, 0, Y.desc, 0, Y.ptr))
        ws.check()
        want = x @ w.T
        u.close(Y.numpy(), want, ((C + 4) * E + part) * (np.abs(x) @ np.abs(w).T) + 1.01 * half * np.abs(want) + 1e-30, "y")
    DW = u.Rows((K, C), dtype, fill=float("nan"))
    size = ig.get_linear_backward_filter_workspace_size(h, xd, DY.desc, WD)
    for lend in (size, 0):
        print("filter", dtype, C, lend, flush=True)
        ws = u.Workspace(size)
        ig.check(ig.linear_backward_filter(h, 1.0, xd, X.data_ptr(), DY.desc, DY.ptr, ws.buf.data_ptr(), lend, 0.0, WD, DW.ptr, 0))
        ws.check()
        want = dy.T @ x
        u.close(DW.numpy(), want, ((M + 4) * E + part) * (np.abs(dy).T @ np.abs(x)) + 1.01 * half * np.abs(want) + 1e-30, "dw")


@pytest.mark.parametrize("C", [64, 1001])
def test_layer_norm(C, buffer):
    u = plain._u()
    ig, h = u.ig, u.handle()
    rng = np.random.default_rng(C)
    x = plain.rounded(plain.normal(rng, 3, C) * 2 + plain.normal(rng, 3, 1), "bf16")
    X, xd = far(ig, buffer, x, "bf16", APART)
    Y = u.Rows((3, C), "f32", fill=float("nan"))
    print("norm", C, flush=True)
    ig.check(ig.layer_norm_forward(h, 1.0, xd, X.data_ptr(), 0, 0, plain.EPS, 0.0, Y.desc, Y.ptr))
    y, m, s = fo.layer_norm(x, None, None, plain.EPS)
    em = (C + 4) * E * np.abs(x).mean(1)
    d = np.abs(x - m[:, None])
    es = s * (2 * (C + 8) * E + s * s * 2 * em * d.mean(1) + s * s * em * em)
    u.close(Y.numpy(), y, em[:, None] * s[:, None] + d * (es + 6 * E * s)[:, None] + 6 * E * np.abs(y) + 1e-30, "y")
