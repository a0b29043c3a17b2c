"""Bfloat16 products whose rows lie on 4-byte boundaries only and end inside a 16-byte piece, with NaN wherever the matrices are not.

Tolerance: products of bfloat16 are exact in float; a sum of n of them in any order is off by at most (n + 4) 2^-24 of their magnitudes, the result is
rounded to float (2^-24) or bfloat16 (2^-8 of it)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import feed_forward_oracle as fo
from tests import test_gpu_feed_forward as plain

E = 2.0 ** -24


def among_nan(u, values, pad, lead):
    """The matrix with NaN in front of it, between its rows and behind it."""
    m = u.Rows(values, "bf16", pad, lead)
    keep = m.view.clone()
    m.buf.fill_(float("nan"))
    m.view.copy_(keep)
    return m


def tolerance(u, out, n, magnitudes, want):
    return (n + 4) * E * magnitudes + u.HALF_STEP[out] * 1.01 * np.abs(want) + 1e-30


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("pad,lead", [(0, 0), (2, 2), (6, 0), (0, 6), (1, 2)])
def test_filter_gradient(pad, lead, out):
    u = plain._u()
    ig, h = u.ig, u.handle()
    for M, C, K in ((1, 2, 2), (33, 38, 54), (70, 130, 66), (333, 62, 1154), (515, 258, 262), (129, 514, 1030)):
        print("filter", M, C, K, pad, lead, out, flush=True)
        rng = np.random.default_rng(M + C)
        x, dy = plain.rounded(plain.normal(rng, M, C), "bf16"), plain.rounded(plain.normal(rng, M, K), "bf16")
        X, DY = among_nan(u, x, pad, lead), among_nan(u, dy, pad, lead)
        DW, DB = u.Rows((K, C), out, fill=float("nan")), u.vector(np.full(K, np.nan))
        W = u.filter_desc(out, K, C)
        size = ig.get_linear_backward_filter_workspace_size(h, X.desc, DY.desc, W)
        for lend in (size, 0):
            ws = u.Workspace(size)
            ig.check(ig.linear_backward_filter(h, 1.0, X.desc, X.ptr, DY.desc, DY.ptr, ws.buf.data_ptr(), lend, 0.0, W, DW.ptr, DB.data_ptr()))
            ws.check()
            want, bias = fo.linear_backward_filter(dy, x)
            u.close(DW.numpy(), want, tolerance(u, out, M, np.abs(dy).T @ np.abs(x), want), "dw")
            u.close(DB.double().cpu().numpy(), bias, (M + 4) * E * np.abs(dy).sum(0) + 1e-30, "dbias")


@pytest.mark.parametrize("pad,lead", [(0, 0), (2, 2), (6, 0), (0, 6), (1, 2)])
def test_forward_and_data_gradient(pad, lead):
    u = plain._u()
    ig, h = u.ig, u.handle()
    for M, C, K in ((1, 2, 8), (8, 258, 64), (100, 1002, 104), (300, 334, 512), (513, 518, 776)):
        print("forward, data", M, C, K, pad, lead, flush=True)
        rng = np.random.default_rng(M + C)
        dy, w = plain.rounded(plain.normal(rng, M, K), "bf16"), plain.rounded(plain.normal(rng, K, C), "bf16")
        DY, W = among_nan(u, dy, pad, lead), among_nan(u, w, 0, lead)
        DX = u.Rows((M, C), "bf16", pad, lead, fill=float("nan"))
        WD = u.filter_desc("bf16", K, C)
        size = ig.get_linear_backward_data_workspace_size(h, WD, DY.desc, DX.desc)
        V = among_nan(u, np.ascontiguousarray(w.T), 0, lead)
        VD = u.filter_desc("bf16", C, K)
        more = ig.get_linear_forward_workspace_size(h, DY.desc, VD, DX.desc)
        want = dy @ w
        for lend in (True, False):
            ws = u.Workspace(max(size, more))
            ig.check(ig.linear_backward_data(h, 1.0, WD, W.ptr, DY.desc, DY.ptr, ws.buf.data_ptr(), size if lend else 0, ig.IGC_ACTIVATION_IDENTITY, None, 0,
                                             0.0, None, 0, DX.desc, DX.ptr))
            ws.check()
            u.close(DX.numpy(), want, tolerance(u, "bf16", K, np.abs(dy) @ np.abs(w), want), "dx")
            DX.view.fill_(float("nan"))
            ig.check(ig.linear_forward(h, 1.0, DY.desc, DY.ptr, VD, V.ptr, ws.buf.data_ptr(), more if lend else 0, 0, ig.IGC_ACTIVATION_IDENTITY, 0.0, None, 0,
                                       DX.desc, 0, DX.ptr))
            ws.check()
            u.close(DX.numpy(), want, tolerance(u, "bf16", K, np.abs(dy) @ np.abs(w), want), "y")
