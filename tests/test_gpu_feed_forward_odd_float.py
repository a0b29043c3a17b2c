"""Float products whose operands' rows end inside a 16-byte piece, with NaN wherever the matrices are not.

Tolerance: a sum of n products in any order is off by at most (n + 4) 2^-24 of the products' magnitudes; taken in three parts a product is off by
less than 2^-21 + 2^-30 of it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import feed_forward_oracle as fo
from tests import test_gpu_feed_forward as plain

E, LEFT_OUT = 2.0 ** -24, 2.0 ** -21 + 2.0 ** -30


def among_nan(u, values, pad, lead):
    """The matrix with NaN in front of it, between its rows and behind it."""
    import torch
    m = u.Rows(values, "f32", pad, lead)
    keep = m.view.clone()
    m.buf.fill_(float("nan"))
    m.view.copy_(keep)
    return m


@pytest.mark.parametrize("lead", [0, 1, 3])
@pytest.mark.parametrize("pad", [0, 1, 5])
def test_filter_gradient(pad, lead):
    u = plain._u()
    ig, h = u.ig, u.handle()
    for M, C, K in ((1, 1, 1), (3, 2, 5), (33, 37, 53), (70, 129, 66), (123, 64, 1155), (265, 127, 301), (515, 259, 261)):
        print("filter", M, C, K, pad, lead, flush=True)
        rng = np.random.default_rng(M + C)
        x, dy = plain.rounded(plain.normal(rng, M, C), "f32"), plain.rounded(plain.normal(rng, M, K), "f32")
        X, DY = among_nan(u, x, pad, lead), among_nan(u, dy, pad, lead)
        DW, DB = u.Rows((K, C), "f32", fill=float("nan")), u.vector(np.full(K, np.nan))
        W = u.filter_desc("f32", K, C)
        size = ig.get_linear_backward_filter_workspace_size(h, X.desc, DY.desc, W)
        for lend in (size, 0):
            ws = u.Workspace(size)
            ig.check(ig.linear_backward_filter(h, 1.0, X.desc, X.ptr, DY.desc, DY.ptr, ws.buf.data_ptr(), lend, 0.0, W, DW.ptr, DB.data_ptr()))
            ws.check()
            want, bias = fo.linear_backward_filter(dy, x)
            u.close(DW.numpy(), want, ((M + 4) * E + LEFT_OUT) * (np.abs(dy).T @ np.abs(x)) + E * np.abs(want) + 1e-30, "dw")
            u.close(DB.double().cpu().numpy(), bias, (M + 4) * E * np.abs(dy).sum(0) + 1e-30, "dbias")


@pytest.mark.parametrize("pad,lead", [(0, 0), (1, 1), (4, 3)])
def test_data_gradient(pad, lead):
    u = plain._u()
    ig, h = u.ig, u.handle()
    for M, C, K in ((1, 1, 4), (8, 257, 64), (100, 1001, 100), (300, 333, 512), (70, 63, 36)):
        print("data", M, C, K, pad, lead, flush=True)
        rng = np.random.default_rng(M + C)
        dy, w = plain.rounded(plain.normal(rng, M, K), "f32"), plain.rounded(plain.normal(rng, K, C), "f32")
        DY, W = among_nan(u, dy, pad, lead), among_nan(u, w, 0, lead)
        DX = u.Rows((M, C), "f32", pad, lead, fill=float("nan"))
        WD = u.filter_desc("f32", K, C)
        size = ig.get_linear_backward_data_workspace_size(h, WD, DY.desc, DX.desc)
        for lend in (size, 0):
            ws = u.Workspace(size)
            ig.check(ig.linear_backward_data(h, 1.0, WD, W.ptr, DY.desc, DY.ptr, ws.buf.data_ptr(), lend, ig.IGC_ACTIVATION_IDENTITY, None, 0, 0.0, None, 0,
                                             DX.desc, DX.ptr))
            ws.check()
            want = dy @ w
            u.close(DX.numpy(), want, ((K + 4) * E + LEFT_OUT) * (np.abs(dy) @ np.abs(w)) + E * np.abs(want) + 1e-30, "dx")
