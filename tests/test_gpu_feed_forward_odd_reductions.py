"""Float products whose reduction ends inside a 16-byte piece, taken as they lie: what follows a row - the next row's infinities, NaN between the
rows and behind the matrix - is no part of its sums.

Tolerance: a sum of n products in any order is off by at most (n + 4) 2^-24 of the products' magnitudes; taken in three parts a product is off by
less than 2^-21 + 2^-30 of it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests import test_gpu_feed_forward as plain
from tests.test_gpu_feed_forward_odd_float import E, LEFT_OUT, among_nan

# tokens, features reduced over (1, 2 and 3 beyond a multiple of 4; one piece, one step of 32, a step's end, many), features of the result
SHAPES = [(1, 1, 5), (3, 2, 40), (8, 3, 129), (1, 31, 200), (33, 33, 64), (64, 65, 131), (2, 95, 257), (70, 126, 100), (5, 601, 300), (130, 262, 270),
          (1, 4743, 1664), (8, 2051, 700), (300, 1003, 515)]


@pytest.mark.parametrize("pad,lead", [(0, 0), (1, 1), (2, 3), (4, 0)])
@pytest.mark.parametrize("data", [False, True], ids=["forward", "data"])
def test_rows_that_end_inside_a_piece(data, pad, lead):
    u = plain._u()
    ig, h = u.ig, u.handle()
    for M, n, N in SHAPES:
        print("data" if data else "forward", M, n, N, pad, lead, flush=True)
        rng = np.random.default_rng(M + n)
        a, b = plain.rounded(plain.normal(rng, M, n), "f32"), plain.rounded(plain.normal(rng, *((n, N) if data else (N, n))), "f32")
        # every other row begins with an infinity, which is its own row's only
        a[1::2, 0] = np.inf
        if not data:
            b[1::2, 0] = np.inf
        A, B, Y = among_nan(u, a, pad, lead), among_nan(u, b, 0, lead), u.Rows((M, N), "f32", pad, lead, fill=float("nan"))
        W = u.filter_desc("f32", *b.shape)
        size = ig.get_linear_backward_data_workspace_size(h, W, A.desc, Y.desc) if data else ig.get_linear_forward_workspace_size(h, A.desc, W, Y.desc)
        for lend in sorted({0, size // 2 // 16 * 16, size}):
            Y.view.fill_(float("nan"))
            ws = u.Workspace(lend)
            if data:
                ig.check(ig.linear_backward_data(h, 1.0, W, B.ptr, A.desc, A.ptr, ws.buf.data_ptr(), lend, -1, None, 0, 0.0, None, 0, Y.desc, Y.ptr))
            else:
                ig.check(ig.linear_forward(h, 1.0, A.desc, A.ptr, W, B.ptr, ws.buf.data_ptr(), lend, 0, -1, 0.0, None, 0, Y.desc, 0, Y.ptr))
            ws.check()
            right = a[0::2], b if data else b[0::2].T
            want = right[0] @ right[1]
            got = Y.view.double().cpu().numpy()
            u.close(got[0::2, :] if data else got[0::2, 0::2], want, ((n + 4) * E + LEFT_OUT) * (np.abs(right[0]) @ np.abs(right[1])) + E * np.abs(want) + 1e-30, "y")
            assert not np.isfinite(got[1::2]).any() and (data or not np.isfinite(got[:, 1::2]).any())
            Y.view.fill_(0)
            Y.numpy()
