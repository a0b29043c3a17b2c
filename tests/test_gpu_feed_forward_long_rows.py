"""Layer norm of rows that 512 and 1024 threads hold, and of rows written in place whose last chunk is not whole: the tolerances of
test_gpu_feed_forward.py."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import feed_forward_oracle as fo
from tests import test_gpu_feed_forward as plain

E = 2.0 ** -24


@pytest.mark.parametrize("layout", [(0, 0), (3, 1)], ids=str)
@pytest.mark.parametrize("types", plain.NORM_TYPES, ids="-".join)
def test_long_rows(types, layout, monkeypatch):
    monkeypatch.setattr(plain, "NORM_SHAPES", [(3, 20000), (2, 32768), (3, 12305), (5, 16380)])
    plain.test_layer_norm_forward(types, layout)
    plain.test_layer_norm_backward(types, layout)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("beta", [0.0, 0.5])
def test_ragged_rows_in_place(dtype, beta):
    u = plain._u()
    ig, h = u.ig, u.handle()
    half = u.HALF_STEP[dtype]
    for M, C in ((9, 9), (70, 100), (5, 255), (6, 1001), (5, 2047), (4, 4099), (3, 8190), (3, 16379), (2, 16391), (2, 32761)):
        rng = np.random.default_rng(C)
        x = plain.rounded(plain.normal(rng, M, C) * 2 + plain.normal(rng, M, 1), dtype)
        X = u.Rows(x, dtype)
        print("in place", dtype, beta, M, C, flush=True)
        ig.check(ig.layer_norm_forward(h, 1.0, X.desc, X.ptr, 0, 0, plain.EPS, beta, X.desc, X.ptr))
        y, m, s = fo.layer_norm(x, None, None, plain.EPS)
        em = (C + 4) * E * np.abs(x).mean(1)
        d = np.abs(x - m[:, None])
        es = s * (2 * (C + 8) * E + s * s * 2 * em * d.mean(1) + s * s * em * em)
        tol = em[:, None] * s[:, None] + d * (es + 6 * E * s)[:, None] + 4 * E * (np.abs(y) + np.abs(beta * x))
        want = y + beta * x
        u.close(X.numpy(), want, tol + 4 * E * np.abs(beta * x) + half * np.abs(want) * 1.01 + 1e-30, "in place")
