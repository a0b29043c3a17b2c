"""Weight decay of AdamW at ordinary products of rate and decay, which are near float's steps: p - rate decay p, rounded once.

Tolerances: half a step of the result, and 2^-22 of the decay (rate, decay and their product are rounded, and it is multiplied by p and added to the update: 4 roundings)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import adamw_oracle as ao
from tests.test_gpu_adamw import B1, B2, EPS, _u, handle, parameters

PRODUCTS = [(1e-6, 0.1), (1e-5, 0.01), (3e-5, 0.1), (1e-3, 0.1), (2e-7, 0.1), (0.5, 1.0)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rate,decay", PRODUCTS)
def test_decay_alone(rate, decay, bits):
    """No gradient yet: the update is zero."""
    import paper_1410_0759_amd as ig
    u = _u()
    for fresh_step in (1, 1000):
        x = u.Tensor(np.random.default_rng(1), 40007, "f32", "f32", bits, copy=True, decay=decay, fresh=True)
        x.g.put(np.zeros(x.n), x.g.dtype)
        p = x.p.numpy()
        ig.check(ig.adamw_step(handle(), parameters(learning_rate=rate, step=fresh_step), u.table([x])), "igcAdamWStep")
        want, got = p * (1 - rate * decay), x.p.numpy()
        tol = np.spacing(np.abs(want).astype(np.float32)).astype(np.float64) / 2 + 2.0 ** -22 * rate * decay * np.abs(p)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (int(bad.sum()), bad.size, p[bad][:3], got[bad][:3], want[bad][:3])


@pytest.mark.parametrize("rate,decay", PRODUCTS[:3])
def test_decay_on_the_average(rate, decay):
    """With updates beside it: over many weights the decay asked for, not a multiple of float's steps.  (Each result is off by half a step at most, as good as evenly spread because the
    updates are: of their sum's deviation, the steps / sqrt 12 times the root of their number, eight times.)"""
    import paper_1410_0759_amd as ig
    u = _u()
    n = 1 << 20
    x = u.Tensor(np.random.default_rng(2), n, decay=decay)
    x.p.put(np.random.default_rng(3).uniform(0.5, 2.0, n), x.p.dtype)
    p, g, (m, v) = x.p.numpy(), x.g.numpy(), x.states()
    ig.check(ig.adamw_step(handle(), parameters(learning_rate=rate, step=7, gradient_scale=0.5), u.table([x])), "igcAdamWStep")
    want = ao.step(p, g, m, v, 7, rate, B1, B2, EPS, decay, 0.5)[0]
    steps = np.spacing(want.astype(np.float32)).astype(np.float64)
    off = (x.p.numpy() - want).sum()
    assert abs(off) < 8 * np.sqrt((steps ** 2).sum() / 12) < 0.05 * rate * decay * p.sum(), (off, rate * decay * p.sum())


def test_weights_that_are_not_finite_stay_so():
    import paper_1410_0759_amd as ig
    u = _u()
    for decay in (0.0, 0.1):
        x = u.Tensor(np.random.default_rng(4), 300, decay=decay)
        p = x.p.numpy()
        p[3], p[5], p[7], p[9] = np.inf, -np.inf, np.nan, 3.4e38
        x.p.put(p, x.p.dtype)
        ig.check(ig.adamw_step(handle(), parameters(), u.table([x])), "igcAdamWStep")
        got = x.p.numpy()
        assert got[3] == np.inf and got[5] == -np.inf and np.isnan(got[7])
        assert np.isfinite(np.delete(got, [3, 5, 7])).all() and abs(got[9] / 3.4e38 - 1) < 2e-4
