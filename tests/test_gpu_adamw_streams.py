"""AdamW over lists of more elements than are read through the caches: tensors on 128-byte boundaries are read past them, others in the same list are not.  Formula and tolerances are
those of the shorter lists."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import adamw_oracle as ao
from tests.test_gpu_adamw import B1, B2, E, RATE, _u, handle, near, parameters

LONG = (1 << 24) + 4097       # (more than are kept in the caches, with a ragged end)


def codes(code, scale, x, tx, form, random, what):
    """code, scale: of the numbers x, known to tx (which is m's error and not a part of m: its two terms may cancel)."""
    want, most = ao.scales(x, form), np.zeros(-(-len(x) // 256) * 256)
    most[:len(x)] = tx
    near(scale, want, 8 * E * want + most.reshape(-1, 256).max(1) / form[0], what + " scale")
    s = np.repeat(scale, 256)[:len(x)]
    there = s > 0
    y, ty = (np.divide(q, s, out=np.zeros(len(x)), where=there) for q in (x, tx))
    ty += 4 * E * np.abs(y)         # (the inverse of the scale, and the product with it)
    lo, hi = (ao.rounded(y + d, form, random) for d in (-ty, ty))
    ok = (code >= np.minimum(lo, hi)) & (code <= np.maximum(lo, hi))
    assert ok.all(), (what, int((~ok).sum()), int(np.argmin(ok)), code[~ok][:3], y[~ok][:3])


def step(tensors, t=7, scale=0.5, seed=99):
    import paper_1410_0759_amd as ig
    u = _u()
    before = [(x.p.numpy(), x.g.numpy(), *x.states()) for x in tensors]
    ig.check(ig.adamw_step(handle(), parameters(step=t, seed=seed, gradient_scale=scale), u.table(tensors)), "igcAdamWStep")
    for i, (x, (p, g, m, v)) in enumerate(zip(tensors, before)):
        what = "tensor %d of %d" % (i, x.n)
        wp, wm, wv = ao.step(p, g, m, v, t, RATE, B1, B2, 1e-8, x.decay, scale)
        tm, tv = 4 * E * (np.abs(B1 * m) + np.abs((1 - B1) * scale * g)), 6 * E * (B2 * v + (1 - B2) * (scale * g) ** 2)
        c1, c2 = 1 / (1 - B1 ** t), 1 / (1 - B2 ** t)
        root = np.sqrt(wv * c2) + 1e-8
        near_root = np.divide(tv * c2, np.sqrt(wv * c2) * 2, out=np.zeros(x.n), where=wv > 0)
        tp = RATE * c1 / root * (tm + np.abs(wm) * (16 * E + 1.01 * near_root / root)) + 4 * E * (np.abs(p) + np.abs(wp))
        got = x.p.numpy()
        near(got, wp, tp + (E if x.p.dtype.itemsize == 4 else 2.0 ** -8) * (np.abs(wp) + tp), what + " p")
        if x.copy is not None:
            import torch
            assert np.array_equal(x.copy.numpy(), torch.from_numpy(got).to(torch.bfloat16).double().numpy()), what + " copy"
        assert np.array_equal(x.g.numpy(), g)
        if x.bits == 32:
            near(x.m.numpy(), wm, tm, what + " m")
            near(x.v.numpy(), wv, tv, what + " v")
        elif x.n:
            rm, rv = ao.random_bits(x.n, seed, t)
            codes(x.m.numpy(), x.ms.numpy(), wm, tm, ao.E4M3, rm, what + " m")
            codes(x.v.numpy(), x.vs.numpy(), wv, tv, ao.E5M2, rv, what + " v")


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_long_lists(grad, param, bits):
    u = _u()
    rng = np.random.default_rng(5)
    print("long list", grad, param, bits, flush=True)
    step([u.Tensor(rng, LONG, param, grad, bits, copy=param == "f32"), u.Tensor(rng, 70001, param, grad, bits, lead=3), u.Tensor(rng, 4099, param, grad, bits, copy=param == "f32"),
          u.Tensor(rng, 0), u.Tensor(rng, 1, param, grad, bits), u.Tensor(rng, 255, "f32", "bf16", 40 - bits)])
