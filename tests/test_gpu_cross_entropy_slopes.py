"""Gradients of cross entropy with the slopes dz of bfloat16 features in two parts, as the handle can be asked for, against the formulas in 64 bits.

Tolerances as where dz is rounded (e = 2^-24), but dz reaches the products with an error of 2^-16 of each element (two roundings of 2^-8) beside its own; a product of n terms is n of the one
part and n of the other, (2 n + 10) e of their magnitudes, and e for each piece of the vocabulary."""
import pytest

pytestmark = pytest.mark.gpu

import torch

from oracle import cross_entropy_oracle as co
from tests.test_gpu_cross_entropy import E, HALF, LAYOUTS, SIZES, Case, _u, near


class Whole(Case):
    def __init__(self, *a, units=256, **more):
        super().__init__(*a, **more)
        ig = _u().ig
        ig.set_cross_entropy_slopes(self.h, ig.IGC_DATA_FLOAT)
        ig.set_compute_units(self.h, units)

    def check(self, dx, dw, alpha=1.0, beta=0.0, pbeta=0.0, dbias=True, pieces=1, got=None):
        got = got or self.backward(dx, dw, dbias, alpha, beta, pbeta)
        _, _, z, tz = self.exact()
        s, d = self.log_sum.double(), self.dloss.double()
        dz = alpha * co.slopes(z, s, self.t, d)
        there = ((self.t >= 0) & (self.t < self.V))[:, None]
        size = torch.where(there, abs(alpha) * d.abs()[:, None] * torch.exp(z - s[:, None]), 0.0)
        tdz = size * (torch.expm1(tz) + 2 * E * (z - s[:, None]).abs() + 8 * E) + 8 * E * dz.abs()
        parts = tdz + 2.0 ** -16 * (dz.abs() + tdz)
        x, w = self.X.view.double(), self.w.double()
        for name, want, tol, scale, out in (
                ("dbias", dz.sum(0), tdz.sum(0) + (self.M + 8) * E * dz.abs().sum(0), pbeta, "f32"),
                ("dx", dz @ w, parts @ w.abs() + (2 * self.V + 10 + 2 * pieces) * E * ((dz.abs() + parts) @ w.abs()), beta, dx),
                ("dw", dz.t() @ x, parts.t() @ x.abs() + (2 * self.M + 10) * E * ((dz.abs() + parts).t() @ x.abs()), pbeta, dw)):
            if name not in got:
                continue
            have, old = got[name]
            if scale:
                want, tol = want + scale * old, tol + 4 * E * (scale * old).abs()
            near(have, want, tol + HALF[out] * (want.abs() + tol) + 1e-37, name + " " + str((self.M, self.C, self.V, self.layout, dx, dw, alpha, beta, pbeta)))


TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")]


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_any_number_of_rows(types):
    for i, (M, C, V) in enumerate(SIZES + [(33, 96, 9000), (70, 96, 300), (1100, 520, 6000), (777, 1000, 10007)]):
        print("slopes in two parts", types, M, C, V, flush=True)
        Whole(M, C, V, "bf16", LAYOUTS[i % 4], bias=i % 2 == 1).check(*types, alpha=1.0 if i % 4 else 0.5, beta=(0.0, 1.0, -2.0)[i % 3], pbeta=(0.0, 0.0, 1.0, 0.5)[i % 4])


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_large_tiles_pieces_and_logits_in_memory(out):
    from tests.kernel_names import launched
    for M, C, V, layout, units, kernel in ((2047, 1000, 16381, (8, 8), 256, "igc::Slopes<"), (5000, 72, 40011, (0, 0), 256, "igc::Slopes<"), (1100, 520, 6000, (3, 1), 8, "slope_kernel"),
                                           (767, 1001, 4097, (1, 1), 8, "slope_kernel")):
        print("slopes in two parts", out, M, C, V, units, flush=True)
        c = Whole(M, C, V, "bf16", layout, bias=True, units=units)
        got, names = launched(lambda: c.backward(out, out, beta=0.5, pbeta=0.0))
        assert any(kernel in n for n in names) and not any("rest_rows" in n or "WithRows" in n for n in names), names
        assert M != 2047 or any("TileConfig<256, 256" in n and "igc::Slopes<" in n for n in names), names
        assert M != 5000 or sum("igc::Slopes<" in n for n in names) == 2, names
        c.check(out, out, beta=0.5, pieces=2, got=got)
        del c, got
    torch.cuda.empty_cache()


def test_one_gradient_at_a_time():
    for M in (20, 70):
        c = Whole(M, 96, 300, "bf16", bias=True)
        for ask in (("bf16", None, False), (None, "f32", False), (None, None, True), (None, "bf16", True), ("f32", None, True)):
            c.check(ask[0], ask[1], dbias=ask[2])


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32")], ids="-".join)
def test_targets_that_repeat(types):
    for M, C, V in ((33, 64, 100), (600, 70, 50), (3000, 40, 2), (2000, 130, 10)):
        for how in (0, 1):
            c = Whole(M, C, V, "bf16", bias=True, lost=0.0)
            m = torch.arange(M, device="cuda")
            c.t = (m % V if how else 0 * m + V // 2).to(torch.int32)
            c.check(*types, alpha=1.0 / M)


def test_entries_that_are_nobodys_target():
    """As exact as the others: by the norm of such rows of dw against 64 bits (2^-16 and the exponential's error; with dz rounded to bfloat16 1.7e-3)."""
    c = Whole(777, 1000, 10007, "bf16", bias=True, lost=0.0)
    got = c.backward(None, "f32", dbias=False)["dw"][0]
    z = c.exact()[2]
    want = co.slopes(z, c.log_sum.double(), c.t, c.dloss.double()).t() @ c.X.view.double()
    free = torch.ones(10007, dtype=torch.bool, device="cuda")
    free[c.t.long()] = False
    assert 9000 < int(free.sum()) < 10007
    assert float((got - want)[free].norm() / want[free].norm()) < 2.0 ** -15


def test_a_heads_gradients():
    """VocabularyHead: float gradients as exact as float's unless it is made for speed."""
    _u()
    from paper_1410_0759_amd import training as tr
    M, D, V = 300, 256, 1000
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(M, D, generator=g, device="cuda").to(torch.bfloat16)
    t = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    off = {}
    for slopes in (torch.float32, torch.bfloat16, None):
        head = tr.VocabularyHead(D, V, **({} if slopes is None else {"slopes": slopes}))
        head.forward(x, t)
        head.backward(scale=1.0 / M)
        z = x.double() @ head.w.double().t()
        want = (co.slopes(z, torch.logsumexp(z, 1), t, torch.ones(M, dtype=torch.float64, device="cuda")) / M).t() @ x.double()
        off[slopes] = float((head.grads["w"] - want).norm() / want.norm())
    assert off[torch.float32] < 2.0 ** -15 and off[None] == off[torch.float32] and off[torch.bfloat16] > 2 * off[torch.float32], off
