"""Gradients of cross entropy with rows longer than the tiles take (2^22 elements): the kernel for any layout puts back what rounding left of dz at the targets as well.

Tolerances are those of the shorter rows; a logit is a sum of the 64 features that are not zero (the others' products are zeros, and add nothing)."""
import pytest

pytestmark = pytest.mark.gpu

import torch

from tests.test_gpu_cross_entropy import E, Case, _u

C, SOME = (1 << 22) + 8, 64


class Long(Case):
    def __init__(self, M, V, **more):
        super().__init__(M, C, V, "bf16", bias=True, **more)
        at = torch.randperm(C, generator=self.g, device="cuda")[:SOME]
        at[0] = C - 1
        keep = self.X.view[:, at].clone()
        self.X.view.zero_()
        self.X.view[:, at] = keep
        self.w.normal_(generator=self.g)
        self.w *= 2.0 / SOME ** 0.5

    def exact(self):
        loss, log_sum, z, _ = super().exact()
        size = self.X.view.double().abs() @ self.w.double().abs().t()
        return loss, log_sum, z, (SOME + 4) * E * size + E * (z.abs() + self.bias.double().abs())


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32")], ids="-".join)
def test_rows_longer_than_the_tiles_take(types):
    from tests.kernel_names import launched
    for M, V, repeat in ((40, 5, False), (70, 3, True)):
        print("long rows", types, M, V, flush=True)
        c = Long(M, V, lost=0.1)
        if repeat:
            c.t = (torch.arange(M, device="cuda") % 2).to(torch.int32)
        got, names = launched(lambda: c.backward(*types))
        assert sum("linear_any_kernel" in n for n in names) == 3, names
        c.check_backward(*types, alpha=1.0 / M, beta=0.5 if repeat else 0.0, pbeta=0.5)
        del c, got
        torch.cuda.empty_cache()
