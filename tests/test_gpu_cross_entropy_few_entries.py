"""Gradients of many rows over a few entries: in two parts, without a long sum for each entry; against the formulas in 64 bits, with the tolerances of slopes in two parts."""
import pytest

pytestmark = pytest.mark.gpu

import torch

from tests.test_gpu_cross_entropy import _u
from tests.test_gpu_cross_entropy_slopes import Whole


def a_case(M, C, V, layout, how):
    print("few entries", M, C, V, how, flush=True)
    c = Whole(M, C, V, "bf16", layout, bias=True, lost=0.1)
    ig = _u().ig
    ig.set_cross_entropy_slopes(c.h, ig.IGC_DATA_BFLOAT16)       # (as handles are at first)
    if how == "same":
        c.t = torch.where(c.t >= 0, V - 1, c.t.long()).to(torch.int32)
    return c


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32")], ids="-".join)
def test_many_rows_of_a_few_entries(types):
    from tests.kernel_names import launched
    for i, (M, C, V, layout) in enumerate([(512, 40, 1, (0, 0)), (3000, 40, 2, (3, 1)), (2000, 130, 10, (0, 0)), (1111, 2048, 16, (8, 8)), (700, 4096, 8, (0, 0)), (20001, 64, 2, (0, 0))]):
        c = a_case(M, C, V, layout, "same" if i % 2 else "any")
        got, names = launched(lambda: c.backward(*types, beta=0.5))
        assert not any("rest_rows" in n for n in names), names
        c.check(*types, beta=0.5, got=got)


def test_nearly_a_million_rows_of_two_entries():
    c = a_case(932003, 72, 2, (0, 0), "any")
    c.check("bf16", "f32")
    torch.cuda.empty_cache()


def test_more_entries_fewer_rows_and_more_features_are_as_they_were():
    from tests.kernel_names import launched
    for M, C, V in ((2000, 130, 17), (700, 4096, 9), (511, 40, 2), (66000, 1017, 2)):
        c = a_case(M, C, V, (0, 0), "any")
        _, names = launched(lambda: c.backward("bf16", "bf16"))
        assert any("rest_rows" in n for n in names), names
        c.check_backward("bf16", "f32")
