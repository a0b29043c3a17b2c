"""Cross entropy and its gradients on the tiles of 256 x 256, named by the profiler, and through float logits in pieces: sizes off the tiles, repeated targets, bias.  Formulas and tolerances
are those of the smaller sizes."""
import pytest

pytestmark = pytest.mark.gpu

import torch

from tests.test_gpu_cross_entropy import Case, _u

LARGE = "TileConfig<256, 256, 2, 4, "


ENDS = {"loss": ("false, false", "RowStatistics"), "slopes": ("false, false", "Slopes"), "data": ("false, true", "WithRows"), "filter": ("true, true", "WithRows")}


def check_names(names, ends):
    for end in ends.split():
        kernel, what = ENDS[end]
        assert any(LARGE + kernel in n and "igc::" + what in n for n in names), (end, names)


def a_case(M, C, V, layout=(0, 0), units=256, repeat=0, **more):
    print("large tiles", M, C, V, layout, units, repeat, flush=True)
    c = Case(M, C, V, "bf16", layout, bias=True, **more)
    _u().ig.set_compute_units(c.h, units)
    if repeat:      # a third of the rows share a few targets, the last entry among them
        m = torch.arange(M, device="cuda")
        c.t = torch.where(m % 3 == 0, V - 1 - m // 3 % repeat, c.t.long()).to(torch.int32)
    return c


# (sizes, what of them takes the large tiles)
SIZES = [((2047, 1000, 16381, (8, 8)), "slopes filter"), ((4090, 4096, 8185, (0, 0)), "slopes data filter"), ((4095, 2056, 16381, (2, 2)), "slopes data"), ((2303, 1024, 16383, (0, 0)), "data filter"),
         ((2305, 1024, 16385, (8, 8)), "data"), ((4095, 2056, 9001, (2, 2)), "data"), ((4095, 4104, 8193, (0, 0)), ""), ((9047, 3136, 2265, (0, 0)), "filter")]


def test_loss():
    from tests.kernel_names import launched
    for size, ends in SIZES:
        c = a_case(*size)
        _, names = launched(c.forward)
        check_names(names, "loss" if "slopes" in ends else "")
        c.check_forward()
        first = c.forward()
        assert all(torch.equal(a, b) for a, b in zip(first, c.forward()))
        del c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_gradients(out):
    from tests.kernel_names import launched
    for size, ends in SIZES:
        c = a_case(*size, repeat=5)
        got, names = launched(lambda: c.backward(out, out))
        check_names(names, ends)
        c.check_backward(out, out, alpha=1.0 / c.M, beta=1.0, pbeta=1.0)
        del c, got
        torch.cuda.empty_cache()


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_gradients_as_planned_for_eight_compute_units(out):
    """Both products with rows added in tiles of 256 x 256, at sizes one off them; the logits in memory."""
    from tests.kernel_names import launched
    for M, C, V, layout, repeat in ((1100, 520, 6000, (0, 0), 3), (1025, 2049, 3001, (2, 2), 0), (767, 1001, 4097, (1, 1), 1), (1023, 264, 12001, (8, 8), 300)):
        c = a_case(M, C, V, layout, 8, repeat)
        got, names = launched(lambda: c.backward(out, out))
        check_names(names, "data filter" if C > 264 else "data")
        assert any("slope_kernel" in n for n in names), names
        c.check_backward(out, out, alpha=0.5, beta=0.5, pbeta=0.0)
        del c, got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M,C,V,pieces", [(2100, 72, 66000, 2), (16, 40, 2200000, 3)])
def test_logits_in_memory_in_pieces(M, C, V, pieces):
    """More float logits than a piece holds, where the planning (for eight compute units) finds them the faster; the last piece smaller than the others."""
    from tests.kernel_names import launched
    c = a_case(M, C, V, (8, 8) if M > 16 else (0, 0), 8, size=1.0)
    _, names = launched(c.forward)
    assert sum("row_parts_kernel" in n for n in names) == pieces, names
    c.check_forward()
    del c
    torch.cuda.empty_cache()
