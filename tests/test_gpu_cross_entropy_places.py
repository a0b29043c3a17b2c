"""Cross entropy with bfloat16 features and vocabularies two bytes off 4-byte boundaries.  Formulas and tolerances are those of operands
on boundaries."""
import pytest

pytestmark = pytest.mark.gpu

import torch

from oracle import cross_entropy_oracle as co
from tests.test_gpu_cross_entropy import Case, _u


def off(w):
    """a copy of w, one element behind a 256-byte boundary"""
    buf = torch.full((w.numel() + 9,), 777.0, dtype=w.dtype, device="cuda")
    to = buf[1:1 + w.numel()].view(w.shape)
    to.copy_(w)
    assert to.data_ptr() % 4 == 2
    return to


PLACES = [(True, False), (False, True), (True, True)]
SIZES = [(1, 1, 1), (4, 64, 1000), (16, 128, 300), (33, 96, 9000), (65, 200, 4100), (130, 64, 5003), (300, 512, 1030), (777, 1000, 10007), (257, 130, 129)]


def a_case(M, C, V, x_off, w_off, **more):
    print("places", M, C, V, x_off, w_off, flush=True)
    c = Case(M, C, V, "bf16", (8, 1) if x_off else (8, 0), bias=True, **more)
    if w_off:
        c.w = off(c.w)
    assert c.X.ptr % 4 == (2 if x_off else 0)
    return c


@pytest.mark.parametrize("x_off,w_off", PLACES)
def test_loss(x_off, w_off):
    for size in SIZES:
        a_case(*size, x_off, w_off).check_forward()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("x_off,w_off", PLACES)
def test_gradients(x_off, w_off, out):
    for i, size in enumerate(SIZES):
        a_case(*size, x_off, w_off).check_backward(out, out, dbias=i % 3 != 0, beta=(0.0, 1.0, -2.0)[i % 3], pbeta=(0.0, 0.0, 1.0, 0.5)[i % 4])


@pytest.mark.parametrize("x_off,w_off", PLACES)
def test_copies_and_large_tiles(x_off, w_off):
    """Many rows: copied first, then on the tiles that operands on boundaries have; a long vocabulary in pieces of its copy."""
    from tests.kernel_names import launched
    for M, C, V, pieces in ((2047, 1000, 16381, 1), (1100, 4096, 20001, 3)):
        c = a_case(M, C, V, x_off, w_off)
        for call, end in ((c.forward, "igc::RowStatistics"), (lambda: c.backward("bf16", "bf16"), "igc::Slopes<")):
            _, names = launched(call)
            tiles = [n for n in names if "linear_tiles_kernel" in n]
            assert any("linear_pack_kernel" in n for n in names) and not any("TileConfig<64," in n for n in tiles), names
            assert sum(end in n for n in names) == (pieces if w_off or pieces == 1 else sum(end in n for n in names)), names
        c.check_forward()
        c.check_backward("bf16", "f32", alpha=1.0 / M, pieces=3)
        del c
    torch.cuda.empty_cache()


def test_more_tiles_than_a_launch_of_the_smallest_holds():
    """40000 x 8 -> 1000001, 4e10 logits: looked at in some rows."""
    c = Case(40000, 8, 1000001, "bf16", bias=True)
    c.w = off(c.w)
    loss, log_sum = c.forward()
    some = torch.cat([torch.arange(20), torch.arange(19990, 20010), torch.arange(39980, 40000)]).cuda()
    wl, ws, _ = co.forward(c.X.view[some].double(), c.w.double(), c.bias.double(), c.t[some])
    assert float((loss[some] - wl).abs().max()) < 1e-4 and float((log_sum[some] - ws).abs().max()) < 1e-4
    torch.cuda.empty_cache()
