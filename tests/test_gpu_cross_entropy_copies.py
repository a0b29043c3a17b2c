"""Cross entropy with vocabularies that are copied first, in pieces."""
import pytest

pytestmark = pytest.mark.gpu

import torch

from tests.test_gpu_cross_entropy import Case, _u


def test_float_vocabularies_in_pieces_of_their_parts():
    """The parts of w, copied, are 512 MB at a time; the room asked for is bounded by them."""
    from tests.kernel_names import launched
    u, ig = _u(), _u().ig
    for M in (1000, 1500):
        c = Case(M, 4096, 60001, "f32", (1, 1), bias=True)
        _, names = launched(c.forward)
        assert sum("RowStatistics" in n or "row_parts_kernel" in n for n in names) == 3, names      # (no logits in memory, or pieces of them)
        c.check_forward()
        assert ig.get_linear_cross_entropy_forward_workspace_size(c.h, c.X.desc, c.wd) < 700 << 20 < 60001 * 4096 * 6
        del c
    torch.cuda.empty_cache()
