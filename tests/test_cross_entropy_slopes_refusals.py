"""The choice of what the slopes go into the products as: host logic, no GPU call."""
import pytest
import torch

import paper_1410_0759_amd as ig
from paper_1410_0759_amd import training as tr
from tests.test_cross_entropy_refusals import BAD, B, F, OK, P, UNSUPPORTED, D, filt, rows, status


def test_choice():
    h = ig.Handle()
    assert ig.get_cross_entropy_slopes(h) == B
    for bad in (D, -1, 17):
        assert status(lambda: ig.set_cross_entropy_slopes(h, bad)) == BAD
    assert ig.get_cross_entropy_slopes(h) == B
    assert status(lambda: ig.set_cross_entropy_slopes(h, F)) == OK and ig.get_cross_entropy_slopes(h) == F
    with pytest.raises(ValueError, match="slopes"):
        tr.VocabularyHead(8, 20, device="cpu", slopes=torch.float64)
    assert ig.get_cross_entropy_slopes(tr.VocabularyHead(8, 20, device="cpu").handle) == F
    assert ig.get_cross_entropy_slopes(tr.VocabularyHead(8, 20, device="cpu", slopes=torch.bfloat16).handle) == B


def test_workspace_and_rows():
    """The query goes by the handle's choice, stays bounded by pieces, and the call asks for what it reports; two parts of more than 2^29 rows are refused."""
    def query(h, M, C, V):
        return ig.get_linear_cross_entropy_backward_workspace_size(h, rows(B, M, C), filt(B, V, C), rows(B, M, C), filt(B, V, C))

    def call(h, M, C, V, room):
        return ig.linear_cross_entropy_backward(h, 1.0, rows(B, M, C), P, filt(B, V, C), P, 0, P, P, 0, P, room, 0.0, rows(B, M, C), P, 0.0, filt(B, V, C), P, 0)

    a, b = ig.Handle(), ig.Handle()
    ig.set_cross_entropy_slopes(b, F)
    assert query(a, 20, 64, 1000) == query(b, 20, 64, 1000)           # (few rows are in two parts anyway)
    need = query(b, 1000, 64, 1000)
    assert need != query(a, 1000, 64, 1000) and call(b, 1000, 64, 1000, need - 1) == BAD
    assert query(b, 8192, 4096, 131072) < 5 << 28 < 2 * 8192 * 131072 * 2      # (of all of dz that would be 4 GB)
    most = 1 << 29
    assert status(lambda: query(b, most, 1, 1)) == OK and status(lambda: query(b, most + 1, 1, 1)) == UNSUPPORTED and call(b, most + 1, 1, 1, 1 << 50) == UNSUPPORTED
    assert status(lambda: query(a, most + 1, 1, 1)) == OK


def test_room_of_a_few_entries():
    """Beyond 2^26 features of x the parts are not held at once: no more room than twice x, and logits and dz in 64 columns."""
    h = ig.Handle()
    for M, C in ((1 << 21, 4096), ((1 << 26) // 64 + 1, 64), (70000, 1000)):
        assert ig.get_linear_cross_entropy_backward_workspace_size(h, rows(B, M, C), filt(B, 2, C), rows(B, M, C), filt(B, 2, C)) < 2 * M * C * 2 + M * 64 * (4 + 2) + (1 << 27)
