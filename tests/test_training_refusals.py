"""What the head, the optimiser and the block in four bits refuse: no GPU call."""
import pytest
import torch

from paper_1410_0759_amd import training as tr


def test_head():
    head = tr.VocabularyHead(8, 20, torch.float32, bias=True, device="cpu")
    x, t = torch.zeros(5, 8), torch.zeros(5, dtype=torch.int32)
    for bad in (torch.zeros(5, 7), torch.zeros(5, 8, dtype=torch.bfloat16), torch.zeros(8), torch.zeros(8, 5).t(), torch.zeros(0, 8), torch.zeros(5, 8, device="meta")):
        with pytest.raises(ValueError, match="x"):
            head.forward(bad, t)
    for bad in (torch.zeros(5, dtype=torch.int64), torch.zeros(4, dtype=torch.int32), torch.zeros(10, dtype=torch.int32)[::2], torch.zeros(5, 1, dtype=torch.int32)):
        with pytest.raises(ValueError, match="targets"):
            head.forward(x, bad)
    with pytest.raises(ValueError, match="GPU"):
        head.forward(x, t)
    with pytest.raises(ValueError, match="no forward pass"):
        head.backward()


def test_optimiser():
    w, g = torch.zeros(4, 8), torch.zeros(4, 8)
    for bad in ({}, {"w": (w, torch.zeros(4, 7))}, {"w": (w.t(), g.t())}, {"w": (w.double(), g)}, {"w": (w, w)}, {"w": (w, g), "v": (w[1:3], torch.zeros(2, 8))}):
        with pytest.raises(ValueError):
            tr.AdamW(bad)
    with pytest.raises(ValueError):
        tr.AdamW({"w": (w, g)}, bits=16)
    opt = tr.AdamW({"w": (w, g)})
    with pytest.raises(ValueError, match="GPU"):
        opt.step()
    with pytest.raises(ValueError, match="other weights"):
        opt.load_state_dict(tr.AdamW({"w": (w[:2], g[:2])}).state_dict())
    opt.load_state_dict(opt.state_dict())
    eight = tr.AdamW({"w": (torch.zeros(64, 64, dtype=torch.bfloat16), torch.zeros(64, 64)), "small": (w, g), "bias": (torch.zeros(5000), torch.zeros(5000))}, bits=8)
    assert {n: s["m"].element_size() for n, s in eight.state.items()} == {"w": 1, "small": 4, "bias": 4}
    assert [(q.count, q.state_bits, q.weight_decay) for q in eight.table] == [(4096, 8, 0.1), (32, 32, 0.1), (5000, 32, 0.0)]
