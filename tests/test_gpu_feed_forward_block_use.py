"""A feed-forward block between several uses: passes without a gradient among passes with one."""
import pytest

pytestmark = pytest.mark.gpu


def _modules():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1410_0759_amd import feed_forward
    return torch, feed_forward


def _data(torch, block, M, n, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(M, block.width, generator=g, device="cuda").to(block.dtype) for _ in range(n)]


def test_a_pass_without_gradient_leaves_the_one_before():
    torch, ff = _modules()
    block = ff.FeedForward(64, 256)
    x, other, dy = _data(torch, block, 33, 3)
    y = block.forward(x).clone()
    want = [block.backward(x, dy).clone()] + [t.clone() for t in block.grads.values()]
    kept = block.forward(x)
    served = block.forward(other, keep=False).clone()
    got = [block.backward(x, dy).clone()] + [t.clone() for t in block.grads.values()]
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert torch.equal(kept, y)                                    # (its result too)
    assert torch.equal(served, block.forward(other))


def test_backward_of_rows_that_were_not_kept_is_refused():
    torch, ff = _modules()
    block = ff.FeedForward(64, 256)
    x, other, dy = _data(torch, block, 12, 3)
    with pytest.raises(ValueError, match="forward"):
        block.backward(x, dy)
    block.forward(x, keep=False)
    with pytest.raises(ValueError, match="forward"):
        block.backward(x, dy)
    block.forward(x)
    block.forward(other)
    with pytest.raises(ValueError, match="forward"):
        block.backward(x, dy)
    block.forward(x[:7])
    want = block.backward(other, dy).clone()
    block.forward(other)
    assert torch.equal(block.backward(other, dy), want)
    block.backward(x[:7], dy[:7])


def test_the_result_as_the_next_input():
    """Twice the same block: without a gradient in place, with one only through a copy."""
    torch, ff = _modules()
    block = ff.FeedForward(64, 256)
    x, dy = _data(torch, block, 21, 2)
    once = block.forward(x).clone()
    want = block.forward(once).clone()
    with pytest.raises(ValueError, match="clone"):
        block.forward(block.forward(x))
    assert torch.equal(block.forward(block.forward(x, keep=False), keep=False), want)
    block.forward(once)
    block.backward(once, dy)
