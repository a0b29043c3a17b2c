"""A feed-forward block between several uses: passes without a gradient among passes with one, streams, threads, many
numbers of tokens."""
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


def test_two_streams_in_turn():
    """Passes of as many tokens on two streams, nothing synchronised between them but by the block: what each gives alone, bit for bit."""
    torch, ff = _modules()
    block = ff.FeedForward(1024, 4096)
    data = _data(torch, block, 2000, 4)
    want = []
    for x, dy in (data[:2], data[2:]):
        want.append([block.forward(x).clone(), block.backward(x, dy).clone()] + [t.clone() for t in block.grads.values()])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(6):
        for s, (x, dy) in zip(streams, (data[:2], data[2:])):
            with torch.cuda.stream(s):
                y = block.forward(x).clone()
                got.append([y, block.backward(x, dy).clone()] + [t.clone() for t in block.grads.values()])
    torch.cuda.synchronize()
    for i, results in enumerate(got):
        assert all(torch.equal(p, q) for p, q in zip(results, want[i % 2])), i


def test_the_first_call_on_another_stream():
    torch, ff = _modules()
    x = torch.randn(64, 2048, device="cuda").to(torch.bfloat16)
    torch.cuda.synchronize()
    block = ff.FeedForward(2048, 8192)
    with torch.cuda.stream(torch.cuda.Stream()):
        got = block.forward(x).clone()            # (behind the weights, which are still being made)
    torch.cuda.synchronize()
    assert torch.equal(got, block.forward(x))


def test_threads():
    """Passes without a gradient from several threads, each on its own stream, with its own number of tokens."""
    import threading
    torch, ff = _modules()
    block = ff.FeedForward(256, 1024)
    sizes = (5, 64, 300)
    xs = [_data(torch, block, M, 1, seed=M)[0] for M in sizes]
    want = [block.forward(x, keep=False).clone() for x in xs]
    torch.cuda.synchronize()
    results, errors = {}, []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                results[i] = [block.forward(xs[i], keep=False).clone() for _ in range(30)]
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(sizes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not errors and len(results) == len(sizes)
    assert all(torch.equal(y, want[i]) for i in results for y in results[i])


def test_many_numbers_of_tokens():
    """Buffers are kept for the last few sizes only, and for what a graph holds."""
    torch, ff = _modules()
    block = ff.FeedForward(64, 256, sizes=3)
    data = {M: _data(torch, block, M, 2, seed=M) for M in range(1, 41)}
    x, dy = data[7]
    want = [block.forward(x).clone(), block.backward(x, dy).clone()] + [t.clone() for t in block.grads.values()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = [block.forward(x), block.backward(x, dy)]
    y = {}
    for M in (*range(1, 7), *range(8, 41), 3):
        y[M] = block.forward(data[M][0], keep=M % 2 == 0).clone()
        assert len(block._buffers) <= 4 and all(size[0] in (7, M, *y) for size in block._buffers)
    for M in (4, 40, 3):
        assert torch.equal(block.forward(data[M][0]), y[M])
    block.backward(*data[4])
    with pytest.raises(ValueError, match="forward"):
        block.backward(*data[6])                                   # (its buffers are gone)
    for t in captured + list(block.grads.values()):
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(captured + list(block.grads.values()), want))
