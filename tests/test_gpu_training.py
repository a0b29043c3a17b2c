"""A block, the vocabulary's loss and the optimiser's step together, and the block in four bits: on the GPU against 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import adamw_oracle as ao


def _modules():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1410_0759_amd import feed_forward, training
    return torch, feed_forward, training


def block_in_double(torch, p, x):
    """The block with autograd; p: leaves in double."""
    mean = x.mean(1, keepdim=True)
    d = x - mean
    h = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * p["scale"] + p["shift"]
    z = h @ p["w1"].t() + p["b1"]
    return z * 0.5 * torch.special.erfc(-z / 2 ** 0.5) @ p["w2"].t() + p["b2"] + x


def setting(torch, ff, tr, dtype, M=70, D=48, H=96, V=301, bias=True, bits=32):
    block, head = ff.FeedForward(D, H, dtype), tr.VocabularyHead(D, V, dtype, bias=bias, seed=5)
    g = torch.Generator(device="cuda").manual_seed(2)
    for n in ("b1", "b2", "shift"):
        getattr(block, n).copy_(0.3 * torch.randn(getattr(block, n).shape, generator=g, device="cuda"))
    weights = {**{n: (getattr(block, n), q) for n, q in block.grads.items()}, "head": (head.w, head.grads["w"])}
    if bias:
        weights["bias"] = (head.bias, head.grads["bias"])
    x = torch.randn(M, D, generator=g, device="cuda").to(dtype)
    t = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    t[::7] = -100
    return block, head, weights, x, t


# as for the block alone: float sums of at most a few hundred terms; in bfloat16 half a dozen roundings on the way, a few deviations of their sum
@pytest.mark.parametrize("dtype,tol", [("float32", 3e-5), ("bfloat16", 4e-2)])
def test_gradients_of_the_loss_through_the_block(dtype, tol):
    torch, ff, tr = _modules()
    block, head, weights, x, t = setting(torch, ff, tr, getattr(torch, dtype))
    loss = head.forward(block.forward(x), t)
    block.backward(x, head.backward(scale=1.0 / 70))
    p = {n: w.double().requires_grad_(True) for n, (w, _) in weights.items()}
    y = block_in_double(torch, p, x.double())
    z = y @ p["head"].t() + p["bias"]
    there = t >= 0
    want = torch.where(there, torch.logsumexp(z, 1) - z.gather(1, t.clamp(min=0).long()[:, None])[:, 0], 0.0)
    (want.sum() / 70).backward()
    want = want.detach()
    assert float((loss - want).abs().max()) <= tol * float(want.abs().max())
    for n, (_, got) in weights.items():
        w = p[n].grad
        assert float((got - w).abs().max()) <= tol * float(w.abs().max()), (n, float((got - w).abs().max() / w.abs().max()))
    first = {n: q.clone() for n, (_, q) in weights.items()}
    head.backward(scale=1.0 / 70, accumulate=True)
    for n in ("head", "bias"):
        assert torch.allclose(weights[n][1], 2 * first[n], rtol=1e-5, atol=1e-5 * float(first[n].abs().max())), n


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_use_these_gradients(dtype, bits):
    """Three steps: every weight as the formula has it from the gradients of that step, the states in 32 bits kept beside; in 8 bits from the states that were read back."""
    torch, ff, tr = _modules()
    block, head, weights, x, t = setting(torch, ff, tr, getattr(torch, dtype))
    opt = tr.AdamW(weights, rate=1e-2, bits=bits, decay=0.05, seed=3)
    m = {n: np.zeros(w.numel()) for n, (w, _) in weights.items()}
    v = {n: np.zeros(w.numel()) for n, (w, _) in weights.items()}
    eight = {n for n in weights if opt.state[n]["m"].element_size() == 1}
    assert eight == (set() if bits == 32 else {"w1", "w2", "head"})
    for step in range(1, 4):
        loss = head.forward(block.forward(x), t)
        block.backward(x, head.backward(scale=1.0 / 70))
        flat = lambda a: a.double().cpu().numpy().reshape(-1)
        before = {n: flat(opt.state[n].get("master", w)) for n, (w, _) in weights.items()}
        grads = {n: flat(g) for n, (_, g) in weights.items()}
        opt.step(scale=0.5)
        for n, (w, _) in weights.items():
            wp, wm, wv = ao.step(before[n], grads[n], m[n], v[n], step, 1e-2, 0.9, 0.999, 1e-8, 0.05 if w.dim() > 1 else 0.0, 0.5)
            got = flat(opt.state[n].get("master", w))
            # 16 x 2^-24 of an update of at most a few rates, 4 x 2^-24 of the weight
            assert np.abs(got - wp).max() <= 1e-2 * 10 * 20 * 2.0 ** -24 + 2.0 ** -21 * np.abs(wp).max(), (n, step, np.abs(got - wp).max())
            if "master" in opt.state[n]:
                assert torch.equal(w.reshape(-1), opt.state[n]["master"].to(torch.bfloat16)), n
            s = opt.state[n]
            m[n], v[n] = flat(s["m"]), flat(s["v"])
            if n in eight:
                m[n], v[n] = (q * np.repeat(flat(s[k]), 256)[:q.size] for q, k in ((m[n], "m_scale"), (v[n], "v_scale")))
    assert opt.steps == 3


def test_a_run_that_goes_on():
    torch, ff, tr = _modules()
    run = []
    for again in (False, True):
        block, head, weights, x, t = setting(torch, ff, tr, torch.bfloat16)
        opt = tr.AdamW(weights, bits=8)

        def steps(n):
            for _ in range(n):
                head.forward(block.forward(x), t)
                block.backward(x, head.backward(scale=1.0 / 70))
                opt.step()

        steps(2)
        if again:
            saved = opt.state_dict()
            opt = tr.AdamW(weights, bits=8)
            opt.load_state_dict(saved)
        steps(2)
        run.append([w.clone() for w, _ in weights.values()])
    assert all(torch.equal(a, b) for a, b in zip(*run))


@pytest.mark.parametrize("dtype,tol", [("float32", 3e-5), ("bfloat16", 3e-2)])
@pytest.mark.parametrize("M", [1, 5, 130])
def test_a_block_in_four_bits(dtype, tol, M):
    """Against the formula with the numbers that the codes stand for."""
    torch, ff, tr = _modules()
    import paper_1410_0759_amd as ig
    block, _, _, x, _ = setting(torch, ff, tr, getattr(torch, dtype), M=M, D=200, H=333)
    served = tr.FourBitFeedForward(block, group=32)
    p = {n: getattr(block, n).double() for n in ("scale", "shift", "b1", "b2")}
    for n, (k, c) in (("w1", (333, 200)), ("w2", (200, 333))):
        w = torch.empty(k, c, device="cuda")
        codes, scales = getattr(served, n)
        h = ig.Handle()
        h.set_stream(torch.cuda.current_stream().cuda_stream)
        ig.check(ig.dequantize_filter4(h, 32, codes.data_ptr(), scales.data_ptr(), ig.FilterDescriptor().set(ig.IGC_DATA_FLOAT, k, c, 1, 1), w.data_ptr()))
        p[n] = w.double()
        assert float((w - getattr(block, n).float()).abs().max()) <= float(getattr(block, n).float().abs().max()) / 6 * 1.01      # half the widest step, a sixth of the largest
    want = block_in_double(torch, p, x.double())
    assert float((served.forward(x).double() - want).abs().max()) <= tol * float(want.abs().max())


def test_captured():
    """Loss, gradients and a served token in graphs, replayed over changed inputs with eager calls between; the optimiser's own counting is refused there."""
    torch, ff, tr = _modules()
    block, head, weights, x, t = setting(torch, ff, tr, torch.bfloat16)
    opt, served = tr.AdamW(weights), tr.FourBitFeedForward(block)
    y = block.forward(x).clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        loss = head.forward(y, t)
        dy = head.backward(scale=0.25)
        out = served.forward(x[:1])
        with pytest.raises(ValueError):
            opt.step()
    for i in range(4):
        y.copy_(torch.randn(y.shape, device="cuda"))
        x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        got = [loss.clone(), dy.clone(), out.clone(), head.grads["w"].clone(), head.grads["bias"].clone()]
        want = [head.forward(y, t), head.backward(scale=0.25), served.forward(x[:1]), head.grads["w"], head.grads["bias"]]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    assert opt.steps == 0


def test_another_stream_and_threads():
    torch, ff, tr = _modules()
    import threading
    block, head, weights, x, t = setting(torch, ff, tr, torch.bfloat16)
    y = block.forward(x).clone()
    want = head.forward(y, t).clone(), head.backward().clone()
    side = torch.cuda.Stream()
    head.forward(y, t)
    with torch.cuda.stream(side):
        dy = head.backward()
    side.synchronize()
    assert torch.equal(dy, want[1])
    served, results = tr.FourBitFeedForward(block), {}
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            results[i] = served.forward(x[i:i + 9])
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(6)]
    [a.start() for a in threads]
    [a.join() for a in threads]
    for i in range(6):
        assert torch.equal(results[i], served.forward(x[i:i + 9])), i


def test_example_runs():
    _, _, tr = _modules()
    tr.main(width=128, hidden=512, entries=300, tokens=100, steps=3)
