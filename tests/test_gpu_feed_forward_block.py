"""The feed-forward block (norm, product with GELU, product with residual, and back) on the GPU: against the formulas in 64 bits,
against differences, captured into a graph, on another stream, with tensors beyond 2 GiB."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import feed_forward_oracle as fo


def _modules():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1410_0759_amd import feed_forward
    from tests import feed_forward_util
    return torch, feed_forward, feed_forward_util


def oracle_block(p, x, dy):
    """(y, gradients) in 64 bits, nothing rounded on the way"""
    h, mean, inv = fo.layer_norm(x, p["scale"], p["shift"], 1e-5)
    a, z = fo.linear(h, p["w1"], p["b1"], fo.GELU, None)
    y, _ = fo.linear(a, p["w2"], p["b2"], fo.IDENTITY, x, beta=1.0)
    g = {}
    g["w2"], g["b2"] = fo.linear_backward_filter(dy, a)
    dz = fo.linear_backward_data(dy, p["w2"], fo.GELU, z, None)
    g["w1"], g["b1"] = fo.linear_backward_filter(dz, h)
    dh = fo.linear_backward_data(dz, p["w1"], fo.IDENTITY, None, None)
    dx, g["scale"], g["shift"] = fo.layer_norm_backward(x, dh, p["scale"], mean, inv)
    return y, dx + dy, g


def _filled(torch, block, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    for n in ("b1", "b2", "shift"):
        getattr(block, n).copy_(0.3 * torch.randn(getattr(block, n).shape, generator=g, device="cuda"))
    block.scale.copy_(1 + 0.2 * torch.randn(block.scale.shape, generator=g, device="cuda"))
    return {n: getattr(block, n).double().cpu().numpy() for n in block.grads}, g


# rounded to bfloat16 on the way: h, z, a (forward), a, dz, dh (backward), each off by half a step, 2^-8 of its size; a result sums over at most five such
# roundings with signs that do not agree, its error against the largest of the row of results: below 2^-8 sqrt(5) times a few deviations of the sum
@pytest.mark.parametrize("dtype,tol", [("f32", 2e-5), ("bf16", 3e-2)])
@pytest.mark.parametrize("M,D,H", [(1, 40, 72), (5, 64, 256), (130, 136, 264), (301, 100, 333)])
def test_block_against_the_formulas(dtype, tol, M, D, H):
    torch, ff, u = _modules()
    block = ff.FeedForward(D, H, u.DTYPES[dtype])
    p, g = _filled(torch, block)
    x, dy = (torch.randn(M, D, generator=g, device="cuda").to(block.dtype) for _ in range(2))
    y = block.forward(x).clone()
    dx = block.backward(x, dy).clone()
    wy, wdx, wg = oracle_block(p, x.double().cpu().numpy(), dy.double().cpu().numpy())
    for name, got, want in [("y", y, wy), ("dx", dx, wdx)] + [(n, block.grads[n], wg[n]) for n in wg]:
        got = got.double().cpu().numpy()
        assert np.all(np.isfinite(got)), name
        assert np.abs(got - want).max() <= tol * np.abs(want).max(), (name, np.abs(got - want).max() / np.abs(want).max())
    first = {n: t.clone() for n, t in block.grads.items()}
    block.backward(x, dy, accumulate=True)
    for n, t in block.grads.items():
        assert torch.allclose(t, 2 * first[n], rtol=1e-5, atol=1e-5 * float(first[n].abs().max())), n


def test_block_gradient_against_differences():
    """Float: the derivative of sum(dy * y) along a direction, central differences of the forward pass with a step of 2^-7; its third-order term
    and the rounding of two sums, 2^-24 of the sum of magnitudes over twice the step, are within 1 % of the gradient's size here."""
    torch, ff, u = _modules()
    block = ff.FeedForward(48, 96, torch.float32)
    _, g = _filled(torch, block)
    x, dy = (torch.randn(20, 48, generator=g, device="cuda") for _ in range(2))
    block.forward(x)
    dx = block.backward(x, dy).clone()
    grads = {n: t.clone() for n, t in block.grads.items()}
    loss = lambda: float((block.forward(x).double() * dy.double()).sum())
    for name, t, grad in [("x", x, dx)] + [(n, getattr(block, n), grads[n]) for n in grads]:
        d = torch.randn(t.shape, generator=g, device="cuda") / t.numel() ** 0.5
        keep, step = t.clone(), 2.0 ** -7
        t.copy_(keep + step * d)
        up = loss()
        t.copy_(keep - step * d)
        down = loss()
        t.copy_(keep)
        want = float((grad.double() * d.double()).sum())
        size = float(grad.double().norm()) / t.numel() ** 0.5
        assert abs((up - down) / (2 * step) - want) <= 0.01 * size * 4, (name, (up - down) / (2 * step), want)


def test_block_in_a_graph():
    """Forward and backward captured; replays with new inputs in the same buffers, eager calls and synchronizations between them, give what
    the eager calls give, bit for bit."""
    torch, ff, u = _modules()
    for dtype, M, D, H in ((torch.bfloat16, 200, 136, 520), (torch.float32, 77, 50, 130), (torch.bfloat16, 3, 512, 2048)):
        block = ff.FeedForward(D, H, dtype)
        _, g = _filled(torch, block)
        x, dy = (torch.randn(M, D, generator=g, device="cuda").to(dtype) for _ in range(2))

        def step():
            block.forward(x)
            block.backward(x, dy)

        b = block._use(x)
        results = lambda: [t.clone() for t in [b.y, b.dx] + list(block.grads.values())]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(4):
            x.copy_(torch.randn(M, D, generator=g, device="cuda"))
            dy.copy_(torch.randn(M, D, generator=g, device="cuda"))
            step()
            torch.cuda.synchronize()
            want = results()
            for t in [b.y, b.dx] + list(block.grads.values()):
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(results(), want))


def test_block_on_another_stream():
    torch, ff, u = _modules()
    block = ff.FeedForward(256, 1024)
    _, g = _filled(torch, block)
    x, dy = (torch.randn(300, 256, generator=g, device="cuda").to(block.dtype) for _ in range(2))
    want = block.forward(x).clone(), block.backward(x, dy).clone()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        busy = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            busy = busy @ busy * 0.01
        xs = (x.float() + 0 * busy[0, 0].nan_to_num(0.0, 0.0, 0.0)).to(block.dtype)      # (ready only when that is done)
        got = block.forward(xs).clone(), block.backward(xs, dy).clone()
    stream.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    with pytest.raises(ValueError):
        block.forward(x.float())
    with pytest.raises(ValueError):
        block.forward(x[:, :100])


def test_tensors_beyond_two_gib():
    """Rows so far apart that the last ones lie past 2^32 bytes: the same results as for the rows side by side."""
    torch, ff, u = _modules()
    ig = u.ig
    h = u.handle()
    M, C, K, stride = 1200, 264, 136, 1 << 21
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(M, C, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn(K, C, generator=g, device="cuda").to(torch.bfloat16)
    far = torch.zeros((M - 1) * stride + C, dtype=torch.bfloat16, device="cuda")
    xf = torch.as_strided(far, (M, C), (stride, 1))
    xf.copy_(x)
    assert (M - 1) * stride * 2 > 1 << 32
    desc = lambda t, dt=ig.IGC_DATA_BFLOAT16: ig.TensorDescriptor().set(dt, t.shape[0], t.shape[1], 1, 1, (t.stride(0), 1, 1, 1))
    wd, dwd = u.filter_desc("bf16", K, C), u.filter_desc("f32", K, C)
    y, ws = (torch.empty(M, K, dtype=torch.bfloat16, device="cuda") for _ in range(2)), torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    y = list(y)
    n = [torch.empty(M, C, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dw, db = [torch.empty(K, C, device="cuda") for _ in range(2)], [torch.empty(K, device="cuda") for _ in range(2)]
    for i, t in enumerate((x, xf)):
        ig.check(ig.linear_forward(h, 1.0, desc(t), t.data_ptr(), wd, w.data_ptr(), ws.data_ptr(), ws.numel(), 0, -1, 0.0, None, 0, desc(y[i]), 0, y[i].data_ptr()))
        ig.check(ig.layer_norm_forward(h, 1.0, desc(t), t.data_ptr(), 0, 0, 1e-5, 0.0, desc(n[i]), n[i].data_ptr()))
        ig.check(ig.linear_backward_filter(h, 1.0, desc(t), t.data_ptr(), desc(y[0]), y[0].data_ptr(), ws.data_ptr(), ws.numel(), 0.0, dwd, dw[i].data_ptr(),
                                           db[i].data_ptr()))
    assert torch.equal(*y) and torch.equal(*n) and torch.equal(*dw) and torch.equal(*db)
    # written there: dx of the norm and the product back to x
    dxf, dx = torch.as_strided(far, (M, C), (stride, 1)), torch.empty(M, C, dtype=torch.bfloat16, device="cuda")
    for t in (dx, dxf):
        ig.check(ig.linear_backward_data(h, 1.0, wd, w.data_ptr(), desc(y[0]), y[0].data_ptr(), ws.data_ptr(), ws.numel(), -1, None, 0, 0.0, None, 0, desc(t),
                                         t.data_ptr()))
    assert torch.equal(dx, dxf)


def test_example_runs(capsys):
    torch, ff, u = _modules()
    ff.main(width=128, hidden=512, tokens=200, steps=6)
    lines = capsys.readouterr().out.strip().splitlines()
    first, last = float(lines[0].split()[-1]), float(lines[-2].split()[-1])
    assert last < first and float(lines[-1].split()[-1]) < 0.1
