"""The optimiser's step on the GPU against its formula in 64 bits.

Tolerances: e = 2^-24, half a step of fp32.  m: at most four roundings (v: six) of numbers no larger than the two terms.  The update: m and v as above, the
constants (a rounding each), a root, a quotient, two products: 16 e of it and what m's and v's own errors make of it; the parameter's product and
difference 4 e of their terms; then half a step of the parameter's type.  Codes: the formula's, or those that the number 8 e to either side has."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import adamw_oracle as ao

E = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
RATE, B1, B2, EPS = 1e-3, 0.9, 0.99, 1e-8


def _u():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from tests import adamw_util
    return adamw_util


def parameters(**more):
    import paper_1410_0759_amd as ig
    return ig.AdamWParameters(**{**dict(learning_rate=RATE, beta1=B1, beta2=B2, epsilon=EPS, gradient_scale=0.5, step=7, seed=99), **more})


def handle():
    import torch
    import paper_1410_0759_amd as ig
    h = ig.Handle()
    h.set_stream(torch.cuda.current_stream().cuda_stream)
    return h


def near(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        i = int(np.argmax(bad))
        raise AssertionError("%s: %d of %d off; [%d] %.9g instead of %.9g, allowed %.3g" % (what, bad.sum(), bad.size, i, got[i], want[i], tol[i]))


def check_codes(code, scale, x, form, random, what):
    """code, scale: of the numbers x (known to 4 e)."""
    want = ao.scales(x, form)
    near(scale, want, 8 * E * want, what + " scale")
    s = np.repeat(scale, 256)[:len(x)]
    y = np.divide(x, s, out=np.zeros(len(x)), where=s > 0)
    lo, hi = (ao.rounded(y * (1 + d), form, random) for d in (-8 * E, 8 * E))
    ok = (code >= np.minimum(lo, hi)) & (code <= np.maximum(lo, hi))
    assert ok.all(), (what, int((~ok).sum()), int(np.argmin(ok)), code[~ok][:3], y[~ok][:3])


def run(tensors, t=7, rate=RATE, scale=0.5, seed=99, **more):
    """One step; all results against the formula."""
    u = _u()
    import paper_1410_0759_amd as ig
    before = [(x.p.numpy(), x.g.numpy(), *x.states()) for x in tensors]
    ig.check(ig.adamw_step(handle(), parameters(**{**dict(step=t, seed=seed, learning_rate=rate, gradient_scale=scale), **more}), u.table(tensors)), "igcAdamWStep")
    for i, (x, (p, g, m, v)) in enumerate(zip(tensors, before)):
        check(x, p, g, m, v, "tensor %d of %d" % (i, x.n), t, rate, scale, seed)


def check(x, p, g, m, v, what, t=7, rate=RATE, scale=0.5, seed=99, first=0):
    """first: the place of x in its tensor."""
    wp, wm, wv = ao.step(p, g, m, v, t, rate, B1, B2, EPS, x.decay, scale)
    tm, tv = 4 * E * (np.abs(B1 * m) + np.abs((1 - B1) * scale * g)), 6 * E * (B2 * v + (1 - B2) * (scale * g) ** 2)
    c1, c2 = 1 / (1 - B1 ** t), 1 / (1 - B2 ** t)
    root = np.sqrt(wv * c2) + EPS
    near_root = np.divide(tv * c2, np.sqrt(wv * c2) * 2, out=np.zeros(x.n), where=wv > 0)
    tu = rate * c1 / root * (tm + np.abs(wm) * (16 * E + 1.01 * near_root / root))
    half = HALF["f32" if x.p.dtype.itemsize == 4 else "bf16"]
    tp = tu + 4 * E * (np.abs(p) + np.abs(wp))
    got = x.p.numpy()
    near(got, wp, tp + half * (np.abs(wp) + tp), what + " p")
    if x.copy is not None:
        import torch
        assert np.array_equal(x.copy.numpy(), torch.from_numpy(got).to(torch.bfloat16).double().numpy()), what + " copy"
    assert np.array_equal(x.g.numpy(), g)
    if x.bits == 32:
        near(x.m.numpy(), wm, tm, what + " m")
        near(x.v.numpy(), wv, tv, what + " v")
    elif x.n:
        rm, rv = ao.random_bits(x.n, seed, t, first)
        check_codes(x.m.numpy(), x.ms.numpy(), wm, ao.E4M3, rm, what + " m")
        check_codes(x.v.numpy(), x.vs.numpy(), wv, ao.E5M2, rv, what + " v")


SIZES = [1, 3, 255, 256, 257, 1000, 1024, 4095, 4096, 4097, 20011]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("param", ["f32", "bf16"])
def test_types_and_sizes(param, grad, bits):
    u = _u()
    rng = np.random.default_rng(len(param) * 100 + len(grad) * 10 + bits)
    for lead in (0, 1, 5):
        print("adamw", param, grad, bits, lead, flush=True)
        run([u.Tensor(rng, n, param, grad, bits, copy=param == "f32" and n % 2 == 1, decay=0.1 * (n % 3), lead=lead) for n in SIZES])


def test_many_tensors_of_all_kinds():
    """Over several launches, tensors without elements among them."""
    u = _u()
    rng = np.random.default_rng(5)
    kinds = [(p, g, b) for p in ("f32", "bf16") for g in ("f32", "bf16") for b in (32, 8)]
    tensors = []
    for i in range(131):
        param, grad, bits = kinds[i % 8]
        n = 0 if i % 13 == 4 else int(rng.integers(1, 9000 if i % 10 == 0 else 600))
        tensors.append(u.Tensor(rng, n, param, grad, bits, copy=param == "f32", lead=i % 7))
    run(tensors)
    run([u.Tensor(rng, 0), u.Tensor(rng, 0, bits=8)])
    import paper_1410_0759_amd as ig
    assert ig.adamw_step(handle(), parameters(), u.table([])) == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_and_tensors_without_gradient(bits):
    u = _u()
    rng = np.random.default_rng(6)
    a, b = u.Tensor(rng, 3000, bits=bits, fresh=True), u.Tensor(rng, 700, bits=bits, fresh=True)
    b.g.bytes.zero_()
    run([a, b], t=1)
    assert not b.m.numpy().any() and not b.v.numpy().any()
    run([a, b], t=2)


def test_large_tensor_and_small_numbers():
    """Over four million elements; blocks of gradients from 1e-36 to 1e15, squares below every float among them."""
    u = _u()
    rng = np.random.default_rng(7)
    for bits in (32, 8):
        run([u.Tensor(rng, 300, bits=bits), u.Tensor(rng, (1 << 22) + 77, bits=bits, lead=3)])
    x = u.Tensor(rng, 256 * 40, bits=8, fresh=True)
    x.g.put(rng.standard_normal(x.n) * np.repeat(10.0 ** rng.uniform(-36, 15, 40), 256), x.g.dtype)
    import paper_1410_0759_amd as ig
    g = x.g.numpy()
    ig.check(ig.adamw_step(handle(), parameters(step=1, gradient_scale=1.0), u.table([x])))
    m = ((1 - B1) * g)
    rm, _ = ao.random_bits(x.n, 99, 1)
    check_codes(x.m.numpy(), x.ms.numpy(), m, ao.E4M3, rm, "m")
    assert np.isfinite(x.p.numpy()).all() and np.isfinite(x.v.numpy()).all()
    used = np.repeat(x.vs.numpy() > 0, 256) & (np.abs(g) > 1e-15)
    assert (x.v.numpy()[used] > 0).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_squares_below_the_normal_numbers(bits):
    """A first step with gradients around 1e-19 and an epsilon below their roots: steps of the rate, whatever the gradient.  (A hundredth of the square has 16 bits left at 1e-19:
    its root is known to 2^-16.)"""
    u = _u()
    import paper_1410_0759_amd as ig
    rng = np.random.default_rng(13)
    x = u.Tensor(rng, 1000, bits=bits, fresh=True, decay=0.0)
    x.g.put(np.copysign(1e-19 * (1 + rng.random(1000)), rng.standard_normal(1000)), x.g.dtype)
    p, g = x.p.numpy(), x.g.numpy()
    ig.check(ig.adamw_step(handle(), parameters(step=1, gradient_scale=1.0, epsilon=1e-30, learning_rate=0.25), u.table([x])))
    near(x.p.numpy(), p - 0.25 * np.sign(g), 0.25 * 2.0 ** -15 + 4 * E * (np.abs(p) + 0.25), "p")


def test_infinite_and_undefined_gradients_stay_where_they_are():
    u = _u()
    rng = np.random.default_rng(8)
    for bits in (32, 8):
        x, y = u.Tensor(rng, 1000, bits=bits), None
        g = x.g.numpy()
        places = [3, 300, 301, 999]
        g[places] = [np.inf, np.nan, -np.inf, np.nan]
        x.g.put(g, x.g.dtype)
        p, (m, v) = x.p.numpy(), x.states()
        import paper_1410_0759_amd as ig
        ig.check(ig.adamw_step(handle(), parameters(), u.table([x])))
        rest = np.ones(1000, bool)
        rest[places] = False
        wp, wm, wv = ao.step(p, g, m, v, 7, RATE, B1, B2, EPS, x.decay, 0.5)
        got = x.p.numpy()
        assert not np.isfinite(got[places]).any() and np.isfinite(got[rest]).all()
        assert np.abs(got[rest] - wp[rest]).max() < 1e-5
        gm, gv = x.states()
        assert np.isfinite(gm[rest]).all() and np.isfinite(gv[rest]).all() and not np.isfinite(gm[places]).any() and not np.isfinite(gv[places]).any()
        if bits == 8:
            rm, rv = ao.random_bits(1000, 99, 7)
            for code, scale, w, form, r in ((x.m.numpy(), x.ms.numpy(), wm, ao.E4M3, rm), (x.v.numpy(), x.vs.numpy(), wv, ao.E5M2, rv)):
                w = np.where(rest, w, 0.0)
                check_codes(np.where(rest, code, 0.0), scale, w, form, r, "codes")


def test_same_bits_again():
    u = _u()
    import paper_1410_0759_amd as ig
    results = []
    for _ in range(2):
        rng = np.random.default_rng(9)
        tensors = [u.Tensor(rng, n, bits=b, copy=True) for n in (5000, 77) for b in (8, 32)]
        ig.check(ig.adamw_step(handle(), parameters(), u.table(tensors)))
        results.append([a.bytes.cpu().numpy().copy() for x in tensors for a in x.arrays()])
    assert all(np.array_equal(a, b) for a, b in zip(*results))


def test_states_in_8_bits_keep_their_averages():
    """A thousand steps of beta2 0.99 with gradients whose size rises fivefold after the first: v and m, averaged over 65536 elements of a kind, follow the
    formula.  An element's code is off by less than a quarter of itself at random (uniform at worst: a variance of 1/4 x 1/4 over the 100 steps that an average
    remembers, at most 100 x the variance of one); the mean over 65536 of them by 0.25 x 10 / 256 = 1 % at one deviation: 5 % allowed."""
    u = _u()
    import torch
    import paper_1410_0759_amd as ig
    rng = np.random.default_rng(10)
    n = 1 << 16
    x = u.Tensor(rng, n, bits=8, fresh=True, decay=0.0)
    base = np.abs(rng.standard_normal(n)) * 0.1 + 1.0
    t, h, tab = 0, handle(), u.table([x])
    m = v = np.zeros(n)
    for g, steps in ((base, 200), (5 * base, 400), (base, 400)):
        x.g.put(g, x.g.dtype)
        gs = x.g.numpy()
        for _ in range(steps):
            t += 1
            ig.check(ig.adamw_step(h, parameters(step=t, gradient_scale=1.0), tab))
            m, v = B1 * m + (1 - B1) * gs, B2 * v + (1 - B2) * gs * gs
        gm, gv = x.states()
        assert abs(gm.mean() / m.mean() - 1) < 0.05 and abs(gv.mean() / v.mean() - 1) < 0.05, (t, gm.mean() / m.mean(), gv.mean() / v.mean())


def test_rate_scale_and_step_on_the_device_and_in_a_graph():
    """Replays of one captured step, the step's number and the rate changed between them, as eager steps with these numbers."""
    u = _u()
    import torch
    import paper_1410_0759_amd as ig
    make = lambda: [u.Tensor(np.random.default_rng(11), n, bits=b, copy=True) for n in (5001, 300) for b in (8, 32)]
    a, b = make(), make()
    rate, scale, step = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = parameters(learning_rate=0.0, step=0, gradient_scale=0.5, device_learning_rate=rate.data_ptr(), device_gradient_scale=scale.data_ptr(), device_step=step.data_ptr())
    tab = u.table(a)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        h = handle()
        ig.check(ig.adamw_step(h, q, tab))
    for t, r, s in ((1, 1e-3, 1.0), (2, 5e-4, 0.25), (3, 1e-4, 2.0), (1000, 1e-2, 1.0)):
        rate.fill_(r)
        scale.fill_(s)
        step.fill_(t)
        graph.replay()
        ig.check(ig.adamw_step(handle(), parameters(learning_rate=float(np.float32(r)), step=t, gradient_scale=0.5 * s), u.table(b)))
        for x, y in zip(a, b):
            for c, d in zip(x.arrays(), y.arrays()):
                assert np.array_equal(c.bytes.cpu().numpy(), d.bytes.cpu().numpy()), t


def test_on_another_stream():
    u = _u()
    import torch
    import paper_1410_0759_amd as ig
    side = torch.cuda.Stream()
    x = u.Tensor(np.random.default_rng(12), 70001, bits=8)
    before = (x.p.numpy(), x.g.numpy(), *x.states())
    side.wait_stream(torch.cuda.current_stream())
    h = ig.Handle()
    h.set_stream(side.cuda_stream)
    ig.check(ig.adamw_step(h, parameters(), u.table([x])))
    side.synchronize()
    check(x, *before, "on another stream")


def test_steps_below_one_on_the_device():
    """A step on the device below 1 counts as 1, for what is rounded too."""
    u = _u()
    import torch
    import paper_1410_0759_amd as ig
    a, b = (u.Tensor(np.random.default_rng(14), 3000, bits=8, fresh=True) for _ in range(2))
    step = torch.full((1,), -3, dtype=torch.int32, device="cuda")
    ig.check(ig.adamw_step(handle(), parameters(step=0, device_step=step.data_ptr()), u.table([a])))
    ig.check(ig.adamw_step(handle(), parameters(step=1), u.table([b])))
    for x, y in zip(a.arrays(), b.arrays()):
        assert np.array_equal(x.bytes.cpu().numpy(), y.bytes.cpu().numpy())


def test_more_elements_than_32_bits_count():
    """Both ends of a tensor of 2^32 + 70001 elements with a copy and states in 8 bits; what lies between has no gradient and stays."""
    u = _u()
    import torch
    import paper_1410_0759_amd as ig
    n, far, part = 2 ** 32 + 70001, 2 ** 32, 70001
    rng = np.random.default_rng(15)
    small = [u.Tensor(rng, part, grad="bf16", bits=8, copy=True) for _ in range(2)]
    zeros = lambda count, dtype: torch.zeros(count, dtype=torch.uint8 if dtype.itemsize == 1 else dtype, device="cuda").view(dtype)
    blocks = -(-n // 256)
    arrays = dict(p=zeros(n, torch.float32), g=zeros(n, torch.bfloat16), copy=zeros(n, torch.bfloat16), m=zeros(n, torch.float8_e4m3fn), v=zeros(n, torch.float8_e5m2),
                  ms=zeros(blocks, torch.float32), vs=zeros(blocks, torch.float32))
    for x, at in zip(small, (0, far)):
        for name, a in arrays.items():
            from_ = at // 256 if name in ("ms", "vs") else at
            a.view(torch.uint8)[from_ * a.element_size():][:getattr(x, name).bytes.numel()] = getattr(x, name).bytes
    table = (ig.AdamWTensor * 1)()
    q = table[0]
    q.param, q.grad, q.copy, q.m, q.v, q.m_scale, q.v_scale = (arrays[k].data_ptr() for k in ("p", "g", "copy", "m", "v", "ms", "vs"))
    q.count, q.weight_decay, q.param_type, q.grad_type, q.state_bits = n, 0.1, ig.IGC_DATA_FLOAT, ig.IGC_DATA_BFLOAT16, 8
    before = [(x.p.numpy(), x.g.numpy(), *x.states()) for x in small]
    ig.check(ig.adamw_step(handle(), parameters(), table))
    for x, at, old in zip(small, (0, far), before):
        for name, a in arrays.items():
            from_ = at // 256 if name in ("ms", "vs") else at
            getattr(x, name).bytes.copy_(a.view(torch.uint8)[from_ * a.element_size():][:getattr(x, name).bytes.numel()])
        check(x, *old, "at %d" % at, first=at)
    for name, a in arrays.items():
        begin, end = (part // 256 + 1, far // 256) if name in ("ms", "vs") else ((part // 256 + 1) * 256, far)
        assert not bool(a.view(torch.uint8)[begin * a.element_size():end * a.element_size()].any()), name
    del arrays, a
    torch.cuda.empty_cache()
