"""Operators around a feed-forward block as a training or serving program calls them: the loss over a vocabulary and its gradient, the optimiser's
step, and products with weights of four bits.

A case is one call (`four_bits_store`: two).  Kinds:
  loss             rows of features to cross entropies over V entries: z = x w^T + bias, log_sum = log sum_v exp z, loss = log_sum - z[target]; 0 for a
                   row without a target (a target outside 0..V-1)
  loss_gradient    dz = dloss (exp(z - log_sum) - [v is the target]), 0 for rows without one; dx = dz w, dw = dz^T x, dbias = column sums of dz
  adamw            m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2, p = p (1 - rate decay) - rate (m c1) / (sqrt(v c2) + eps), g: gradient times a scale,
                   c: 1 / (1 - b^step); bfloat16 copies of the matrices with it.  The matrices' m and v in floats, or in 8 bits: e4m3 and e5m2 in units of a
                   scale per 256 elements, rounded up or down at random by a counter's hash
  four_bits_store  a filter into four bits (e2m1) with a scale for each group of a row's features, and back
  four_bits        y = f(x w^T + bias) + r with such a filter
Sizes: M rows, C features in, V entries or K features out; `pad` elements between the rows of every matrix.  `dtype`: of x and w; `out`: of y.  An
optimiser's tensors are those of `layers` feed-forward blocks of `width` and `hidden`: two matrices, their biases, a norm's scale and shift.
"""
import math
import random

import torch

own = False

_T = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
RATE, BETA1, BETA2, EPSILON, DECAY, STEP, SCALE, SEED = 3e-5, 0.9, 0.999, 1e-8, 0.1, 1000, 0.75, 12345
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BORDERS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)
UP_AT = (1, 3, 5)    # a number on these borders has the even code above it


def _loss(name, kind, dtype, M, C, V, pad=0, bias=False):
    c = {"kind": kind, "dtype": dtype, "M": M, "C": C, "V": V, "pad": pad, "bias": bias}
    return dict(c, name=name) if name else c


def _adamw(name, layers, width, hidden, bits, grad):
    c = {"kind": "adamw", "layers": layers, "width": width, "hidden": hidden, "bits": bits, "grad": grad}
    return dict(c, name=name) if name else c


def _four(name, kind, dtype, out, M, C, K, group, act="none", pad=0, residual=False):
    c = {"kind": kind, "dtype": dtype, "C": C, "K": K, "group": group}
    if kind == "four_bits":
        c.update({"out": out, "M": M, "act": act, "pad": pad, "residual": residual})
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: how likely the next tokens of four sequences were
        _loss("loss_4_tokens", "loss", "bf16", 4, 4096, 32768),
        # training, the largest: a batch of tokens over a large vocabulary
        _loss("loss_batch", "loss", "bf16", 8192, 4096, 131072),
        # a float classifier with a bias on a ragged batch, rows of a wider buffer, nothing divides
        _loss("loss_odd_float", "loss", "f32", 1023, 1001, 5003, pad=3, bias=True),
        # training: the gradient of such a batch
        _loss("loss_back_batch", "loss_gradient", "bf16", 4096, 4096, 65536),
        # the last, short batch of an odd vocabulary with a bias
        _loss("loss_back_odd", "loss_gradient", "bf16", 777, 1000, 10007, pad=8, bias=True),
        # a small model's step: forty-eight tensors, most of them tiny: the latency of a call
        _adamw("adamw_small", 8, 128, 512, 32, "f32"),
        # a large model's step on float gradients
        _adamw("adamw_large", 4, 4096, 16384, 32, "f32"),
        # the same with the matrices' states in 8 bits and gradients in 16; odd widths, so that most tensors lie on odd places
        _adamw("adamw_8_bits", 3, 4001, 16001, 8, "bf16"),
        # making a served model: a block's first filter into four bits
        _four("four_bits_store", "four_bits_store", "bf16", "", 0, 4096, 16384, 128),
        # serving: one token through a block's first product
        _four("four_bits_1_token", "four_bits", "bf16", "bf16", 1, 4096, 16384, 128, act="gelu"),
        # serving: a ragged batch of sequences, one token each, a float model's odd second product with the residual
        _four("four_bits_odd", "four_bits", "f32", "f32", 37, 5001, 2003, 32, pad=1, residual=True),
        # a prompt
        _four("four_bits_prompt", "four_bits", "bf16", "bf16", 2048, 4096, 8192, 64, act="gelu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A number of features: a multiple of 64, of 8, or any."""
    n = _log(rng, lo, hi)
    step = rng.choice((1, 8, 64, 64))
    return max(lo, n // step * step)


def draw(rng):
    kind = rng.choice(("loss", "loss", "loss_gradient", "loss_gradient", "adamw", "adamw", "four_bits_store", "four_bits", "four_bits", "four_bits"))
    pad = rng.choice((0, 0, 1, 8))
    if kind.startswith("loss"):
        dtype = rng.choice(("bf16", "bf16", "f32"))
        C, V = _width(rng, 64, 8192), _width(rng, 100, 131072)
        most = 1 << (36 if dtype == "f32" else 39)
        while 64 * C * V > most:
            C //= 2
        M = _log(rng, 1, min(8192, max(64, most // (C * V) // (3 if kind == "loss_gradient" else 1)), (1 << 30) // V))
        return _loss(None, kind, dtype, M, C, V, pad, rng.random() < 0.5)
    if kind == "adamw":
        width, hidden = _width(rng, 16, 4096), _width(rng, 16, 16384)
        return _adamw(None, _log(rng, 1, max(1, min(32, (1 << 28) // (width * hidden)))), width, hidden, rng.choice((8, 8, 32)), rng.choice(("f32", "bf16")))
    group, dtype = rng.choice((32, 64, 128)), rng.choice(("bf16", "bf16", "f32"))
    C, K = _width(rng, 64, 16384), _width(rng, 64, 16384)
    while C * K > 4096 * 16384:
        C, K = max(64, C // 2), max(64, K // 2)
    if kind == "four_bits_store":
        return _four(None, kind, dtype, "", 0, C, K, group)
    M = _log(rng, 1, rng.choice((16, 256, 4096)))
    return _four(None, kind, dtype, "f32" if dtype == "f32" else rng.choice(("bf16", "bf16", "f32")), M, C, K, group,
                 rng.choice(("none", "relu", "gelu", "silu")), pad, rng.random() < 0.5)


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _matrix(rows, cols, dtype, pad, fill):
    """rows x cols of `fill`, rounded to dtype, in rows cols + pad apart."""
    wide = torch.zeros(rows, cols + pad, dtype=_T[dtype], device="cuda")
    wide[:, :cols] = fill.to(_T[dtype])
    return wide[:, :cols]


def _loss_inputs(case, g):
    M, C, V = case["M"], case["C"], case["V"]
    # features after a norm, drawn towards their target's row as a trained model's are: some of the targets are likely, others not
    w = _matrix(V, C, case["dtype"], 0, torch.randn(V, C, generator=g, device="cuda") * (2.0 / math.sqrt(C)))
    target = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn(M, C, generator=g, device="cuda") + (3 * torch.rand(M, 1, generator=g, device="cuda")) * w[target.long()].float()
    a = {"x": _matrix(M, C, case["dtype"], case["pad"], x), "w": w}
    # padding and prompts have no target
    a["target"] = torch.where(torch.rand(M, generator=g, device="cuda") < 0.1, torch.full_like(target, -100), target)
    if case["bias"]:
        a["bias"] = torch.randn(V, generator=g, device="cuda")
    if case["kind"] == "loss_gradient":
        # an average over the rows, each with a weight of its own; the logarithms of the sums as a forward pass leaves them
        a["dloss"] = (0.5 + torch.rand(M, generator=g, device="cuda")) / M
        parts = [torch.logsumexp(xs.double() @ a["w"].double().t() + a["bias"].double() if case["bias"] else xs.double() @ a["w"].double().t(), 1)
                 for xs in a["x"].split(max(1, (1 << 28) // V))]
        a["log_sum"] = torch.cat(parts).float()
    return a


def _shapes(case):
    """[(size, whether a matrix)] of the optimiser's tensors."""
    D, H = case["width"], case["hidden"]
    return [(H * D, True), (H, False), (D * H, True), (D, False), (D, False), (D, False)] * case["layers"]


def _blocks(n):
    return (n + 255) // 256


def _to_blocks(t, fill=0.0):
    """One tensor's elements in rows of 256."""
    n = t.numel()
    return torch.nn.functional.pad(t, (0, _blocks(n) * 256 - n), value=fill).view(-1, 256)


def _adamw_inputs(case, g):
    shapes = _shapes(case)
    n, nm = sum(s for s, _ in shapes), sum(s for s, mat in shapes if mat)

    def flat(size, dtype=torch.float32):
        return torch.empty(size, dtype=dtype, device="cuda")

    # all tensors of a kind lie behind each other in one buffer
    a = {"p": flat(n), "g": flat(n, _T[case["grad"]]), "copy": flat(nm, torch.bfloat16), "m": flat(n if case["bits"] == 32 else n - nm)}
    a["v"] = flat(a["m"].numel())
    if case["bits"] == 8:
        nb = sum(_blocks(s) for s, mat in shapes if mat)
        a.update({"m8": flat(nm, torch.float8_e4m3fn), "v8": flat(nm, torch.float8_e5m2), "m_scale": flat(nb), "v_scale": flat(nb)})
    at = {k: 0 for k in a}
    views = []

    def take(name, size):
        at[name] += size
        return a[name][at[name] - size:at[name]]

    for size, mat in shapes:
        # gradients of very different size from place to place; the states of many steps of such gradients
        spread = torch.exp(1.5 * torch.randn(size, generator=g, device="cuda")) * 1e-4
        t = {"p": take("p", size), "g": take("g", size), "decay": DECAY if mat else 0.0}
        t["p"].normal_(0 if mat else 0.5, 0.02 if mat else 0.1, generator=g)
        t["g"].copy_(torch.randn(size, generator=g, device="cuda") * spread)
        m, v = 0.3 * torch.randn(size, generator=g, device="cuda") * spread, spread.square() * (0.5 + torch.rand(size, generator=g, device="cuda"))
        if mat:
            t["copy"] = take("copy", size)
            t["copy"].copy_(t["p"])
        if mat and case["bits"] == 8:
            t.update({"m8": take("m8", size), "v8": take("v8", size), "m_scale": take("m_scale", _blocks(size)), "v_scale": take("v_scale", _blocks(size))})
            for q, s, most, code in ((m, "m_scale", 448.0, "m8"), (v, "v_scale", 57344.0, "v8")):
                rows = _to_blocks(q)
                t[s].copy_(rows.abs().amax(1) / most)
                t[code].copy_((rows / t[s][:, None]).clamp(-most, most).to(t[code].dtype).view(-1)[:size])
        else:
            t["m"], t["v"] = take("m", size), take("v", size)
            t["m"].copy_(m)
            t["v"].copy_(v)
        views.append(t)
    return dict(a, tensors=views)


def _to_codes(w, group):
    """e2m1 codes (K x C) and bfloat16 scales (groups x K) of a filter: the smallest bfloat16 that lets the group's largest be 6, the nearest code."""
    K, C = w.shape
    groups = -(-C // group)
    rows = torch.nn.functional.pad(w.double(), (0, groups * group - C)).view(K, groups, group)
    want = rows.abs().amax(2) / 6
    near = want.to(torch.float32).to(torch.bfloat16)
    above = (near.view(torch.int16) + 1).view(torch.bfloat16)
    scale = torch.where(near.double() < want, above, near)
    at = torch.tensor(BORDERS, dtype=torch.float64, device=w.device)
    edges = scale.double()[:, :, None] * at
    size = rows.abs()
    code = torch.zeros_like(rows, dtype=torch.uint8)
    code = sum(((size >= edges[:, :, i, None]) if i in UP_AT else (size > edges[:, :, i, None])).to(torch.uint8) for i in range(7))
    code = torch.where((scale == 0)[:, :, None], torch.zeros_like(code), code) | ((rows < 0) & (code > 0)).to(torch.uint8) * 8
    return code.view(K, groups * group)[:, :C].contiguous(), scale.t().contiguous()


def _pack(code):
    """K x C codes as the library keeps them: blocks of 128 features in 64 bytes; word 4 g + i of a block holds features 32 i + 8 g to 32 i + 8 g + 7."""
    K, C = code.shape
    blocks = -(-C // 128)
    c = torch.nn.functional.pad(code, (0, blocks * 128 - C)).view(K, blocks, 4, 4, 4, 2).permute(0, 1, 3, 2, 4, 5)
    return (c[..., 0] | c[..., 1] << 4).reshape(K, blocks * 64).contiguous()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["kind"].startswith("loss"):
        return _loss_inputs(case, g)
    if case["kind"] == "adamw":
        return _adamw_inputs(case, g)
    K, C, dtype = case["K"], case["C"], case["dtype"]
    # rows of different size, a few features far larger than the rest
    w = torch.randn(K, C, generator=g, device="cuda") * (0.5 + torch.rand(K, 1, generator=g, device="cuda")) / math.sqrt(C)
    w = torch.where(torch.rand(C, generator=g, device="cuda") < 0.005, 4 * w, w).to(_T[dtype])
    if case["kind"] == "four_bits_store":
        return {"w": w}
    code, scale = _to_codes(w, case["group"])
    M, pad, out = case["M"], case["pad"], case["out"]
    a = {"x": _matrix(M, C, dtype, pad, torch.randn(M, C, generator=g, device="cuda") + 0.1), "codes": _pack(code), "scales": scale,
         "bias": 0.5 * torch.randn(K, generator=g, device="cuda")}
    if case["residual"]:
        a["r"] = _matrix(M, K, out, pad, torch.randn(M, K, generator=g, device="cuda"))
    return a


def prepare(case, seed):
    a = _inputs(case, seed)
    return {"case": case, "a": a, "plan": _plan(case, a) if own else None}


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _plan(case, a):
    """Handle, descriptors, output buffers and workspace, as a program makes them once for a layer."""
    import paper_1410_0759_amd as ig
    DT = {torch.float32: ig.IGC_DATA_FLOAT, torch.bfloat16: ig.IGC_DATA_BFLOAT16}
    p = {"ig": ig, "handle": ig.Handle()}
    hd = p["handle"]
    hd.set_stream(torch.cuda.current_stream().cuda_stream)

    def desc(t):
        return ig.TensorDescriptor().set(DT[t.dtype], t.shape[0], t.shape[1], 1, 1, (t.stride(0), 1, 1, 1))

    def fresh(rows, cols, dtype):
        return torch.empty(rows, cols + case["pad"], dtype=_T[dtype], device="cuda")[:, :cols]

    kind, size = case["kind"], 0
    if kind.startswith("loss"):
        M, C, V, dtype = case["M"], case["C"], case["V"], case["dtype"]
        p["xdesc"], p["wdesc"] = desc(a["x"]), ig.FilterDescriptor().set(DT[_T[dtype]], V, C, 1, 1)
        if kind == "loss":
            p["loss"], p["log_sum"] = (torch.empty(M, device="cuda") for _ in range(2))
            size = ig.get_linear_cross_entropy_forward_workspace_size(hd, p["xdesc"], p["wdesc"])
        else:
            p["dx"], p["dw"] = fresh(M, C, dtype), torch.empty(V, C, dtype=_T[dtype], device="cuda")
            p["dbias"] = torch.empty(V, device="cuda") if case["bias"] else None
            p["dxdesc"] = desc(p["dx"])
            size = ig.get_linear_cross_entropy_backward_workspace_size(hd, p["xdesc"], p["wdesc"], p["dxdesc"], p["wdesc"])
    elif kind == "adamw":
        p["parameters"] = ig.AdamWParameters(learning_rate=RATE, beta1=BETA1, beta2=BETA2, epsilon=EPSILON, gradient_scale=SCALE, step=STEP, seed=SEED)
        p["tensors"] = (ig.AdamWTensor * len(a["tensors"]))()
        for q, t in zip(p["tensors"], a["tensors"]):
            q.param, q.param_type, q.grad, q.grad_type = t["p"].data_ptr(), ig.IGC_DATA_FLOAT, t["g"].data_ptr(), DT[t["g"].dtype]
            q.count, q.weight_decay, q.copy = t["p"].numel(), t["decay"], _ptr(t.get("copy"))
            q.state_bits = 8 if "m8" in t else 32
            q.m, q.v = (t["m8"].data_ptr(), t["v8"].data_ptr()) if "m8" in t else (t["m"].data_ptr(), t["v"].data_ptr())
            q.m_scale, q.v_scale = _ptr(t.get("m_scale")), _ptr(t.get("v_scale"))
    else:
        p["wdesc"] = ig.FilterDescriptor().set(DT[_T[case["dtype"]]], case["K"], case["C"], 1, 1)
        if kind == "four_bits_store":
            code_bytes, scale_bytes = ig.get_filter4_size(p["wdesc"], case["group"])
            p["codes"], p["scales"] = (torch.empty(b, dtype=torch.uint8, device="cuda") for b in (code_bytes, scale_bytes))
            p["back"] = torch.empty(case["K"], case["C"], device="cuda")
            p["backdesc"] = ig.FilterDescriptor().set(ig.IGC_DATA_FLOAT, case["K"], case["C"], 1, 1)
        else:
            p["xdesc"], p["y"] = desc(a["x"]), fresh(case["M"], case["K"], case["out"])
            p["ydesc"], p["rdesc"] = desc(p["y"]), desc(a["r"]) if "r" in a else None
            size = ig.get_linear4_forward_workspace_size(hd, p["xdesc"], p["wdesc"], case["group"], p["ydesc"])
            p["act"] = {"none": ig.IGC_ACTIVATION_IDENTITY, "relu": ig.IGC_ACTIVATION_RELU, "gelu": ig.IGC_ACTIVATION_GELU, "silu": ig.IGC_ACTIVATION_SILU}[case["act"]]
    p["ws"] = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    p["ws_bytes"] = size
    return p


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _run_own(state):
    case, a, p = state["case"], state["a"], state["plan"]
    ig, hd, kind = p["ig"], p["handle"], case["kind"]
    if kind == "loss":
        ig.check(ig.linear_cross_entropy_forward(hd, p["xdesc"], _ptr(a["x"]), p["wdesc"], _ptr(a["w"]), _ptr(a.get("bias")), _ptr(a["target"]), _ptr(p["ws"]), p["ws_bytes"],
                                                 _ptr(p["loss"]), _ptr(p["log_sum"])), "igcLinearCrossEntropyForward")
        return {"loss": p["loss"], "log_sum": p["log_sum"]}
    if kind == "loss_gradient":
        ig.check(ig.linear_cross_entropy_backward(hd, 1.0, p["xdesc"], _ptr(a["x"]), p["wdesc"], _ptr(a["w"]), _ptr(a.get("bias")), _ptr(a["target"]), _ptr(a["log_sum"]),
                                                  _ptr(a["dloss"]), _ptr(p["ws"]), p["ws_bytes"], 0.0, p["dxdesc"], _ptr(p["dx"]), 0.0, p["wdesc"], _ptr(p["dw"]),
                                                  _ptr(p["dbias"])), "igcLinearCrossEntropyBackward")
        return {"dx": p["dx"], "dw": p["dw"], "dbias": p["dbias"]} if case["bias"] else {"dx": p["dx"], "dw": p["dw"]}
    if kind == "adamw":
        ig.check(ig.adamw_step(hd, p["parameters"], p["tensors"]), "igcAdamWStep")
        return _adamw_results(a)
    if kind == "four_bits_store":
        ig.check(ig.quantize_filter4(hd, p["wdesc"], _ptr(a["w"]), case["group"], _ptr(p["codes"]), _ptr(p["scales"])), "igcQuantizeFilter4")
        ig.check(ig.dequantize_filter4(hd, case["group"], _ptr(p["codes"]), _ptr(p["scales"]), p["backdesc"], _ptr(p["back"])), "igcDequantizeFilter4")
        return {"w": p["back"]}
    ig.check(ig.linear4_forward(hd, 1.0, p["xdesc"], _ptr(a["x"]), p["wdesc"], case["group"], _ptr(a["codes"]), _ptr(a["scales"]), _ptr(p["ws"]), p["ws_bytes"],
                                _ptr(a["bias"]), p["act"], 1.0 if "r" in a else 0.0, p["rdesc"], _ptr(a.get("r")), p["ydesc"], _ptr(p["y"])), "igcLinear4Forward")
    return {"y": p["y"]}


def _adamw_results(a):
    return {n: t for n, t in a.items() if n not in ("g", "tensors")}


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _logits(a):
    z = a["x"].float() @ a["w"].float().t()
    return z + a["bias"] if "bias" in a else z


def _hash(x):
    """32 mixed bits of 32 (held in 64)."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(n):
    """Of a tensor's elements: 32 each, from the seed, the step and the element's place."""
    key = _hash(SEED ^ _hash(STEP))
    return _hash(torch.arange(n, device="cuda", dtype=torch.int64) ^ key)


def _rounded(value, scale, bits, kept, dtype, least):
    """value / scale with `kept` bits behind the leading one, up or down by 16 random bits, as dtype; one that is not zero at least `least`."""
    most = torch.finfo(dtype).max
    drop = 23 - kept
    rows = torch.where(scale[:, None] > 0, _to_blocks(value) * (1 / scale)[:, None], torch.zeros((), device="cuda")).view(-1)[:value.numel()]
    up = (rows.view(torch.int32) + (bits << (drop - 16)).to(torch.int32)) & ~((1 << drop) - 1)
    y = up.view(torch.float32).clamp(-most, most)
    if least:
        y = torch.where(value > 0, y.clamp(min=least), y)
    return y.to(dtype)


def _adamw_plain(t):
    g = t["g"].float() * SCALE
    eight = "m8" in t
    n = g.numel()
    if eight:
        m = (_to_blocks(t["m8"].float()) * t["m_scale"][:, None]).view(-1)[:n]
        v = (_to_blocks(t["v8"].float()) * t["v_scale"][:, None]).view(-1)[:n]
    else:
        m, v = t["m"], t["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    update = m * (1 / (1 - BETA1 ** STEP)) / (torch.sqrt(v * (1 / (1 - BETA2 ** STEP))) + EPSILON)
    t["p"].copy_(t["p"] * (1 - RATE * t["decay"]) - RATE * update)
    if "copy" in t:
        t["copy"].copy_(t["p"])
    if not eight:
        t["m"].copy_(m)
        t["v"].copy_(v)
        return
    bits = _random_bits(n)
    t["m_scale"].copy_(_to_blocks(m).abs().amax(1) * (1 / 448.0))
    t["v_scale"].copy_(_to_blocks(v).amax(1) * (1 / 57344.0))
    t["m8"].copy_(_rounded(m, t["m_scale"], bits & 0xFFFF, 3, torch.float8_e4m3fn, 0.0))
    t["v8"].copy_(_rounded(v, t["v_scale"], bits >> 16, 2, torch.float8_e5m2, 2.0 ** -16))


def _values(codes, scales, C, group):
    """The filter (K x C) that packed codes and scales stand for, in floats."""
    K, blocks = codes.shape[0], codes.shape[1] // 64
    code = torch.stack((codes & 15, codes >> 4), -1).view(K, blocks, 4, 4, 4, 2).permute(0, 1, 3, 2, 4, 5).reshape(K, blocks * 128)[:, :C].long()
    return _of_codes(code, scales, group)


def _of_codes(code, scales, group):
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device="cuda")
    return table[code] * scales.t().float().repeat_interleave(group, 1)[:, :code.shape[1]]


def _plain(state):
    case, a = state["case"], state["a"]
    kind = case["kind"]
    if kind == "loss":
        z = _logits(a)
        most = z.amax(1)
        log_sum = most + torch.log(torch.exp(z - most[:, None]).sum(1))
        there = a["target"] >= 0
        picked = z.gather(1, a["target"].long().clamp(min=0)[:, None])[:, 0]
        return {"loss": torch.where(there, log_sum - picked, torch.zeros_like(picked)), "log_sum": log_sum}
    if kind == "loss_gradient":
        dz = torch.exp(_logits(a) - a["log_sum"][:, None])
        there = a["target"] >= 0
        dz.scatter_add_(1, a["target"].long().clamp(min=0)[:, None], torch.full((case["M"], 1), -1.0, device="cuda"))
        dz = dz * torch.where(there, a["dloss"], torch.zeros_like(a["dloss"]))[:, None]
        out = {"dx": (dz @ a["w"].float()).to(a["x"].dtype), "dw": (dz.t() @ a["x"].float()).to(a["w"].dtype)}
        return dict(out, dbias=dz.sum(0)) if case["bias"] else out
    if kind == "adamw":
        [_adamw_plain(t) for t in a["tensors"]]
        return _adamw_results(a)
    if kind == "four_bits_store":
        code, scale = _to_codes(a["w"], case["group"])
        return {"w": _of_codes(code.long(), scale, case["group"])}
    y = _act(case["act"], a["x"].float() @ _values(a["codes"], a["scales"], case["C"], case["group"]).t() + a["bias"])
    return {"y": (y + a["r"].float() if "r" in a else y).to(_T[case["out"]])}


def run(state):
    return _run_own(state) if own else _plain(state)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------
def _exact_loss(case, a):
    """A few rows at a time; the gradient as that of sum(dloss * loss), with the logarithms of the sums as given."""
    w, bias = a["w"].double(), a["bias"].double() if "bias" in a else torch.zeros(case["V"], dtype=torch.float64, device="cuda")
    step = max(1, (1 << 28) // case["V"])
    if case["kind"] == "loss":
        sums, losses = [], []
        for x, t in zip(a["x"].split(step), a["target"].split(step)):
            z = torch.addmm(bias, x.double(), w.t())
            sums.append(torch.logsumexp(z, 1))
            at = t.long()
            losses.append(torch.where(at < 0, 0.0, sums[-1] - z[torch.arange(len(at), device="cuda"), at.clamp(min=0)]))
        return {"loss": torch.cat(losses), "log_sum": torch.cat(sums)}
    dx, dw, dbias = [], torch.zeros_like(w), torch.zeros_like(bias)
    for x, t, s, d in zip(*(a[n].split(step) for n in ("x", "target", "log_sum", "dloss"))):
        d = torch.where(t < 0, 0.0, d.double())
        p = torch.addmm(bias, x.double(), w.t()).sub_(s.double()[:, None]).exp_().mul_(d[:, None])
        rows = (t >= 0).nonzero()[:, 0]
        p[rows, t[rows].long()] -= d[rows]
        dx.append(torch.mm(p, w))
        dw.addmm_(p.t(), x.double())
        dbias += torch.mv(p.t(), torch.ones(len(d), dtype=torch.float64, device="cuda"))
    out = {"dx": torch.cat(dx), "dw": dw}
    return dict(out, dbias=dbias) if case["bias"] else out


def _exact_eight(value, most, man, least, tiny, bits):
    """Blocks' scales, and the codes' values: steps of 2^-man of the power of two below, up where the part behind them and the random part reach one; below
    the format's smallest normal number `least` then the nearest of its steps of `tiny`."""
    n = value.numel()
    whole = torch.zeros(_blocks(n) * 256, dtype=torch.float64, device="cuda")
    whole[:n] = value
    scale = (whole.view(-1, 256).abs().max(1).values / most).float()
    y = (whole.view(-1, 256) / scale.double().clamp(min=1e-300)[:, None]).reshape(-1)[:n]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1e-300))) - man)
    y = torch.sign(y) * step * torch.floor(y.abs() / step + bits.double() / 65536)
    return scale, torch.where(y.abs() < least, torch.round(y / tiny) * tiny, y.clamp(-most, most))


def _exact_adamw(case, a):
    out = {}

    def put(name, value):
        out.setdefault(name, []).append(value)

    for t in a["tensors"]:
        n = t["p"].numel()
        g, p = t["g"].double() * SCALE, t["p"].double()
        m, v = (t["m8"], t["v8"]) if "m8" in t else (t["m"], t["v"])
        m, v = m.double(), v.double()
        if "m8" in t:
            m, v = (s.double().repeat_interleave(256)[:n] * q for s, q in ((t["m_scale"], m), (t["v_scale"], v)))
        m = torch.lerp(g, m, BETA1)
        v = torch.lerp(g.square(), v, BETA2)
        root = (v / -math.expm1(STEP * math.log(BETA2))).sqrt()
        p = p - RATE * (t["decay"] * p + m / -math.expm1(STEP * math.log(BETA1)) / (root + EPSILON))
        put("p", p)
        if "copy" in t:
            put("copy", p)
        if "m8" not in t:
            put("m", m)
            put("v", v)
            continue
        bits = _mixed(torch.arange(n, device="cuda") ^ _mixed(SEED ^ _mixed(STEP)))
        m_scale, m8 = _exact_eight(m, 448.0, 3, 2.0 ** -6, 2.0 ** -9, bits & 0xFFFF)
        v_scale, v8 = _exact_eight(v, 57344.0, 2, 2.0 ** -14, 2.0 ** -16, bits >> 16)
        put("m8", m8)
        put("v8", torch.where(v > 0, v8.clamp(min=2.0 ** -16), v8))
        put("m_scale", m_scale.double())
        put("v_scale", v_scale.double())
    return {k: torch.cat(v) for k, v in out.items()}


def _mixed(x):
    """The hash, in steps written out."""
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        x = x ^ (x >> shift)
        x = x * factor % (1 << 32)
    return x ^ (x >> 16)


def _exact_store(a, group):
    """Each value of the table tried: the nearest one, of two as near the one with the even code."""
    K, C = a["w"].shape
    out = torch.empty(K, C, dtype=torch.float64, device="cuda")
    for c in range(0, C, group):
        w = a["w"][:, c:c + group].double()
        want = w.abs().max(1, keepdim=True).values / 6
        e = torch.floor(torch.log2(want.clamp(min=1e-300))) - 7
        s = torch.where(want > 0, torch.ceil(want / torch.exp2(e)) * torch.exp2(e), 0.0)   # (eight significant bits)
        best, off = torch.zeros_like(w), w.abs()
        for i in (2, 4, 6, 1, 3, 5, 7):
            d = (w.abs() - E2M1[i] * s).abs()
            near = d < off
            best, off = torch.where(near, E2M1[i] * s, best), torch.minimum(d, off)
        out[:, c:c + group] = torch.copysign(best, w)
    return {"w": out}


def exact(case, seed):
    a = _inputs(case, seed)
    kind = case["kind"]
    if kind.startswith("loss"):
        return _exact_loss(case, a)
    if kind == "adamw":
        return _exact_adamw(case, a)
    if kind == "four_bits_store":
        return _exact_store(a, case["group"])
    C, group = case["C"], case["group"]
    table = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    codes = a["codes"].view(case["K"], -1, 4, 4, 4)      # block, g, i, byte of the word
    z = a["bias"].double().repeat(case["M"], 1)
    for c in range(0, C, 8):
        block, i, g = c // 128, c % 128 // 32, c % 32 // 8
        byte = codes[:, block, g, i].long()
        code = torch.stack((byte % 16, byte // 16), 2).view(case["K"], 8)[:, :C - c]
        w = torch.where(code >= 8, -table[code % 8], table[code % 8])
        z.addmm_(a["x"][:, c:c + 8].double(), (w * a["scales"][c // group].double()[:, None]).t())
    act = {"none": lambda: z, "relu": lambda: torch.relu(z), "gelu": lambda: z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0)), "silu": lambda: z * torch.sigmoid(z)}
    return {"y": act[case["act"]]() + (a["r"].double() if "r" in a else 0.0)}


def work(case):
    kind = case["kind"]
    if kind.startswith("loss"):
        M, C, V, i = case["M"], case["C"], case["V"], _SIZE[case["dtype"]]
        b = i * (M * C + V * C) + 4 * (V if case["bias"] else 0) + 4 * M
        if kind == "loss":
            return {"bytes": b + 8 * M, "flops": 2 * M * C * V}
        return {"bytes": 2 * b + 8 * M, "flops": 6 * M * C * V}
    if kind == "adamw":
        mats, rest = (sum(s for s, mat in _shapes(case) if mat is q) for q in (True, False))
        one = 8 + _SIZE[case["grad"]]
        return {"bytes": mats * (one + 2 + (16 if case["bits"] == 32 else 4 + 16 / 256)) + rest * (one + 16), "flops": 20 * (mats + rest)}
    K, C = case["K"], case["C"]
    held = K * -(-C // 128) * 64 + 2 * K * -(-C // case["group"])
    if kind == "four_bits_store":
        return {"bytes": _SIZE[case["dtype"]] * K * C + held + held + 4 * K * C, "flops": 10 * K * C}
    M, i, o = case["M"], _SIZE[case["dtype"]], _SIZE[case["out"]]
    return {"bytes": held + i * M * C + 4 * K + o * M * K * (1 + case["residual"]), "flops": 2 * M * C * K}
