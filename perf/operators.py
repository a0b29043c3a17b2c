"""Operators of a feed-forward block as a training or serving program calls them: layer norm and the matrix product with
bias, activation and residual, each forward and backward.

A case is one call.  Rows are tokens; `pad` elements lie between the rows of every matrix (a slice of a wider buffer).
Kinds:
  norm_forward    y = (x - mean) / sqrt(variance + eps) * scale + shift, and the rows' mean and 1/sqrt(variance + eps)
  norm_backward   dx (+ the gradient `r` that reaches x past the norm, where `residual`), dscale, dshift
  linear_forward  y = f(x w^T + bias) + r; with `keep` also z = x w^T + bias, which training keeps for the backward pass
  linear_data     dx = (dy w) f'(z) (+ r): f is the activation in front of the product, z what it was applied to
  linear_filter   dw = dy^T x, dbias = column sums of dy
Sizes: M rows, C features in, K features out (norms: M rows of C).  `dtype`: the type of x, w, dy; `out`: of y, dx, dw (z and
r go with it); scales, shifts, biases and their gradients are float (double where x is).
"""
import math
import random

import torch

own = False

EPS = 1e-5
_T = {"f32": torch.float32, "bf16": torch.bfloat16, "f64": torch.float64}
_SIZE = {"f32": 4, "bf16": 2, "f64": 8}


def _norm(name, kind, dtype, out, M, C, pad=0, residual=False):
    c = {"kind": kind, "dtype": dtype, "out": out, "M": M, "C": C, "pad": pad}
    if kind == "norm_backward":
        c["residual"] = residual
    return dict(c, name=name) if name else c


def _linear(name, kind, dtype, out, M, C, K, act="none", pad=0, residual=False, keep=False):
    c = {"kind": kind, "dtype": dtype, "out": out, "M": M, "C": C, "K": K, "pad": pad}
    if kind != "linear_filter":
        c["act"], c["residual"] = act, residual
    if kind == "linear_forward":
        c["keep"] = keep
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: the norm in front of a block, four sequences with one new token each: the latency of a call
        _norm("norm_4_tokens", "norm_forward", "bf16", "bf16", 4, 4096),
        # training: the norm of a whole batch of tokens, a float residual stream into a bfloat16 block
        _norm("norm_batch", "norm_forward", "f32", "bf16", 16384, 4096),
        # a narrow model on a ragged batch, rows of a wider buffer, nothing divides
        _norm("norm_odd", "norm_forward", "f32", "f32", 5003, 1001, pad=3),
        # training: the gradient of a block's norm joins the one that went past it
        _norm("norm_back_batch", "norm_backward", "bf16", "bf16", 8192, 8192, residual=True),
        # the last, short batch of an odd width
        _norm("norm_back_odd", "norm_backward", "f32", "f32", 3001, 777),
        # serving: eight sequences, one token each, through the block's first product
        _linear("product_8_tokens", "linear_forward", "bf16", "bf16", 8, 4096, 16384, act="gelu"),
        # training, the largest: the block's first product over a batch, its pre-activation kept
        _linear("product_batch", "linear_forward", "bf16", "bf16", 8192, 4096, 16384, act="gelu", keep=True),
        # float, a prompt of odd length through an odd second product with the residual added
        _linear("product_odd_float", "linear_forward", "f32", "f32", 1023, 2050, 1000, residual=True, pad=1),
        # training: gradient through the block's second product and the GELU in front of it
        _linear("data_batch", "linear_data", "bf16", "bf16", 8192, 16384, 4096, act="gelu"),
        # float training of a small model: gradient through a product with a rectifier in front
        _linear("data_float", "linear_data", "f32", "f32", 4096, 2048, 1024, act="relu"),
        # training: gradients of a product's weights and bias, kept in float for the optimiser
        _linear("filter_batch", "linear_filter", "bf16", "f32", 8192, 4096, 4096),
        # a ragged batch and widths that nothing divides
        _linear("filter_odd", "linear_filter", "bf16", "bf16", 3333, 1001, 1503),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A number of features: a multiple of 64, of 8, or any."""
    n = _log(rng, lo, hi)
    step = rng.choice((1, 8, 64, 64))
    return max(lo, n // step * step)


def draw(rng):
    kind = rng.choice(("norm_forward", "norm_backward", "linear_forward", "linear_forward", "linear_data", "linear_filter"))
    pad = rng.choice((0, 0, 1, 8))
    if kind.startswith("norm"):
        dtype, out = rng.choice((("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f64", "f64")))
        C = _width(rng, 33, 16384)
        M = _log(rng, 1, min(65536, (1 << 26) // C))
        return _norm(None, kind, dtype, out, M, C, pad, residual=rng.random() < 0.5)
    dtype, out = rng.choice((("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")))
    C, K = _width(rng, 64, 16384), _width(rng, 64, 16384)
    while C * K > 4096 * 16384:
        C, K = max(64, C // 2), max(64, K // 2)
    M = _log(rng, 1, min(8192, (1 << 36) // (C * K), (1 << 27) // max(C, K)))   # (a quarter of the largest case's work at most)
    act = rng.choice(("none", "relu", "gelu", "silu", "tanh", "sigmoid"))
    return _linear(None, kind, dtype, out, M, C, K, act, pad, residual=rng.random() < 0.5, keep=rng.random() < 0.5)


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _matrix(rows, cols, dtype, pad, fill):
    """rows x cols of `fill` (float or double), rounded to dtype, in rows cols + pad apart."""
    wide = torch.zeros(rows, cols + pad, dtype=_T[dtype], device="cuda")
    wide[:, :cols] = fill.to(_T[dtype])
    return wide[:, :cols]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    M, C, dtype, out, pad, kind = case["M"], case["C"], case["dtype"], case["out"], case["pad"], case["kind"]
    wide = torch.float64 if dtype == "f64" else torch.float32

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=wide)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda", dtype=wide)

    if kind.startswith("norm"):
        # a residual stream: rows of different size, an offset per feature, a few features far larger than the rest
        size = 0.5 + uniform(C)
        size = torch.where(uniform(C) < 0.005, 20 * size, size)
        x = (normal(M, C) * size + 0.3 * normal(C)) * (0.25 + 2 * uniform(M, 1))
        a = {"x": _matrix(M, C, dtype, pad, x), "scale": 1 + 0.2 * normal(C), "shift": 0.1 * normal(C)}
        if kind == "norm_backward":
            xd = a["x"].double()
            mean = xd.mean(1)
            var = (xd - mean[:, None]).square().mean(1)
            a["mean"], a["invstd"] = mean.to(wide), (1 / (var + EPS).sqrt()).to(wide)
            a["dy"] = _matrix(M, C, out, pad, 1e-3 * normal(M, C) * (0.1 + uniform(M, 1)))
            if case["residual"]:
                a["r"] = _matrix(M, C, dtype, pad, 1e-3 * normal(M, C))
            del a["shift"]
        return a
    K = case["K"]
    if kind == "linear_forward":
        a = {"x": _matrix(M, C, dtype, pad, normal(M, C)), "w": _matrix(K, C, dtype, 0, normal(K, C) / math.sqrt(C)), "bias": 0.5 * normal(K)}
        if case["residual"]:
            a["r"] = _matrix(M, K, out, pad, normal(M, K))
        return a
    a = {"dy": _matrix(M, K, dtype, pad, 1e-2 * normal(M, K) * (0.1 + uniform(M, 1)))}
    if kind == "linear_filter":
        a["x"] = _matrix(M, C, dtype, pad, normal(M, C) + 0.2)
        return a
    a["w"] = _matrix(K, C, dtype, 0, normal(K, C) / math.sqrt(C))
    if case["act"] != "none":
        a["z"] = _matrix(M, C, out, pad, 1.5 * normal(M, C))
    if case["residual"]:
        a["r"] = _matrix(M, C, out, pad, 1e-2 * normal(M, C))
    return a


def prepare(case, seed):
    a = _inputs(case, seed)
    return {"case": case, "a": a, "plan": _plan(case, a) if own else None}


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _plan(case, a):
    """Handle, descriptors, output buffers and workspace, as a program makes them once for a layer."""
    import paper_1410_0759_amd as ig
    DT = {torch.float32: ig.IGC_DATA_FLOAT, torch.bfloat16: ig.IGC_DATA_BFLOAT16, torch.float64: ig.IGC_DATA_DOUBLE}
    p = {"ig": ig, "handle": ig.Handle()}
    p["handle"].set_stream(torch.cuda.current_stream().cuda_stream)

    def desc(t):
        return ig.TensorDescriptor().set(DT[t.dtype], t.shape[0], t.shape[1], 1, 1, (t.stride(0), 1, 1, 1))

    def fresh(rows, cols, dtype):
        return torch.empty(rows, cols + case["pad"], dtype=_T[dtype], device="cuda")[:, :cols]

    kind, M, C, dtype, out = case["kind"], case["M"], case["C"], case["dtype"], case["out"]
    wide = _T["f64" if dtype == "f64" else "f32"]
    for n in ("x", "dy", "z", "r"):
        p[n + "desc"] = desc(a[n]) if n in a else None
    if "w" in a:
        p["wdesc"] = ig.FilterDescriptor().set(DT[a["w"].dtype], case["K"], C, 1, 1)
    size = 0
    if kind == "norm_forward":
        p["y"] = fresh(M, C, out)
        p["ydesc"] = desc(p["y"])
        p["mean"], p["invstd"] = (torch.empty(M, dtype=wide, device="cuda") for _ in range(2))
    elif kind == "norm_backward":
        p["dx"] = fresh(M, C, dtype)
        p["dxdesc"] = desc(p["dx"])
        p["dscale"], p["dshift"] = (torch.empty(C, dtype=wide, device="cuda") for _ in range(2))
        size = ig.get_layer_norm_backward_workspace_size(p["handle"], p["xdesc"], p["dydesc"], p["dxdesc"])
    elif kind == "linear_forward":
        p["y"] = fresh(M, case["K"], out)
        p["ydesc"] = desc(p["y"])
        if case["keep"]:
            p["z"] = fresh(M, case["K"], out)
        size = ig.get_linear_forward_workspace_size(p["handle"], p["xdesc"], p["wdesc"], p["ydesc"])
    elif kind == "linear_data":
        p["dx"] = fresh(M, C, out)
        p["dxdesc"] = desc(p["dx"])
        size = ig.get_linear_backward_data_workspace_size(p["handle"], p["wdesc"], p["dydesc"], p["dxdesc"])
    else:
        p["dw"] = torch.empty(case["K"], C, dtype=_T[out], device="cuda")
        p["dbias"] = torch.empty(case["K"], dtype=torch.float32, device="cuda")
        p["dwdesc"] = ig.FilterDescriptor().set(DT[_T[out]], case["K"], C, 1, 1)
        size = ig.get_linear_backward_filter_workspace_size(p["handle"], p["xdesc"], p["dydesc"], p["dwdesc"])
    p["ws"] = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    p["ws_bytes"] = size
    p["act"] = {"none": ig.IGC_ACTIVATION_IDENTITY, "sigmoid": ig.IGC_ACTIVATION_SIGMOID, "relu": ig.IGC_ACTIVATION_RELU, "tanh": ig.IGC_ACTIVATION_TANH,
                "gelu": ig.IGC_ACTIVATION_GELU, "silu": ig.IGC_ACTIVATION_SILU}[case.get("act", "none")]
    return p


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _run_own(state):
    case, a, p = state["case"], state["a"], state["plan"]
    ig, kind = p["ig"], case["kind"]
    beta = 1.0 if "r" in a else 0.0
    if kind == "norm_forward":
        ig.check(ig.layer_norm_forward(p["handle"], 1.0, p["xdesc"], _ptr(a["x"]), _ptr(a["scale"]), _ptr(a["shift"]), EPS, 0.0, p["ydesc"], _ptr(p["y"]),
                                       _ptr(p["mean"]), _ptr(p["invstd"])), "igcLayerNormForward")
        return {"y": p["y"], "mean": p["mean"], "invstd": p["invstd"]}
    if kind == "norm_backward":
        ig.check(ig.layer_norm_backward(p["handle"], 1.0, p["xdesc"], _ptr(a["x"]), p["dydesc"], _ptr(a["dy"]), _ptr(a["scale"]), _ptr(a["mean"]), _ptr(a["invstd"]),
                                        _ptr(p["ws"]), p["ws_bytes"], beta, p["rdesc"], _ptr(a.get("r")), p["dxdesc"], _ptr(p["dx"]), 0.0,
                                        _ptr(p["dscale"]), _ptr(p["dshift"])), "igcLayerNormBackward")
        return {"dx": p["dx"], "dscale": p["dscale"], "dshift": p["dshift"]}
    if kind == "linear_forward":
        ig.check(ig.linear_forward(p["handle"], 1.0, p["xdesc"], _ptr(a["x"]), p["wdesc"], _ptr(a["w"]), _ptr(p["ws"]), p["ws_bytes"], _ptr(a["bias"]), p["act"], beta,
                                   p["rdesc"], _ptr(a.get("r")), p["ydesc"], _ptr(p.get("z")), _ptr(p["y"])), "igcLinearForward")
        return {"y": p["y"], "z": p["z"]} if case["keep"] else {"y": p["y"]}
    if kind == "linear_data":
        ig.check(ig.linear_backward_data(p["handle"], 1.0, p["wdesc"], _ptr(a["w"]), p["dydesc"], _ptr(a["dy"]), _ptr(p["ws"]), p["ws_bytes"], p["act"],
                                         p["zdesc"], _ptr(a.get("z")), beta, p["rdesc"], _ptr(a.get("r")), p["dxdesc"], _ptr(p["dx"])), "igcLinearBackwardData")
        return {"dx": p["dx"]}
    ig.check(ig.linear_backward_filter(p["handle"], 1.0, p["xdesc"], _ptr(a["x"]), p["dydesc"], _ptr(a["dy"]), _ptr(p["ws"]), p["ws_bytes"], 0.0,
                                       p["dwdesc"], _ptr(p["dw"]), _ptr(p["dbias"])), "igcLinearBackwardFilter")
    return {"dw": p["dw"], "dbias": p["dbias"]}


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _act(name, z):
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "tanh":
        return torch.tanh(z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_derivative(name, z):
    if name == "sigmoid":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 - s)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "tanh":
        t = torch.tanh(z)
        return 1 - t * t
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain(state):
    case, a = state["case"], state["a"]
    kind, out = case["kind"], _T[case["out"]]
    f = {n: t if t.dtype == torch.float64 else t.float() for n, t in a.items()}
    if kind == "norm_forward":
        mean = f["x"].mean(1, keepdim=True)
        d = f["x"] - mean
        invstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        return {"y": (d * invstd * f["scale"] + f["shift"]).to(out), "mean": mean[:, 0], "invstd": invstd[:, 0]}
    if kind == "norm_backward":
        s = f["invstd"][:, None]
        h = (f["x"] - f["mean"][:, None]) * s
        q = f["dy"] * f["scale"]
        dx = s * (q - q.mean(1, keepdim=True) - h * (q * h).mean(1, keepdim=True))
        if "r" in f:
            dx = dx + f["r"]
        return {"dx": dx.to(_T[case["dtype"]]), "dscale": (f["dy"] * h).sum(0), "dshift": f["dy"].sum(0)}
    if kind == "linear_forward":
        z = f["x"] @ f["w"].t() + f["bias"]
        y = _act(case["act"], z)
        if "r" in f:
            y = y + f["r"]
        return {"y": y.to(out), "z": z.to(out)} if case["keep"] else {"y": y.to(out)}
    if kind == "linear_data":
        dx = f["dy"] @ f["w"]
        if "z" in f:
            dx = dx * _act_derivative(case["act"], f["z"])
        if "r" in f:
            dx = dx + f["r"]
        return {"dx": dx.to(out)}
    return {"dw": (f["dy"].t() @ f["x"]).to(out), "dbias": f["dy"].sum(0)}


def run(state):
    return _run_own(state) if own else _plain(state)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------
def _phi(z):
    """The normal distribution function, without the cancellation of 1 + erf."""
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _f(name, z):
    return {"none": lambda: z, "sigmoid": lambda: torch.sigmoid(z), "relu": lambda: torch.relu(z), "tanh": lambda: torch.tanh(z),
            "gelu": lambda: z * _phi(z), "silu": lambda: z * torch.sigmoid(z)}[name]()


def _f_slope(name, z):
    """f' of every element as the gradient of the sum of f."""
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        return torch.autograd.grad(_f(name, z).sum(), z)[0]


def exact(case, seed):
    d = {n: t.double() for n, t in _inputs(case, seed).items()}
    kind, C = case["kind"], case["C"]
    if kind == "norm_forward":
        mean = d["x"].sum(1) / C
        var = torch.var(d["x"], dim=1, correction=0)
        s = (var + EPS).rsqrt()
        return {"y": torch.addcmul(d["shift"], d["x"] * s[:, None] - (mean * s)[:, None], d["scale"]), "mean": mean, "invstd": s}
    if kind == "norm_backward":
        # the gradient of sum(dy * y) with respect to x has three parts: the direct one, through the mean and through the
        # deviation; mean and 1/deviation are taken as given
        s, m = d["invstd"], d["mean"]
        c = d["x"].sub(m[:, None])
        q = d["dy"].mul(d["scale"])
        along = torch.einsum("rc,rc->r", q, c) * s.pow(3) / C
        dx = q.mul(s[:, None]) - (q.sum(1) * s / C)[:, None] - c * along[:, None]
        if "r" in d:
            dx = d["r"] + dx
        return {"dx": dx, "dscale": torch.mv((d["dy"] * c).t(), s), "dshift": torch.mv(d["dy"].t(), torch.ones_like(s))}
    if kind == "linear_forward":
        z = torch.addmm(d["bias"], d["x"], d["w"].t())
        y = _f(case["act"], z) + d.get("r", 0.0)
        return {"y": y, "z": z} if case["keep"] else {"y": y}
    if kind == "linear_data":
        dx = torch.mm(d["w"].t(), d["dy"].t()).t()
        if "z" in d:
            dx = dx * _f_slope(case["act"], d["z"])
        return {"dx": dx + d.get("r", 0.0)}
    return {"dw": torch.mm(d["x"].t(), d["dy"]).t(), "dbias": torch.mv(d["dy"].t(), torch.ones(case["M"], dtype=torch.float64, device="cuda"))}


def work(case):
    M, C, i, o = case["M"], case["C"], _SIZE[case["dtype"]], _SIZE[case["out"]]
    kind, wide = case["kind"], 8 if case["dtype"] == "f64" else 4
    if kind == "norm_forward":
        return {"bytes": M * C * (i + o) + wide * (2 * C + 2 * M), "flops": 8 * M * C}
    if kind == "norm_backward":
        return {"bytes": M * C * (2 * i + o + (i if case["residual"] else 0)) + wide * (3 * C + 2 * M), "flops": 14 * M * C}
    K = case["K"]
    flops = 2 * M * C * K
    if kind == "linear_forward":
        return {"bytes": i * (M * C + K * C) + 4 * K + o * M * K * (1 + case["residual"] + case["keep"]), "flops": flops}
    if kind == "linear_data":
        return {"bytes": i * (M * K + K * C) + o * M * C * (1 + case["residual"] + (case["act"] != "none")), "flops": flops}
    return {"bytes": i * (M * K + M * C) + o * K * C + 4 * K, "flops": flops + M * K}
