"""A feed-forward block trained against the next token's probability and served in four bits, on the library's functions:

    loss = cross entropy of (block(x) w^T + bias) over a vocabulary;  an AdamW step over all weights;  then the block's two filters in four bits

PyTorch serves for device memory and streams only.  Results and workspaces are allocated by PyTorch on the current stream for each call, so a result is the caller's, and a
call can be captured into a graph.  Weights, gradients and states are used in place: calls that share them follow each other (one stream, or streams that wait for each
other).  ``python -m paper_1410_0759_amd.training`` trains a small block for some steps and then runs single tokens through it.
"""
import contextlib
import threading

import torch

from . import binding as ig
from .feed_forward import FeedForward, _DATA, _desc


class _Module:
    """A handle, used by one call at a time, on the weights' device and the current stream."""

    def __init__(self, device):
        self.device, self.handle, self._lock = torch.device(device), ig.Handle(), threading.RLock()

    @contextlib.contextmanager
    def _call(self):
        if self.device.type != "cuda":
            raise ValueError("the calls need their weights on a GPU")
        with self._lock, torch.cuda.device(self.device):
            self.handle.set_stream(torch.cuda.current_stream().cuda_stream)
            yield self.handle

    def _rows(self, name, t, width, dtype, rows=None):
        if t.dim() != 2 or t.shape[0] < 1 or t.shape[1] != width or (t.shape[1] > 1 and t.stride(1) != 1) or t.dtype != dtype or rows not in (None, t.shape[0]):
            raise ValueError("%s: %srows of %d adjacent features of type %s" % (name, "" if rows is None else "%d " % rows, width, dtype))
        if t.device != self.device:
            raise ValueError("%s: on the weights' device, %s" % (name, self.device))

    def _vector(self, name, t, n, dtype):
        if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous() or t.dtype != dtype or t.device != self.device:
            raise ValueError("%s: %d adjacent numbers of type %s on the weights' device, %s" % (name, n, dtype, self.device))

    @staticmethod
    def _space(size):
        return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


class VocabularyHead(_Module):
    """The last product and the cross entropy of its logits, which are never held.  Weights of the compute type, float gradients.
    slopes: what the logits' gradients go into the products as, where the weights are bfloat16: torch.float32, as exact as float gradients are to be, or torch.bfloat16,
    for up to 1.7 times the speed."""

    def __init__(self, width, entries, dtype=torch.bfloat16, bias=False, device="cuda", seed=0, slopes=torch.float32):
        device = torch.device("cuda", torch.cuda.current_device()) if str(device) == "cuda" else torch.device(device)
        super().__init__(device)
        if slopes not in _DATA:
            raise ValueError("VocabularyHead: slopes in float32 or bfloat16")
        ig.set_cross_entropy_slopes(self.handle, _DATA[slopes])
        g = torch.Generator(device=device).manual_seed(seed)
        self.width, self.entries, self.dtype = width, entries, dtype
        self.w = (torch.randn(entries, width, generator=g, device=device) / width ** 0.5).to(dtype)
        self.bias = torch.zeros(entries, device=device) if bias else None
        self.grads = {n: torch.zeros(t.shape, device=device) for n, t in (("w", self.w), ("bias", self.bias)) if t is not None}
        self.w_desc = ig.FilterDescriptor().set(_DATA[dtype], entries, width, 1, 1)
        self.dw_desc = ig.FilterDescriptor().set(ig.IGC_DATA_FLOAT, entries, width, 1, 1)
        self._kept = None

    def _bias(self):
        return 0 if self.bias is None else self.bias.data_ptr()

    def forward(self, x, targets, keep=True):
        """Each row's loss; 0 where its target (32-bit) is no entry.  keep: for ``backward``; x and targets have to stay as they are until then."""
        self._rows("x", x, self.width, self.dtype)
        self._vector("targets", targets, x.shape[0], torch.int32)
        with self._call() as hd:
            loss, log_sum = (torch.empty(x.shape[0], device=self.device) for _ in range(2))
            xd = _desc(x)
            size = ig.get_linear_cross_entropy_forward_workspace_size(hd, xd, self.w_desc)
            ws = self._space(size)
            ig.check(ig.linear_cross_entropy_forward(hd, xd, x.data_ptr(), self.w_desc, self.w.data_ptr(), self._bias(), targets.data_ptr(), ws.data_ptr(), size, loss.data_ptr(),
                                                     log_sum.data_ptr()), "igcLinearCrossEntropyForward")
            if keep:
                self._kept = x, targets, log_sum, torch.cuda.current_stream()
            return loss

    def backward(self, dloss=None, scale=1.0, accumulate=False):
        """Gradient with respect to the x of the last forward pass that kept its results, of ``scale`` times the sum of its losses (each times its dloss, where given); ``grads``
        receives (accumulate: is increased by) the weights' gradients."""
        if self._kept is None:
            raise ValueError("backward: no forward pass kept its results")
        x, targets, log_sum, stream = self._kept
        if dloss is not None:
            self._vector("dloss", dloss, x.shape[0], torch.float32)
        with self._call() as hd:
            here = torch.cuda.current_stream()
            if here != stream and not torch.cuda.is_current_stream_capturing():
                here.wait_stream(stream)
                log_sum.record_stream(here)      # (memory of the other stream's: not given away before this one is done with it)
            dx = torch.empty(x.shape, dtype=x.dtype, device=self.device)
            xd, dxd = _desc(x), _desc(dx)
            size = ig.get_linear_cross_entropy_backward_workspace_size(hd, xd, self.w_desc, dxd, self.dw_desc)
            ws = self._space(size)
            ig.check(ig.linear_cross_entropy_backward(hd, scale, xd, x.data_ptr(), self.w_desc, self.w.data_ptr(), self._bias(), targets.data_ptr(), log_sum.data_ptr(),
                                                      0 if dloss is None else dloss.data_ptr(), ws.data_ptr(), size, 0.0, dxd, dx.data_ptr(), 1.0 if accumulate else 0.0, self.dw_desc,
                                                      self.grads["w"].data_ptr(), self.grads["bias"].data_ptr() if self.bias is not None else 0), "igcLinearCrossEntropyBackward")
            return dx


class AdamW(_Module):
    """Steps over named weights: {name: (weight, gradient)}, packed tensors of one device.  A bfloat16 weight has a float master, made here, whose rounding it is after every step.
    bits 8: matrices of at least 4096 elements keep their states in 8 bits.  decay: of matrices only."""

    SMALL = 4096

    def __init__(self, weights, rate=1e-3, betas=(0.9, 0.999), epsilon=1e-8, decay=0.1, bits=32, seed=0):
        if not weights or bits not in (8, 32):
            raise ValueError("AdamW: at least one weight, and states in 8 or 32 bits")
        super().__init__(next(iter(weights.values()))[0].device)
        self.rate, self.betas, self.epsilon, self.seed, self.steps = rate, betas, epsilon, seed, 0
        self.weights, self.state = dict(weights), {}
        self.table = (ig.AdamWTensor * len(weights))()
        taken = []
        for (name, (w, g)), q in zip(weights.items(), self.table):
            for what, t in (("weight", w), ("gradient", g)):
                if t.dtype not in _DATA or not t.is_contiguous() or t.shape != w.shape or t.device != self.device:
                    raise ValueError("%s: a packed %s of float or bfloat16 on %s" % (name, what, self.device))
            n, eight = w.numel(), bits == 8 and w.dim() > 1 and w.numel() >= self.SMALL
            taken += [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), name) for t in (w, g) if n]
            new = lambda size, dtype=torch.float32: torch.zeros(size, dtype=dtype, device=self.device)
            s = self.state[name] = {"m": new(n, torch.float8_e4m3fn if eight else torch.float32), "v": new(n, torch.float8_e5m2 if eight else torch.float32)}
            if eight:
                s["m_scale"], s["v_scale"] = new(-(-n // 256)), new(-(-n // 256))
            if w.dtype == torch.bfloat16:
                s["master"] = w.reshape(-1).float()
            ptr = lambda t: 0 if t is None or n == 0 else t.data_ptr()
            q.param, q.copy = (ptr(s["master"]), ptr(w)) if "master" in s else (ptr(w), 0)
            q.grad, q.m, q.v, q.m_scale, q.v_scale = (ptr(t) for t in (g, s["m"], s["v"], s.get("m_scale"), s.get("v_scale")))
            q.count, q.weight_decay, q.state_bits = n, decay if w.dim() > 1 else 0.0, 8 if eight else 32
            q.param_type, q.grad_type = ig.IGC_DATA_FLOAT, _DATA[g.dtype]
        taken.sort()
        for a, b in zip(taken, taken[1:]):
            if b[0] < a[1]:
                raise ValueError("AdamW: %s and %s share memory" % (a[2], b[2]))

    def step(self, scale=1.0, rate=None):
        """One step with ``scale`` times the gradients.  (Not while a graph is captured: its replays would all be the step of that number.)"""
        with self._call() as hd:
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("AdamW.step counts its steps on the host: capture igcAdamWStep with the step's number on the device")
            q = ig.AdamWParameters(learning_rate=self.rate if rate is None else rate, beta1=self.betas[0], beta2=self.betas[1], epsilon=self.epsilon, gradient_scale=scale,
                                   step=self.steps + 1, seed=self.seed)
            ig.check(ig.adamw_step(hd, q, self.table), "igcAdamWStep")
            self.steps += 1

    def state_dict(self):
        """Copies of the states, for ``load_state_dict`` of a run that goes on."""
        return {"steps": self.steps, "seed": self.seed, "state": {n: {k: t.clone() for k, t in s.items()} for n, s in self.state.items()}}

    def load_state_dict(self, saved):
        if {n: {k: (t.shape, t.dtype) for k, t in s.items()} for n, s in saved["state"].items()} != {n: {k: (t.shape, t.dtype) for k, t in s.items()} for n, s in self.state.items()}:
            raise ValueError("load_state_dict: states of other weights")
        self.steps, self.seed = saved["steps"], saved["seed"]
        for n, s in saved["state"].items():
            for k, t in s.items():
                self.state[n][k].copy_(t)
            if "master" in s:
                self.weights[n][0].copy_(s["master"].view(self.weights[n][0].shape))


class FourBitFeedForward(_Module):
    """A block to serve from: y = gelu(layer_norm(x) w1^T + b1) w2^T + b2 + x, with the filters of a FeedForward in four bits."""

    def __init__(self, block, group=128):
        super().__init__(block.w1.device)
        self.width, self.hidden, self.dtype, self.group = block.width, block.hidden, block.dtype, group
        self.scale, self.shift, self.b1, self.b2 = (t.clone() for t in (block.scale, block.shift, block.b1, block.b2))
        self.w1_desc, self.w2_desc = (ig.FilterDescriptor().set(_DATA[self.dtype], k, c, 1, 1) for k, c in ((self.hidden, self.width), (self.width, self.hidden)))
        with self._call() as hd:
            self.w1, self.w2 = (self._store(hd, d, w) for d, w in ((self.w1_desc, block.w1), (self.w2_desc, block.w2)))

    def _store(self, hd, desc, w):
        codes, scales = (torch.empty(n, dtype=torch.uint8, device=self.device) for n in ig.get_filter4_size(desc, self.group))
        ig.check(ig.quantize_filter4(hd, desc, w.data_ptr(), self.group, codes.data_ptr(), scales.data_ptr()), "igcQuantizeFilter4")
        return codes, scales

    def _product(self, hd, x, desc, w, bias, activation, r, y):
        xd, yd = _desc(x), _desc(y)
        size = ig.get_linear4_forward_workspace_size(hd, xd, desc, self.group, yd)
        ws = self._space(size)
        ig.check(ig.linear4_forward(hd, 1.0, xd, x.data_ptr(), desc, self.group, w[0].data_ptr(), w[1].data_ptr(), ws.data_ptr(), size, bias.data_ptr(), activation,
                                    0.0 if r is None else 1.0, None if r is None else _desc(r), 0 if r is None else r.data_ptr(), yd, y.data_ptr()), "igcLinear4Forward")

    def forward(self, x):
        self._rows("x", x, self.width, self.dtype)
        with self._call() as hd:
            new = lambda n: torch.empty(x.shape[0], n, dtype=self.dtype, device=self.device)
            h, a, y = new(self.width), new(self.hidden), new(self.width)
            ig.check(ig.layer_norm_forward(hd, 1.0, _desc(x), x.data_ptr(), self.scale.data_ptr(), self.shift.data_ptr(), FeedForward.EPS, 0.0, _desc(h), h.data_ptr(), 0, 0),
                     "igcLayerNormForward")
            self._product(hd, h, self.w1_desc, self.w1, self.b1, ig.IGC_ACTIVATION_GELU, None, a)
            self._product(hd, a, self.w2_desc, self.w2, self.b2, ig.IGC_ACTIVATION_IDENTITY, x, y)
            return y


def main(width=512, hidden=2048, entries=1000, tokens=1000, steps=30, rate=1e-3):
    block, head = FeedForward(width, hidden), VocabularyHead(width, entries)
    optimizer = AdamW({**{n: (getattr(block, n), g) for n, g in block.grads.items()}, "head": (head.w, head.grads["w"])}, rate=rate, bits=8)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(tokens, width, generator=g, device="cuda").to(block.dtype)
    targets = torch.randint(0, entries, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    for step in range(steps):
        loss = head.forward(block.forward(x), targets)
        block.backward(x, head.backward(scale=1.0 / tokens))
        optimizer.step()
        if step % 10 == 0 or step == steps - 1:
            print("step %2d: cross entropy %.4f" % (step, float(loss.mean())), flush=True)
    served = FourBitFeedForward(block)
    one = torch.cat([served.forward(x[i:i + 1]) for i in range(4)])
    print("cross entropy of four tokens, each alone: %.4f in bfloat16, %.4f in four bits" % (
        float(head.forward(block.forward(x[:4], keep=False).clone(), targets[:4], keep=False).mean()), float(head.forward(one, targets[:4], keep=False).mean())))


if __name__ == "__main__":
    main()
