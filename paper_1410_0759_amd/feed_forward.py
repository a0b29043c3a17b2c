"""A feed-forward block of a transformer on the library's functions, trained and served:

    h = layer_norm(x);  z = h w1^T + b1;  y = gelu(z) w2^T + b2 + x

PyTorch serves for device memory and streams only.  A block keeps its descriptors, output buffers and workspaces for the numbers of tokens that it met
last, so that a step makes no allocation after the first of its size and can be captured into a graph.  ``python -m paper_1410_0759_amd.feed_forward``
trains one on a fixed random batch for a few steps and then runs single tokens through it.
"""
import contextlib
import threading

import torch

from . import binding as ig

_DATA = {torch.float32: ig.IGC_DATA_FLOAT, torch.bfloat16: ig.IGC_DATA_BFLOAT16}


def _desc(t):
    return ig.TensorDescriptor().set(_DATA[t.dtype], t.shape[0], t.shape[1], 1, 1, (t.stride(0), 1, 1, 1))


class _Buffers:
    """What a batch of M tokens needs.  keep: also the forward pass's results that the backward pass reads, and the gradients."""

    def __init__(self, block, M, keep):
        D, H, dt, dev = block.width, block.hidden, block.dtype, block.w1.device
        new = lambda n, dtype=dt: torch.empty(M, n, dtype=dtype, device=dev)
        self.h, self.a, self.y = new(D), new(H), new(D)
        self.narrow, self.wide = _desc(self.h), _desc(self.a)         # rows of D, rows of H
        hd, w1, w2 = block.handle, block.w1_desc, block.w2_desc
        sizes = [ig.get_linear_forward_workspace_size(hd, self.narrow, w1, self.wide),
                 ig.get_linear_forward_workspace_size(hd, self.wide, w2, self.narrow)]
        if keep:
            self.x = None                                               # the rows that the results are of
            self.z, self.dz, self.dh, self.dx = new(H), new(H), new(D), new(D)
            self.mean, self.invstd = (torch.empty(M, device=dev) for _ in range(2))
            sizes += [ig.get_linear_backward_data_workspace_size(hd, w2, self.narrow, self.wide),
                      ig.get_linear_backward_data_workspace_size(hd, w1, self.wide, self.narrow),
                      ig.get_linear_backward_filter_workspace_size(hd, self.narrow, self.wide, block.dw1_desc),
                      ig.get_linear_backward_filter_workspace_size(hd, self.wide, self.narrow, block.dw2_desc),
                      ig.get_layer_norm_backward_workspace_size(hd, self.narrow, self.narrow, self.narrow)]
        self.room = max(sizes)                                          # (calls of one stream follow each other: one workspace for all)
        self.ws = torch.empty(max(self.room, 16), dtype=torch.uint8, device=dev)
        self.tensors = [t for t in vars(self).values() if isinstance(t, torch.Tensor)]
        self.stream = torch.cuda.current_stream()                       # that they are allocated on
        self.captured = False                                           # a graph may read and write them at any time


class FeedForward:
    """Weights of the compute type, float master gradients.

    Calls run on the current stream of the weights' device.  Buffers, workspace and gradients are shared: a call on another stream than the call
    before first waits for what that stream holds by then, its reads of results included.  (Not while a graph is captured: its replays among
    other calls are the caller's to order.)  Calls from several threads are made one after the other; a result is the next call's to overwrite
    all the same, and a backward pass belongs to the last forward pass, whoever made it.

    sizes: buffers are kept for so many numbers of tokens, passes with and without gradient counted apart; those not used for longest go, a pending
    backward pass with them.  Buffers that were used while a graph was captured stay for the block's life, which has to be the graph's."""

    EPS = 1e-5

    def __init__(self, width, hidden, dtype=torch.bfloat16, device="cuda", seed=0, sizes=16):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda k, c: (torch.randn(k, c, generator=g, device=device) / c ** 0.5).to(dtype)
        self.width, self.hidden, self.dtype, self.sizes = width, hidden, dtype, max(1, sizes)
        self.w1, self.w2 = rand(hidden, width), rand(width, hidden)
        self.b1, self.b2 = torch.zeros(hidden, device=device), torch.zeros(width, device=device)
        self.scale, self.shift = torch.ones(width, device=device), torch.zeros(width, device=device)
        self.handle = ig.Handle()
        filt = lambda t, dt: ig.FilterDescriptor().set(dt, t.shape[0], t.shape[1], 1, 1)
        self.w1_desc, self.w2_desc = filt(self.w1, _DATA[dtype]), filt(self.w2, _DATA[dtype])
        self.dw1_desc, self.dw2_desc = filt(self.w1, ig.IGC_DATA_FLOAT), filt(self.w2, ig.IGC_DATA_FLOAT)
        like = lambda t: torch.zeros(t.shape, device=device)
        self.grads = {n: like(getattr(self, n)) for n in ("w1", "b1", "w2", "b2", "scale", "shift")}
        self._buffers, self._lock = {}, threading.RLock()
        self._stream = torch.cuda.current_stream(self.w1.device) if self.w1.is_cuda else None      # of the last call; the weights are made on it

    def _check(self, name, t, rows=None):
        """Rows as the library's functions read them; they are not told more than the distance between rows."""
        if t.dim() != 2 or t.shape[1] != self.width or t.stride(1) != 1 or t.dtype != self.dtype or rows not in (None, t.shape[0]):
            raise ValueError("%s: %srows of %d adjacent features of type %s" % (name, "" if rows is None else "%d " % rows, self.width, self.dtype))
        if t.device != self.w1.device:
            raise ValueError("%s: on the weights' device, %s" % (name, self.w1.device))

    @contextlib.contextmanager
    def _call(self, x, dy=None):
        """The arguments checked; the block for one call at a time, on its device."""
        self._check("x", x)
        if dy is not None:
            self._check("dy", dy, x.shape[0])
        if not self.w1.is_cuda:
            raise ValueError("the block's calls need its weights on a GPU")
        with self._lock, torch.cuda.device(self.w1.device):
            yield

    def _use(self, x, keep=True):
        """The buffers for x, with the handle on the current stream and that behind the calls before."""
        stream = torch.cuda.current_stream()
        captured = torch.cuda.is_current_stream_capturing()
        if not captured:
            if stream != self._stream:
                stream.wait_stream(self._stream)
            self._stream = stream
        self.handle.set_stream(stream.cuda_stream)
        size = x.shape[0], keep
        b = self._buffers.pop(size, None) or _Buffers(self, *size)
        self._buffers[size] = b                  # (the last one used at the end)
        if captured:
            b.captured = True
        else:
            others = [k for k, v in self._buffers.items() if not v.captured]
            for k in others[:max(0, len(others) - self.sizes)]:
                del self._buffers[k]
        if not captured and stream != b.stream:
            for t in b.tensors:
                t.record_stream(stream)      # (memory of another stream's: not given away before this one is done with it)
        return b

    def forward(self, x, keep=True):
        """The block's result (a buffer of the block, overwritten by the next call with as many tokens and the same ``keep``).  keep: for ``backward``; x
        is held until the next such call and has to stay as it is until then.  Without, nothing that ``backward`` reads is touched."""
        with self._call(x):
            return self._forward(x, keep)

    def _forward(self, x, keep):
        b, hd, xd = self._use(x, keep=keep), self.handle, _desc(x)
        mean, invstd, z = (t.data_ptr() for t in (b.mean, b.invstd, b.z)) if keep else (0, 0, 0)
        if keep:
            if x.untyped_storage().data_ptr() == b.y.untyped_storage().data_ptr():
                raise ValueError("x: the block's own result buffer, which this pass would overwrite, and backward reads x; clone it")
            b.x = None
        ig.check(ig.layer_norm_forward(hd, 1.0, xd, x.data_ptr(), self.scale.data_ptr(), self.shift.data_ptr(), self.EPS, 0.0, b.narrow,
                                       b.h.data_ptr(), mean, invstd), "igcLayerNormForward")
        ig.check(ig.linear_forward(hd, 1.0, b.narrow, b.h.data_ptr(), self.w1_desc, self.w1.data_ptr(), b.ws.data_ptr(), b.room, self.b1.data_ptr(),
                                   ig.IGC_ACTIVATION_GELU, 0.0, None, 0, b.wide, z, b.a.data_ptr()), "igcLinearForward")
        ig.check(ig.linear_forward(hd, 1.0, b.wide, b.a.data_ptr(), self.w2_desc, self.w2.data_ptr(), b.ws.data_ptr(), b.room, self.b2.data_ptr(),
                                   ig.IGC_ACTIVATION_IDENTITY, 1.0, xd, x.data_ptr(), b.narrow, 0, b.y.data_ptr()), "igcLinearForward")
        if keep:
            b.x = x
        return b.y

    def backward(self, x, dy, accumulate=False):
        """Gradient with respect to x, given that with respect to the result (dy: laid out in rows as x is, any distance apart) of the last forward pass
        that kept its results for as many tokens, which has to have been of these rows, in this place; ``grads`` receives (accumulate: is
        increased by) the parameters' gradients."""
        with self._call(x, dy):
            return self._backward(x, dy, accumulate)

    def _backward(self, x, dy, accumulate):
        b, hd, xd, dyd = self._use(x), self.handle, _desc(x), _desc(dy)
        if b.x is None or (b.x.data_ptr(), b.x.stride()) != (x.data_ptr(), x.stride()):
            raise ValueError("backward: the last forward pass of %d tokens that kept its results was not of these rows" % x.shape[0])
        g, keep = {n: t.data_ptr() for n, t in self.grads.items()}, 1.0 if accumulate else 0.0
        ws, room = b.ws.data_ptr(), b.room
        ig.check(ig.linear_backward_filter(hd, 1.0, b.wide, b.a.data_ptr(), dyd, dy.data_ptr(), ws, room, keep, self.dw2_desc, g["w2"], g["b2"]),
                 "igcLinearBackwardFilter")
        ig.check(ig.linear_backward_data(hd, 1.0, self.w2_desc, self.w2.data_ptr(), dyd, dy.data_ptr(), ws, room, ig.IGC_ACTIVATION_GELU, b.wide,
                                         b.z.data_ptr(), 0.0, None, 0, b.wide, b.dz.data_ptr()), "igcLinearBackwardData")
        ig.check(ig.linear_backward_filter(hd, 1.0, b.narrow, b.h.data_ptr(), b.wide, b.dz.data_ptr(), ws, room, keep, self.dw1_desc, g["w1"], g["b1"]),
                 "igcLinearBackwardFilter")
        ig.check(ig.linear_backward_data(hd, 1.0, self.w1_desc, self.w1.data_ptr(), b.wide, b.dz.data_ptr(), ws, room, ig.IGC_ACTIVATION_IDENTITY,
                                         None, 0, 0.0, None, 0, b.narrow, b.dh.data_ptr()), "igcLinearBackwardData")
        ig.check(ig.layer_norm_backward(hd, 1.0, xd, x.data_ptr(), b.narrow, b.dh.data_ptr(), self.scale.data_ptr(), b.mean.data_ptr(),
                                        b.invstd.data_ptr(), ws, room, 1.0, dyd, dy.data_ptr(), b.narrow, b.dx.data_ptr(), keep, g["scale"],
                                        g["shift"]), "igcLayerNormBackward")
        return b.dx


def main(width=512, hidden=2048, tokens=1000, steps=20, rate=0.02):
    block = FeedForward(width, hidden)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(tokens, width, generator=g, device="cuda").to(block.dtype)
    target = torch.randn(tokens, width, generator=g, device="cuda")
    master = {n: getattr(block, n).float() for n in block.grads}
    loss = None
    for step in range(steps):
        d = block.forward(x).float() - target
        loss = float((d * d).mean())
        block.backward(x, (d * (2.0 / tokens)).to(block.dtype))
        for n, w in master.items():
            w -= rate * block.grads[n]
            getattr(block, n).copy_(w)
        if step % 5 == 0 or step == steps - 1:
            print("step %2d: mean squared error %.4f" % (step, loss), flush=True)
    whole = block.forward(x).clone()
    one = torch.cat([block.forward(x[i:i + 1], keep=False).clone() for i in range(4)])
    print("single tokens, largest difference from the batch: %.4f" % float((one.float() - whole[:4].float()).abs().max()))


if __name__ == "__main__":
    main()
