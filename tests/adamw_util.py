"""Tensors of an optimiser's step at odd places in buffers full of guards."""
import numpy as np
import torch

import paper_1410_0759_amd as ig

DATA = {torch.float32: ig.IGC_DATA_FLOAT, torch.bfloat16: ig.IGC_DATA_BFLOAT16}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GUARD = 0x5A


class Array:
    """n elements, `lead` elements behind a 256-byte boundary, guard bytes around."""

    def __init__(self, n, dtype, lead=0, values=None):
        size = torch.empty(0, dtype=dtype).element_size()
        self.buf = torch.full((lead * size + n * size + 512,), GUARD, dtype=torch.uint8, device="cuda")
        self.bytes = self.buf[lead * size:lead * size + n * size]
        self.at, self.n = lead * size, n
        self.t = self.bytes.view(dtype) if lead * size % 4 == 0 or size < 4 else None
        if values is not None and n:
            self.put(values, dtype)
        self.dtype = dtype

    def put(self, values, dtype):
        self.bytes.copy_(torch.from_numpy(np.ascontiguousarray(values)).to(dtype).cuda().view(torch.uint8))

    @property
    def ptr(self):
        return self.bytes.data_ptr()

    def numpy(self):
        torch.cuda.synchronize()
        assert bool((self.buf[:self.at] == GUARD).all()) and bool((self.buf[self.at + self.bytes.numel():] == GUARD).all()), "store outside the tensor"
        return self.bytes.clone().view(self.dtype).double().cpu().numpy()


class Tensor:
    """One tensor of the list, with its inputs as float64."""

    def __init__(self, rng, n, param="f32", grad="f32", bits=32, copy=False, decay=0.1, lead=0, fresh=False):
        self.n, self.bits, self.decay = n, bits, decay
        size = np.exp(rng.standard_normal(n))
        self.p = Array(n, TYPES[param], lead, rng.standard_normal(n) * 0.5)
        self.g = Array(n, TYPES[grad], lead, rng.standard_normal(n) * size)
        self.copy = Array(n, torch.bfloat16, lead) if copy else None
        blocks = -(-n // 256)
        m, v = (np.zeros(n), np.zeros(n)) if fresh else (0.3 * rng.standard_normal(n) * size, size ** 2 * (0.5 + rng.random(n)))
        if bits == 8:
            from oracle import adamw_oracle as ao
            self.ms, self.vs = (Array(blocks, torch.float32, lead, ao.scales(x, f)) for x, f in ((m, ao.E4M3), (v, ao.E5M2)))
            per = lambda a: np.repeat(a.numpy(), 256)[:n]
            quotient = lambda x, s: np.divide(x, s, out=np.zeros(n), where=s > 0)
            self.m = Array(n, torch.float8_e4m3fn, lead, np.clip(quotient(m, per(self.ms)), -448, 448))
            self.v = Array(n, torch.float8_e5m2, lead, np.clip(quotient(v, per(self.vs)), 0, 57344))
        else:
            self.ms = self.vs = None
            self.m, self.v = Array(n, torch.float32, lead, m), Array(n, torch.float32, lead, v)

    def arrays(self):
        return [a for a in (self.p, self.g, self.copy, self.m, self.v, self.ms, self.vs) if a is not None]

    def states(self):
        m, v = self.m.numpy(), self.v.numpy()
        if self.bits == 8:
            m, v = m * np.repeat(self.ms.numpy(), 256)[:self.n], v * np.repeat(self.vs.numpy(), 256)[:self.n]
        return m, v

    def entry(self, q):
        ptr = lambda a: 0 if a is None or self.n == 0 else a.ptr
        q.param, q.grad, q.copy, q.m, q.v, q.m_scale, q.v_scale = (ptr(a) for a in (self.p, self.g, self.copy, self.m, self.v, self.ms, self.vs))
        q.count, q.weight_decay, q.param_type, q.grad_type, q.state_bits = self.n, self.decay, DATA[self.p.dtype], DATA[self.g.dtype], self.bits


def table(tensors):
    t = (ig.AdamWTensor * len(tensors))()
    for q, x in zip(t, tensors):
        x.entry(q)
    return t
