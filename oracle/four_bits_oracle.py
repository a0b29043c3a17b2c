"""Filters in four bits, in 64 bits (include/igconv.h, igcQuantizeFilter4)."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bfloat16_not_below(x):
    """The smallest number of eight significant bits not below x >= 0 (within bfloat16's normal range; its steps below that)."""
    x = np.asarray(x, dtype=np.float64)
    e = np.floor(np.log2(np.where(x > 0, x, 1.0)))
    e = np.where(2.0 ** e > x, e - 1, np.where(2.0 ** (e + 1) <= x, e + 1, e)) if x.any() else e
    step = 2.0 ** np.maximum(e - 7, -133)
    return np.where(x > 0, np.ceil(x / step) * step, 0.0)


def quantize(w, group):
    """(codes K x C, scales groups x K) of w (float64, K x C)."""
    K, C = w.shape
    codes, scales = np.zeros((K, C), np.uint8), []
    for c in range(0, C, group):
        part = w[:, c:c + group]
        s = bfloat16_not_below(np.abs(part).max(1) / 6)
        scales.append(s)
        far = np.abs(np.abs(part)[:, :, None] - s[:, None, None] * VALUES)
        near = far.min(2, keepdims=True)
        code = np.argmax((far == near) * np.where(np.arange(8) % 2 == 0, 2, 1), axis=2)     # (of two as near the even one)
        code = np.where(s[:, None] > 0, code, 0)
        codes[:, c:c + group] = code + np.where((part < 0) & (code > 0), 8, 0)
    return codes, np.array(scales)


def values(codes, scales, group):
    v = np.concatenate([VALUES, -VALUES])[codes]
    return v * np.repeat(scales, group, axis=0)[:codes.shape[1]].T


def pack(codes):
    K, C = codes.shape
    blocks = -(-C // 128)
    out = np.zeros((K, blocks * 64), np.uint8)
    for c in range(C):
        block, i, g, e = c // 128, c % 128 // 32, c % 32 // 8, c % 8
        out[:, block * 64 + (4 * g + i) * 4 + e // 2] |= codes[:, c] << (4 * (e % 2))
    return out
