"""An AdamW step in 64 bits, and what its states in 8 bits stand for (include/igconv.h, igcAdamWStep)."""
import numpy as np

BLOCK = 256
# (largest number, bits behind the leading one, smallest normal number, the steps below it, least of what is not zero)
E4M3 = (448.0, 3, 2.0 ** -6, 2.0 ** -9, 0.0)
E5M2 = (57344.0, 2, 2.0 ** -14, 2.0 ** -16, 2.0 ** -16)


def step(p, g, m, v, t, rate, beta1, beta2, epsilon, decay, scale=1.0):
    """(p, m, v) after the step t; all float64."""
    g = scale * g
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - rate * decay) - rate * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + epsilon), m, v


def hashed(x):
    x = np.asarray(x, dtype=np.uint64)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x7FEB352D)) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x846CA68B)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(n, seed, t, first=0):
    """16 bits for each element of m, and of v, from the element `first` on."""
    i = np.arange(first, first + n, dtype=np.uint64)
    i = (i & np.uint64(0xFFFFFFFF)) ^ (((i >> np.uint64(32)) * np.uint64(0x9E3779B9)) & np.uint64(0xFFFFFFFF))
    r = hashed(i ^ hashed(np.uint64(seed) ^ hashed(np.uint64(t))))
    return (r & np.uint64(0xFFFF)).astype(np.float64), (r >> np.uint64(16)).astype(np.float64)


def scales(x, form):
    """Of blocks of 256, over the finite elements."""
    padded = np.zeros(-(-len(x) // BLOCK) * BLOCK)
    padded[:len(x)] = np.where(np.isfinite(x), np.abs(x), 0.0)
    s = padded.reshape(-1, BLOCK).max(1) / form[0]
    return np.where(s < 2.0 ** -100, 0.0, s)


def rounded(y, form, random):
    """y in units of its scale, to the format: up by 16 random bits."""
    most, kept, least, tiny, floor = form
    a = np.abs(y)
    unit = 2.0 ** (np.floor(np.log2(np.where(a > 0, a, 1.0))) - kept)
    r = unit * np.floor(a / unit + random / 65536)
    r = np.where(r < least, np.round(r / tiny) * tiny, np.minimum(r, most))
    return np.copysign(np.where(a > 0, np.maximum(r, floor), 0.0), y)
