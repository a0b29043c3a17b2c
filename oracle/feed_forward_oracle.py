"""Layer norm and the matrix products of a feed-forward block in 64 bits, straight from their formulas (numpy, matrices of
rows).  TEST INFRASTRUCTURE ONLY."""
import math

import numpy as np

IDENTITY, SIGMOID, RELU, TANH, GELU, SILU = -1, 0, 1, 2, 3, 4
ACTIVATIONS = {"none": IDENTITY, "sigmoid": SIGMOID, "relu": RELU, "tanh": TANH, "gelu": GELU, "silu": SILU}

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def layer_norm(x, scale, shift, eps):
    """(y, mean, 1 / deviation)"""
    mean = x.sum(1) / x.shape[1]
    d = x - mean[:, None]
    s = 1 / np.sqrt((d * d).sum(1) / x.shape[1] + eps)
    y = d * s[:, None]
    if scale is not None:
        y = y * scale
    if shift is not None:
        y = y + shift
    return y, mean, s


def layer_norm_backward(x, dy, scale, mean, s):
    """(dx, dscale, dshift) with mean and 1 / deviation as given"""
    h = (x - mean[:, None]) * s[:, None]
    q = dy if scale is None else dy * scale
    dx = s[:, None] * (q - q.mean(1, keepdims=True) - h * (q * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def activation(act, v):
    if act == SIGMOID:
        return 1 / (1 + np.exp(-v))
    if act == RELU:
        return np.maximum(v, 0)
    if act == TANH:
        return np.tanh(v)
    if act == GELU:
        return v * 0.5 * _erfc(-v / math.sqrt(2))
    if act == SILU:
        return v / (1 + np.exp(-v))
    return v


def activation_slope(act, v):
    if act == SIGMOID:
        s = 1 / (1 + np.exp(-v))
        return s * (1 - s)
    if act == RELU:
        return (v > 0).astype(np.float64)
    if act == TANH:
        return 1 - np.tanh(v) ** 2
    if act == GELU:
        return 0.5 * _erfc(-v / math.sqrt(2)) + v * np.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if act == SILU:
        s = 1 / (1 + np.exp(-v))
        return s + v * s * (1 - s)
    return np.ones_like(v)


def linear(x, w, bias, act, r, alpha=1.0, beta=0.0):
    """(y, z)"""
    z = alpha * (x @ w.T)
    if bias is not None:
        z = z + bias
    y = activation(act, z)
    return (y if r is None else y + beta * r), z


def linear_backward_data(dy, w, act, z, r, alpha=1.0, beta=0.0):
    dx = alpha * (dy @ w)
    if act != IDENTITY:
        dx = dx * activation_slope(act, z)
    return dx if r is None else dx + beta * r


def linear_backward_filter(dy, x, alpha=1.0, beta=0.0, dw=None, dbias=None):
    """(dw, dbias); dw and dbias: what they held before"""
    gw, gb = alpha * (dy.T @ x), alpha * dy.sum(0)
    if dw is not None:
        gw, gb = gw + beta * dw, gb + beta * dbias
    return gw, gb
