"""The 8-bit integer layers in fp64 numpy: the definitions written out, no code shared with the GPU library."""
from __future__ import annotations

import numpy as np


def quantize(x, residual=None, gamma=None, eps=None):
    """(h, y, scale, y / scale) of rows; ``eps`` None: without the norm (y = x).  The codes are y / scale rounded to the nearest whole
    number; a row of zeros has scale 0 and codes 0."""
    h = x if residual is None else x + residual
    y = h
    if eps is not None:
        y = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
        if gamma is not None:
            y = y * gamma
    scale = np.abs(y).max(-1) / 127.0
    with np.errstate(divide="ignore", invalid="ignore"):
        v = np.where(scale[:, None] > 0, 127.0 * y / np.abs(y).max(-1, keepdims=True), 0.0)
    return h, y, scale, v


def activate(z, name):
    if name in (None, "none"):
        return z
    if name == "relu":
        return np.where(z > 0, z, 0.0)
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (z + 0.044715 * z ** 3)))
    if name == "tanh":
        return np.tanh(z)
    assert name == "sigmoid"
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z))


def gemm(A, scale_a, B, scale_b, bias=None, residual=None, activation=None):
    """(result, scaled product) of [.., M, K] by [.., N, K] whole numbers (exact in fp64: at most 2^31)."""
    t = (A @ np.swapaxes(B, -1, -2)) * scale_a[..., :, None] * scale_b[..., None, :]
    y = activate(t if bias is None else t + bias, activation)
    return (y if residual is None else y + residual), t
