"""Shared helpers of the tests of the key-value cache: caches in any layout, and the bounds of the outputs.

Bounds (u = 2^-24, half a step of fp32; h = half a step of the output's type relative to it).
  turned rows  the angle is known to 2^-50 of itself in 64 bits; its fraction of a turn is rounded to fp32 (pi u of angle), sine and cosine are off by at most a
               step (2 u), the two products and their sum by 2 u of |a| + |b|: together below 8 u (|a| + |b|), and h at the store.
  8-bit rows   code: 1/2 + 127 * (twice what the row is off, of its maximum, + 5 u).  Turned rows: |a| + |b| <= 2 sqrt(2) max|y|, so 127 * (2 * 2.83 * 8 u + 5 u) < 4e-4.
               scale: 2.83 * 8 u + u < 2^-19 of it.
  attention    a score: D additions of at most 2 u (the matrix instruction may truncate) of sum|alpha q k|, and a handful of roundings of itself: ds = (D + 8) 2 u dot + 8 u peak + 16 u cap.
               a weight: ds ln-wise, 2^-22 of ex2, 2^-21 for the arguments' subtraction (|s| log2(e) up to 8 above the maximum), and its rounding: 2^-18 (bf16 twice), 2^-22 (fp16
               twice), 2^-11 (fp16 once, over 8 bits).  The sum over n positions: a chain of n / 32 + 64 additions of 2 u.  The quotient has the weights' errors twice.
               8 bits: weights are held as fp16 in units of which the largest scale is 64 or more, so one below 2^-14 units, where fp16's steps end, is off by up to 2^-25 units:
               2^-31 of the largest scale, times codes up to 127: 2^-31 max|v| for each position (the sum that they are divided by is 1 or more).
               lse: ds + 2^-20 + 4 u |lse|.
"""
from __future__ import annotations

import numpy as np
import torch

from tests import parity as P

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24
CODE_TOL_TURNED, SCALE_TOL_TURNED = 0.5 + 4e-4, 2.0 ** -19


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def half_step(t):
    return torch.finfo(t).eps / 2


def turned_bound(y, x, pairs, adjacent, angle, t):
    """Of rotary rows y, from x (both [tokens, heads, D]); t: the type that they were rounded to, or None."""
    size = np.zeros_like(y)
    first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if adjacent else (slice(0, pairs), slice(pairs, 2 * pairs))
    both = np.abs(x[..., first]) + np.abs(x[..., second])
    off = 8 * U + np.abs(angle)[:, None, :] * 2.0 ** -50
    size[..., first] = size[..., second] = both * off
    return size if t is None else size * (1 + half_step(t)) + half_step(t) * np.abs(y) + torch.finfo(t).smallest_normal * half_step(t)


def raw_angle(positions, freqs, sections):
    positions = np.atleast_2d(np.asarray(positions))
    return positions[np.repeat(np.arange(len(sections)), sections)].T * np.asarray(freqs)


def attention_bounds(out, lse, weight, n, D, dtype, quantized, softcap=0.0):
    mass, peak, dot, most = weight
    ds = ((D + 8) * 2 * U * dot + 8 * U * peak + 16 * U * softcap)
    rounding = 2.0 ** -11 if quantized and dtype == torch.bfloat16 else 2.0 ** -18 if dtype == torch.bfloat16 else 2.0 ** -22
    each = 2 * (ds + 2.0 ** -22 + 2.0 ** -21) + rounding + (n / 32 + 64) * 2 * U
    small = n * 2.0 ** -31 * most if quantized else 0 * most
    bound = (1 + half_step(dtype)) * (each[..., None] * mass + small[..., None]) + half_step(dtype) * np.abs(out) + torch.finfo(dtype).smallest_normal * half_step(dtype)
    return bound, ds + 2.0 ** -20 + 4 * U * np.abs(np.where(np.isfinite(lse), lse, 0))


class Cache:
    """A cache inside canaries, in one of several layouts, full of what must not matter (NaN, or large codes with NaN scales)."""

    def __init__(self, pages, heads, page, D, name, quantized, device, layout="heads first"):
        self.page, self.quantized, self.t = page, quantized, TYPES[name]
        held = torch.int8 if quantized else self.t

        def make(dtype, fill, last):
            if layout == "heads first":
                base = P.guarded((pages, heads, page, *last), dtype, fill, device)
                t = base
            elif layout == "rows first":        # [pages, page, heads, D]
                base = P.guarded((pages, page, heads, *last), dtype, fill, device)
                t = base.transpose(1, 2)
            else:                               # "padded": rows of a wider allocation
                base = P.guarded((pages, heads, page + 1, *[n + 16 for n in last]), dtype, fill, device)
                t = base[:, :, :page] if not last else base[:, :, :page, 16:]
            t._base_tensor = base
            return t

        self.k, self.v = (make(held, -128 if quantized else float("nan"), (D,)) for _ in "kv")
        self.ks, self.vs = (make(torch.float32, float("nan"), ()) if quantized else None for _ in "kv")

    def tensors(self):
        return {"k": self.k, "v": self.v, "k_scale": self.ks, "v_scale": self.vs}

    def scales(self):
        return {"k_scale": self.ks, "v_scale": self.vs}

    def check_canaries(self, label=""):
        for name, t in self.tensors().items():
            if t is not None:
                P.check_canaries({name: t._base_tensor}, label)

    def put(self, side, page, row, values, g=None):
        """Values [n, heads, D] into rows of pages; 8 bits: as codes with scales.  Returns what is held, in 64 bits."""
        cache, scale = (self.k, self.ks) if side == "k" else (self.v, self.vs)
        if not self.quantized:
            cache[page, :, row] = values.to(self.t)
            return f64(cache[page, :, row])
        s = values.abs().amax(-1) / 127
        codes = (values / s[..., None].clamp_min(1e-30)).round().to(torch.int8)
        cache[page, :, row] = codes
        scale[page, :, row] = s
        return f64(codes) * f64(s)[..., None]

    def values(self, side):
        """What the cache's rows stand for, in 64 bits [pages, heads, page, D]."""
        cache, scale = (self.k, self.ks) if side == "k" else (self.v, self.vs)
        return f64(cache) if scale is None else f64(cache) * f64(scale)[..., None]
