"""Shared helpers of the tests of the 8-bit integer layers: padded tensors inside canaries, and the bounds of the outputs.

Bounds (u = 2^-24, half a step of fp32; t = scale_a scale_b S the scaled product, S its exact integer sum).
  codes   127 h gamma / max|h gamma|: h, h gamma and the quotient are one rounding each, and max carries two of its element: 5 u of at most 127, in
          front of the rounding to a whole number: |q - v| <= 1/2 + 127 * 5 u.
  scale   without the norm one rounding (the division by 127).  With it: the sum of squares is at most 8 + 4 + 1 + 5 + 16 + 8 additions
          deep (chunk, chunks, the element behind them, lanes, warps, CTAs), with h's rounding twice 44 u, half of that behind the root; mean, + eps,
          the reciprocal root (2 steps of fp32 = 4 u), the maximum (2 u), product, division: 22 + 1 + 1 + 4 + 2 + 1 + 1 = 32 u = 2^-19.
  product S to fp32, its product with scale_b, the fused multiply-add: (2 |t| + |z|) u, z = t + bias.  Activations change that by at most
          1.13 and add: sigmoid (and GELU's) relative 2^-21 (1 + |x|) of sigmoid(x), x GELU's inner argument with 5 u of its own;
          |x| sigmoid(x) <= 0.3 for x < 0 and (1 - sigmoid) takes the place of |x| for x > 0: below |z| 2^-20 in all; tanhf 2 steps.
          tanhf and GELU vanish with z, sigmoid does not: its error near z = 0 is that of ex2 (2^-22), the addition of 1 (2^-24) and rcp
          (2^-23) times sigmoid(z) itself, so |act(z)| belongs to the sum of what the error is proportional to.
          With the residual's addition: 2^-20 (|t| + |bias| + |act| + |residual|), plus half a step of the output's type.
"""
from __future__ import annotations

import numpy as np
import torch

from tests import parity as P

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODE_TOL = 0.5 + 127 * 5 * 2.0 ** -24
SCALE_TOL_PLAIN, SCALE_TOL_NORM = 2.0 ** -24, 2.0 ** -19
SENTINEL = {torch.int8: -128, torch.float32: -77.0, torch.bfloat16: -77.0, torch.float16: -77.0}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def put(a, dtype, device, extra=0):
    """A numpy array as a device tensor whose rows start on 16-byte boundaries (``extra`` more 16-byte units behind each row); what
    stands between the rows is NaN (or a large code): nothing may read it."""
    n, per = a.shape[-1], 16 // torch.empty((), dtype=dtype).element_size()
    t = torch.full((*a.shape[:-1], ((n + per - 1) // per + extra) * per), 127 if dtype == torch.int8 else float("nan"), dtype=dtype, device=device)[..., :n]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a)).to(device))
    return t


def out(shape, dtype, device, extra=0):
    """An output buffer inside canaries, its padding and itself filled with a sentinel."""
    n, per = shape[-1], 16 // torch.empty((), dtype=dtype).element_size()
    base = P.guarded((*shape[:-1], ((n + per - 1) // per + extra) * per), dtype, SENTINEL[dtype], device)
    t = base[..., :n]
    t._base_tensor = base
    return t


def check_surroundings(tensors, label=""):
    """Nothing outside the outputs' elements was written."""
    for name, t in tensors.items():
        if t is None:
            continue
        base = getattr(t, "_base_tensor", t)
        P.check_canaries({name: base}, label)
        pad = base[..., t.shape[-1]:]
        assert bool((pad == SENTINEL[t.dtype]).all()), f"{label}: columns behind {name} were written"


def product_bound(y, t, dtype, bias=None, residual=None):
    act = y if residual is None else y - residual
    size = np.abs(t) + np.abs(act) + (0 if bias is None else np.abs(bias)) + (0 if residual is None else np.abs(residual))
    return (torch.finfo(dtype).eps / 2 + 2.0 ** -24) * np.abs(y) + 2.0 ** -20 * size + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
