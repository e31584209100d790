"""Paged attention where its number formats end, against the definition in 64 bits: queries near the largest number over an 8-bit cache, weights far below the largest one, soft-caps of any size.

Bounds (u = 2^-24, half a step of fp32), beside what tests/kv.py derives:
  queries over 8 bits  an element enters as a multiple of 2^-21 of a power of two that is at most its row's largest, max: off by at most 2^-22 max.  A score: 2^-22 |alpha| max sum|k|, and its
                       factor (alpha, power of two, scale, log2 e) is rounded four times: 4 u of itself (inside 8 u peak).
  weights              over 8 bits as there; fp16 over 16 bits: the largest is held as 2^7, and fp16's steps end at 2^-24, so the two parts together are off by up to 2^-25: 2^-32 of the largest weight,
                       2^-32 max|v| for each position.
  soft-cap             relative to the score: 16 u (both of its branches are below 2^-21 = 8 u of it, and its argument is rounded three times).
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from tests import kv, parity as P
from tests.test_gpu_paged_attention import TYPES, Call

pytestmark = pytest.mark.gpu

FORMS = [(1, 8, 2, 128), (3, 4, 1, 64), (5, 5, 1, 256), (8, 8, 1, 128)]   # new tokens, query heads, key heads, D: 4 .. 64 query rows
MAX_BF16 = torch.finfo(torch.bfloat16).max


def check(c):
    """As Call.check, with the bounds above (the soft-cap's in place of one that is relative to the cap)."""
    quantized, dtype = c.cache.quantized, c.out.dtype
    q, keys = kv.f64(c.q), c.cache.values("k")
    want, lse, weight = orc.attention(q, keys, c.cache.values("v"), c.table, c.lengths, c.alpha, c.cap, None if c.slopes is None else kv.f64(c.slopes), c.window)
    ds = np.zeros_like(lse)
    if quantized:
        held = np.abs(np.nan_to_num(keys)).sum(-1).max()
        ds += 2.0 ** -22 * abs(c.alpha) * np.abs(q).max(-1) * held
    if c.cap:
        ds += 16 * kv.U * weight[1]
    bound, lse_bound = kv.attention_bounds(want, lse, weight, int(c.lengths.max()), c.D, dtype, quantized)
    small = c.lengths.max() * 2.0 ** -32 * weight[3] if dtype == torch.float16 and not quantized else np.zeros_like(lse)
    bound = bound + (1 + kv.half_step(dtype)) * (2 * ds[..., None] * weight[0] + small[..., None])
    got, got_lse, seen = kv.f64(c.out), kv.f64(c.lse), np.isfinite(lse)
    assert np.isfinite(got).all() and np.array_equal(np.isfinite(got_lse), seen)
    assert np.all(np.abs(got_lse - lse)[seen] <= (lse_bound + ds)[seen])
    worst = np.max(np.abs(got - want) / bound)
    assert worst <= 1, worst


@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("T,Hq,H,D", FORMS)
@pytest.mark.parametrize("largest", [2.0 ** 125, 2.0 ** 126, 1.9921875 * 2.0 ** 126, 2.0 ** 127, 1.5 * 2.0 ** 127, MAX_BF16])
def test_large_queries_over_8_bits(largest, T, Hq, H, D, cap, cuda_device):
    """A row's largest elements, of both signs, up to the type's largest number; alpha brings the scores back."""
    c = Call([300, 45, 64], T, Hq, H, D, 16, "bf16", True, cuda_device, seed=D, alpha=2.0 ** -126, cap=cap)
    x = kv.f64(c.q)
    x /= np.abs(x).max(-1, keepdims=True)
    x[..., 7::16], x[..., 3::16] = 1, -1
    c.q.copy_(torch.from_numpy((x * largest).astype(np.float32)).to(cuda_device))   # (exact: the rounding to bf16 is the copy's)
    assert c.q.abs().max() == largest
    for side in "kv":   # codes up to 127 with scales of about 2^-7
        scale = c.cache.ks if side == "k" else c.cache.vs
        scale.mul_(2.0 ** torch.round(-torch.log2(scale) - 7))
    c.run()
    check(c)


def test_an_outlying_query_element_over_8_bits(cuda_device):
    """One element 2^15 times as large as the others meets keys that are zero there."""
    for name in ("bf16", "f16"):
        c = Call([300, 45], 1, 8, 2, 128, 16, name, True, cuda_device, seed=3)
        c.q[..., 5] = 2.0 ** 15
        c.cache.k[..., 5] = 0
        c.run()
        check(c)


@pytest.mark.parametrize("name,quantized", TYPES)
@pytest.mark.parametrize("T,Hq,H,D", FORMS)
@pytest.mark.parametrize("gap", [10.0, 13.0, 15.0, 16.5, 18.0])
def test_small_weights_behind_a_dominating_position(gap, T, Hq, H, D, name, quantized, cuda_device):
    """The first position outweighs each other by e^gap, and its value is zero: thousands of small like weights are the output.  As many sequences as give a CTA whole ones, so that a
    warp that holds the first position holds a quarter of the others or more; all of them on the same pages."""
    n, B = 3000, 320
    c = Call([n], T, Hq, H, D, 16, name, quantized, cuda_device, seed=1, alpha=1.0)
    where = [torch.from_numpy(x).to(cuda_device) for x in (c.table[0, np.arange(n) // 16].astype(np.int64), np.arange(n) % 16)]
    g = torch.Generator(device=cuda_device).manual_seed(2)
    keys, values = torch.zeros(n, H, D, device=cuda_device), 1 + 0.25 * torch.rand(n, H, D, device=cuda_device, generator=g)
    keys[0, :, 0] = 1.0
    values[0] = 0
    c.cache.put("k", *where, keys)
    c.cache.put("v", *where, values)
    c.q = torch.zeros(B, T, Hq, D, dtype=c.q.dtype, device=cuda_device)
    c.q[..., 0] = gap
    c.out, c.lse = P.guarded((B, T, Hq, D), c.q.dtype, -77.0, cuda_device), P.guarded((B, T, Hq), torch.float32, -77.0, cuda_device)
    c.device_table, c.device_lengths = c.device_table.repeat(B, 1), c.device_lengths.repeat(B)
    c.run()
    some = [0, 1, B // 2, B - 1]
    c.q, c.out, c.lse, c.table, c.lengths = c.q[some], c.out[some], c.lse[some], c.table.repeat(4, 0), c.lengths.repeat(4)
    check(c)


@pytest.mark.parametrize("name,quantized", TYPES)
@pytest.mark.parametrize("T,Hq,H,D", FORMS[:2] + FORMS[3:])
@pytest.mark.parametrize("cap", [1e-40, 1e-30, 0.5, 6.0, 30.0, 3000.0, 1e5, 1e7, 1e8, 1e20, 3e38])
def test_caps_of_all_sizes(cap, T, Hq, H, D, name, quantized, cuda_device):
    c = Call([400, 0, 33, 129], T, Hq, H, D, 24, name, quantized, cuda_device, seed=D, cap=cap, scale=3.0, slopes=T == 3)
    c.run()
    check(c)
