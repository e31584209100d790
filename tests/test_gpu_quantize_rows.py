"""Rows to int8 with a scale each (comfuse_quantize_rows), alone and behind a residual addition and an RMSNorm, against fp64: types, row
lengths around the chunk, warp, CTA and cluster sizes, padded leading dimensions, in place, rows of zeros, with infinities, NaNs,
subnormal and huge values, streams and captured graphs."""
import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import q8_oracle as orc
from tests import q8

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _check(x, q, scale, dtype, residual=None, gamma=None, h=None, values=None, norm=True, label=""):
    f = lambda t: None if t is None else q8.f64(t)  # noqa: E731
    ref_h, _, ref_s, v = orc.quantize(f(x), f(residual), f(gamma), EPS if norm else None)
    s, c = f(scale), f(q)
    assert np.all(np.abs(s - ref_s) <= (q8.SCALE_TOL_NORM if norm else q8.SCALE_TOL_PLAIN) * ref_s + 2.0 ** -149), label
    assert np.all(np.abs(c - v) <= q8.CODE_TOL), (label, np.abs(c - v).max())
    assert np.abs(c).max() <= 127
    if h is not None:
        want = (x.float() + residual.float() if residual is not None else x.float()).to(dtype)
        assert torch.equal(h, want), label
    if values is not None:
        assert torch.equal(values, (q.float() * scale[:, None]).to(torch.bfloat16)), label


def _run(M, N, name, norm, residual, gamma, device, seed, extra=0, with_h=True, with_values=True):
    g = np.random.default_rng(seed)
    dtype = q8.TYPES[name]
    x = q8.put(g.standard_normal((M, N)) * g.choice([0.1, 1.0, 20.0], size=(1, N)), dtype, device, extra)
    r = q8.put(g.standard_normal((M, N)), dtype, device, 2 * extra) if residual else None
    w = q8.put(1 + 0.1 * g.standard_normal(N), dtype, device).contiguous() if gamma else None
    h = q8.out((M, N), dtype, device, extra) if norm and with_h else None
    q, v = q8.out((M, N), torch.int8, device, extra), q8.out((M, N), torch.bfloat16, device, extra) if with_values else None
    s = q8.out((M,), torch.float32, device)
    if norm:
        cf.rmsnorm_quantize_rows(x, q, s, residual=r, gamma=w, h=h, values=v, eps=EPS)
    else:
        cf.quantize_rows(x, q, s, values=v)
    torch.cuda.synchronize()
    label = f"{M}x{N} {name} norm={norm} residual={residual} gamma={gamma}"
    _check(x, q, s, dtype, r, w, h, v, norm, label)
    q8.check_surroundings({"q": q, "scale": s, "h": h, "values": v}, label)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N", [(1, 1), (1, 7), (3, 8), (5, 9), (2, 255), (130, 256), (4, 257), (7, 511), (3, 1000), (9, 1024), (2, 1025), (33, 1536), (1, 4096), (300, 4096), (2, 4099),
                                 (5, 8191), (301, 8200), (1, 16384), (150, 16385), (3, 32768), (2, 65535), (1, 65536), (75, 65536)])
def test_sizes(M, N, name, cuda_device):
    _run(M, N, name, True, True, True, cuda_device, M + N)
    _run(M, N, name, False, False, False, cuda_device, M + N + 1)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("gamma", [False, True])
@pytest.mark.parametrize("N", [100, 2056])
def test_what_may_be_absent(N, gamma, residual, cuda_device):
    _run(17, N, "bf16", True, residual, gamma, cuda_device, N, extra=3)
    _run(17, N, "f32", True, residual, gamma, cuda_device, N, extra=1, with_h=False, with_values=False)


def test_many_rows(cuda_device):
    _run(70001, 40, "bf16", True, True, True, cuda_device, 5)
    _run(20011, 1032, "f16", False, False, False, cuda_device, 6)


@pytest.mark.parametrize("N", [264, 5000])
@pytest.mark.parametrize("into", ["residual", "x"])
def test_in_place(N, into, cuda_device):
    g = np.random.default_rng(N)
    x, r = (q8.put(g.standard_normal((40, N)), torch.bfloat16, cuda_device) for _ in range(2))
    keep_x, keep_r = x.clone(), r.clone()
    q, s = q8.out((40, N), torch.int8, cuda_device), q8.out((40,), torch.float32, cuda_device)
    h = r if into == "residual" else x
    cf.rmsnorm_quantize_rows(x, q, s, residual=r, h=h, eps=EPS)
    torch.cuda.synchronize()
    _check(keep_x, q, s, torch.bfloat16, keep_r, None, h, None)
    assert torch.equal(x if into == "residual" else r, keep_x if into == "residual" else keep_r)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("N", [40, 1400, 20000])
def test_rows_out_of_the_ordinary(N, norm, cuda_device):
    """Zeros, one element, subnormal and tiny values, huge ones, infinities and NaNs: each in a row of its own, beside ordinary rows."""
    g = np.random.default_rng(N)
    x = g.standard_normal((12, N)).astype(np.float32)
    x[1] = 0.0
    x[2] = 0.0
    x[2, N - 1] = -3.0
    x[3] *= np.float32(1e-40)
    x[4] *= np.float32(1e-37)
    x[5] *= np.float32(1e18 if norm else 1e38) * np.float32(0.5 if norm else 0.02)
    x[6, N // 2] = np.inf
    x[7, 0] = np.nan
    x[8, N - 1] = -np.inf
    x[9] = np.float32(2.0) ** -20
    X = q8.put(x, torch.float32, cuda_device)
    q, s, v = q8.out((12, N), torch.int8, cuda_device), q8.out((12,), torch.float32, cuda_device), q8.out((12, N), torch.bfloat16, cuda_device)
    if norm:
        cf.rmsnorm_quantize_rows(X, q, s, values=v, eps=EPS)
    else:
        cf.quantize_rows(X, q, s, values=v)
    torch.cuda.synchronize()
    bad = [6, 7, 8]
    assert torch.isnan(s[bad]).all() and (q[bad] == 0).all() and torch.isnan(v[bad].float()).all()
    assert s[1] == 0 and (q[1] == 0).all() and (v[1] == 0).all()
    good = [i for i in range(12) if i not in bad and i != 3]
    i = torch.tensor(good, device=cuda_device)
    _check(X[i], q[i], s[i], torch.float32, values=v[i], norm=norm)
    # subnormal values: the codes are exact, the scale is one of fp32's few subnormal numbers (half a step off at most)
    _, _, ref_s, ref_v = orc.quantize(x[3:4].astype(np.float64), eps=EPS if norm else None)
    assert np.all(np.abs(q8.f64(q[3:4]) - ref_v) <= q8.CODE_TOL + (127 * 2.0 ** -149 / np.abs(x[3]).max() if norm else 0))
    assert abs(float(s[3]) - ref_s[0]) <= 2.0 ** -149 + q8.SCALE_TOL_NORM * ref_s[0]
    q8.check_surroundings({"q": q, "scale": s, "values": v})


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("N", [5, 200, 801, 1500, 17000])
def test_rows_that_are_not_finite(N, name, norm, cuda_device):
    """One infinity or NaN, of either sign, at any place of a row, makes that row NaN and no other."""
    g = np.random.default_rng(N)
    M = 40
    x = g.standard_normal((M, N)).astype(np.float32)
    bad = {}
    for i in range(0, M, 3):
        bad[i] = [np.inf, -np.inf, np.nan, -np.nan][(i // 3) % 4]
        x[i, [0, N - 1, N // 2, (i * 37) % N][(i // 12) % 4]] = bad[i]
    X = q8.put(x, q8.TYPES[name], cuda_device)
    q, s, v = q8.out((M, N), torch.int8, cuda_device), q8.out((M,), torch.float32, cuda_device), q8.out((M, N), torch.bfloat16, cuda_device)
    if norm:
        cf.rmsnorm_quantize_rows(X, q, s, values=v, eps=EPS)
    else:
        cf.quantize_rows(X, q, s, values=v)
    torch.cuda.synchronize()
    i = torch.tensor(sorted(bad), device=cuda_device)
    j = torch.tensor([k for k in range(M) if k not in bad], device=cuda_device)
    assert torch.isnan(s[i]).all() and (q[i] == 0).all() and torch.isnan(v[i].float()).all()
    _check(X[j], q[j], s[j], q8.TYPES[name], values=v[j], norm=norm)


@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_the_middle_of_two_codes_goes_to_the_even_one(name, cuda_device):
    """max = 127 / 2^k: the codes of multiples of 2^-k / 2 lie exactly between two whole numbers."""
    x = torch.zeros(8, 256, device=cuda_device)
    x[:, 0] = 127
    x[:, 1:254] = (torch.arange(253, device=cuda_device) - 126) / 2
    x *= 2.0 ** torch.arange(-4, 4, device=cuda_device)[:, None]
    q, s = torch.empty(8, 256, dtype=torch.int8, device=cuda_device), torch.empty(8, device=cuda_device)
    cf.quantize_rows(x.to(q8.TYPES[name]), q, s)
    want = torch.zeros(256, device=cuda_device)
    want[0], want[1:254] = 127, ((torch.arange(253, device=cuda_device) - 126) / 2).round()   # (ties to even)
    assert (q == want).all() and torch.equal(s, 2.0 ** torch.arange(-4, 4, device=cuda_device))


def test_offsets_beyond_32_bits(cuda_device):
    """More than 2^32 bytes of rows: the last ones are read and written where they stand."""
    M, N = 70000, 65536
    x = torch.zeros(M, N, dtype=torch.bfloat16, device=cuda_device)
    q, s = torch.empty(M, N, dtype=torch.int8, device=cuda_device), torch.empty(M, device=cuda_device)
    rows = [0, 32767, 32768, 65535, 65536, M - 1]
    for k in rows:
        x[k] = torch.randn(N, device=cuda_device)
    cf.rmsnorm_quantize_rows(x, q, s, h=x, eps=EPS)
    i = torch.tensor(rows, device=cuda_device)
    _check(x[i], q[i], s[i], torch.bfloat16)
    assert int((s != 0).sum()) == len(rows) and not q[1:32767].any() and not q[65537:M - 1].any()


@pytest.mark.parametrize("N", [1, 40, 500, 3000, 65536])
def test_squares_beyond_fp32(N, cuda_device):
    """Rows whose sum of squares, or whose single squares, leave fp32's range, in every element or in some."""
    g = np.random.default_rng(N)
    x = g.standard_normal((6, N)).astype(np.float32)
    x[0] *= np.float32(1e19)
    x[1] *= np.float32(3e37)
    x[2, N // 2] = np.float32(3e38)
    x[3, N - 1] = np.float32(1e18)
    x[4] = np.float32(2.0 ** 50)
    X = q8.put(x, torch.float32, cuda_device)
    q, s = q8.out((6, N), torch.int8, cuda_device), q8.out((6,), torch.float32, cuda_device)
    cf.rmsnorm_quantize_rows(X, q, s, eps=EPS)
    torch.cuda.synchronize()
    _check(X, q, s, torch.float32)


def test_another_stream_and_a_captured_graph(cuda_device):
    """Calls on a side stream; two captured calls replayed with new data, eager calls of other sizes between the replays."""
    g = np.random.default_rng(3)
    N = 4096
    x, r = (q8.put(g.standard_normal((64, N)), torch.bfloat16, cuda_device) for _ in range(2))
    q, s, h = q8.out((64, N), torch.int8, cuda_device), q8.out((64,), torch.float32, cuda_device), q8.out((64, N), torch.bfloat16, cuda_device)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cf.rmsnorm_quantize_rows(x, q, s, residual=r, h=h, eps=EPS, stream=side)
    side.synchronize()
    _check(x, q, s, torch.bfloat16, r, None, h)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cf.rmsnorm_quantize_rows(x, q, s, residual=r, h=h, eps=EPS)
        cf.quantize_rows(h, q, s)
    for seed in (1, 2):
        x.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal((64, N))))
        _run(3, 1000, "f16", True, True, True, cuda_device, seed)
        graph.replay()
        torch.cuda.synchronize()
        _check(h, q, s, torch.bfloat16, norm=False)


def test_the_binding_finds_the_current_stream(cuda_device):
    b = cf._bound_q8()
    side = torch.cuda.Stream()
    current = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    assert b.stream(current, 0) == current()
    with torch.cuda.stream(side):
        assert b.stream(current, 0) == side.cuda_stream == current()
    assert b.stream(side, 0) == side.cuda_stream
    assert b.stream(current, 0) == current()


def test_the_same_call_gives_the_same_bits(cuda_device):
    g = np.random.default_rng(8)
    x, r = (q8.put(g.standard_normal((200, 9000)), torch.bfloat16, cuda_device) for _ in range(2))
    got = []
    for _ in range(3):
        q, s = q8.out((200, 9000), torch.int8, cuda_device), q8.out((200,), torch.float32, cuda_device)
        cf.rmsnorm_quantize_rows(x, q, s, residual=r)
        got.append((q.clone(), s.clone()))
    for q, s in got[1:]:
        assert torch.equal(q, got[0][0]) and torch.equal(s, got[0][1])
