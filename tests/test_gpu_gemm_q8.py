"""The int8 product with a scale for each row and channel (comfuse_gemm_q8) against fp64, whose sums are exact: one row to many, every cut
of the form for few rows (groups of 16 to 128 rows, 1 to 8 shares of the contraction) and of the tile kernel, sizes that fit
nothing, batches, types, activations, extreme codes, NaN scales, in place, streams and captured graphs."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import q8_oracle as orc
from tests import q8

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run_case(M, N, K, name, device, batch=None, activation=None, bias=True, residual=True, seed=0, extra=0, in_place=False):
    g = np.random.default_rng(seed)
    dtype = q8.TYPES[name]
    lead = () if batch is None else (batch,)
    a, b = (g.integers(-128, 128, size=(*lead, n, K)) for n in (M, N))
    sa, sb = (np.exp(g.normal(size=(*lead, n))).astype(np.float32) * np.float32(k) for n, k in ((M, 1 / 74), (N, K ** -0.5 / 74)))
    w = q8.put(g.standard_normal(N), dtype, device).contiguous() if bias else None
    r = q8.put(g.standard_normal((*lead, M, N)), dtype, device, extra) if residual else None
    A, B = q8.put(a, torch.int8, device, extra), q8.put(b, torch.int8, device, 2 * extra)
    y = r if in_place else q8.out((*lead, M, N), dtype, device, extra)
    ref_r = None if r is None else q8.f64(r)
    cf.gemm_q8(A, torch.from_numpy(sa).to(device), B, torch.from_numpy(sb).to(device), y, bias=w, residual=r, activation=activation)
    torch.cuda.synchronize()
    label = f"{batch} x {M} x {N} x {K} {name} {activation}"
    ref_b = None if w is None else q8.f64(w)
    ref, t = orc.gemm(a.astype(np.float64), sa.astype(np.float64), b.astype(np.float64), sb.astype(np.float64), ref_b, ref_r, activation)
    off = np.abs(q8.f64(y) - ref) - q8.product_bound(ref, t, dtype, ref_b, ref_r)
    assert off.max() <= 0, (label, off.max(), np.unravel_index(off.argmax(), off.shape))
    if not in_place:
        q8.check_surroundings({"Y": y}, label)


SIZES = [(1, 1, 1), (1, 4096, 4096), (2, 5, 17), (3, 130, 31), (15, 128, 128), (16, 127, 129), (17, 129, 640), (31, 257, 1000), (33, 1000, 2049), (64, 640, 1300), (65, 256, 300), (100, 1001, 700),
         (128, 384, 2056), (129, 200, 515), (200, 1300, 4100), (256, 640, 256), (257, 3, 4), (300, 777, 1032), (513, 1024, 64), (700, 72, 5000), (1000, 1000, 100),
         (100, 128, 1024), (70, 4001, 500), (100, 1030, 8192), (127, 2050, 8200), (250, 120, 3000), (12, 8200, 4100), (8, 20000, 2700), (60, 40000, 260), (90, 300, 20000), (520, 4000, 300), (5000, 100, 700),
         (3000, 1700, 300), (2817, 2001, 131), (40000, 8, 64)]


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_sizes(M, N, K, name, cuda_device):
    run_case(M, N, K, name, cuda_device, seed=M + N + K)


@pytest.mark.parametrize("activation", [None, "relu", "gelu_tanh", "tanh", "sigmoid"])
@pytest.mark.parametrize("M,N,K", [(7, 300, 520), (2900, 1800, 140)])
def test_activations_and_absent_operands(M, N, K, activation, cuda_device):
    for name, bias, residual in (("bf16", True, False), ("f32", False, True), ("f16", False, False), ("f32", True, True)):
        run_case(M, N, K, name, cuda_device, activation=activation, bias=bias, residual=residual, seed=N, extra=1)


@pytest.mark.parametrize("batch,M,N,K", [(1, 5, 40, 64), (3, 1, 1000, 300), (5, 33, 129, 65), (96, 126, 126, 64), (7, 600, 1500, 80), (96, 20, 504, 64),
                                         (60, 50, 520, 300), (30, 40, 1020, 70), (96, 16, 500, 70)])
def test_batches(batch, M, N, K, cuda_device):
    run_case(M, N, K, "f32", cuda_device, batch=batch, seed=batch)
    run_case(M, N, K, "bf16", cuda_device, batch=batch, seed=batch + 1, extra=3, activation="gelu_tanh")


@pytest.mark.parametrize("K", [64, 250, 300, 900, 1200])
def test_rings_and_epilogue_warps_by_the_contraction(K, cuda_device):
    """Tiles of 256 columns in every cut of the ring and of the epilogue: by type, length, residual, activation and the size of the result."""
    for name in ("bf16", "f32"):
        run_case(2900, 1801, K, name, cuda_device, residual=False, seed=K)
        run_case(2817, 1807, K, name, cuda_device, residual=True, seed=K + 1, extra=1)
        run_case(2900, 1799, K, name, cuda_device, residual=True, activation="sigmoid", seed=K + 2)
    run_case(130, 504, K, "f32", cuda_device, batch=96, residual=False, seed=K + 3)
    if K == 64:
        run_case(7001, 4001, K, "f32", cuda_device, residual=False, seed=5)


@pytest.mark.parametrize("M,N,K,batch", [(20, 300, 600, None), (2900, 1800, 140, None), (9, 33, 300, 4)])
def test_in_place(M, N, K, batch, cuda_device):
    run_case(M, N, K, "bf16", cuda_device, batch=batch, in_place=True, extra=1)


@pytest.mark.parametrize("M", [3, 150, 9000])
def test_the_longest_sums_are_exact(M, cuda_device):
    """131071 products of -128 by -128 stay within int32; every other code too."""
    K, N = (131071, 5) if M < 9000 else (4000, 600)
    a, b = torch.full((M, (K + 15) // 16 * 16), 99, dtype=torch.int8, device=cuda_device), torch.full((N, (K + 15) // 16 * 16), 77, dtype=torch.int8, device=cuda_device)
    a[:, :K], b[:, :K] = -128, -128
    b[1, :K] = 127
    ones = lambda n: torch.ones(n, device=cuda_device)  # noqa: E731
    y = torch.empty(M, (N + 3) // 4 * 4, device=cuda_device)[:, :N]
    cf.gemm_q8(a[:, :K], ones(M), b[:, :K], ones(N), y)
    want = torch.full((M, N), float(K * 16384), device=cuda_device)
    want[:, 1] = float(-K * 128 * 127)
    assert torch.equal(y, want)    # (rounded to fp32 once on both sides)


def test_scales_that_are_not_numbers_stay_in_their_rows_and_channels(cuda_device):
    for M in (5, 3000):
        K, N = 256, 1700
        a, b = (torch.randint(-127, 128, (n, K), dtype=torch.int8, device=cuda_device) for n in (M, N))
        sa, sb = torch.ones(M, device=cuda_device), torch.ones(N, device=cuda_device)
        sa[2], sb[3] = float("nan"), float("inf")
        y = torch.empty(M, 1704, device=cuda_device)[:, :N]
        cf.gemm_q8(a, sa, b, sb, y)
        bad = ~torch.isfinite(y)
        assert bad[2].all() and bad[:, 3].all() and torch.isnan(y[2]).all()
        bad[2], bad[:, 3] = False, False
        assert not bad.any()


def test_a_quantised_row_of_nan_gives_a_row_of_nan(cuda_device):
    x = torch.randn(4, 320, device=cuda_device).to(torch.bfloat16)
    x[1, 7] = float("nan")
    x[3] = 0
    q, s = torch.empty(4, 320, dtype=torch.int8, device=cuda_device), torch.empty(4, device=cuda_device)
    cf.quantize_rows(x, q, s)
    w, sw = torch.randint(-127, 128, (24, 320), dtype=torch.int8, device=cuda_device), torch.ones(24, device=cuda_device)
    y = torch.empty(4, 24, dtype=torch.bfloat16, device=cuda_device)
    cf.gemm_q8(q, s, w, sw, y)
    assert torch.isnan(y[1]).all() and (y[3] == 0).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2]).all()


def test_unaligned_views(cuda_device):
    """Operands that start inside a larger tensor, on 16-byte (not 32-byte) boundaries: slices of weights, of a batch, of an output."""
    for M in (24, 3000):
        K, N = 400, 1704
        a, b = (torch.randint(-127, 128, (n, K + 48), dtype=torch.int8, device=cuda_device)[:, 16:16 + K] for n in (M + 3, N))
        a = a[3:]
        sa, sb = torch.rand(M + 3, device=cuda_device)[3:], torch.rand(N, device=cuda_device)
        big = torch.full((M, N + 24), -5.0, dtype=torch.bfloat16, device=cuda_device)
        res = torch.randn(M, N + 8, dtype=torch.bfloat16, device=cuda_device)[:, 8:]
        y = big[:, 8:8 + N]
        cf.gemm_q8(a, sa, b, sb, y, residual=res)
        ref, t = orc.gemm(q8.f64(a), q8.f64(sa), q8.f64(b), q8.f64(sb), None, q8.f64(res))
        assert (np.abs(q8.f64(y) - ref) <= q8.product_bound(ref, t, torch.bfloat16, None, q8.f64(res))).all()
        assert (big[:, :8] == -5).all() and (big[:, 8 + N:] == -5).all()


def test_split_sums_do_not_change_a_bit(cuda_device):
    """Integer sums: the row by itself (8 shares) and among many (no shares) give the same bits."""
    K, N = 4096, 512
    a, b = (torch.randint(-127, 128, (n, K), dtype=torch.int8, device=cuda_device) for n in (9000, N))
    sa, sb = torch.rand(9000, device=cuda_device), torch.rand(N, device=cuda_device)
    y = torch.empty(9000, N, dtype=torch.bfloat16, device=cuda_device)
    cf.gemm_q8(a, sa, b, sb, y, activation="gelu_tanh")
    for M in (1, 16, 40, 100, 200, 600):
        z = torch.empty(M, N, dtype=torch.bfloat16, device=cuda_device)
        cf.gemm_q8(a[:M], sa[:M], b, sb, z, activation="gelu_tanh")
        assert torch.equal(z, y[:M]), M


def test_offsets_beyond_32_bits(cuda_device):
    """A result, and a batch of operands, of more than 2^32 bytes."""
    g = torch.Generator(device=cuda_device).manual_seed(3)
    rand = lambda *s: torch.randint(-127, 128, s, dtype=torch.int8, device=cuda_device, generator=g)  # noqa: E731
    M, N, K = 70000, 33000, 64
    a, b = rand(M, K), rand(N, K)
    sa, sb = torch.rand(M, device=cuda_device, generator=g), torch.rand(N, device=cuda_device, generator=g)
    y = torch.empty(M, N, dtype=torch.bfloat16, device=cuda_device)
    cf.gemm_q8(a, sa, b, sb, y)
    for rows in (slice(0, 3), slice(65000, 65100), slice(M - 50, M)):
        want = (a[rows].double() @ b.double().mT) * sa[rows].double()[:, None] * sb.double()
        assert ((y[rows].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -20)).all()
    del y
    batch, M, N, K = 70, 3, 512, 131056
    a, b = rand(batch, M, K), rand(batch, N, K)
    sa, sb = torch.rand(batch, M, device=cuda_device, generator=g), torch.rand(batch, N, device=cuda_device, generator=g)
    y = torch.empty(batch, M, N, device=cuda_device)
    cf.gemm_q8(a, sa, b, sb, y)
    want = torch.stack([(a[i].double() @ b[i].double().mT) for i in (0, 35, 69)]) * sa[[0, 35, 69], :, None].double() * sb[[0, 35, 69], None].double()
    assert ((y[[0, 35, 69]].double() - want).abs() <= want.abs() * 2.0 ** -20).all()


CHILD = """
import torch
from tests import test_gpu_gemm_q8 as t
import paper_2608_03537_b200 as cf
d = torch.device("cuda:0")
for M, N, K in t.SIZES[:-3]:
    t.run_case(M, N, K, "bf16", d, seed=M)
t.run_case(33, 129, 65, "f32", d, batch=5)
t.run_case(300, 700, 129, "f16", d, activation="tanh", extra=1)
assert cf.last_device_status() == cf.OK
"""


def test_the_tile_kernel_at_small_sizes(cuda_device):
    """With the form for few rows off every size runs on the tile kernel: one tile, partial tiles, short and long contractions."""
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT, COMFUSE_FEW_ROWS="0"), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-3000:]


CHECKED = """
import torch
import paper_2608_03537_b200 as cf
from tests import test_gpu_gemm_q8 as t, test_gpu_quantize_rows as r
assert cf.LIB_PATH.endswith("libcomfuse_checked.so"), cf.LIB_PATH
d = torch.device("cuda:0")
for M, N, K in t.SIZES:
    t.run_case(M, N, K, "bf16", d, seed=M)
    t.run_case(M, N, K, "f32", d, seed=N, activation="gelu_tanh")
for M, N in ((1, 7), (3, 1000), (300, 4099), (5, 65536), (9000, 250)):
    r._run(M, N, "bf16", True, True, True, d, N)
    r._run(M, N, "f32", False, False, False, d, N)
assert cf.last_device_status() == cf.OK
"""


def test_no_bounds_predicate_fails_in_the_checked_build(cuda_device):
    lib = os.path.join(ROOT, "paper_2608_03537_b200", "libcomfuse_checked.so")
    if not os.path.exists(lib):
        from paper_2608_03537_b200 import build
        build.build(checked=True)
    r = subprocess.run([sys.executable, "-c", CHECKED], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT, COMFUSE_LIB=lib), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-3000:]


def test_another_stream_and_captured_graphs(cuda_device):
    """Two graphs that hold calls of both forms, replayed in turn with new activations, and a call on a side stream meanwhile."""
    K, N = 1024, 768
    g = torch.Generator(device=cuda_device).manual_seed(5)
    rand = lambda *s: torch.randint(-127, 128, s, dtype=torch.int8, device=cuda_device, generator=g)  # noqa: E731
    w, sw = rand(N, K), torch.rand(N, device=cuda_device)
    sets = []
    for M in (20, 12000):
        a, sa, y = rand(M, K), torch.rand(M, device=cuda_device), torch.empty(M, N, dtype=torch.bfloat16, device=cuda_device)
        cf.gemm_q8(a, sa, w, sw, y)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cf.gemm_q8(a, sa, w, sw, y, activation="relu")
        sets.append((a, sa, y, graph))
    side = torch.cuda.Stream()
    b, sb, z = rand(50, K), torch.rand(50, device=cuda_device), torch.empty(50, N, device=cuda_device)
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(2):
        for a, sa, y, graph in sets:
            a.copy_(rand(*a.shape))
            graph.replay()
        cf.gemm_q8(b, sb, w, sw, z, stream=side)
        torch.cuda.synchronize()
        want = (b.double() @ w.double().mT) * sb.double()[:, None] * sw.double()
        assert ((z.double() - want).abs() <= want.abs() * 2.0 ** -20).all()
        for a, sa, y, graph in sets:
            want = ((a.double() @ w.double().mT) * sa.double()[:, None] * sw.double()).clamp_min(0)
            assert ((y.double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -20)).all()


FIRST = """
import torch
import paper_2608_03537_b200 as cf
d = torch.device("cuda:0")
K, N = 8192, 1024
w, sw = torch.randint(-127, 128, (N, K), dtype=torch.int8, device=d), torch.rand(N, device=d)
sets = [(torch.randn(M, K, device=d), torch.zeros(M, K, dtype=torch.int8, device=d), torch.zeros(M, device=d), torch.zeros(M, N, device=d)) for M in (1, 40, 250, 3000)]
graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=side):
    for x, q, s, y in sets:
        cf.quantize_rows(x, q, s)
        cf.gemm_q8(q, s, w, sw, y)
graph.replay()
torch.cuda.synchronize()
for x, q, s, y in sets:
    want = (q.double() @ w.double().mT) * s.double()[:, None] * sw.double()
    assert bool((s > 0).all()) and ((y.double() - want).abs() <= want.abs() * 2.0 ** -20).all(), x.shape
assert cf.last_device_status() == cf.OK
"""


def test_the_first_calls_of_a_process_may_be_captured(cuda_device):
    """Nothing that a form sets up on its first call (attributes, how many clusters fit) disturbs a capture."""
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-3000:]


def test_threads_with_streams_of_their_own(cuda_device):
    """Calls from several threads at once, each on its stream: every form, eager."""
    from concurrent.futures import ThreadPoolExecutor
    K, N = 2048, 1000
    w, sw = torch.randint(-127, 128, (N, K), dtype=torch.int8, device=cuda_device), torch.rand(N, device=cuda_device)

    def work(M):
        torch.cuda.set_device(cuda_device)
        side = torch.cuda.Stream()
        x = torch.randn(M, K, device=cuda_device)
        q, s, y = torch.empty(M, K, dtype=torch.int8, device=cuda_device), torch.empty(M, device=cuda_device), torch.empty(M, N, device=cuda_device)
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(50):
            cf.quantize_rows(x, q, s, stream=side)
            cf.gemm_q8(q, s, w, sw, y, stream=side)
        side.synchronize()
        want = (q.double() @ w.double().mT) * s.double()[:, None] * sw.double()
        return bool(((y.double() - want).abs() <= want.abs() * 2.0 ** -20).all())

    torch.cuda.synchronize()
    with ThreadPoolExecutor(4) as pool:
        assert all(pool.map(work, (1, 40, 300, 3000)))
