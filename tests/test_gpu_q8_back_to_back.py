"""Chains of 8-bit calls that hand their results on through the same buffers, with nothing between them: each kernel is on the SMs while
the two in front of it still run, and has to see what the last one wrote, not what stood in the buffer before.  Every call's inputs
differ, so a code, a scale, a gain or a bias of the call before shows; the bits have to be those of the same calls made one by one."""
import pytest
import torch

import paper_2608_03537_b200 as cf

pytestmark = pytest.mark.gpu

CALLS = 40


def _rand(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _chain(M, N, K, name, device, both):
    """(run, results): `run(between)` makes CALLS pairs of calls through one set of codes and scales; `both` has B's codes and scales written
    in front of each product too (keys that have just been computed)."""
    g = torch.Generator(device=device).manual_seed(M + N + K)
    t = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]
    loud = 2.0 ** torch.arange(CALLS, device=device).remainder(9)[:, None, None]   # scales of neighbours differ by powers of two and more
    x, w = (_rand(g, CALLS, M, K) * loud).to(t), (_rand(g, CALLS, N, K) / loud).to(t)
    q, s = torch.zeros(M, K, dtype=torch.int8, device=device), torch.zeros(M, device=device)
    p, u = torch.zeros(N, K, dtype=torch.int8, device=device), torch.zeros(N, device=device)
    cf.quantize_rows(w[0], p, u)
    y = torch.zeros(CALLS, M, N, dtype=t, device=device)

    def run(between):
        for i in range(CALLS):
            if both:
                cf.quantize_rows(w[i], p, u)
                between()
            cf.quantize_rows(x[i], q, s)
            between()
            cf.gemm_q8(q, s, p, u, y[i])
            between()
    return run, y


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("M,N,K,name", [(1, 16, 128, "f32"), (1, 256, 64, "bf16"), (3, 48, 256, "f16"), (8, 128, 1024, "bf16"), (16, 64, 256, "f32"), (16, 1024, 512, "bf16"),
                                        (40, 128, 256, "bf16"), (100, 512, 1024, "f32"), (700, 256, 64, "bf16"), (3000, 512, 128, "f32")])
def test_products_see_the_codes_and_scales_just_written(M, N, K, name, both, cuda_device):
    run, y = _chain(M, N, K, name, cuda_device, both)
    run(torch.cuda.synchronize)
    want = y.clone()
    assert len({float(want[i].double().abs().sum()) for i in range(CALLS)}) == CALLS   # (the calls' results differ)
    for _ in range(5):
        y.zero_()
        run(lambda: None)
        assert torch.equal(y, want)
    y.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(lambda: None)
    for _ in range(3):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)


@pytest.mark.parametrize("M,N", [(1, 64), (5, 256), (40, 1008), (300, 4096), (3, 16384)])
def test_norms_see_the_rows_and_gains_just_written(M, N, cuda_device):
    """A residual stream through CALLS norms, whose gains are the first rows of the stream itself: h in place, over and over."""
    g = torch.Generator(device=cuda_device).manual_seed(M + N)
    t = torch.bfloat16
    x = _rand(g, CALLS, M, N).to(t)
    h = torch.zeros(CALLS + 1, M, N, dtype=t, device=cuda_device)
    h[0] = _rand(g, M, N).to(t)
    q, s = torch.zeros(CALLS, M, N, dtype=torch.int8, device=cuda_device), torch.zeros(CALLS, M, device=cuda_device)

    def run(between):
        for i in range(CALLS):   # reads what call i - 1 wrote: as the residual, and its first row as the gains
            cf.rmsnorm_quantize_rows(x[i], q[i], s[i], residual=h[i], gamma=h[i, 0], h=h[i + 1])
            between()
    run(torch.cuda.synchronize)
    want = h.clone(), q.clone(), s.clone()
    for _ in range(10):
        h[1:].zero_()
        run(lambda: None)
        assert torch.equal(h, want[0]) and torch.equal(q, want[1]) and torch.equal(s, want[2])


@pytest.mark.parametrize("M", [1, 40, 600])
def test_products_see_the_bias_and_residual_just_written(M, cuda_device):
    """Y of one product is the residual of the next, and its first row the bias."""
    K = N = 256
    g = torch.Generator(device=cuda_device).manual_seed(M)
    a, b = (torch.randint(-127, 128, (n, K), dtype=torch.int8, device=cuda_device, generator=g) for n in (M, N))
    sa, sb = (torch.rand(n, device=cuda_device, generator=g) * 1e-2 for n in (M, N))
    y = torch.zeros(CALLS + 1, M, N, device=cuda_device)
    y[0] = _rand(g, M, N)

    def run(between):
        for i in range(CALLS):
            cf.gemm_q8(a, sa, b, sb, y[i + 1], bias=y[i, 0], residual=y[i], activation="tanh")
            between()
    run(torch.cuda.synchronize)
    want = y.clone()
    for _ in range(10):
        y[1:].zero_()
        run(lambda: None)
        assert torch.equal(y, want)
