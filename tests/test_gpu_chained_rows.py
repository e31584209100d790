"""Chains of the library's bf16 calls in which each reads what the call in front of it wrote in every way that is not a GEMM operand: as the residual,
the row vectors (bias, gamma, beta) and the mask.  A kernel is on the SMs while the two in front of it still run, so an operand read too
early, or from an older line of the L1, is the one that stood there before.  Queued without a pause the chain has to give the bits of
the same calls made one by one."""
import pytest
import torch

import paper_2608_03537_b200 as cf

pytestmark = pytest.mark.gpu

CALLS = 12
bf = torch.bfloat16


def _rand(device, seed, *shape, std=1.0):
    return (torch.randn(*shape, device=device, generator=torch.Generator(device=device).manual_seed(seed)) * std).to(bf)


def _same_queued(run, out):
    run(torch.cuda.synchronize)
    want = out.clone()
    assert torch.isfinite(want).all() and all(not torch.equal(want[i], want[i + 1]) for i in range(1, CALLS))
    for _ in range(12):
        out[1:].zero_()
        torch.cuda.synchronize()
        torch.cuda._sleep(500_000)      # the host queues the calls while this runs
        run(lambda: None)
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("kind", [cf.EPI_BIAS_RES_LAYERNORM, cf.EPI_BIAS_GELU_RES_RMSNORM_MAX])
@pytest.mark.parametrize("M,N,K", [(1, 256, 128), (20, 768, 256), (64, 1024, 64), (300, 256, 64), (40, 4096, 256), (520, 4096, 1024), (1500, 768, 64)])
def test_residual_and_row_vectors_of_the_call_before(M, N, K, kind, cuda_device):
    a, b = _rand(cuda_device, 1, M, K), _rand(cuda_device, 2, K, N, std=K ** -0.5)
    y = torch.zeros(CALLS + 1, M, N, dtype=bf, device=cuda_device)
    y[0] = _rand(cuda_device, 3, M, N)
    fixed = 1 + _rand(cuda_device, 11, N, std=0.1)
    ln = kind == cf.EPI_BIAS_RES_LAYERNORM
    top, arg = torch.empty(M, device=cuda_device), torch.empty(M, dtype=torch.int32, device=cuda_device)
    ws = torch.empty(256 << 20, dtype=torch.uint8, device=cuda_device)

    def run(between):
        for i in range(CALLS):
            # Row vectors in every other call only: with fixed ones |y| <= 1.5 sqrt(N) <= 96 whatever came in, with y's row as gains and offsets it is
            # at most 64 * 96 + 96, so that no sum leaves fp16's range, in which the form of two kernels keeps the row.
            row = y[i, 0]
            cf.gemm_epilogue(a, b, y[i + 1], kind, bias=row, residual=y[i], gamma=row if i % 2 else fixed, beta=(row if i % 2 else fixed) if ln else None,
                             row_max=None if ln else top, row_argmax=None if ln else arg, workspace=ws)
            between()
    _same_queued(run, y)


@pytest.mark.parametrize("M,N", [(1, 256), (40, 504), (200, 1024), (700, 2048)])
def test_mask_of_the_call_before(M, N, cuda_device):
    K = 64
    q, k = _rand(cuda_device, 4, M, K), _rand(cuda_device, 5, K, N)
    y = torch.zeros(CALLS + 1, M, N, dtype=bf, device=cuda_device)
    y[0] = _rand(cuda_device, 6, M, N)

    def run(between):
        for i in range(CALLS):
            cf.gemm_epilogue(q, k, y[i + 1], cf.EPI_SCALE_MASK_SOFTMAX, alpha=K ** -0.5 * (1 + i), mask=cf.MASK_ADDITIVE, mask_tensor=y[i])
            between()
    _same_queued(run, y)


@pytest.mark.parametrize("M", [1, 16, 40, 64, 300, 3000])
def test_rows_and_vectors_of_the_mlp_before(M, cuda_device):
    hidden = 512
    w1, w2, b1 = _rand(cuda_device, 7, 128, hidden, std=0.1), _rand(cuda_device, 8, hidden, 128, std=0.05), _rand(cuda_device, 9, hidden)
    fixed = 1 + _rand(cuda_device, 11, 128, std=0.1)
    o = torch.zeros(CALLS + 1, M, 128, dtype=bf, device=cuda_device)
    o[0] = _rand(cuda_device, 10, M, 128)

    def run(between):
        for i in range(CALLS):
            row = o[i, 0]
            cf.b2b_gemm(o[i], w1, b1, w2, row, o[i + 1], gamma=row if i % 2 else fixed, beta=row if i % 2 else fixed)
            between()
    _same_queued(run, o)
