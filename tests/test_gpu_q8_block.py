"""The 8-bit layers as they are used together: an MLP block of a transformer (norm and residual -> product with GELU -> rows to int8 ->
product with the residual), eager and captured, against the definition in 64 bits step by step, and beside the library's bf16 layers."""
import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import q8_oracle as orc
from tests import q8

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _block(M, N, H, name, device, seed):
    g = torch.Generator(device=device).manual_seed(seed)
    t = q8.TYPES[name]
    rand = lambda *s: torch.randn(*s, device=device, generator=g)  # noqa: E731
    b = dict(x=rand(M, N).to(t), r=rand(M, N).to(t), gamma=(1 + 0.1 * rand(N)).to(t), b1=(0.1 * rand(H)).to(t), b2=(0.1 * rand(N)).to(t), t=t)
    for k, n, m in (("1", H, N), ("2", N, H)):
        w = rand(n, m) * m ** -0.5
        s = w.abs().amax(1) / 127
        b["W" + k], b["s" + k] = (w / s[:, None]).round().to(torch.int8), s
    b["q"], b["sq"] = torch.empty(M, N, dtype=torch.int8, device=device), torch.empty(M, device=device)
    b["p"], b["sp"] = torch.empty(M, H, dtype=torch.int8, device=device), torch.empty(M, device=device)
    b["h"], b["u"], b["y"] = torch.empty(M, N, dtype=t, device=device), torch.empty(M, H, dtype=t, device=device), torch.empty(M, N, dtype=t, device=device)
    return b


def _run(b, stream=None):
    cf.rmsnorm_quantize_rows(b["x"], b["q"], b["sq"], residual=b["r"], gamma=b["gamma"], h=b["h"], eps=EPS, stream=stream)
    cf.gemm_q8(b["q"], b["sq"], b["W1"], b["s1"], b["u"], bias=b["b1"], activation="gelu_tanh", stream=stream)
    cf.quantize_rows(b["u"], b["p"], b["sp"], stream=stream)
    cf.gemm_q8(b["p"], b["sp"], b["W2"], b["s2"], b["y"], bias=b["b2"], residual=b["h"], stream=stream)


def _check(b):
    """Each step against the definition on what the step before it handed over, so that the bounds are those of one step."""
    f = q8.f64
    _, _, s, v = orc.quantize(f(b["x"]), f(b["r"]), f(b["gamma"]), EPS)
    assert np.all(np.abs(f(b["q"]) - v) <= q8.CODE_TOL) and np.all(np.abs(f(b["sq"]) - s) <= q8.SCALE_TOL_NORM * s)
    assert torch.equal(b["h"], (b["x"].float() + b["r"].float()).to(b["t"]))
    u, t = orc.gemm(f(b["q"]), f(b["sq"]), f(b["W1"]), f(b["s1"]), f(b["b1"]), None, "gelu_tanh")
    assert np.all(np.abs(f(b["u"]) - u) <= q8.product_bound(u, t, b["t"], f(b["b1"])))
    _, _, s, v = orc.quantize(f(b["u"]))
    assert np.all(np.abs(f(b["p"]) - v) <= q8.CODE_TOL) and np.all(np.abs(f(b["sp"]) - s) <= q8.SCALE_TOL_PLAIN * s)
    y, t = orc.gemm(f(b["p"]), f(b["sp"]), f(b["W2"]), f(b["s2"]), f(b["b2"]), f(b["h"]))
    assert np.all(np.abs(f(b["y"]) - y) <= q8.product_bound(y, t, b["t"], f(b["b2"]), f(b["h"])))


@pytest.mark.parametrize("M,N,H,name", [(1, 256, 1024, "bf16"), (40, 1024, 4096, "bf16"), (333, 512, 2048, "f16"), (5000, 256, 1040, "bf16"), (7, 64, 80, "f32")])
def test_block(M, N, H, name, cuda_device):
    b = _block(M, N, H, name, cuda_device, M)
    _run(b)
    torch.cuda.synchronize()
    _check(b)


def test_block_captured_and_replayed_with_new_tokens(cuda_device):
    b, other = _block(40, 512, 2048, "bf16", cuda_device, 1), _block(2000, 512, 2048, "bf16", cuda_device, 2)
    _run(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(b)
        _run(other)
    side = torch.cuda.Stream()
    third = _block(16, 256, 512, "bf16", cuda_device, 3)
    side.wait_stream(torch.cuda.current_stream())
    for seed in (5, 6):
        new = _block(40, 512, 2048, "bf16", cuda_device, seed)
        b["x"].copy_(new["x"])
        graph.replay()
        _run(third, stream=side)    # beside the graph, on buffers of its own
        torch.cuda.synchronize()
        for c in (b, other, third):
            _check(c)


def test_residual_stream_in_place_over_two_layers(cuda_device):
    """h over the residual, the product over its own residual: the same bits as with buffers of their own."""
    a, b = _block(33, 512, 1024, "bf16", cuda_device, 4), _block(33, 512, 1024, "bf16", cuda_device, 4)
    for _ in range(2):
        _run(a)
        a["r"], a["y"] = a["y"], torch.empty_like(a["y"])
        cf.rmsnorm_quantize_rows(b["x"], b["q"], b["sq"], residual=b["r"], gamma=b["gamma"], h=b["r"], eps=EPS)
        cf.gemm_q8(b["q"], b["sq"], b["W1"], b["s1"], b["u"], bias=b["b1"], activation="gelu_tanh")
        cf.quantize_rows(b["u"], b["p"], b["sp"])
        cf.gemm_q8(b["p"], b["sp"], b["W2"], b["s2"], b["r"], bias=b["b2"], residual=b["r"])
    assert torch.equal(a["r"], b["r"])


def test_values_feed_the_bf16_layers(cuda_device):
    """What the 8 bits stand for, through the library's bf16 GEMM with the dequantised weight, is close to the 8-bit product: the
    accuracy of a layer's quantisation read without its integers.  bf16 holds weights and values to 2^-8 relative each."""
    M, N, K = 64, 256, 512
    b = _block(M, K, N, "bf16", cuda_device, 9)
    v = torch.empty(M, K, dtype=torch.bfloat16, device=cuda_device)
    cf.rmsnorm_quantize_rows(b["x"], b["q"], b["sq"], residual=b["r"], gamma=b["gamma"], h=b["h"], values=v, eps=EPS)
    y8, y16 = (torch.empty(M, N, dtype=torch.bfloat16, device=cuda_device) for _ in range(2))
    cf.gemm_q8(b["q"], b["sq"], b["W1"], b["s1"], y8, activation="relu")
    w = (b["W1"].float() * b["s1"][:, None]).to(torch.bfloat16)
    spec = cf.make_spec([("acc", -1, -1, -1, 0.0), ("relu", 0, -1, -1, 0.0)], 1)
    cf.gemm_spec(v, w, y16, spec, b_nk=True)
    torch.cuda.synchronize()
    off = (y8.double() - y16.double()).abs()
    # two operands 2^-9 off each at most, one rounding of each result 2^-9: 2^-9 (2 sum|v w| + 2 |y|)
    size = v.double().abs() @ w.double().abs().mT
    assert (off <= 2.0 ** -9 * (2 * size + 2 * y8.double().abs()) * 1.01).all()
