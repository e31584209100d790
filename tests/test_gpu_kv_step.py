"""A transformer's attention block as it decodes: norm -> 8-bit projection -> turned, quantised and cached -> attention over the cache -> 8-bit projection onto the residual stream, step
after step; and a prompt's cached prefix read back for the library's attention over short sources."""
import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import kv_oracle as orc
from tests import kv

pytestmark = pytest.mark.gpu


def _block(device, B, Hq, H, D, quantized, page=16, width=6):
    g = torch.Generator(device=device).manual_seed(B)
    rand = lambda *s: torch.randn(*s, device=device, generator=g)  # noqa: E731
    N = 256
    b = dict(B=B, Hq=Hq, H=H, D=D, page=page, x=rand(B, N).bfloat16(), gamma=(1 + 0.1 * rand(N)).bfloat16(), quantized=quantized)
    for k, n, m in (("qkv", (Hq + 2 * H) * D, N), ("o", N, Hq * D)):
        w = rand(n, m) * m ** -0.5
        s = w.abs().amax(1) / 127
        b["W" + k], b["s" + k] = (w / s[:, None]).round().to(torch.int8), s
    b["cache"] = kv.Cache(B * width + 1, H, page, D, "bf16", quantized, device)
    b["table"] = (torch.randperm(B * width, device=device, generator=g).to(torch.int32)).view(B, width)
    b["lengths"] = torch.zeros(B, dtype=torch.int32, device=device)
    b["freqs"] = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=device) / (D // 2))
    b["q8"], b["sq"] = torch.empty(B, N, dtype=torch.int8, device=device), torch.empty(B, device=device)
    b["p8"], b["sp"] = torch.empty(B, Hq * D, dtype=torch.int8, device=device), torch.empty(B, device=device)
    b["u"], b["q"], b["o"] = torch.empty(B, (Hq + 2 * H) * D, dtype=torch.bfloat16, device=device), torch.empty(B, Hq, D, dtype=torch.bfloat16, device=device), torch.empty(B, Hq, D, dtype=torch.bfloat16, device=device)
    b["positions"], b["slots"] = torch.zeros(B, dtype=torch.int32, device=device), torch.zeros(B, dtype=torch.int64, device=device)
    b["workspace"] = torch.empty(cf.PAGED_ATTENTION_WORKSPACE_BYTES, dtype=torch.uint8, device=device)
    return b


def _step(b):
    """One new token of each sequence.  (positions, slots and lengths are the program's own bookkeeping.)"""
    n = b["lengths"].long()
    b["positions"].copy_(n)
    b["slots"].copy_(torch.gather(b["table"].long(), 1, (n // b["page"])[:, None])[:, 0] * b["page"] + n % b["page"])
    b["lengths"].add_(1)
    cf.rmsnorm_quantize_rows(b["x"], b["q8"], b["sq"], gamma=b["gamma"])
    cf.gemm_q8(b["q8"], b["sq"], b["Wqkv"], b["sqkv"], b["u"])
    q, k, v = b["u"].view(b["B"], -1, b["D"]).split((b["Hq"], b["H"], b["H"]), dim=1)
    c = b["cache"]
    cf.cache_write(k, v, c.k, c.v, b["slots"], q=q, q_out=b["q"], positions=b["positions"], freqs=b["freqs"], **c.scales())
    cf.paged_attention(b["q"], c.k, c.v, b["table"], b["lengths"], b["o"], workspace=b["workspace"], **c.scales())
    cf.quantize_rows(b["o"].view(b["B"], -1), b["p8"], b["sp"])
    cf.gemm_q8(b["p8"], b["sp"], b["Wo"], b["so"], b["x"], residual=b["x"])


def _check(b):
    """The attention of the last step on what the cache holds (each other step has tests of its own), and its queries."""
    q, k, v = b["u"].view(b["B"], -1, b["D"]).split((b["Hq"], b["H"], b["H"]), dim=1)
    angle = kv.raw_angle(b["positions"].cpu().numpy(), b["freqs"].cpu().numpy(), (b["D"] // 2,))
    want = orc.rotary(kv.f64(q), b["positions"].cpu().numpy(), b["freqs"].cpu().numpy())
    assert np.all(np.abs(kv.f64(b["q"]) - want) <= kv.turned_bound(want, kv.f64(q), b["D"] // 2, False, angle, torch.bfloat16))
    lengths = b["lengths"].cpu().numpy()
    out, lse, weight = orc.attention(kv.f64(b["q"])[:, None], b["cache"].values("k"), b["cache"].values("v"), b["table"].cpu().numpy(), lengths, b["D"] ** -0.5)
    bound, _ = kv.attention_bounds(out, lse, weight, int(lengths.max()), b["D"], torch.bfloat16, b["quantized"])
    assert np.all(np.abs(kv.f64(b["o"])[:, None] - out) <= bound)


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("B,Hq,H,D", [(1, 8, 2, 64), (5, 4, 4, 128), (40, 8, 1, 64)])
def test_decoding(B, Hq, H, D, quantized, cuda_device):
    b = _block(cuda_device, B, Hq, H, D, quantized)
    b["lengths"][B // 2:] += 0
    for step in range(37):
        _step(b)
        if step in (0, 15, 16, 36):
            torch.cuda.synchronize()
            _check(b)
    assert torch.isfinite(b["x"].float()).all()


@pytest.mark.parametrize("quantized", [False, True])
def test_decoding_as_a_graph_is_decoding(quantized, cuda_device):
    eager, captured = _block(cuda_device, 6, 8, 2, 64, quantized), _block(cuda_device, 6, 8, 2, 64, quantized)
    _step(eager)
    _step(captured)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(captured)
    for _ in range(30):
        _step(eager)
        graph.replay()
    torch.cuda.synchronize()
    _check(captured)
    assert torch.equal(eager["x"], captured["x"]) and torch.equal(eager["o"], captured["o"]) and torch.equal(eager["lengths"], captured["lengths"])


def test_a_prefix_read_back_for_attention_over_it(cuda_device):
    """A cached prefix in 8 bits, read back and given to the attention of many queries (one key per row); the same answer, within both calls' bounds, as new tokens over the cache."""
    H, D, n, T, page = 2, 128, 256, 64, 64
    c = kv.Cache(5, H, page, D, "bf16", True, cuda_device)
    g = torch.Generator(device=cuda_device).manual_seed(1)
    k, v = torch.randn(2, n, H, D, device=cuda_device, generator=g).bfloat16()
    q = torch.randn(1, T, H, D, device=cuda_device, generator=g).bfloat16()
    table = torch.tensor([[3, 0, 4, 1]], dtype=torch.int32, device=cuda_device)
    pos = torch.arange(n, device=cuda_device)
    slots = table[0].long()[pos // page] * page + pos % page
    cf.cache_write(k, v, c.k, c.v, slots, **c.scales())
    back = [torch.empty_like(k) for _ in "kv"]
    cf.cache_read(c.k, c.v, slots, *back, **c.scales())
    keys, values = (t.transpose(0, 1).contiguous() for t in back)
    queries = q[0].transpose(0, 1).contiguous()
    O = torch.empty(H, T, D, dtype=torch.bfloat16, device=cuda_device)
    cf.b2b_attention(queries, keys, values, O, alpha=D ** -0.5, keys_row_major=True)
    out, ws = torch.empty_like(q[:, -1]), torch.empty(cf.PAGED_ATTENTION_WORKSPACE_BYTES, dtype=torch.uint8, device=cuda_device)
    cf.paged_attention(q[:, -1], c.k, c.v, table, torch.tensor([n], dtype=torch.int32, device=cuda_device), out, workspace=ws, **c.scales())
    # values up to about 4: rounded to bf16 on the way (2^-9), weights to bf16 (2^-9), outputs twice (2^-9 of at most 1); averages of 256 of them
    assert (O[:, -1].float() - out[0].float()).abs().max() <= 4 * 4 * 2.0 ** -9


CHILD = r"""
import threading
import torch
import paper_2608_03537_b200 as cf
from tests import test_gpu_kv_step as steps

dev = torch.device("cuda:0")
torch.cuda.set_device(0)
blocks = [steps._block(dev, 6, 8, 2, 64, q) for q in (False, True)]
for b in blocks:
    b["x"].add_(1)
torch.cuda.synchronize()
# the first calls of the process, captured
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    for b in blocks:
        steps._step(b)
for _ in range(5):
    graph.replay()
torch.cuda.synchronize()
for b in blocks:
    assert int(b["lengths"][0]) == 5
    steps._check(b)
# and from several threads, each on its own stream and block
own = [steps._block(dev, 3 + i, 8, 2, 64, i % 2 == 1) for i in range(4)]
torch.cuda.synchronize()
errors = []
def work(b):
    try:
        torch.cuda.set_device(0)
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                steps._step(b)
            torch.cuda.current_stream().synchronize()
    except BaseException as e:
        errors.append(e)
threads = [threading.Thread(target=work, args=(b,)) for b in own]
[t.start() for t in threads]
[t.join() for t in threads]
assert not errors, errors
for b in own:
    steps._check(b)
assert cf.last_device_status() == cf.OK
print("steps ok")
"""


def test_captured_as_the_first_calls_of_a_process_and_from_several_threads(cuda_device):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=root, env=dict(os.environ, PYTHONPATH=root), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "steps ok" in r.stdout, r.stdout + r.stderr[-3000:]
