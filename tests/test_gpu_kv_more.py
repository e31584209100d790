"""Key-value cache calls beside those of the operators' own tests: every 8-bit width, a long sequence against the definition, places behind 2^31 bytes in 8 bits, decoding of sequences that
differ in length, and the same bits from every repeated call."""
import pytest
import torch

import paper_2608_03537_b200 as cf
from tests import kv, test_gpu_kv_step as steps
from tests.test_gpu_paged_attention import TYPES, Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("D", [16, 32, 48, 80, 112, 144, 160, 192, 208, 224, 240])
def test_8_bit_widths(D, name, cuda_device):
    c = Call([300, 0, 77, 1], 2, 12, 2, D, 16, name, True, cuda_device, seed=D, slopes=True)
    c.run()
    c.check()


@pytest.mark.parametrize("D", [8, 40, 72, 136, 248])
def test_8_bit_widths_that_are_refused(D, cuda_device):
    """Rows of codes are read in pieces of 16."""
    c = kv.Cache(3, 2, 16, D, "bf16", True, cuda_device)
    table, lengths = torch.zeros(1, 2, dtype=torch.int32, device=cuda_device), torch.ones(1, dtype=torch.int32, device=cuda_device)
    q, k, slots = torch.zeros(1, 4, D, device=cuda_device).bfloat16(), torch.zeros(1, 2, D, device=cuda_device).bfloat16(), torch.zeros(1, dtype=torch.int64, device=cuda_device)
    for call in (lambda: cf.paged_attention_workspace_size(q, c.k, c.v, table, **c.scales()), lambda: cf.paged_attention(q, c.k, c.v, table, lengths, q.clone(), **c.scales()),
                 lambda: cf.cache_write(k, k, c.k, c.v, slots, **c.scales()), lambda: cf.cache_read(c.k, c.v, slots, k, k.clone(), **c.scales())):
        with pytest.raises(cf.ComfuseError) as e:
            call()
        assert e.value.status == cf.ERR_ALIGNMENT
    torch.cuda.synchronize()
    c.check_canaries()


@pytest.mark.parametrize("name,quantized", TYPES)
def test_a_long_sequence(name, quantized, cuda_device):
    c = Call([131072, 70000], 1, 8, 2, 64, 64, name, quantized, cuda_device, seed=5)
    c.run()
    c.check()


@pytest.mark.parametrize("name,quantized", TYPES)
@pytest.mark.parametrize("T,Hq,H,D,cap,window", [(1, 32, 8, 128, 0.0, 0), (5, 16, 2, 256, 30.0, 0), (3, 12, 12, 64, 0.0, 100), (16, 4, 1, 128, 5.0, 0)])
def test_the_same_bits_again(T, Hq, H, D, cap, window, name, quantized, cuda_device):
    c = Call([3000, 0, 517, 64, 1200], T, Hq, H, D, 24, name, quantized, cuda_device, seed=D, cap=cap, window=window)
    got = []
    for _ in range(8):
        c.out.fill_(-77.0)
        c.run()
        got.append((c.out.clone(), c.lse.clone()))
    assert all(torch.equal(got[0][0], o) and torch.equal(got[0][1], l) for o, l in got)


def test_8_bits_behind_32_bits(cuda_device):
    """Codes behind 2^31 bytes of a cache, scales behind 2^23 rows: written, read back and attended, as in a cache of four pages."""
    pages, page, D, H = 150000, 64, 128, 2
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("not enough free memory")
    g = torch.Generator(device=cuda_device).manual_seed(1)
    k, v = torch.randn(2, 250, H, D, device=cuda_device, generator=g).bfloat16()
    q = torch.randn(1, 8, D, device=cuda_device, generator=g).bfloat16()
    pos = torch.arange(250, device=cuda_device)
    got = []
    for n, table in ((pages, [pages - 1, pages - 3, 2, pages - 2]), (4, [0, 1, 2, 3])):
        cache = [torch.zeros(n, H, page, D, dtype=torch.int8, device=cuda_device) for _ in "kv"]
        scales = dict(zip(("k_scale", "v_scale"), (torch.zeros(n, H, page, device=cuda_device) for _ in "kv")))
        t = torch.tensor([table], dtype=torch.int32, device=cuda_device)
        slots = t[0].long()[pos // page] * page + pos % page
        cf.cache_write(k, v, *cache, slots, **scales)
        back = [torch.zeros_like(k) for _ in "kv"]
        cf.cache_read(*cache, slots, *back, **scales)
        out, ws = torch.zeros_like(q), torch.empty(cf.PAGED_ATTENTION_WORKSPACE_BYTES, dtype=torch.uint8, device=cuda_device)
        cf.paged_attention(q, *cache, t, torch.tensor([250], dtype=torch.int32, device=cuda_device), out, workspace=ws, **scales)
        assert n == 4 or torch.count_nonzero(scales["k_scale"]) == 250 * H
        got.append((*back, out))
        del cache, scales
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][2].abs().sum() > 0
    assert (got[0][0].float() - k.float()).abs().max() <= k.abs().max().float() * (0.5 / 127 + 2.0 ** -8)


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("B,Hq,H,D", [(7, 8, 2, 64), (40, 4, 4, 128)])
def test_decoding_of_sequences_of_different_lengths(B, Hq, H, D, quantized, cuda_device):
    """Sequences that have 0 to 55 tokens in the cache before the first step."""
    b = steps._block(cuda_device, B, Hq, H, D, quantized)
    g = torch.Generator(device=cuda_device).manual_seed(3)
    lengths = torch.randint(0, 56, (B,), device=cuda_device, generator=g)
    lengths[0], lengths[1], lengths[B - 1] = 0, 55, 16
    at = torch.cat([b["table"][i].long()[torch.arange(int(n), device=cuda_device) // b["page"]] * b["page"] + torch.arange(int(n), device=cuda_device) % b["page"] for i, n in enumerate(lengths)])
    k, v = torch.randn(2, len(at), H, D, device=cuda_device, generator=g).bfloat16()
    cf.cache_write(k, v, b["cache"].k, b["cache"].v, at, **b["cache"].scales())
    b["lengths"].copy_(lengths)
    for step in range(37):
        steps._step(b)
        if step in (0, 9, 36):
            torch.cuda.synchronize()
            steps._check(b)
    assert torch.equal(b["lengths"].long(), lengths + 37) and torch.isfinite(b["x"].float()).all()
