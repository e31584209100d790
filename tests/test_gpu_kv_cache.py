"""Keys and values written into a paged cache, in 16 and 8 bits, and read back, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import kv_oracle as orc
from tests import kv, parity as P, q8

pytestmark = pytest.mark.gpu


def _tokens(tokens, Hq, H, D, name, device, seed):
    g = torch.Generator(device=device).manual_seed(seed)
    base = torch.randn(tokens, Hq + 2 * H, D, device=device, generator=g).to(kv.TYPES[name])
    return base.split((Hq, H, H), dim=1)   # (views of one projection's output)


def _slots(tokens, pages, page, device, seed):
    """Places anywhere, each once; some tokens are padding."""
    r = np.random.RandomState(seed)
    s = r.permutation(pages * page)[:tokens].astype(np.int64)
    if tokens > 4:
        s[1], s[tokens // 2], s[-1] = -1, pages * page, -2 ** 62
    return torch.from_numpy(s).to(device)


def _check_written(cache, k, v, slots, positions=None, freqs=None, sections=None, adjacent=False):
    page = cache.page
    s = slots.cpu().numpy()
    real = (s >= 0) & (s < cache.k.shape[0] * page)
    where = (s[real] // page, slice(None), s[real] % page)
    held = {w: (t.detach().cpu()) for w, t in cache.tensors().items() if t is not None}
    for w, x in (("k", k), ("v", v)):
        x = kv.f64(x)[real]
        y, angle = x, None
        turned = w == "k" and positions is not None
        if turned:
            parts = sections or (len(freqs),)
            pos = np.atleast_2d(positions.cpu().numpy())[:, real]
            angle = kv.raw_angle(pos, freqs.cpu().numpy(), parts)
            y = orc.rotary(x, pos, freqs.cpu().numpy(), parts, adjacent)
        if not cache.quantized:
            got = kv.f64(held[w][where])
            if turned:
                assert np.all(np.abs(got - y) <= kv.turned_bound(y, x, len(freqs), adjacent, angle, cache.t))
            else:
                assert np.array_equal(got, y, equal_nan=True)
            continue
        scale, v64 = orc.quantize(y)
        codes, got = kv.f64(held[w][where]), kv.f64(held[w + "_scale"][where])
        assert np.array_equal(np.isnan(got), np.isnan(scale))
        fine = ~np.isnan(scale)
        assert np.all(np.abs(got - scale)[fine] <= (kv.SCALE_TOL_TURNED if turned else q8.SCALE_TOL_PLAIN) * scale[fine])
        assert np.all(np.abs(codes - v64) <= (kv.CODE_TOL_TURNED if turned else q8.CODE_TOL)) and np.all(codes[~fine] == 0)
    # every other row of the cache is as it was
    rest = np.ones((cache.k.shape[0], page), bool)
    rest[where[0], where[2]] = False
    page_i, row_i = np.nonzero(rest)
    for w, t in held.items():
        other = t[page_i, :, row_i]
        assert bool((other == -128).all()) if t.dtype == torch.int8 else bool(torch.isnan(other).all())
    cache.check_canaries()


CASES = [  # tokens, Hq, H, D, pairs, axes, adjacent, page, layout
    (1, 32, 8, 128, 64, 1, False, 16, "heads first"), (1, 1, 1, 16, 8, 1, True, 1, "heads first"), (5, 6, 3, 64, 32, 1, False, 24, "rows first"), (64, 16, 2, 128, 32, 1, False, 64, "padded"),
    (33, 4, 4, 80, 40, 3, False, 7, "heads first"), (100, 5, 5, 96, 20, 2, False, 100, "rows first"), (777, 3, 1, 256, 128, 1, True, 128, "heads first"), (9, 2, 2, 48, 5, 1, True, 8, "padded"),
    (3000, 2, 1, 64, 32, 1, False, 16, "heads first"), (20, 0, 3, 112, 56, 1, False, 33, "rows first"), (12, 0, 2, 128, 0, 1, False, 16, "heads first"), (2500, 8, 8, 16, 8, 1, False, 64, "heads first")]


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,Hq,H,D,pairs,axes,adjacent,page,layout", CASES)
def test_write_and_read(tokens, Hq, H, D, pairs, axes, adjacent, page, layout, name, quantized, cuda_device):
    pages = tokens // page + 3
    cache = kv.Cache(pages, H, page, D, name, quantized, cuda_device, layout)
    q, k, v = _tokens(tokens, Hq, H, D, name, cuda_device, tokens + D)
    slots = _slots(tokens, pages, page, cuda_device, D)
    kw, sections, positions, freqs = {}, None, None, None
    if pairs:
        positions = torch.randint(0, 100000, (axes, tokens), dtype=torch.int32, device=cuda_device)
        freqs = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64, device=cuda_device) / pairs)
        if axes == 1:
            positions = positions[0]
        else:
            sections = (pairs - (axes - 1) * (pairs // axes),) + (pairs // axes,) * (axes - 1)
        kw = dict(positions=positions, freqs=freqs, sections=sections, adjacent=adjacent)
    q_out = P.guarded(q.shape, q.dtype, -77.0, cuda_device) if Hq else None
    cf.cache_write(k, v, cache.k, cache.v, slots, **cache.scales(), **kw, **(dict(q=q, q_out=q_out) if Hq else {}))
    torch.cuda.synchronize()
    _check_written(cache, k, v, slots, positions, freqs, sections, adjacent)
    if Hq:
        alone = torch.empty_like(q_out)
        cf.rotary(q, positions, freqs, alone, sections=sections, adjacent=adjacent)
        assert torch.equal(q_out, alone)   # (the same arithmetic; checked against the definition by itself)
        P.check_canaries({"q_out": q_out})
    # read back, twice the same slot among them
    again = torch.cat((slots, slots[:1]))
    back = [P.guarded((tokens + 1, H, D), kv.TYPES[name], -77.0, cuda_device) for _ in "kv"]
    cf.cache_read(cache.k, cache.v, again, *back, **cache.scales())
    torch.cuda.synchronize()
    P.check_canaries({"k": back[0], "v": back[1]})
    s = again.cpu().numpy()
    real = (s >= 0) & (s < pages * page)
    for w, got in zip("kv", back):
        got = kv.f64(got)
        assert np.all(got[~real] == -77.0)
        want = cache.values(w)[s[real] // page, :, s[real] % page]
        assert np.all(np.abs(got[real] - want) <= ((kv.half_step(cache.t) + kv.U) * np.abs(want) + torch.finfo(cache.t).smallest_normal * kv.half_step(cache.t) if quantized else 0))


@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_odd_values_in_8_bits(name, cuda_device):
    """Zeros, denormals, the largest numbers, infinities and NaN; rows of one magnitude and ties."""
    t = kv.TYPES[name]
    k = torch.zeros(8, 1, 32, device=cuda_device).to(t)
    tiny = torch.finfo(t).smallest_normal * torch.finfo(t).eps
    k[1] = tiny
    k[2, 0, 3] = torch.finfo(t).max
    k[3, 0, 31] = float("inf")
    k[4, 0, 16] = float("nan")
    k[5] = torch.arange(-16, 16, device=cuda_device).to(t)
    k[6, 0] = torch.arange(32, device=cuda_device).to(t) * 0.5
    k[6, 0, 0] = 127
    k[7, 0, 8] = -float("inf")
    v = k.flip(0).contiguous()
    cache = kv.Cache(2, 1, 4, 32, name, True, cuda_device)
    slots = torch.arange(8, device=cuda_device)
    cf.cache_write(k, v, cache.k, cache.v, slots, **cache.scales())
    torch.cuda.synchronize()
    page, row = slots.cpu().numpy() // 4, slots.cpu().numpy() % 4
    for x, codes, scale in ((k, cache.k, cache.ks), (v, cache.v, cache.vs)):
        s, q = orc.quantize(kv.f64(x))
        got_s, got_q = kv.f64(scale)[page, :, row], kv.f64(codes)[page, :, row]
        assert np.array_equal(np.isnan(got_s), np.isnan(s))
        # a scale below fp32's normal numbers is flushed or off by a denormal's step
        assert np.all((np.abs(got_s - s) <= q8.SCALE_TOL_PLAIN * s + 2.0 ** -126)[~np.isnan(s)])
        assert np.all(np.abs(got_q - q) <= q8.CODE_TOL)
        ties = np.abs(q - np.rint(q)) == 0.5
        assert np.array_equal(got_q[ties], np.rint(q[ties]))


def test_offsets_beyond_32_bits(cuda_device):
    """Rows behind 2^31 elements of a cache."""
    pages, H, page, D = 150000, 1, 64, 256
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("not enough free memory")
    cache = torch.zeros(pages, H, page, D, dtype=torch.bfloat16, device=cuda_device)
    k, v = torch.randn(2, 3, H, D, device=cuda_device).bfloat16()
    slots = torch.tensor([pages * page - 1, 7, pages * page - 65], device=cuda_device)
    small = torch.zeros(2, H, page, D, dtype=torch.bfloat16, device=cuda_device)
    cf.cache_write(k, k, cache, cache, slots)
    out = torch.zeros_like(k)
    cf.cache_read(cache, cache, slots, out, out.clone())
    assert torch.equal(out, k)
    assert torch.equal(cache[-1, 0, -1], k[0, 0]) and torch.equal(cache[-2, 0, -1], k[2, 0])
    del cache, small


def test_captured_and_on_another_stream(cuda_device):
    cache = kv.Cache(6, 2, 16, 64, "bf16", True, cuda_device)
    q, k, v = _tokens(20, 4, 2, 64, "bf16", cuda_device, 1)
    k, v, slots = k.contiguous(), v.contiguous(), _slots(20, 6, 16, cuda_device, 1)
    out = [torch.zeros_like(k) for _ in "kv"]

    def step(stream=None):
        cf.cache_write(k, v, cache.k, cache.v, slots, **cache.scales(), stream=stream)
        cf.cache_read(cache.k, cache.v, slots, *out, **cache.scales(), stream=stream)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    k.normal_()
    graph.replay()
    torch.cuda.synchronize()
    captured = [o.clone() for o in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured, out))
    _check_written(cache, k, v, slots)


def test_refusals(cuda_device):
    cache = kv.Cache(4, 2, 16, 64, "bf16", False, cuda_device)
    q8c = kv.Cache(4, 2, 16, 64, "bf16", True, cuda_device)
    q, k, v = (t.contiguous() for t in _tokens(5, 4, 2, 64, "bf16", cuda_device, 1))
    slots = torch.arange(5, device=cuda_device)
    pos, freqs = torch.arange(5, dtype=torch.int32, device=cuda_device), torch.ones(32, dtype=torch.float64, device=cuda_device)
    write = lambda k=k, v=v, kc=cache.k, vc=cache.v, s=slots, **kw: cf.cache_write(k, v, kc, vc, s, **kw)  # noqa: E731
    for kw in (dict(k=k.half()), dict(v=v[:, :1]), dict(s=slots.int()), dict(s=slots[:4]), dict(kc=q8c.k), dict(kc=q8c.k, vc=q8c.v), dict(k_scale=q8c.ks, v_scale=q8c.vs), dict(kc=q8c.k, vc=q8c.v, k_scale=q8c.ks),
               dict(q=q), dict(q=q, q_out=q), dict(q=q, q_out=q[:, :2], positions=pos, freqs=freqs), dict(positions=pos), dict(s=slots.cpu()), dict(kc=cache.k[:, :1]), dict(k=k.float(), v=v.float()),
               dict(kc=cache.k.float(), vc=cache.v.float())):
        with pytest.raises(AssertionError):
            write(**kw)
    wide = torch.zeros(4, 2, 16, 68, dtype=torch.bfloat16, device=cuda_device)
    for kw in (dict(kc=wide[..., :64], vc=wide[..., :64]), dict(positions=pos, freqs=freqs.repeat(2)), dict(kc=wide.flatten()[4:4 + 4 * 2 * 16 * 64].view(4, 2, 16, 64)), dict(k=k[:1].expand(5, 2, 64)),
               dict(k=k[:0], v=v[:0], s=slots[:0])):
        with pytest.raises(cf.ComfuseError):
            write(**kw)
    with pytest.raises(AssertionError):
        cf.cache_read(cache.k, cache.v, slots, k, v[:4])
    torch.cuda.synchronize()
    assert torch.isnan(cache.k).all() and torch.isnan(cache.v).all()
