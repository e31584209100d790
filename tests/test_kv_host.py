"""What the key-value cache's entry points refuse before they touch a device, the sizes of the attention's workspace, and properties of the kernels that are read from their source (no GPU
needed)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import kv_oracle as orc

FAKE, OTHER, ODD, OFF4 = (ctypes.c_void_p(n) for n in (4096, 8192, 4104, 4098))
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_03537_b200", "csrc")
PASSED = (cf.ERR_CUDA, cf.ERR_ARCH)   # the checks let it through: no device here
L = cf.lib()
ref = ctypes.byref


@pytest.fixture
def no_device():
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up: only without a device")


def _set(s, kw, *names):
    for k in list(kw):
        if hasattr(s, k):
            v = kw.pop(k)
            if isinstance(v, tuple):
                v = type(getattr(s, k))(*v)
            setattr(s, k, v)
    return s


def _rotary_of(**kw):
    r = cf.Rotary(4096, 4096, 0, 32, 1, (ctypes.c_int32 * 4)(32, 0, 0, 0), 0, 0)
    return _set(r, kw)


def _cache_of(**kw):
    three = ctypes.c_int64 * 3
    c = cf.KvCache(4096, 8192, None, None, 6, 2, 16, 64, cf.DTYPE_BF16, 0, three(2048, 1024, 64), three(2048, 1024, 64), three(0, 0, 0), three(0, 0, 0))
    return _set(c, kw)


QUANTIZED = dict(quantized=1, k_scale=4096, v_scale=4096, k_scale_strides=(32, 16, 1), v_scale_strides=(32, 16, 1))


def _rotary(x=FAKE, out=OTHER, rotary=None, **kw):
    two = ctypes.c_int64 * 2
    d = _set(cf.RotaryDesc(5, 3, 64, cf.DTYPE_BF16, two(192, 64), two(192, 64)), kw)
    return L.comfuse_rotary(ref(d), ref(rotary if rotary is not None else _rotary_of(**kw)), x, out, None)


def test_rotary_takes(no_device):
    before = cf.launch_count()
    for kw in (dict(), dict(out=FAKE), dict(dtype=cf.DTYPE_F32), dict(axes=3, sections=(10, 0, 22, 0), axis_stride=5), dict(adjacent=1, inverse=1), dict(pairs=1, sections=(1, 0, 0, 0)), dict(tokens=1, x_strides=(0, 64)),
               dict(heads=1, out_strides=(192, 3)), dict(D=512, x_strides=(1536, 512), out_strides=(1536, 512))):
        assert _rotary(**kw) in PASSED, kw
    assert cf.launch_count() == before


def test_rotary_refuses():
    for kw in (dict(x=None), dict(out=None), dict(tokens=0), dict(heads=0), dict(D=0), dict(dtype=3), dict(pairs=33, sections=(33, 0, 0, 0)), dict(pairs=0, sections=(0, 0, 0, 0)), dict(axes=0), dict(axes=5), dict(axes=2),
               dict(sections=(31, 0, 0, 0)), dict(sections=(16, 16, 0, 0)), dict(axes=2, sections=(33, -1, 0, 0), axis_stride=5), dict(axes=2, sections=(16, 16, 0, 0), axis_stride=-1), dict(adjacent=2), dict(inverse=-1),
               dict(positions=None), dict(freqs=None), dict(x_strides=(192, 56)), dict(x_strides=(-192, 64)), dict(out_strides=(0, 64)), dict(out=FAKE, out_strides=(384, 64))):
        assert (_rotary(**kw) if kw != dict(axes=2) else _rotary(axes=2, sections=(32, 0, 0, 1))) == cf.ERR_INVALID_ARG, kw
    for kw in (dict(D=60, pairs=30, sections=(30, 0, 0, 0)), dict(x=ODD), dict(out=ODD), dict(x_strides=(196, 64)), dict(out_strides=(192, 68)), dict(positions=4098), dict(freqs=4100), dict(dtype=cf.DTYPE_F32, x_strides=(194, 64))):
        assert _rotary(**kw) == cf.ERR_ALIGNMENT, kw
    assert _rotary(D=520, x_strides=(1560, 520), out_strides=(1560, 520)) == cf.ERR_UNSUPPORTED
    two = ctypes.c_int64 * 2
    d = cf.RotaryDesc(5, 3, 64, cf.DTYPE_BF16, two(192, 64), two(192, 64))
    assert L.comfuse_rotary(None, ref(_rotary_of()), FAKE, OTHER, None) == cf.ERR_INVALID_ARG
    assert L.comfuse_rotary(ref(d), None, FAKE, OTHER, None) == cf.ERR_INVALID_ARG


def _write(k=FAKE, v=FAKE, q=None, q_out=None, slots=FAKE, turned=True, **kw):
    two = ctypes.c_int64 * 2
    d = _set(cf.CacheWriteDesc(5, 0 if q is None else 4, two(128, 64), two(128, 64), two(256, 64), two(256, 64)), {a: kw.pop(a) for a in ("tokens", "q_heads", "q_strides", "q_out_strides") if a in kw} |
             {a[1:]: kw.pop(a) for a in ("_k_strides", "_v_strides") if a in kw})
    r = _rotary_of(**{a: kw.pop(a) for a in ("pairs", "sections", "inverse") if a in kw})
    c = _cache_of(**kw)
    return L.comfuse_cache_write(ref(d), ref(c), ref(r) if turned else None, k, v, q, q_out, slots, None)


def _read(k=FAKE, v=FAKE, slots=FAKE, **kw):
    two = ctypes.c_int64 * 2
    d = _set(cf.CacheReadDesc(5, 0, two(128, 64), two(128, 64)), {a: kw.pop(a) for a in ("tokens", "reserved") if a in kw})
    return L.comfuse_cache_read(ref(d), ref(_cache_of(**kw)), slots, k, v, None)


def _attention(q=FAKE, table=FAKE, lengths=FAKE, slopes=None, out=OTHER, lse=None, workspace=FAKE, bytes=1 << 25, size=False, **kw):
    three = ctypes.c_int64 * 3
    d = cf.PagedAttentionDesc(3, 2, 8, 10, three(1024, 512, 64), three(1024, 512, 64), 10, 0, 0, 0.125, 0.0)
    _set(d, kw)
    c = _cache_of(**kw)
    if size:
        n = ctypes.c_size_t(7)
        return L.comfuse_paged_attention_workspace_size(ref(d), ref(c), ref(n)), n.value
    return L.comfuse_paged_attention(ref(d), ref(c), q, table, lengths, slopes, out, lse, workspace, bytes, None)


def test_cache_calls_take(no_device):
    before = cf.launch_count()
    for kw in (dict(), dict(q=FAKE, q_out=FAKE), dict(turned=False), QUANTIZED, dict(QUANTIZED, dtype=cf.DTYPE_F16), dict(k_strides=(2048, 64, 128)), dict(heads=1, k_strides=(1024, 0, 64)), dict(tokens=1, _k_strides=(0, 64))):
        assert _write(**kw) in PASSED, kw
    for kw in (dict(), QUANTIZED, dict(v_strides=(4096, 1024, 64))):
        assert _read(**kw) in PASSED, kw
    for kw in (dict(), QUANTIZED, dict(slopes=FAKE, lse=FAKE), dict(window=5, max_length=100, softcap=3.0), dict(tokens=1, q_strides=(512, 0, 64), out_strides=(512, 0, 64)), dict(max_length=64, workspace=None, bytes=0),
               dict(batch=1, table_stride=0)):
        assert _attention(**kw) in PASSED, kw
    assert cf.launch_count() == before


BAD_CACHES = [(cf.ERR_INVALID_ARG, [dict(k=None), dict(v=None), dict(pages=0), dict(heads=0), dict(page_size=0), dict(D=0), dict(dtype=cf.DTYPE_F32), dict(quantized=2), dict(quantized=1), dict(k_scale=4096),
                                    dict(QUANTIZED, v_scale=None), dict(k_strides=(2048, 1024, 56)), dict(v_strides=(-2048, 1024, 64)), dict(QUANTIZED, k_scale_strides=(32, 16, 0)), dict(k_strides=(2048, 0, 64))]),
              (cf.ERR_ALIGNMENT, [dict(D=60), dict(QUANTIZED, D=56), dict(k=4104), dict(v=8200), dict(k_strides=(2048, 1028, 64)), dict(QUANTIZED, k_strides=(2048, 1032, 64)), dict(QUANTIZED, k_scale=4098)]),
              (cf.ERR_UNSUPPORTED, [dict(page_size=65537)])]


def test_caches_are_refused():
    for status, cases in BAD_CACHES:
        for kw in cases:
            # (k and v are the cache's here: the calls' own are not touched)
            c = _cache_of(**kw)
            two, three = ctypes.c_int64 * 2, ctypes.c_int64 * 3
            D = c.D
            w = cf.CacheWriteDesc(5, 0, two(1024, 512), two(1024, 512), two(0, 0), two(0, 0))
            r = cf.CacheReadDesc(5, 0, two(1024, 512), two(1024, 512))
            a = cf.PagedAttentionDesc(3, 2, 8 * max(1, c.heads), 10, three(8192, 4096, 512), three(8192, 4096, 512), 10, 0, 0, 0.125, 0.0)
            assert L.comfuse_cache_write(ref(w), ref(c), None, FAKE, FAKE, None, None, FAKE, None) == status, (kw, D)
            assert L.comfuse_cache_read(ref(r), ref(c), FAKE, FAKE, FAKE, None) == status, kw
            assert L.comfuse_paged_attention(ref(a), ref(c), FAKE, FAKE, FAKE, None, OTHER, None, FAKE, 1 << 25, None) == status, kw
    assert L.comfuse_cache_read(ref(r), None, FAKE, FAKE, FAKE, None) == cf.ERR_INVALID_ARG
    assert _write(D=264, k_strides=(2 ** 20, 2 ** 16, 264), v_strides=(2 ** 20, 2 ** 16, 264)) == cf.ERR_UNSUPPORTED


def test_cache_write_and_read_refuse():
    for kw in (dict(k=None), dict(slots=None), dict(tokens=0), dict(q=FAKE), dict(q_out=FAKE), dict(q=FAKE, q_out=FAKE, turned=False), dict(inverse=1), dict(pairs=40, sections=(40, 0, 0, 0)), dict(_k_strides=(0, 64)),
               dict(_v_strides=(128, 32)), dict(q=FAKE, q_out=FAKE, q_out_strides=(512, 64)), dict(q=FAKE, q_out=OTHER, q_strides=(256, 0)), dict(q_heads=-1)):
        assert _write(**kw) == cf.ERR_INVALID_ARG, kw
    for kw in (dict(k=ODD), dict(v=ODD), dict(slots=ctypes.c_void_p(4100)), dict(q=ODD, q_out=FAKE), dict(q=FAKE, q_out=ODD), dict(_k_strides=(132, 64))):
        assert _write(**kw) == cf.ERR_ALIGNMENT, kw
    for kw in (dict(k=None), dict(v=None), dict(slots=None), dict(tokens=0), dict(reserved=1)):
        assert _read(**kw) == cf.ERR_INVALID_ARG, kw
    for kw in (dict(k=ODD), dict(v=ODD), dict(slots=ctypes.c_void_p(4100))):
        assert _read(**kw) == cf.ERR_ALIGNMENT, kw


def test_attention_refuses():
    for kw in (dict(q=None), dict(table=None), dict(lengths=None), dict(out=None), dict(batch=0), dict(tokens=0), dict(q_heads=0), dict(q_heads=7), dict(table_width=0), dict(max_length=-1), dict(window=-1),
               dict(alpha=float("inf")), dict(softcap=-1.0), dict(softcap=float("nan")), dict(table_stride=9), dict(q_strides=(1024, 512, 0)), dict(out_strides=(1024, 512, 56)),
               dict(out=FAKE, out_strides=(2048, 512, 64)), dict(out=FAKE, out_strides=(1024, 512, 128))):
        assert _attention(**kw) == cf.ERR_INVALID_ARG, kw
    long = dict(table_width=4096, table_stride=4096)   # room for sequences that are cut
    for kw in (dict(q=ODD), dict(out=ODD), dict(table=OFF4), dict(lengths=OFF4), dict(slopes=OFF4), dict(lse=OFF4), dict(long, workspace=ODD), dict(q_strides=(1028, 512, 64))):
        assert _attention(**kw) == cf.ERR_ALIGNMENT, kw
    for kw in (dict(tokens=65), dict(table_width=2 ** 28, table_stride=2 ** 28), dict(batch=2 ** 30)):
        assert _attention(**kw) == cf.ERR_UNSUPPORTED, kw
    need = _attention(size=True, **long)[1]
    for kw in (dict(long, workspace=None), dict(long, bytes=need - 1)):
        assert _attention(**kw) == cf.ERR_WORKSPACE, kw
    assert L.comfuse_paged_attention_workspace_size(None, ref(_cache_of()), ref(ctypes.c_size_t())) == cf.ERR_INVALID_ARG
    assert _attention(size=True, q_heads=7)[0] == cf.ERR_INVALID_ARG


def test_workspace_is_bounded():
    assert _attention(size=True, max_length=64) == (cf.OK, 0)   # nothing to be cut
    r = np.random.RandomState(1)
    for _ in range(300):
        heads, group = int(r.randint(1, 17)), int(r.randint(1, 33))
        q8 = bool(r.randint(2))
        D = int(r.choice([16, 64, 80, 128, 256]))
        st, n = _attention(size=True, **(QUANTIZED if q8 else {}), D=D, heads=heads, q_heads=heads * group, tokens=int(r.randint(1, 65)), batch=int(2 ** r.uniform(0, 8)), table_width=int(2 ** r.uniform(0, 14)),
                           window=int(r.choice([0, 100])), table_stride=1 << 20)
        assert st == cf.OK and 0 <= n <= cf.PAGED_ATTENTION_WORKSPACE_BYTES and n % 16 == 0


z = torch.zeros
bf = torch.bfloat16


class _Stream:
    cuda_stream = 0


def _bound(name, *args):
    """A call through the binding with CPU tensors (whose device is -1); the library is never reached by what is refused."""
    return getattr(cf._bound_kv(device=False), name)(*args, -1, _Stream())


def test_binding_refuses():
    x, pos, freqs = z(4, 2, 32), z(4, dtype=torch.int32), z(16, dtype=torch.float64)
    rotary = lambda x=x, pos=pos, freqs=freqs, sections=None, out=x: _bound("rotary", x, pos, freqs, sections, False, False, out)  # noqa: E731
    for kw, text in ((dict(x=x.double()), "x has another"), (dict(x=x[0]), "x has a shape"), (dict(pos=pos.long()), "positions has another"), (dict(pos=pos[:3]), "positions has a shape"), (dict(freqs=freqs.float()), "freqs has another"),
                     (dict(pos=z(5, 4, dtype=torch.int32)), "axes"), (dict(pos=z(2, 4, dtype=torch.int32)), "sections"), (dict(sections=(16, 0)), "axes"), (dict(sections=(15,)), "add up"), (dict(sections=(-1,)), "add up"),
                     (dict(out=x.to(bf)), "out has another"), (dict(out=x[:, :1]), "out has a shape"), (dict(out=z(4, 2, 64)[..., ::2]), "dense")):
        with pytest.raises(AssertionError, match=text):
            rotary(**kw)
    with pytest.raises(TypeError):
        rotary(sections=3)
    k, kc, slots = z(4, 2, 32, dtype=bf), z(3, 2, 8, 32, dtype=bf), z(4, dtype=torch.int64)
    codes, scale = z(3, 2, 8, 32, dtype=torch.int8), z(3, 2, 8)
    read = lambda kc=kc, vc=kc, ks=None, vs=None, s=slots, k=k, v=k: _bound("cache_read", kc, vc, ks, vs, s, k, v)  # noqa: E731
    for kw, text in ((dict(kc=kc[0]), "k_cache has a shape"), (dict(kc=kc.half()), "k_cache has another"), (dict(vc=kc[:2]), "v_cache has a shape"), (dict(kc=codes), "v_cache has another"), (dict(kc=codes, vc=codes), "has k_scale"),
                     (dict(ks=scale, vs=scale), "belong to"), (dict(kc=codes, vc=codes, ks=scale, vs=scale.half()), "v_scale has another"), (dict(kc=codes, vc=codes, ks=scale[:, :1], vs=scale), "k_scale has a shape"),
                     (dict(s=slots.int()), "slots has another"), (dict(s=slots[:2]), "slots has a shape"), (dict(k=k.float()), "k has another"), (dict(k=k[:, :1]), "k has a shape"), (dict(v=k[:3]), "v has a shape")):
        with pytest.raises(AssertionError, match=text):
            read(**kw)
    with pytest.raises(AssertionError, match="together"):
        _bound("cache_write", k, k, kc, kc, None, None, slots, k, None, None, None, None, False, False)
    with pytest.raises(AssertionError, match="missing"):
        _bound("cache_write", k, k, kc, kc, None, None, slots, k, k, None, None, None, False, False)
    q, table, n = z(2, 4, 32, dtype=bf), z(2, 5, dtype=torch.int32), z(2, dtype=torch.int32)

    def attend(q=q, kc=kc, table=table, alpha=1.0, cap=0.0, window=0, most=None, n=n, slopes=None, out=q, lse=None, ws=None):
        return _bound("paged_attention", q, kc, kc, None, None, table, alpha, cap, window, most, n, slopes, out, lse, ws)

    for kw, text in ((dict(q=q.float()), "q has another"), (dict(q=q[0]), "q has a shape"), (dict(q=q[..., :16]), "q has a shape"), (dict(kc=kc.half()), "k_cache has another"), (dict(table=table.long()), "page_table has another"),
                     (dict(table=table[:1]), "page_table has a shape"), (dict(n=n.long()), "lengths has another"), (dict(n=z(3, dtype=torch.int32)), "lengths has a shape"), (dict(out=q.half()), "out has another"),
                     (dict(out=q[:, None]), "out has a shape"), (dict(slopes=z(5)), "slopes has a shape"), (dict(lse=z(2, 1, 4)), "lse has a shape"), (dict(lse=z(4, 2).T), "dense"), (dict(window=-1), "window"),
                     (dict(most=0), "max_length"), (dict(ws=z(4, 4).T), "dense")):
        with pytest.raises(AssertionError, match=text):
            attend(**kw)


def test_structures_are_those_of_the_header(tmp_path):
    """Sizes and offsets, asked of the C compiler."""
    structs = {"comfuse_rotary_t": cf.Rotary, "comfuse_rotary_desc_t": cf.RotaryDesc, "comfuse_kv_cache_t": cf.KvCache, "comfuse_cache_write_desc_t": cf.CacheWriteDesc, "comfuse_cache_read_desc_t": cf.CacheReadDesc,
               "comfuse_paged_attention_desc_t": cf.PagedAttentionDesc}
    lines = [f'printf("%zu\\n", sizeof({c}));' + "".join(f'printf("%zu\\n", offsetof({c}, {f}));' for f, *_ in s._fields_) for c, s in structs.items()]
    src = tmp_path / "t.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"comfuse.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }")
    import subprocess
    subprocess.run([os.environ.get("CC") or "gcc", "-I", os.path.join(os.path.dirname(os.path.dirname(CSRC)), "include"), str(src), "-o", str(tmp_path / "t")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()]
    want = [x for s in structs.values() for x in (ctypes.sizeof(s), *(getattr(s, f).offset for f, *_ in s._fields_))]
    assert got == want


STORE = re.compile(r"\b(?:st_16|st_8|store_piece<\w+>|Elem<\w+>::put)\(|(?:c\.scale|p\.lse|part)\[[^\n]*?\] =|\*reinterpret_cast<uint32_t\*>\(to\) =|\*lse =")
STORES = {"kv_cache.cu": 12, "paged_attention.cuh": 10}


@pytest.mark.parametrize("name", sorted(STORES))
def test_every_store_has_its_predicate(name):
    """The checked build evaluates a predicate in front of every store to global memory."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    kernel = text[text.index("__global__"):text.index("cudaLaunchConfig_t")]
    found = list(STORE.finditer(kernel))
    assert len(found) == STORES[name], [m.group() for m in found]
    for m in found:
        depth = 0
        for line in kernel[:m.start()].splitlines()[:-16:-1] + [kernel[:m.start()].splitlines()[-1]]:
            depth += line.count("}") - line.count("{")
            if "COMFUSE_IN_BOUNDS" in line and depth <= 0:
                break
        else:
            pytest.fail(f"{name}: no predicate in front of {kernel[m.start():m.start() + 60]!r}")


# ---- the oracle itself
def test_oracle_rotary_is_a_rotation():
    r = np.random.RandomState(0)
    x, pos, freqs = r.standard_normal((5, 2, 12)), r.randint(0, 1000, (2, 5)), np.array([1.0, 0.3, 0.01, 2.0])
    for adjacent in (False, True):
        y = orc.rotary(x, pos, freqs, (1, 3), adjacent)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 8:], x[..., 8:])
        assert np.allclose(orc.rotary(y, pos, freqs, (1, 3), adjacent, inverse=True), x)
        i, j = (6, 7) if adjacent else (3, 7)
        a = pos[1] * 2.0
        assert np.allclose(y[:, 0, i], x[:, 0, i] * np.cos(a) - x[:, 0, j] * np.sin(a))
        # the score of a turned query and key depends on the distance alone (one axis)
        q, k = (orc.rotary(x, p, freqs, None, adjacent) for p in (pos[0], pos[0] - 7))
        far = [orc.rotary(x, p + 1000, freqs, None, adjacent) for p in (pos[0], pos[0] - 7)]
        assert np.allclose((q * k).sum(-1), (far[0] * far[1]).sum(-1))


def test_oracle_attention_is_the_softmax():
    r = np.random.RandomState(1)
    q, kc = r.standard_normal((2, 2, 4, 8)), r.standard_normal((3, 2, 4, 8))
    table, lengths = np.array([[2, 0], [1, -1]]), np.array([7, 0])
    out, lse, _ = orc.attention(q, kc, kc, table, lengths, 0.5)
    keys = np.concatenate([kc[2, 1], kc[0, 1]])[:7]
    s = 0.5 * keys @ q[0, 1, 3]
    assert np.allclose(out[0, 1, 3], np.exp(s - lse[0, 1, 3]) @ keys) and np.isclose(np.exp(lse[0, 1, 3]), np.exp(s).sum())
    assert np.isclose(np.exp(lse[0, 0, 3]), np.exp(0.5 * keys[:6] @ q[0, 0, 3]).sum())
    assert np.all(out[1] == 0) and np.all(lse[1] == -np.inf)
    one, lse1, _ = orc.attention(q, kc, kc, table, lengths, 0.5, window=1)
    assert np.allclose(one[0, 1, 3], keys[6]) and np.isclose(lse1[0, 1, 3], s[6])
