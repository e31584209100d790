"""What the 8-bit entry points refuse, before they touch a device (no GPU needed): the C entry points, the Python binding's checks of types,
shapes and devices, and what the kernels do behind an expired wait, read from their source."""
import ctypes
import os
import re

import pytest
import torch

import paper_2608_03537_b200 as cf

FAKE, ODD, OFF4 = (ctypes.c_void_p(4096 + n) for n in (0, 8, 2))
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_03537_b200", "csrc")


def _quantize(x=FAKE, residual=None, gamma=None, h=None, q=FAKE, scale=FAKE, values=None, **kw):
    d = cf.QuantizeDesc(cf.QUANTIZE_RMSNORM, cf.DTYPE_BF16, 4, 100, 104, 104, 104, 112, 104, 1e-5, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return cf.lib().comfuse_quantize_rows(ctypes.byref(d), x, residual, gamma, h, q, scale, values, None)


PASSED = (cf.ERR_CUDA, cf.ERR_ARCH)   # the checks let it through: no device here


@pytest.fixture
def no_device():
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up: only without a device")


def test_quantize_rows_takes(no_device):
    before = cf.launch_count()
    assert _quantize() in PASSED
    assert _quantize(residual=FAKE, gamma=FAKE, h=FAKE, values=FAKE) in PASSED                  # h in place of the residual and of x
    assert _quantize(kind=cf.QUANTIZE_PLAIN, eps=0.0, values=FAKE) in PASSED
    assert _quantize(dtype=cf.DTYPE_F32) in PASSED and _quantize(dtype=cf.DTYPE_F16) in PASSED
    assert _quantize(scale=ctypes.c_void_p(4100)) in PASSED                                     # scales are 4-byte aligned
    assert _quantize(rows=1, N=65536, ldx=65536, ldq=65536) in PASSED
    assert _quantize(ldr=0, ldh=0, ldv=0) in PASSED                                             # of tensors that are not given
    assert cf.launch_count() == before


def test_quantize_rows_refuses():
    assert cf.lib().comfuse_quantize_rows(None, FAKE, None, None, None, FAKE, FAKE, None, None) == cf.ERR_INVALID_ARG
    for kw in (dict(rows=0), dict(N=0), dict(rows=-1), dict(kind=2), dict(dtype=3), dict(dtype=-1), dict(reserved=1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(ldx=96), dict(ldq=96), dict(residual=FAKE, ldr=96), dict(h=FAKE, ldh=96), dict(values=FAKE, ldv=96), dict(x=None), dict(q=None),
               dict(scale=None), dict(kind=cf.QUANTIZE_PLAIN), dict(kind=cf.QUANTIZE_PLAIN, eps=0.0, residual=FAKE), dict(kind=cf.QUANTIZE_PLAIN, eps=0.0, gamma=FAKE),
               dict(kind=cf.QUANTIZE_PLAIN, eps=0.0, h=FAKE), dict(h=FAKE, ldh=112), dict(residual=FAKE, h=FAKE, ldr=112)):
        assert _quantize(**kw) == cf.ERR_INVALID_ARG, kw
    for kw in (dict(ldx=108), dict(ldq=104), dict(residual=FAKE, ldr=108), dict(h=ctypes.c_void_p(8192), ldh=108), dict(values=FAKE, ldv=108), dict(x=ODD), dict(residual=ODD), dict(gamma=ODD),
               dict(h=ODD), dict(q=ODD), dict(values=ODD), dict(scale=OFF4), dict(dtype=cf.DTYPE_F32, ldx=102)):
        assert _quantize(**kw) == cf.ERR_ALIGNMENT, kw
    assert _quantize(N=65537, ldx=65544, ldq=65552) == cf.ERR_UNSUPPORTED


def _gemm(A=FAKE, sa=FAKE, B=FAKE, sb=FAKE, bias=None, residual=None, Y=FAKE, **kw):
    d = cf.GemmQ8Desc(1, 5, 100, 60, 64, 64, 104, 104, 0, 0, 0, 0, cf.DTYPE_BF16, 0, 0, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return cf.lib().comfuse_gemm_q8(ctypes.byref(d), A, sa, B, sb, bias, residual, Y, None)


BATCHED = dict(batch=3, batch_stride_a=320, batch_stride_b=6400, batch_stride_r=520, batch_stride_y=520)


def test_gemm_q8_takes(no_device):
    before = cf.launch_count()
    assert _gemm() in PASSED
    assert _gemm(bias=FAKE, residual=FAKE, activation=cf.OPS["tanh"]) in PASSED                 # Y is the residual itself
    assert _gemm(**BATCHED, residual=FAKE, dtype=cf.DTYPE_F32) in PASSED
    assert _gemm(K=131071, lda=131072, ldb=131072) in PASSED
    assert _gemm(N=65536, ldy=65536) in PASSED
    assert _gemm(sa=ctypes.c_void_p(4100), sb=ctypes.c_void_p(4108)) in PASSED
    assert cf.launch_count() == before


def test_gemm_q8_refuses():
    assert cf.lib().comfuse_gemm_q8(None, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None) == cf.ERR_INVALID_ARG
    for kw in (dict(batch=0), dict(M=0), dict(N=0), dict(K=0), dict(M=-5), dict(dtype=3), dict(flags=1), dict(reserved=1), dict(activation=cf.OPS["exp"]), dict(activation=1), dict(A=None),
               dict(sa=None), dict(B=None), dict(sb=None), dict(Y=None), dict(lda=48), dict(ldb=48), dict(ldy=96), dict(residual=FAKE, ldr=96), dict(residual=FAKE, ldr=112),
               dict(BATCHED, batch_stride_a=304), dict(BATCHED, batch_stride_b=6384), dict(BATCHED, batch_stride_y=512),
               dict(BATCHED, residual=FAKE, batch_stride_r=512), dict(BATCHED, residual=FAKE, batch_stride_r=528), dict(BATCHED, batch_stride_a=0)):
        assert _gemm(**kw) == cf.ERR_INVALID_ARG, kw
    for kw in (dict(lda=72), dict(ldb=72), dict(ldy=108), dict(residual=ctypes.c_void_p(8192), ldr=108), dict(A=ODD), dict(B=ODD), dict(Y=ODD), dict(bias=ODD), dict(residual=ODD), dict(sa=OFF4),
               dict(sb=OFF4), dict(BATCHED, batch_stride_a=328), dict(BATCHED, batch_stride_b=6408), dict(BATCHED, batch_stride_y=524)):
        assert _gemm(**kw) == cf.ERR_ALIGNMENT, kw
    assert _gemm(K=131072, lda=131072, ldb=131072) == cf.ERR_UNSUPPORTED                        # sums may leave int32
    assert _gemm(N=65537, ldy=65544) == cf.ERR_UNSUPPORTED
    for M in (2 ** 31 - 256, 2 ** 31 - 1):                                                      # a tile's last row is counted in 32 bits
        assert _gemm(M=M) == cf.ERR_UNSUPPORTED


bf, i8, f32 = torch.bfloat16, torch.int8, torch.float32
z = torch.zeros


class _Stream:
    cuda_stream = 0


def _bound(name, *args):
    """A call through the binding with CPU tensors (whose device is -1); the library is never reached by what is refused."""
    return getattr(cf._bound_q8(device=False), name)(*args)


@pytest.mark.parametrize("args,text", [
    ((z(4, 16), z(4, 16, dtype=bf)), "element type"),                                # q is not int8
    ((z(4, 16, dtype=torch.float64), z(4, 16, dtype=i8)), "element type"),
    ((z(4, 16), z(4, 32, dtype=i8)), "shape"),
    ((z(4, 16), z(5, 16, dtype=i8)), "shape"),
    ((z(2, 4, 16), z(2, 4, 16, dtype=i8)), "shape"),                                 # two dimensions
    ((z(4, 32)[:, ::2], z(4, 16, dtype=i8)), "dense"),
])
def test_binding_refuses_rows(args, text):
    x, q = args
    with pytest.raises(AssertionError, match=text):
        _bound("quantize_rows", 0, x, None, None, None, q, z(4), None, 0.0, -1, _Stream())


def test_binding_refuses_other_rows():
    x, q, s = z(4, 16, dtype=bf), z(4, 16, dtype=i8), z(4)
    call = lambda residual=None, gamma=None, h=None, scale=s, values=None, device=-1: _bound("quantize_rows", 1, x, residual, gamma, h, q, scale, values, 1e-5, device, _Stream())  # noqa: E731
    for kw, text in ((dict(residual=z(4, 16)), "residual has another element type"), (dict(residual=z(1, 16, dtype=bf)), "residual has a shape"), (dict(gamma=z(16)), "gamma has another"),
                     (dict(gamma=z(1, 16, dtype=bf)), "gamma has a shape"), (dict(h=z(4, 16, dtype=torch.float16)), "h has another"), (dict(scale=z(4, dtype=bf)), "scale has another"),
                     (dict(scale=z(4, 1)), "scale has a shape"), (dict(scale=z(8)[::2]), "dense"), (dict(values=z(4, 16)), "values has another"), (dict(device=0), "x is not on the current device")):
        with pytest.raises(AssertionError, match=text):
            call(**kw)
    with pytest.raises(AssertionError, match="x has a shape"):
        _bound("quantize_rows", 0, z(16), None, None, None, z(16, dtype=i8), z(1), None, 0.0, -1, _Stream())
    with pytest.raises(TypeError):
        _bound("quantize_rows", 0)


def test_binding_refuses_products():
    def call(A=z(5, 64, dtype=i8), sa=z(5), B=z(24, 64, dtype=i8), sb=z(24), Y=z(5, 24, dtype=bf), bias=None, residual=None, device=-1):
        return _bound("gemm_q8", A, sa, B, sb, Y, bias, residual, 0, device, _Stream())
    for kw, text in ((dict(A=z(5, 64, dtype=bf)), "A has another"), (dict(B=z(24, 64, dtype=torch.uint8)), "B has another"), (dict(B=z(24, 48, dtype=i8)), "B has a shape"),
                     (dict(Y=z(5, 32, dtype=bf)), "Y has a shape"), (dict(Y=z(5, 24, dtype=torch.int32)), "Y has another"), (dict(sa=z(6)), "scale_a has a shape"), (dict(sb=z(5)), "scale_b has a shape"),
                     (dict(sb=z(24, dtype=torch.float64)), "scale_b has another"), (dict(bias=z(24)), "bias has another"), (dict(bias=z(5, dtype=bf)), "bias has a shape"),
                     (dict(residual=z(5, 24)), "residual has another"), (dict(A=z(2, 5, 64, dtype=i8)), "B has a shape"), (dict(B=z(64, 24, dtype=i8).T), "dense"), (dict(device=1), "A is not on")):
        with pytest.raises(AssertionError, match=text):
            call(**kw)


def test_unknown_activations_are_refused():
    with pytest.raises(ValueError, match="silu"):
        cf.gemm_q8(None, None, None, None, None, activation="silu")
    assert set(cf.ACTIVATIONS) == {None, "none", "relu", "gelu_tanh", "tanh", "sigmoid"}


def test_both_ways_to_describe_a_tensor_agree():
    """Through the class's DLPack exchange interface, where it has one, and through the tensor's Python interface."""
    b = cf._bound_q8(device=False)
    base = torch.zeros(6, 40, dtype=bf)
    some = [base, base[1:4, 8:24], base.view(2, 3, 40)[:, 1:], z(7, dtype=i8), z(3, 4, 5, dtype=torch.float16).transpose(0, 1), z(2, 2), z(0, 4), z(2, 3, dtype=torch.int32),
            z(4, dtype=torch.float64), torch.nn.Parameter(z(3, 8)), z(3, 8).requires_grad_(True)]
    class Plain:   # nothing but the Python interface
        def __init__(self, t):
            self.t, self.dtype, self.shape = t, t.dtype, t.shape
            self.stride, self.get_device, self.data_ptr = t.stride, t.get_device, t.data_ptr
    for t in some:
        fast, slow = b.describe(t), b.describe(Plain(t))
        kind = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2, torch.int8: 3}.get(t.dtype, -1)
        assert fast[:4] == slow[:4] == (kind, -1, t.data_ptr(), tuple(t.shape))
        assert all(f == s or n <= 1 for f, s, n in zip(fast[4], slow[4], t.shape))   # (the stride of a dimension of one element may read as 1)
    with pytest.raises(AttributeError):
        b.describe(3)


# per file: the barriers that must be drained behind an expired wait -- the last commit in front of the release of tensor memory, landing loads
DRAINED = {"gemm_q8.cu": ["bar_drain"], "gemm_q8_few.cu": ["bar_acc", "bar_full("]}


@pytest.mark.parametrize("name", sorted(DRAINED))
def test_copies_and_umma_in_flight_are_drained(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    drains = re.findall(r"mbar_drain\(([\w()%+ ]+)", text)
    assert [next(b for b in DRAINED[name] if d.startswith(b)) for d in drains] == DRAINED[name]
    assert text.index("mbar_drain(" + DRAINED[name][0]) < text.index("tmem_release")
    if name == "gemm_q8.cu":      # loads of a pair are not counted one by one: the CTA stays behind the last barrier
        assert text.rindex("linger_behind_expired_wait(w)") > text.rindex("cluster_sync_all();") > text.rindex("mbar_drain(")


def test_every_kernel_that_releases_tensor_memory_is_listed():
    users = {f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h")) and f != "sm100_primitives.cuh" and "tmem_release" in open(os.path.join(CSRC, f)).read()}
    assert users == set(DRAINED)
