"""Every cut that the 8-bit calls can take, by name.  A call's form (a handful of rows, few rows, pairs; a warp, a CTA or a cluster a row) and
how it is cut over CTAs follow from its sizes by estimates; COMFUSE_VERBOSE=1 tells which one a call took.  Each case below names its own and
is compared with fp64, in all three types, by the ordinary and by the checked library: a changed estimate that leaves a cut without a
case fails here.  Sizes are ragged; those of the form for few rows give the same cut however many clusters of the GPU's CTAs fit at once."""
import collections
import os
import re
import shutil
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import q8_oracle as orc
from paper_2608_03537_b200 import build as cf_build
from tests import q8

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPE = {"bf16": 0, "f16": 1, "f32": 2}

# (rows a CTA, shares of the contraction): sizes without and with a long epilogue (an activation beyond ReLU, or a residual)
FEW = {
    (16, 1): ((17, 5, 30), (18, 3, 35)), (16, 2): ((9, 7391, 6139), (137, 764, 2988)), (16, 3): ((17, 5, 1737), (18, 9, 1702)), (16, 4): ((17, 1, 1943), (17, 1, 2013)),
    (16, 6): ((17, 1, 3139), (19, 5, 2983)), (16, 8): ((18, 1, 4051), (23, 3, 4014)),
    (32, 1): ((798, 267, 46), (808, 265, 30)), (32, 2): ((529, 312, 3262), (515, 270, 4005)), (32, 3): ((17, 184, 1896), (17, 395, 1708)), (32, 4): ((17, 131, 2055), (17, 266, 2189)),
    (32, 6): ((17, 1, 3794), (17, 156, 3075)), (32, 8): ((17, 1, 4126), (17, 1, 13474)),
    (64, 1): ((33, 9774, 38), (33, 9579, 42)), (64, 2): ((855, 389, 3996), (613, 513, 5528)), (64, 3): ((604, 386, 3636), (783, 259, 4799)), (64, 4): ((532, 259, 3668), (410, 394, 5959)),
    (64, 6): ((33, 1078, 2999), (33, 1588, 3606)), (64, 8): ((35, 1039, 4066), (33, 1179, 4696)),
    (128, 1): ((66, 10219, 40), (68, 9596, 34)), (128, 2): ((606, 1174, 5518), (953, 798, 8658)), (128, 3): ((787, 675, 4708), (998, 546, 6774)),
    (128, 4): ((491, 786, 6016), (616, 541, 12532)), (128, 6): ((66, 2088, 3180), None), (128, 8): ((66, 1040, 6131), (72, 1035, 12916)),
}
# a decoding step of a hundred sequences through wide layers: whole tiles, and sizes that fit nothing
WIDE = [(100, 16384, 4096), (128, 8192, 8192), (97, 16389, 4111), (127, 8191, 8200)]
HANDFUL = {(8, 1): (7, 20003, 2001), (8, 2): (1, 10007, 1500), (8, 4): (8, 5003, 1030), (8, 8): (3, 1001, 1300), (16, 1): (13, 20003, 1300), (16, 2): (16, 10007, 1500), (16, 4): (9, 5003, 700),
           (16, 8): (15, 1001, 2050)}
# (columns, stages, boxes, epilogue warps): sizes and activation
PAIRS = {(128, 6, 2, 8): [(520, 1030, 70, None), (400, 1500, 33, "tanh")], (256, 4, 1, 16): [(2900, 1801, 140, "sigmoid"), (2817, 1807, 1500, "gelu_tanh")],
         (256, 4, 2, 8): [(2900, 1799, 900, None), (2817, 1807, 1000, "relu")], (256, 5, 1, 8): [(2817, 1801, 1200, None), (2900, 1799, 1700, "gelu_tanh")]}
# rows to int8: M, N
ROWS = [(37, 250), (2050, 500), (2049, 1001), (5, 603), (7, 2105), (600, 8203), (2001, 2507), (600, 9001), (1, 16381), (40, 8207), (150, 16003), (301, 8195), (100, 65501), (200, 30011)]


def product(M, N, K, name, device, activation=None, bias=False, residual=False, seed=0, extra=0):
    g = torch.Generator(device=device).manual_seed(seed)
    t = q8.TYPES[name]
    wide = (K + 15) // 16 * 16
    a, b = (torch.randint(-128, 128, (n, wide), dtype=torch.int8, device=device, generator=g)[:, :K] for n in (M, N))
    sa, sb = (torch.randn(n, device=device, generator=g).exp() * k for n, k in ((M, 1 / 74), (N, K ** -0.5 / 74)))
    pad = (N + 7) // 8 * 8
    w = torch.randn(N, device=device, generator=g).to(t) if bias else None
    r = torch.randn(M, pad, device=device, generator=g).to(t)[:, :N] if residual else None
    y = q8.out((M, N), t, device, extra)
    cf.gemm_q8(a, sa, b, sb, y, bias=w, residual=r, activation=activation)
    torch.cuda.synchronize()
    f = q8.f64
    sums = (a.double() @ b.double().mT) * sa.double()[:, None] * sb.double()   # (the sums are exact: whole numbers below 2^31)
    scaled = sums.cpu().numpy()
    z = orc.activate(scaled if w is None else scaled + f(w), activation)
    if r is not None:
        z = z + f(r)
    label = f"{M} x {N} x {K} {name} {activation} bias={bias} residual={residual}"
    off = np.abs(f(y) - z) - q8.product_bound(z, scaled, t, None if w is None else f(w), None if r is None else f(r))
    assert off.max() <= 0, (label, off.max(), np.unravel_index(off.argmax(), off.shape))
    q8.check_surroundings({"Y": y}, label)


def cases(name):
    """(what the call has to say, M, N, K, activation, bias, residual)"""
    long = [("gelu_tanh", False, False), (None, True, True), ("sigmoid", True, True)]
    short = [(None, False, False), ("relu", True, False)]
    for i, ((rows, shares), sizes) in enumerate(FEW.items()):
        for size, ways, is_long in ((sizes[0], short, 0), (sizes[1], long, 1)):
            if size is not None:
                for way in (ways if rows == 128 else [ways[i % len(ways)]]):
                    yield ("few rows", rows, shares, is_long), *size, *way
    for size in WIDE:
        for ways, is_long in ((short, 0), (long, 1)):
            for way in ways[:2]:
                yield ("few rows", 128, None, is_long), *size, *way
    for i, ((rows, shares), size) in enumerate(HANDFUL.items()):
        yield ("a handful of rows", rows, shares), *size, *(long + short)[i % 5]
    for cut, sizes in PAIRS.items():
        for M, N, K, act in sizes:
            if name == "f32" and K == 900:
                K = 800
            yield ("pairs", *cut), M, N, K, act, True, K % 100 == 0


def run(name):
    d = torch.device("cuda:0")
    for i, (_, M, N, K, act, bias, residual) in enumerate(cases(name)):
        print(f"case {i}", file=sys.stderr, flush=True)
        product(M, N, K, name, d, act, bias, residual, seed=i)
    from tests import test_gpu_quantize_rows as rows
    for i, (M, N) in enumerate(ROWS):
        rows._run(M, N, name, True, i % 2 == 0, i % 3 != 0, d, i)
        rows._run(M, N, name, False, False, False, d, i + 100)
    assert cf.last_device_status() == cf.OK


def _child(name, lib=None):
    env = dict(os.environ, PYTHONPATH=ROOT, COMFUSE_VERBOSE="1")
    code = "import sys\nfrom tests import test_gpu_q8_cuts as t\n"
    if lib:
        env["COMFUSE_LIB"] = lib
        code += f"assert t.cf.LIB_PATH == {lib!r}\n"
    r = subprocess.run([sys.executable, "-c", code + f"t.run({name!r})"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-3000:]
    return r.stderr


def _products(text):
    """Per case the form and cut that its call says."""
    told = {}
    for part in re.split(r"^case ", text, flags=re.M)[1:]:
        i = int(part.split()[0])
        lines = re.findall(r"^comfuse: gemm_q8 dtype=(\d): ([^,]+), (.*)$", part, flags=re.M)
        assert len(lines) == 1, (i, lines)
        dtype, form, rest = lines[0]
        told[i] = (int(dtype), (form, *(int(n) for n in re.findall(r"\w+=(\d+)", rest))))
    return told


def _rows_told(text):
    return {tuple(m) for m in re.findall(r"^comfuse: quantize_rows dtype=(\d) norm=(\d): ([^,]+), chunks=(\d) ctas=(\d)", text, flags=re.M)}


def _check(name, text):
    told = _products(text)
    all_cases = list(cases(name))
    assert sorted(told) == list(range(len(all_cases)))
    for i, case in enumerate(all_cases):
        dtype, cut = told[i]
        assert dtype == TYPE[name]
        assert len(cut) == len(case[0]) and all(w is None or w == c for w, c in zip(case[0], cut)), (case, cut)
    rows = collections.defaultdict(set)
    for dtype, norm, form, chunks, ctas in _rows_told(text):
        assert int(dtype) == TYPE[name]
        rows[int(norm), form].add((int(chunks), int(ctas)))
    assert {c for c, _ in rows[1, "a warp a row"]} == {1, 2} and {c for c, _ in rows[0, "a warp a row"]} == {1, 2, 4}
    for norm in (0, 1):
        assert {s for _, s in rows[norm, "CTAs a row"]} == {1, 2, 4, 8}
        assert {c for c, _ in rows[norm, "CTAs a row"]} == ({1, 2, 4, 8} if norm == 0 and name != "f32" else {1, 2, 4})


@pytest.mark.parametrize("name", list(TYPE))
def test_every_cut(name, cuda_device):
    _check(name, _child(name))


@pytest.mark.parametrize("name", list(TYPE))
def test_every_cut_in_the_checked_build(name, cuda_device):
    """The checked library of these sources: built anew where they have changed, not whatever stands there."""
    lib = os.path.join(os.path.dirname(cf_build.LIB_PATH), "libcomfuse_checked.so")
    if shutil.which(cf_build._nvcc()) is None:
        if not os.path.exists(lib):
            pytest.skip("no checked library and no compiler")
    else:
        assert cf_build.build(checked=True) == lib
    _check(name, _child(name, lib))


# fp32 behind a short contraction: epilogue warps, for M, N, K, residual, 16-byte units behind a row of Y
F32_WARPS = [(16, 2900, 1800, 140, False, 2), (16, 2600, 2048, 250, False, 0), (16, 14000, 2000, 64, False, 0),
             (8, 2900, 1801, 140, False, 0), (8, 2900, 1804, 140, False, 1), (8, 2900, 1800, 140, False, 1),      # rows that are not whole 32-byte sectors, or start within one
             (8, 2560, 1792, 64, False, 0),                                                                       # one round of tiles
             (8, 8192, 4096, 64, False, 0), (8, 16384, 1912, 64, False, 0),                                       # more than the L2 holds
             (8, 2900, 1800, 140, True, 0), (8, 2900, 1800, 264, False, 0)]


def run_f32_warps():
    for i, (_, M, N, K, residual, extra) in enumerate(F32_WARPS):
        print(f"case {i}", file=sys.stderr, flush=True)
        product(M, N, K, "f32", torch.device("cuda:0"), residual=residual, seed=i, extra=extra)


def test_epilogue_warps_of_fp32_follow_the_result(cuda_device):
    """Sixteen where the call's bytes stay in the L2, rows are whole sectors and there is more than one round of tiles; else eight."""
    r = subprocess.run([sys.executable, "-c", "from tests import test_gpu_q8_cuts as t\nt.run_f32_warps()"], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT, COMFUSE_VERBOSE="1"),
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-3000:]
    told = _products(r.stderr)
    assert [told[i][1][0] for i in range(len(F32_WARPS))] == ["pairs"] * len(F32_WARPS)
    assert [told[i][1][4] for i in range(len(F32_WARPS))] == [c[0] for c in F32_WARPS]
