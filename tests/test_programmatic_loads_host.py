"""How kernels read global memory, from their source.  With programmatic launch a kernel is on the SMs while the kernels in front of it still
write: griddepcontrol.wait makes their results visible to ordinary loads.  The read-only path (__ldg, ld.global.nc) is defined for
data that nobody writes while the kernel runs; its loads may be moved in front of the wait, and may find a line that a kernel before the
previous one left in the L1.  So no kernel that waits takes it."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_03537_b200", "csrc")
READ_ONLY = re.compile(r"__ldg\s*\(|ld\.global(\.\w+|::\w+)*\.nc\b|__restrict__")
Q8 = ["gemm_q8.cu", "gemm_q8_few.cu", "gemm_q8_tokens.cu", "quantize_rows.cu", "q8_common.cuh", "q8_params.h"]


def _code(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


@pytest.mark.parametrize("name", Q8)
def test_8_bit_layers_take_ordinary_loads(name):
    assert not READ_ONLY.findall(_code(name))


def test_the_8_bit_files_are_listed():
    assert sorted(f for f in os.listdir(CSRC) if re.match(r"q8_|gemm_q8|quantize", f) and f != "q8_api.cu") == sorted(Q8)


WAITING = sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh")) and "griddepcontrol.wait" in _code(f) or f.endswith((".cu", ".cuh")) and "griddep_wait()" in _code(f))
SHARED = ["epilogue_common.cuh", "fused_launch.cuh", "fused_program.cu"]   # device code of kernels that wait, in files that do not say so


@pytest.mark.parametrize("name", WAITING + SHARED)
def test_kernels_that_wait_take_ordinary_loads(name):
    text = _code(name)
    if name != "row_kernels.cu":
        assert not READ_ONLY.findall(text)
        return
    # two of its kernels are launched without the attribute, behind everything; the others wait
    for kernel in re.split(r"(?=__global__)", text)[1:]:
        waits = "griddepcontrol.wait" in kernel
        assert not (waits and READ_ONLY.findall(kernel)), kernel[:120]
    plain = re.findall(r"(\w+)(?:<[^<>]*>)?<<<", text)
    assert sorted(plain) == ["bias_gelu_kernel", "row_epilogue_kernel"]


def test_kernels_that_wait_are_found():
    assert {"few_rows.cu", "few_rows_mlp.cu", "row_kernels.cu", "fused_pair.cuh", "softmax_rows.cuh", "b2b_mlp.cu", *Q8[:4]} <= set(WAITING)
