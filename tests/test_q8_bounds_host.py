"""The checked build evaluates a predicate in front of every store to global memory that the 8-bit kernels make, from their source: whole
pieces, what stands behind the last whole piece of a row, scales, and the tiles that leave by TMA."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_03537_b200", "csrc")
STORE = re.compile(r"\b(st_16|st_8|store_chunk<\w+>|Elem<\w+>::put|tma_store_3d)\(|(?:p\.scale|qrow|vrow|hrow)\[\w+\] =")
STORES = {"quantize_rows.cu": 7, "gemm_q8.cu": 2, "gemm_q8_few.cu": 3, "gemm_q8_tokens.cu": 1}


@pytest.mark.parametrize("name", sorted(STORES))
def test_every_store_has_its_predicate(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    kernel = text[text.index("__global__"):text.index("cudaLaunchConfig_t")]
    found = list(STORE.finditer(kernel))
    assert len(found) == STORES[name], [m.group() for m in found]
    for m in found:
        # back over at most four lines to the predicate; a block that was closed in between is not the store's
        depth = 0
        for line in kernel[:m.start()].splitlines()[:-6:-1]:
            depth += line.count("}") - line.count("{")
            if "COMFUSE_IN_BOUNDS" in line and depth <= 0:
                break
        else:
            pytest.fail(f"{name}: no predicate in front of {kernel[m.start():m.start() + 60]!r}")
