"""Which kernels free tensor memory, over all the names under which that is done.  test_expired_waits_host.py and test_q8_host.py each list the
files of one name and check what those kernels do behind an expired wait; here no third name, and no file outside the two lists, gets by."""
import os
import re

from tests import test_expired_waits_host as bf16, test_q8_host as q8

CSRC = bf16.CSRC
FREES = {"tmem_dealloc", "tmem_dealloc_pair", "tmem_release"}


def _code(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def _sources():
    return [f for f in sorted(os.listdir(CSRC)) if f.endswith((".cu", ".cuh", ".h"))]


def test_the_instruction_stands_in_the_primitives_alone():
    assert [f for f in _sources() if "tcgen05.dealloc" in _code(f)] == ["sm100_primitives.cuh"]


def test_no_other_function_of_the_headers_frees_tensor_memory():
    text = _code("sm100_primitives.cuh")
    functions = re.findall(r"__device__ __forceinline__ [\w ]*?\b(\w+)\(([^()]*)\) \{(.*?)\n\}", text, flags=re.S)
    found = {name for name, _, body in functions if "tcgen05.dealloc" in body or re.search(r"\b(%s)\(" % "|".join(FREES), body)}
    assert found == FREES
    assert not any(re.search(r"#\s*define\b.*(%s)" % "|".join(FREES), _code(f)) for f in _sources())


def test_every_file_that_frees_tensor_memory_is_in_one_list():
    users = {f for f in _sources() if f != "sm100_primitives.cuh" and re.search(r"\b(%s)\b" % "|".join(FREES), _code(f))}
    lists = [set(bf16.DRAINED), set(bf16.PAIRS), set(q8.DRAINED)]
    assert users == set().union(*lists) and sum(map(len, lists)) == len(users)
    assert {f for f in _sources() if f != "sm100_primitives.cuh" and re.search(r"\btmem_alloc\w*\(", _code(f))} == users   # whoever allocates frees
