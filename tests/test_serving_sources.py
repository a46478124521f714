"""Rules of the serving kernels that no run can show, checked on their sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_07899_b200", "csrc")


def code_of(name):
    """The source without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return re.sub(r"/\*.*?\*/", "", re.sub(r"//[^\n]*", "", text), flags=re.S)


def overlapping_sources():
    """The files whose kernels come up while the kernel before them on the stream still runs."""
    names = [n for n in sorted(os.listdir(CSRC)) if n.endswith((".cu", ".cuh"))]
    return [n for n in names if re.search(r"\blaunch_next\s*\(|griddepcontrol", code_of(n))]


def test_the_serving_kernels_are_found():
    assert set(overlapping_sources()) >= {"kv_attention.cu", "kv_join.cu", "kv_prompt.cu", "kv_store.cu", "linear_i8.cu", "serve.cuh"}


@pytest.mark.parametrize("name", overlapping_sources())
def test_kernels_that_overlap_with_their_producer_read_nothing_as_constant(name):
    """The read-only path asks for data that nobody writes in the kernel's whole life, which begins while the kernel before
    it still writes this one's inputs; and a load that is not volatile may be moved before the wait for that kernel."""
    code = code_of(name)
    for what in (r"__ldg\s*\(", r"\bld_nc_16\s*\(", r"ld\.global\.nc", r"__restrict__", r"__ldc[gsav]\s*\(", r"__ldlu\s*\("):
        assert not re.search(what, code), what
    for asm in re.findall(r"asm\s*(?:volatile\s*)?\(\s*\"ld\.global[^;]*;[^;]*;", code):
        assert re.match(r"asm\s*volatile", asm) and '"memory"' in asm, asm
