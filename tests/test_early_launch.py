"""Kernels that may be placed while the grid before them still runs read what
that grid may have written by ordinary loads: the non-coherent path (__ldg) is
for data that is constant as long as the kernel is there."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_22167_gb300", "csrc")
NON_COHERENT = re.compile(r"__ldg\b|ld\.global(\.\w+)*\.nc\b")


def _code(name):
    src = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", src, flags=re.S)


@pytest.mark.parametrize("name", ["norm_rope.cu", "page_ops.cu", "tree_attn.cu"])
def test_no_non_coherent_loads_of_what_kernels_write(name):
    src = _code(name)
    assert "grid_dep_launch()" in src
    if name == "norm_rope.cu":  # weights and angles, which no kernel writes
        src, n = re.subn(r"void load4\(.*?\n}\n", "", src, flags=re.S)
        assert n == 1
    assert not NON_COHERENT.search(src)
