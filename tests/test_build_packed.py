"""What the packed kernels' sources rely on in the code that the compiler makes of them."""

import os
import re

import pytest

from paper_2602_21196_amd import build as B
from test_build import _assembly, _outside_asm


@pytest.mark.parametrize("name", ["varlen_fwd.hip", "varlen_bwd.hip"])
def test_copies_keep_m0_and_no_kernel_spills(name):
    """The written-out copies use m0, which nothing around them may; and the sums stay in
    registers, which the kernels' comments and layouts were made for."""
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    text = _assembly(name)
    assert re.search(r"s_mov_b32 m0,", text)
    found = [line.strip() for line in _outside_asm(text) if re.search(r"\bm0\b", line)]
    assert not found, found[:5]
    spills = [int(n) for n in re.findall(r"\.vgpr_spill_count:\s*(\d+)", text)]
    assert spills and not any(spills), spills
