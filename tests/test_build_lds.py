"""The packed kernels' LDS addresses stay within what each kernel declares: behind it the
hardware may have some bytes left over, or drop writes and read zeros."""

import os
import re

import pytest

from paper_2602_21196_amd import build as B
from test_build import _assembly

LDS = 160 * 1024          # of a CU: no address is larger
# What an address is formed by; larger literals are no places in LDS.
FORMS = r"\tv_(?:add|add3|lshl_add|lshl_or|or|or3|xor|xad|mov)_\w+ .*?\b0x([0-9a-f]+)\b"


def _beyond(text):
    """Per kernel: its declared bytes, and the instructions that name a place behind them."""
    size = {name: int(n) for n, name in re.findall(
        r"\.group_segment_fixed_size: (\d+).*?\n\s+\.name:\s+(\w+)", text, flags=re.S)}
    found = {}
    for name, n in size.items():
        body = text[text.index(f"\n{name}:"):]
        body = body[:body.index("\n.Lfunc_end")]
        far = [m.group(0) for m in re.finditer(FORMS, body) if n <= int(m.group(1), 16) < LDS
               and re.search(r"\tds_", body)]
        far += [m.group(0) for m in re.finditer(r"\tds_.*? offset:(\d+)", body)
                if int(m.group(1)) >= n]
        found[name] = (n, far)
    return found


def test_places_behind_the_end_are_found():
    body = ("\nk:\n\tv_add_u32_e32 v1, 0x10000, v1\n\tds_write_b32 v1, v2 offset:512\n"
            "\tv_mov_b32_e32 v3, 0xff800000\n.Lfunc_end0:\n")
    meta = "    .group_segment_fixed_size: {}\n    .name:           k\n"
    assert len(_beyond(body + meta.format(65536))["k"][1]) == 1
    assert len(_beyond(body + meta.format(512))["k"][1]) == 2
    assert _beyond(body + meta.format(66048))["k"] == (66048, [])


@pytest.mark.parametrize("name", ["varlen_fwd.hip", "varlen_bwd.hip", "norm_rope.hip"])
def test_no_place_behind_the_declared_lds(name):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    found = _beyond(_assembly(name))
    assert found
    assert not {k: v for k, v in found.items() if v[1]}
