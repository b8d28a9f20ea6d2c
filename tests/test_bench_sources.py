"""The sources by which the benchmark tells whether a measured record is of the kernel that
runs now: all that the kernel is compiled from."""

import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2602_21196_amd", "csrc")
# Declarations of launchers for the host, no device code.
HOST_ONLY = {"kernels.h"}


def _included(name):
    with open(os.path.join(CSRC, name)) as f:
        found = re.findall(r'#include "([\w.]+)"', f.read())
    out = {name}
    for n in found:
        if n not in HOST_ONLY:
            out |= _included(n)
    return out


def test_records_name_every_source_of_their_kernel():
    for kernel, names in bench.KERNEL_SOURCES.items():
        assert set(names) == _included(names[0]), kernel


def test_a_change_of_any_source_is_a_change_of_the_hash(tmp_path, monkeypatch):
    csrc = tmp_path / "paper_2602_21196_amd" / "csrc"
    csrc.mkdir(parents=True)
    for names in bench.KERNEL_SOURCES.values():
        for n in names:
            with open(os.path.join(CSRC, n), "rb") as f:
                (csrc / n).write_bytes(f.read())
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    before = {k: bench.source_sha(k) for k in bench.KERNEL_SOURCES}
    with open(csrc / "attn_bwd_tile.h", "a") as f:
        f.write("// another product\n")
    for k, sha in before.items():
        assert (bench.source_sha(k) != sha) == (k != "attn_fwd"), k
