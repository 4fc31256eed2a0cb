"""Spills of the norm kernels (CPU only): none where a lane takes one step of 8 elements, and no more than the stated ones in the kernels
of longer rows, which are compiled for 1024 lanes and so for 128 registers.  (A spill and its reload pass through memory beside the
rows, and the compiler's wait for it is one for the rows on their way.)"""

import os
import re

import pytest

from paper_2510_08726_amd import build as libbuild

ASM = os.path.join(libbuild.unit_dir("rmsnorm"), f"rmsnorm-hip-amdgcn-amd-amdhsa-{libbuild.ARCH}.s")
SOURCES = ["rmsnorm.hip", "kernel_common.h", "launch.h"]
# (kernel, steps of a lane, 8 bits, widths that are no multiple of 8) -> registers spilled at most, over the types.
MOST = {("add", 2, 1, 0): 25, ("add", 4, 0, 0): 70, ("add", 4, 0, 1): 268, ("add", 4, 1, 0): 208, ("add", 4, 1, 1): 225,
        ("bwd", 2, 0, 1): 5, ("bwd", 4, 0, 0): 177, ("bwd", 4, 0, 1): 404}


@pytest.fixture(scope="module")
def spills():
    newest = max(os.path.getmtime(os.path.join(libbuild.CSRC, s)) for s in SOURCES)
    if not os.path.exists(ASM) or os.path.getmtime(ASM) < newest:
        import __graft_entry__
        __graft_entry__.build()
    found = {}
    for entry in re.split(r"\n  - \.agpr_count", open(ASM).read())[1:]:
        name = re.search(r"\.name:\s+(\S+)", entry).group(1)
        found[name] = int(re.search(r"\.vgpr_spill_count:\s+(\d+)", entry).group(1))
    return found


def test_no_more_spills_than_stated(spills):
    kinds = {}
    for name, n in spills.items():
        m = re.search(r"rmsnorm_add_(bwd_)?kernelI\w+?Li(\d)ELb(\d)E(?:Lb(\d)E)?E", name)
        if not m:
            assert n == 0, name
            continue
        bwd = m.group(1) is not None
        key = ("bwd" if bwd else "add", int(m.group(2)), 0 if bwd else int(m.group(3)), int(m.group(3) if bwd else m.group(4)))
        kinds.setdefault(key, []).append(n)
    assert len(kinds) == 12 + 6 and all(len(n) == 5 for n in kinds.values())
    for key, n in kinds.items():
        assert max(n) <= MOST.get(key, 0), (key, n)
