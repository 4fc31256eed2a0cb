"""Guards on the device code of the training operators (CPU only).

The waves of a backward pass count the copies that they have in flight to LDS; a spill in a tile loop
would wait for the copies of later tiles, and cost what they overlap.  The forward kernels
with the log-sum-exp hold their operands in fixed registers, as the others of prefill.hip do, and are
checked for the same hazards.
"""

import os
import re

import pytest

from paper_2510_08726_amd import build as libbuild
import test_isa_hazards as hazards
from test_serve_codegen import kernels, tile_loop

ASM = "{0}-hip-amdgcn-amd-amdhsa-" + libbuild.ARCH + ".s"
SOURCES = ["prefill.hip", "attn_bwd.hip", "rmsnorm.hip", "kernel_common.h", "launch.h"]


def asm_files():
    files = [os.path.join(libbuild.unit_dir(f"prefill{k}"), ASM.format("prefill")) for k in range(4, 8)]
    return files + [os.path.join(libbuild.unit_dir(u), ASM.format(u)) for u in ("attn_bwd", "rmsnorm")]


@pytest.fixture(scope="module")
def asm():
    files = asm_files()
    newest = max(os.path.getmtime(os.path.join(libbuild.CSRC, s)) for s in SOURCES)
    if not all(os.path.exists(f) and os.path.getmtime(f) >= newest for f in files):
        import __graft_entry__
        __graft_entry__.build()
    return {f: open(f).read() for f in files}


def test_the_kernels_built(asm):
    names = [n for t in asm.values() for n in re.findall(r"^\s*\.amdhsa_kernel\s+(\S+)", t, flags=re.M)]
    count = lambda s: sum(s in n for n in names)     # noqa: E731
    assert count("prefill_lse_kernel") == 32                      # 2 head dims x 2 types x 8 masks and modifiers
    assert count("10bwd_kernel") == 20                            # 2 x 2 x 5
    assert count("bwd_rows_kernel") == 4 and count("bwd_sum_kernel") == 4
    assert count("rmsnorm_add_kernel") == 60                      # 5 pairs of types x 3 lengths x 8 bits x odd
    assert count("rmsnorm_add_bwd_kernel") == 30 and count("rmsnorm_dweight_kernel") == 1
    assert count("quant8_load_kernel") == 6
    assert len(names) == 32 + 20 + 8 + 60 + 30 + 1 + 6


def test_no_packed_fp32(asm):
    for f, t in asm.items():
        assert not re.search(r"v_pk_(?:add|mul|fma)_f32", t), f


def test_tile_loops_of_the_backward_pass_have_no_spills(asm):
    text = next(t for f, t in asm.items() if "attn_bwd" in f)
    found = 0
    for name, lines in kernels(text).items():
        if "10bwd_kernel" not in name:
            continue
        label = {m.group(1): i for i, l in enumerate(lines) if (m := re.match(r"^(\.LBB\w+):", l))}
        for i, l in enumerate(lines):
            m = re.search(r"\bs_c?branch\w*\s+(\.LBB\w+)", l)
            if not m or label.get(m.group(1), i) >= i:
                continue
            body = lines[label[m.group(1)]:i + 1]
            n = sum("v_mfma" in x for x in body)
            # A loop over tiles of one kind: the four products of one tile, of a key block or (dS in two halves) a row block.
            # (Of D = 128 8 MFMAs each, of D = 64 4; the loop around several kinds holds more.)
            per = 8 if "ILi128E" in name else 4
            if n == 4 * per and len(body) < 700:
                spilled = sum("scratch_" in x for x in body)
                # With ALiBi at D = 128 the masked tiles of key blocks, two of a head, reload up to three.
                assert spilled <= (3 if "ILi128E" in name and "Lb1ELb1ELb0E" in name and len(body) > 600 else 0), (name, l, spilled)
                found += 1
    assert found >= 80
    assert tile_loop(next(v for k, v in kernels(text).items() if "10bwd_kernel" in k))


def test_forward_kernels_have_no_mfma_hazards(asm, tmp_path):
    problems, n = [], 0
    for f, text in asm.items():
        if "prefill" not in f:
            continue
        # (The parser goes by the kernels' name.)
        copy = tmp_path / "prefill.s"
        copy.write_text(text.replace("prefill_lse_kernel", "prefill_kernel"))
        for name, (insts, labels) in hazards.kernels(copy).items():
            n += 1
            problems += [f"{name}: {m}" for m in hazards.check_kernel(insts, labels)]
    assert n == 32
    assert not problems, "\n".join(problems[:20])
