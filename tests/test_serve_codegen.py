"""Guards on the device code of the operators around the 4-bit cache (CPU only).

The decode kernel's waves count the copies that they have in flight to LDS
(s_waitcnt vmcnt) and nothing else: a spill to scratch, or any other load or
store between the copies, would be counted with them, and a tile read before
it has arrived.  The tests read the assembly that build() keeps.
"""

import os
import re

import pytest

from paper_2510_08726_amd import build as libbuild


@pytest.fixture(scope="module")
def asm():
    files = libbuild.serve_asm_files()
    if not all(os.path.exists(f) for f in files):
        import __graft_entry__
        __graft_entry__.build()
    return "\n".join(open(f).read() for f in files)


def kernels(asm):
    """Name -> the lines of each kernel."""
    out, name = {}, None
    for line in asm.split("\n"):
        m = re.match(r"^(_ZN4attn\S+):", line)
        if m:
            name = m.group(1)
            out[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name:
            out[name].append(line.split(";")[0].rstrip())
    return out


def tile_loop(lines):
    """The innermost loop that holds matrix instructions."""
    label = {m.group(1): i for i, l in enumerate(lines) if (m := re.match(r"^(\.LBB\w+):", l))}
    best = None
    for i, l in enumerate(lines):
        m = re.search(r"\bs_c?branch\w*\s+(\.LBB\w+)", l)
        if m and label.get(m.group(1), i) < i:
            body = lines[label[m.group(1)]:i + 1]
            if any("v_mfma" in x for x in body) and (best is None or len(body) < len(best)):
                best = body
    return best


def test_the_kernels_built(asm):
    names = [n for n in re.findall(r"^\s*\.amdhsa_kernel\s+(\S+)", asm, flags=re.M)]
    count = lambda s: sum(s in n for n in names)     # noqa: E731
    # 2 head dims x 2 types x 2 column counts x ALiBi x SoftCap; the others per head dim and type
    assert count("17decode_kv4_kernel") == 32 and count("decode_kv4_combine_kernel") == 4
    assert count("kv4_append_kernel") == 4 and count("kv4_load_kernel") == 4 and count("kv_slots_kernel") == 1
    # 16-byte vectors: few heads, several, several streamed; shorter ones and elements: few, several; 2 pairings
    assert count("rope_kernel") == 2 * (2 * (3 + 2 + 2) + 3 + 2)
    assert len(names) == 32 + 4 + 9 + 38


def test_no_scratch(asm):
    sizes = re.findall(r"\.private_segment_fixed_size:\s+(\d+)", asm)
    assert len(sizes) == 83 and set(sizes) == {"0"}
    assert not re.search(r"^\s*scratch_", asm, flags=re.M)


def test_no_packed_fp32(asm):
    assert not re.search(r"^\s*v_pk_(add|mul|fma)_f32", asm, flags=re.M)


def test_tile_loop_waits_for_copies_alone(asm):
    seen = 0
    for name, lines in kernels(asm).items():
        if "17decode_kv4_kernel" not in name:
            continue
        seen += 1
        body = tile_loop(lines)
        wide = "ILi128E" in name
        ops = [l.split()[0] for l in body if l.startswith("\t") and l.split() and not l.split()[0].startswith(".")]
        memory = [o for o in ops if o.startswith(("global_", "buffer_", "flat_"))]
        assert sorted(memory) == (["global_load_lds_dword"] + ["global_load_lds_dwordx4"] * (4 if wide else 2)), name
        waits = {int(m) for m in re.findall(r"s_waitcnt vmcnt\((\d+)\)", "\n".join(body))}
        ring = 2 if wide and "Li1ELb" in name else 4
        # The wait of the last tile may sit on a path of its own, outside the loop's body.
        assert waits <= {k * (5 if wide else 3) for k in range(ring)}, (name, waits)
        assert (ring - 1) * (5 if wide else 3) in waits, (name, waits)
        assert not any("vmcnt" in l and not re.search(r"s_waitcnt vmcnt\(\d+\)$", l) for l in body), name
    assert seen == 32
