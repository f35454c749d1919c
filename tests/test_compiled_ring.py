"""The attention over the 4-bit cache keeps tiles in flight into a ring in LDS and waits for a counted
number of them (s_waitcnt vmcnt), which is right only while a tile's loads are exactly the
instructions that the count assumes, each with its LDS address in m0 just before it; its other form
holds a tile in registers that every load fills whole.  Read from the library built here, on the CPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2509_18344_amd import _binding

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
HERE = os.path.dirname(_binding.__file__)
VM, RING = 6, 4  # loads of a tile, tiles of a wavefront's ring


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Instructions of every k_kv4_partial, by its template arguments (QW, QG, G, RING)."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("needs the ROCm toolchain")
    tmp = tmp_path_factory.mktemp("ring")
    lib = shutil.copy(os.path.join(HERE, "libsubspec.so"), tmp / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp, check=True, capture_output=True, timeout=60)
    found = {}
    for f in sorted(tmp.glob("*gfx950*")):
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", "--no-leading-addr", str(f)],
                              check=True, capture_output=True, text=True, timeout=120).stdout
        if "k_kv4_partial" not in text:
            continue
        key = None
        for line in text.splitlines():
            m = re.match(r".*<(\w+)>:$", line)
            if m:
                key = None
                if "k_kv4_partial" in m.group(1):
                    key = (*(int(v) for v in re.findall(r"Li(\d+)E", m.group(1))), "Lb1E" in m.group(1))
            elif key and line.split():
                found.setdefault(key, []).append(line.split("//")[0].split())
    assert len(found) == 12, sorted(found)
    return found


def test_the_rings_waits_count_the_tiles_loads(kernels):
    for key, code in kernels.items():
        if not key[3]:
            continue
        ops = [" ".join(i) for i in code]
        names = [i[0] for i in code]
        # three tiles ahead of the loop and one in it: a tile's own loads, or as many of one word
        assert names.count("global_load_lds_dwordx4") == RING * 4 and names.count("global_load_lds_dword") == RING * (2 + VM), key
        waits = [k for k, o in enumerate(ops) if re.match(r"s_waitcnt vmcnt\(%d\)$" % ((RING - 1) * VM), o)]
        assert len(waits) == 1, (key, waits)
        first = next(k for k, o in enumerate(ops) if o.startswith("global_load_lds"))
        memory = [n for n in names[first:] if n.startswith(("global_load", "buffer_", "flat_", "scratch_")) and "lds" not in n]
        assert not memory, (key, memory)  # nothing else that the counts would have to know of
        # LDS reads of the last step are back before a load may overwrite them
        loop = max(k for k in range(waits[0]) if names[k].startswith("ds_") or "lgkmcnt(0)" in ops[k])
        assert "lgkmcnt(0)" in ops[loop], (key, ops[loop])


def test_m0_is_written_for_its_load_alone(kernels):
    for key, code in kernels.items():
        ops = [" ".join(i) for i in code]
        for k, o in enumerate(ops):
            if "m0" in re.split(r"\W+", o):
                assert re.match(r"s_mov_b32 m0, s\d+$", o) and ops[k + 1] == "s_nop 0" and ops[k + 2].startswith("global_load_lds"), \
                    (key, ops[k:k + 3])
            if o.startswith("global_load_lds"):
                assert ops[k - 2].startswith("s_mov_b32 m0,"), (key, ops[k - 2:k + 1])


def test_assembly_that_writes_m0_says_so():
    seen = 0
    for f in sorted(os.listdir(os.path.join(HERE, "csrc"))):
        with open(os.path.join(HERE, "csrc", f)) as src:
            for stmt in re.findall(r"asm volatile\((.*?)\);", src.read(), re.S):
                if re.search(r"\bm0\b,", stmt.split("::")[0]):
                    seen += 1
                    assert '"m0"' in stmt.rsplit(":", 1)[1], (f, stmt)
    assert seen >= 2


def test_a_tile_in_registers_is_loaded_whole(kernels):
    for (qw, _, g, ring), code in kernels.items():
        if ring:
            continue
        names = [i[0] for i in code]
        # codes, scales and minima 16 bytes a load: the first tile, the next of committed positions and the
        # next under the masks; the queries' rows; the masks' words
        assert names.count("global_load_dwordx4") == 3 * ((2 + 2 * g) + (2 + g + 1)) + 4 * qw, (qw, g)
        assert names.count("global_load_dword") == 4 and not {"global_load_dwordx2", "global_load_dwordx3"} & set(names)
