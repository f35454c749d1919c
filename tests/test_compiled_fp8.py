"""The 8-bit product's tiles are copied into a ring in LDS by loads written as assembly, and waited for
by a counted number of them (s_waitcnt vmcnt): right only while each load's LDS address is in m0 just
before it and the counts are those of the stages in flight.  Read from the library built here, on the CPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2509_18344_amd import _binding

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
HERE = os.path.dirname(_binding.__file__)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Instructions of every k_fp8_tiles and k_fp8_small, by name and template arguments."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("needs the ROCm toolchain")
    tmp = tmp_path_factory.mktemp("fp8")
    lib = shutil.copy(os.path.join(HERE, "libsubspec.so"), tmp / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp, check=True, capture_output=True, timeout=60)
    found = {}
    for f in sorted(tmp.glob("*gfx950*")):
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", "--no-leading-addr", str(f)],
                              check=True, capture_output=True, text=True, timeout=120).stdout
        if "k_fp8_tiles" not in text and "k_fp8_small" not in text:
            continue
        key = None
        for line in text.splitlines():
            m = re.match(r".*<(\w+)>:$", line)
            if m:
                name = re.search(r"k_fp8_(tiles|small)I", m.group(1))
                key = (name.group(1), *(int(v) for v in re.findall(r"Li(\d+)E", m.group(1)))) if name else None
                if key:
                    key += ("Lb1E" in m.group(1),)
            elif key and line.split():
                found.setdefault(key, []).append(" ".join(line.split("//")[0].split()))
    assert len(found) == 13, sorted(found)
    return found


def test_m0_is_written_for_its_load_alone(kernels):
    for key, ops in kernels.items():
        loads = [k for k, o in enumerate(ops) if o.startswith("global_load_lds")]
        assert loads, key
        for k in loads:
            assert re.match(r"s_mov_b32 m0, \S+$", ops[k - 2]) and ops[k - 1] == "s_nop 0", (key, ops[k - 2:k + 1])
        assert sum("m0" in re.split(r"\W+", o) for o in ops) == len(loads), key
        assert not any(o.startswith("scratch_") for o in ops), key  # a spill would count as a load too


def test_waits_count_the_stages_in_flight(kernels):
    for key, ops in kernels.items():
        if key[0] == "tiles":
            mf, nf, wm, wn, stages = key[1:6]
            copies = -(-(4 * mf * wm + 4 * nf * wn) // 8)
            loads = copies + 1
        else:
            mf, nf, wm, wn, wk, stages = key[1:7]
            waves, runs, words = wm * wn * wk, 4 * mf * wm + 4 * nf * wn, -(-(32 * mf * wm + 32 * nf * wn) // 64)
            assert wk * runs % waves == 0, key
            loads = wk * runs // waves + -(-wk * words // waves)
        want = (stages - 2) * loads
        meets = [ops[k - 1] for k, o in enumerate(ops) if o == "s_barrier"]
        assert any(re.match(r"s_waitcnt vmcnt\(%d\) lgkmcnt\(0\)$" % want, w) for w in meets), (key, want, meets)
        assert any(w == "s_waitcnt vmcnt(0) lgkmcnt(0)" for w in meets), (key, meets)  # the last stages
        assert all("lgkmcnt(0)" in w for w in meets), (key, meets)
