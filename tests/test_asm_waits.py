"""The counted wait of the kernels that decode over 8-bit caches (as test_asm.py has it for E4M3 and whole heads), in both
formats, for heads narrower than the kernel and in phases: gfx950 assembly, no GPU."""
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2607_08991_amd import build

T, FORM = {"t": "uint16_t", "f": "float"}, {"1": "e4m3", "2": "int8"}
ROWS = [(k, t, f, dim, full) for k in ("rows", "rows_phases") for t in ("uint16_t", "float") for f in ("e4m3", "int8")
        for dim in (64, 128, 256) for full in (True, False)]
BOTH = [("both", "uint16_t", f, dim, full) for f in ("e4m3", "int8") for dim in (64, 128, 256) for full in (True, False)]


def instance(case):
    kind, t, form, dim, full = case
    f, full = {"e4m3": "sats::kE4m3", "int8": "sats::kInt8"}[form], str(full).lower()
    if kind == "both":
        return f"template __global__ void sats::attend8_phases_kernel<{f}, {dim}, {full}>(sats::AttendArgs, sats::PhaseArgs);\n"
    name, args = ("rows8_phases", "sats::AttendArgs, sats::PhaseArgs") if kind == "rows_phases" else ("rows8", "sats::AttendArgs")
    return f"template __global__ void sats::attend_{name}_kernel<{t}, {f}, {dim}, {full}>({args});\n"


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    """The vector memory instructions, waits and labels of each kernel, in order."""
    folder = tmp_path_factory.mktemp("asm")
    cases = ROWS + BOTH
    groups = [cases[i::8] for i in range(8)]

    def compile_group(i):
        src, out = str(folder / f"k{i}.hip"), str(folder / f"k{i}.s")
        with open(src, "w") as f:
            f.write('#include <hip/hip_runtime.h>\n#include "attend8.hpp"\n' + "".join(map(instance, groups[i])))
        cmd = [a for a in build.command(out) if a not in build.SOURCES and a not in ("-shared", "-fPIC")]
        subprocess.run(cmd + ["-I", build.CSRC, "--cuda-device-only", "-S", src], check=True, capture_output=True)
        return out

    kernels = {}
    with ThreadPoolExecutor(8) as pool:
        files = list(pool.map(compile_group, range(8)))
    for file in files:
        name = None
        for line in open(file):
            m = re.match(r"_ZN4sats\d+attend_(rows8|rows8_phases)_kernelI(\w)Li(\d)ELi(\d+)ELb(\d)E\w*:", line)
            b = re.match(r"_ZN4sats\d+attend8_phases_kernelILi(\d)ELi(\d+)ELb(\d)E\w*:", line)
            if m:
                name = ("rows" if m[1] == "rows8" else "rows_phases", T[m[2]], FORM[m[3]], int(m[4]), m[5] == "1")
            elif b:
                name = ("both", "uint16_t", FORM[b[1]], int(b[2]), b[3] == "1")
            if m or b:
                kernels[name] = []
            elif ".Lfunc_end" in line:
                name = None
            elif name and re.search(r"\b(buffer_load|s_waitcnt)|ASMEND", line):
                kernels[name].append(line.strip())
    return kernels


@pytest.mark.parametrize("case", ROWS + BOTH, ids=lambda c: "-".join(map(str, c)))
def test_the_wait_for_values_counts_loads_that_are_there(listings, case):
    """In each half of the loop: a block's own loads, the wait, its values; the wait leaves on their way what was issued since
    the values that it is for, and no more.  (Other loads beside these only make it wait for more.)"""
    ins, dim = listings[case], case[3]
    own, into = 2 * (dim // 64 + 2), 2 * dim // 64  # of a block: K's codes, its scales and V's; its values
    want = into + 2 * own
    waits = [i for i, l in enumerate(ins) if re.fullmatch(rf"s_waitcnt vmcnt\({want}\)", l) and "ASMEND" in ins[i - 1] and "ASMEND" in ins[i + 1]]
    assert len(waits) == 2, [l for l in ins if "vmcnt" in l]

    def loads(part):
        part = [l for l in part if "buffer_load" in l]
        return sum("lds" in l for l in part), sum("lds" not in l for l in part)

    assert loads(ins[waits[0]:waits[1]]) == (into, own)
    # in front of it two blocks whole and the next one's own (where ways part the listing has some of them twice)
    before = loads(ins[:waits[0]])
    assert before[0] >= 2 * into and before[1] >= 3 * own, before
