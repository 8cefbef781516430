"""What the compiler makes of places whose speed or correctness hangs on the order
of memory instructions (gfx950 assembly of single kernels; no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2607_08991_amd import build

SM_GATEUP = [("uint16_t", mt) for mt in (1, 2, 3, 4)] + [("float", mt) for mt in (1, 2, 3, 4)]


@pytest.fixture(scope="module")
def sm_gateup(tmp_path_factory):
    """Memory and barrier instructions of each sm_gateup_kernel, in order."""
    folder = tmp_path_factory.mktemp("asm")
    src, out = str(folder / "k.hip"), str(folder / "k.s")
    with open(src, "w") as f:
        f.write('#include <hip/hip_runtime.h>\n#include "prefill.hpp"\n')
        for t, mt in SM_GATEUP:
            f.write(f"template __global__ void sats::sm_gateup_kernel<{t}, {mt}>(sats::PfArgs, int);\n")
    cmd = [a for a in build.command(out) if a not in build.SOURCES and a not in ("-shared", "-fPIC")]
    subprocess.run(cmd + ["-I", build.CSRC, "--cuda-device-only", "-S", src], check=True, capture_output=True)
    kernels, name = {}, None
    for line in open(out):
        m = re.match(r"_ZN4sats16sm_gateup_kernelI(\w)Li(\d)E\w*:", line)
        if m:
            name = ({"t": "uint16_t", "f": "float"}[m[1]], int(m[2]))
            kernels[name] = []
        elif "s_endpgm" in line:
            name = None
        elif name and re.search(r"\b(buffer_load|s_waitcnt|s_barrier)", line):
            kernels[name].append(line.strip())
    return kernels


@pytest.mark.parametrize("t,mt", SM_GATEUP)
def test_the_route_lookup_delays_no_stage(sm_gateup, t, mt):
    """sm_gateup_kernel reads a row's id first, then issues four of its five stages or
    more (three loads each), and only then waits for the id and reads its table entry,
    in front of the first barrier (whose wait counts that load)."""
    ins = sm_gateup[(t, mt)]
    first_stage = next(i for i, l in enumerate(ins) if l.endswith("lds"))
    assert any("buffer_load_dword " in l for l in ins[:first_stage])
    assert not any("vmcnt" in l for l in ins[:first_stage]), ins[:first_stage]
    entry = next(i for i, l in enumerate(ins) if "buffer_load_ubyte" in l)
    barrier = next(i for i, l in enumerate(ins) if "s_barrier" in l)
    assert entry < barrier
    assert sum(l.endswith("lds") for l in ins[:barrier]) == 15
    issued = sum(l.endswith("lds") for l in ins[:entry])
    waits = [int(m[1]) for l in ins[:entry] for m in [re.search(r"vmcnt\((\d+)\)", l)] if m]
    assert issued >= 12 and waits == [issued], ins[:entry]  # (only the id is waited for)


@pytest.fixture(scope="module")
def rows8_loops(tmp_path_factory):
    """The vector memory instructions and waits of the loops of the kernels that decode over 8-bit caches."""
    folder = tmp_path_factory.mktemp("asm8")
    src, out = str(folder / "k.hip"), str(folder / "k.s")
    with open(src, "w") as f:
        f.write('#include <hip/hip_runtime.h>\n#include "attend8.hpp"\n')
        for t in ("uint16_t", "float"):
            for dim in (64, 128, 256):
                f.write(f"template __global__ void sats::attend_rows8_kernel<{t}, sats::kE4m3, {dim}, true>(sats::AttendArgs);\n")
    cmd = [a for a in build.command(out) if a not in build.SOURCES and a not in ("-shared", "-fPIC")]
    subprocess.run(cmd + ["-I", build.CSRC, "--cuda-device-only", "-S", src], check=True, capture_output=True)
    kernels, name = {}, None
    for line in open(out):
        m = re.match(r"_ZN4sats19attend_rows8_kernelI(\w)Li1ELi(\d+)E\w*:", line)
        if m:
            name = ({"t": "uint16_t", "f": "float"}[m[1]], int(m[2]))
            kernels[name] = []
        elif ".Lfunc_end" in line:
            name = None
        elif name and re.search(r"\b(buffer_load|s_waitcnt|ds_read_b64_tr_b8)|ASMEND", line):
            kernels[name].append(line.strip())
    return kernels


@pytest.mark.parametrize("t", ["uint16_t", "float"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_the_wait_for_values_counts_loads_that_are_there(rows8_loops, t, dim):
    """Values come into LDS while a wave works; before it reads them it waits until at most as many loads are on their
    way as were issued since: those of the next block, and of the one after without its values.  Fewer issued than
    that would be a wait that ends too soon."""
    ins = rows8_loops[(t, dim)]
    kinds = lambda part: (sum("lds" in l for l in part if "buffer_load" in l), sum("buffer_load" in l and "lds" not in l for l in part))  # noqa: E731
    own = 2 * (dim // 64 + 2)                   # of a block: K's codes, its scales and V's
    into = 2 * dim // 64                        # its values
    want = into + 2 * own
    waits = [i for i, l in enumerate(ins) if re.fullmatch(rf"s_waitcnt vmcnt\({want}\)", l) and "ASMEND" in ins[i - 1] and "ASMEND" in ins[i + 1]]
    assert len(waits) == 2, [l for l in ins if "vmcnt" in l]
    # in front of the loop: two blocks whole; in each half of it: a block's own loads, the wait, and then its values
    first = waits[0]
    before, mid = kinds(ins[:first]), kinds(ins[first:waits[1]])
    assert before == (2 * into, 3 * own) and mid == (into, own), (before, mid)
