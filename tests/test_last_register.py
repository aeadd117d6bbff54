"""No kernel shifts 64 bits by its wavefronts' last register, which gfx950 does not always do: the library, and what the check finds."""
import os
import shutil
import subprocess

import pytest

from paper_2602_11688_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SHIFT = '''
extern "C" __global__ void NAME(unsigned long long* out) {
    unsigned long long x;
    asm volatile("v_mov_b32 REG, %1\\n\\ts_nop 4\\n\\tINS %0, REG, AMOUNT" : "=&v"(x) : "v"(threadIdx.x) : "REG", "LAST");
    out[threadIdx.x] = x;
}
'''


def test_the_library():
    assert build.shifts_by_the_last_register(build.LIB, HIPCC) == []


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
def test_what_is_found(tmp_path):
    source, want = "#include <hip/hip_runtime.h>\n", set()
    for ins in ("v_lshlrev_b64", "v_lshrrev_b64", "v_ashrrev_i64", "v_lshl_add_u64"):
        for reg, last in ((127, 127), (126, 127), (127, 135), (135, 135), (63, 63), (62, 62), (31, 32)):
            name = f"{ins}_{reg}_{last}"
            add = ins == "v_lshl_add_u64"
            text = SHIFT.replace("INS %0, REG, AMOUNT", f"{ins} %0, %0, REG, %0" if add else "INS %0, REG, -1")
            source += text.replace("NAME", name).replace("INS", ins).replace("REG", f"v{reg}").replace("LAST", f"v{last}").replace('"=&v"(x)', '"+v"(x)' if add else '"=&v"(x)')
            if reg == last and reg % 8 == 7 and not add:
                want.add(name)
    (tmp_path / "shifts.hip").write_text(source)
    out = str(tmp_path / "shifts.so")
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-shared", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", str(tmp_path / "shifts.hip"), "-o", out],
                   check=True, capture_output=True)
    found = build.shifts_by_the_last_register(out, HIPCC)
    assert {name for name, _ in found} == want and len(found) == len(want) == 9
