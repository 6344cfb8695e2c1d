"""Host-side guard on the generated code of every kernel (needs hipcc, no GPU): no 64-bit shift takes its amount from the last register of the
wavefront's allocation.

Such a shift now and then reads v0 in place of it on this chip.  `v_lshlrev_b64 v[46:47], v71, 1` of a kernel with 72 registers gave 1 << v0 in all lanes
of 1 to 3 in 100 of the wavefronts that were the second on their SIMD, so that lanes read another row than theirs (a loop of the adapters' shrink kernel, left
out for it: 86 of 400 runs differed; with 80, 88, 96 or 128 registers, nothing else changed, none of 4000 did).  Waits around the instruction change nothing, and no
parity test finds it reliably.  Registers are allotted by eights."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2312_08583_amd import build as B

SHIFT = re.compile(r"^\s*v_(?:lshlrev_b64|lshrrev_b64|ashrrev_i64)(?:_e64)? v\[\d+:\d+\], v(\d+),")


def shifts_by_the_last_register(assembly: str):
    """(kernel, instruction) of each; kernels of the assembly."""
    found, kernels, name, shifts = [], 0, None, []
    for line in assembly.splitlines():
        label = re.match(r"^(\w+):", line)
        if label and not line.startswith(".L"):
            name, shifts = label.group(1), []
        elif SHIFT.match(line):
            shifts.append((int(SHIFT.match(line).group(1)), line.split(";")[0].strip()))
        elif ".amdhsa_next_free_vgpr" in line:
            kernels += 1
            last = (int(line.split()[-1]) + 7) // 8 * 8 - 1
            found += [(name, text) for amount, text in shifts if amount == last]
    return found, kernels


def _kernel(shift: str, registers: int) -> str:
    return "k:\n\tv_mov_b32_e32 v0, 1\n\t%s\n\ts_endpgm\n\t.amdhsa_kernel k\n\t\t.amdhsa_next_free_vgpr %d\n\t.end_amdhsa_kernel\n" % (shift, registers)


@pytest.mark.parametrize("shift,registers,found", [
    ("v_lshlrev_b64 v[46:47], v71, 1", 72, True), ("v_lshlrev_b64 v[46:47], v71, 1", 66, True), ("v_lshrrev_b64 v[0:1], v7, s[4:5]", 8, True),
    ("v_ashrrev_i64 v[2:3], v15, v[4:5]", 13, True), ("v_lshlrev_b64 v[46:47], v71, 1", 73, False), ("v_lshlrev_b64 v[70:71], v3, 1", 72, False),
    ("v_lshlrev_b64 v[46:47], 3, v[70:71]", 72, False), ("v_lshlrev_b32_e32 v46, v71, v1", 72, False)])
def test_the_form_is_found(shift, registers, found):
    bad, kernels = shifts_by_the_last_register(_kernel(shift, registers))
    assert kernels == 1 and bad == ([("k", shift)] if found else [])


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_no_kernel_has_it(tmp_path):
    flags = [f for f in B.FLAGS if f != "-fPIC"]

    def scan(source):
        out = tmp_path / (source + ".s")
        subprocess.run(["hipcc", *flags, "-S", "--cuda-device-only", os.path.join(B.CSRC, source), "-o", str(out)], check=True, stderr=subprocess.DEVNULL)
        return shifts_by_the_last_register(out.read_text())

    with ThreadPoolExecutor(max_workers=8) as ex:
        results = dict(zip(B.SOURCES, ex.map(scan, B.SOURCES)))
    assert sum(kernels for _, kernels in results.values()) > 200
    assert not any(bad for bad, _ in results.values()), {s: bad for s, (bad, _) in results.items() if bad}
