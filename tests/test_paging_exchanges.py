"""Swaps of half waves in the kernels of beam selection and of the choice of pages read no register that inline asm has just written: a vector instruction's result has to be two wait states old, and
for asm the compiler does not see to that.  The distance is counted in the assembly, with the library's flags and without those that change what lies between."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2209_09130_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
PLAIN = ["--offload-arch=gfx950", "-std=c++17", "-ffp-contract=off"]
FLAGS = {"library": [f for f in build.FLAGS if f not in ("-shared", "-fPIC")], "O3": PLAIN + ["-O3"], "O2": PLAIN + ["-O2"], "O1": PLAIN + ["-O1"]}


def registers(text):
    found = set()
    for one, low, high in re.findall(r"\bv(\d+)\b|\bv\[(\d+):(\d+)\]", text):
        found |= {int(one)} if one else set(range(int(low), int(high) + 1))
    return found


def close_pairs(assembly):
    """(number of swaps, [(asm instruction, swap, wait states between them)] of less than two)."""
    in_asm, recent, swaps, close = False, [], 0, []
    for line in assembly.splitlines():
        s = line.strip()
        if s.startswith(";;#ASMSTART"):
            in_asm = True
        elif s.startswith(";;#ASMEND"):
            in_asm = False
        elif s.endswith(":") or s.split(";")[0].strip().endswith(":") or not s.split(";")[0].strip() or s.startswith((".", "//")):
            continue                                         # (what stands in front of a label may run in front of what stands behind it)
        else:
            s = s.split(";")[0].strip()
            name, _, rest = s.partition(" ")
            operands = rest.split(",")
            if "permlane" in name and "swap" in name:
                swaps += 1
                close += [(t, s, n) for dst, n, t in recent if dst & registers(rest) and n < 2]
            states = int(operands[0], 0) + 1 if name == "s_nop" else 1
            written = registers(operands[0]) if name.startswith("v_") else set()
            recent = [(dst - written, n + states, t) for dst, n, t in recent if n + states < 2]
            if in_asm and name.startswith("v_"):
                recent.append((written, 0, s))
    return swaps, close


def test_distances_are_counted():
    text = ";;#ASMSTART\nv_max3_f32 v1, v2, v3, v4\n;;#ASMEND\n{}v_permlane32_swap_b32_e32 v7, v1\n"
    assert [n for _, _, n in close_pairs(text.format(""))[1]] == [0]
    assert [n for _, _, n in close_pairs(text.format("s_nop 0\n"))[1]] == [1]
    assert close_pairs(text.format("s_nop 1\n")) == (1, []) and close_pairs(text.format("v_add_u32 v9, v9, v9\ns_nop 0\n")) == (1, [])
    assert close_pairs(text.format("v_mov_b32_e32 v1, v5\n")) == (1, [])       # (no asm's result any more: the compiler counts those)


@pytest.mark.skipif(not shutil.which(HIPCC), reason="hipcc is not installed")
@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("source", ["page_select.hip", "beam.hip"])
def test_swaps_wait_for_what_asm_has_written(source, flags, tmp_path):
    out = tmp_path / "kernels.s"
    subprocess.run([HIPCC, *FLAGS[flags], "--cuda-device-only", "-S", "-o", str(out), os.path.join(build.CSRC, source)], check=True, stderr=subprocess.DEVNULL)
    swaps, close = close_pairs(out.read_text())
    assert swaps > 10 and not close, close[:5]
