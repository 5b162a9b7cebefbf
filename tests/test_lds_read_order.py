"""The hand-written LDS reads of the 8-bit products, checked in the code that hipcc makes of them.  LDS operations end in the order of their issue, so a
wait for all but the last n of them makes the earlier ones' registers good; until then such a register is neither read nor written (the
compiler takes the output of inline assembly as written at once).  Scalar loads share the counter and end in any order: none may be issued meanwhile.
(Other vector memory operations only make the waits for loads to LDS stricter.)  A write of M0 has its wait state before a load that takes its
LDS address from it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2504_19925_amd import build
from tests.test_lds_read_waits import _vgprs, m0_without_wait

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def code_of(lines):
    """(instruction, operands, whether by hand) of every line that is one."""
    by_hand = False
    for line in lines:
        s = line.split("//")[0].strip()
        if s.startswith(";;#ASM"):
            by_hand = s == ";;#ASMSTART"
            continue
        s = s.split(";")[0].strip()
        if re.match(r"_Z\w+:", s):
            yield "entry", [s], False
            continue
        m = re.match(r"([a-z]+_\w+) ?(.*)", s)
        if m and not s.endswith(":"):
            yield m.group(1), [o.strip() for o in re.split(r", (?![^\[]*\])", m.group(2))], by_hand


def early_uses(lines):
    """(instruction, operands) that touch a register whose hand-written read may be in flight, and the number of such reads."""
    flying, found, reads = [], [], 0        # destination registers of LDS operations in the order of their issue
    for name, ops, by_hand in code_of(lines):
        if name == "s_waitcnt":
            m = re.search(r"lgkmcnt\((\d+)\)", ops[0])
            if m:
                flying = flying[len(flying) - min(int(m.group(1)), len(flying)):]
            continue
        if name in ("entry", "s_endpgm"):
            flying = []
            continue
        busy = {r for regs in flying for r in regs}
        if any(busy.intersection(_vgprs(o)) for o in ops) or (busy and re.match("s_(buffer_)?load", name)):
            found.append((name, ops))
        if name.startswith("ds_"):
            hand = by_hand and name.startswith("ds_read")
            reads += hand
            flying.append(list(_vgprs(ops[0])) if hand else [])
    return found, reads


def test_the_checks_find_what_they_look_for():
    hand = lambda s: [";;#ASMSTART", s, ";;#ASMEND"]   # noqa: E731
    a, b = hand("ds_read_b128 v[0:3], v9 offset:16"), hand("ds_read_b128 v[4:7], v9")
    use = "v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[0:7], v[8:15], a[0:3], v20, v21 op_sel_hi:[0,0,0]"
    assert early_uses(["_Zk:"] + a + b + ["s_waitcnt lgkmcnt(1)", use])[0]
    assert early_uses(["_Zk:"] + a + b + ["s_waitcnt lgkmcnt(0)", use]) == ([], 2)
    assert early_uses(["_Zk:"] + a + b + ["s_waitcnt lgkmcnt(1)", "v_mov_b32_e32 v30, v2"]) == ([], 2)
    assert early_uses(["_Zk:"] + a + ["s_waitcnt vmcnt(0)", "v_mov_b32_e32 v2, v30"])[0]
    assert early_uses(["_Zk:"] + a + ["ds_write_b32 v40, v41", "s_waitcnt lgkmcnt(1)", "v_mov_b32_e32 v2, v30"]) == ([], 1)
    assert early_uses(["_Zk:"] + a + ["s_load_dword s3, s[0:1], 0x0"])[0] and not early_uses(["_Zk:", "s_load_dword s3, s[0:1], 0x0"] + a)[0]


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
def test_registers_of_reads_in_flight_are_left_alone(tmp_path):
    out = tmp_path / "gemm8.s"
    flags = [f for f in build.FLAGS if f not in ("-fPIC", "-shared")]
    subprocess.run([HIPCC] + flags + ["--cuda-device-only", "-S", os.path.join(build.CSRC, "gemm8.hip"), "-o", str(out)], check=True, capture_output=True)
    lines = out.read_text().splitlines()
    found, reads = early_uses(lines)
    assert reads > 500 and not found, found[:5]
    found, loads = m0_without_wait(lines)
    assert loads > 200 and not found, found[:5]
