"""The hand-counted wait states of the MLA score products (prefix_attn.hip), in the compiled gfx950 code.

S^T is formed by assembly MFMAs, whose hazards the compiler does not see.  It may put anything between them,
a copy or a spill of their operands too, so the code is followed instruction by instruction:

  * each such MFMA has at least 2 wait states of its own before it, for a VALU write of a source and for the
    MFMA before it, whose result it adds to in exactly the same registers;
  * nothing but that next MFMA touches a result until at least 20 wait states after the last one (a product of 16
    passes needs that many, one of 8 passes 12; an s_nop N counts N + 1, any other instruction 1).

CPU only (hipcc cross-compiles)."""
import os
import shutil
import subprocess

import pytest

from asm_waitstates import _parse, _regs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SRC = os.path.join(ROOT, "paper_2609_36938_amd", "csrc", "prefix_attn.hip")
OP = "v_mfma_f32_32x32x16_bf16"
BEFORE, AFTER = 2, 20


def check(text):
    """(assembly MFMAs seen, violations).  Code is followed as it stands in the file, over labels and branches."""
    seen, bad = 0, []
    asm, waited = False, 0
    age = {}  # registers of results, and the wait states since their last MFMA
    for line in text.splitlines():
        s = line.strip()
        if s.startswith(";;#ASMSTART"):
            asm, waited = True, 0
            continue
        if s.startswith(";;#ASMEND"):
            asm = False
            continue
        if s.startswith(".Lfunc_end"):
            age = {}
        s = s.split(";")[0].strip()
        if not s or s.endswith(":") or s.startswith("."):
            continue
        op, dst, src, acc = _parse(s)
        steps = int(s.split()[1], 0) + 1 if op == "s_nop" else 1
        ours = asm and op == OP
        if ours:
            seen += 1
            if waited < BEFORE:
                bad.append(f"{s}: {waited} wait states before it")
            c = s.split(",")[-1].strip()
            if c != "0" and _regs(c) != dst:
                bad.append(f"{s}: adds to other registers")
            touched = src - acc
            if not acc:
                touched = touched | dst  # a new sum over an old one
        else:
            touched = src | dst if op[:2] != "s_" else set()
        early = [r for r in touched if age.get(r, AFTER) < AFTER]
        if early:
            bad.append(f"{s}: v{early[0]} {age[early[0]]} wait states after its MFMA")
        for r in age:
            age[r] += steps
        if ours:
            age.update({r: 0 for r in dst})
        waited += steps
    return seen, bad


GOOD = """;;#ASMSTART
s_nop 1
v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], 0
;;#ASMEND
ds_read_b128 v[20:23], v30
v_mfma_f32_32x32x16_bf16 a[0:15], v[40:43], v[44:47], a[0:15]
;;#ASMSTART
s_nop 1
v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[28:31], v[0:15]
;;#ASMEND
;;#ASMSTART
s_nop 15
s_nop 7
;;#ASMEND
v_mul_f32_e32 v0, v0, v60
"""


def test_the_rules():
    assert check(GOOD) == (2, [])
    for old, new in (("s_nop 1\nv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[28:31]",
                      "s_nop 0\nv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[28:31]"),
                     ("v[28:31], v[0:15]", "v[28:31], v[1:16]"),
                     ("ds_read_b128 v[20:23], v30", "v_mov_b32_e32 v99, v3"),
                     ("ds_read_b128 v[20:23], v30", "scratch_store_dwordx4 off, v[12:15], s0"),
                     ("ds_read_b128 v[20:23], v30", "v_mov_b32_e32 v3, v99"),
                     ("s_nop 15\ns_nop 7", "s_nop 15"), ("s_nop 15\ns_nop 7\n", "")):
        assert old in GOOD and check(GOOD.replace(old, new, 1))[1], (old, new)


@pytest.mark.skipif(not shutil.which(HIPCC) and not os.path.exists(HIPCC), reason="hipcc not installed")
def test_compiled_products(tmp_path):
    from paper_2609_36938_amd.build import FLAGS
    out = tmp_path / "prefix_attn.s"
    r = subprocess.run([HIPCC] + FLAGS + ["--cuda-device-only", "-S", SRC, "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    seen, bad = check(out.read_text())
    assert seen >= 2 * 3 * 36                # both kernels: the first tile, the loop, the second way through
    assert not bad, "\n".join(bad[:20])
