"""What the compiler made of the scaled matrix instruction, in the assembly of the
library's own kernels: results share no register with an 8-bit operand or an exponent
of the same instruction.  It reads an 8-bit operand in two passes, and a result that
lies in one has been seen to be read back as the operand."""
import os
import re
import subprocess

import pytest

from paper_2609_37062_amd import build

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")


def _registers(operand):
    m = re.match(r"([va])(?:\[(\d+):(\d+)\]|(\d+))$", operand)
    if not m:
        return set()  # (a constant)
    lo = int(m[2] or m[4])
    return {(m[1], i) for i in range(lo, int(m[3] or lo) + 1)}


def _scaled(text):
    """(line, result, a, b, c, exponents, whether a or b is of 8 bits) of each."""
    for line in re.findall(r"^\s*(v_mfma_scale_f32_\S+ [^;\n]*)", text, re.M):
        ops = re.split(r",\s*(?![^\[]*\])", line.split(None, 1)[1])
        ops[-1], *mods = ops[-1].split()
        d, a, b, c, sa, sb = (_registers(o) for o in ops[:6])
        wide = any(f"{m}:4" not in mods for m in ("cbsz", "blgp"))
        yield line, d, a, b, c, sa | sb, wide


def test_the_reading_of_a_line():
    one = "v_mfma_scale_f32_16x16x128_f8f6f4 v[2:5], v[74:77], v[2:9], 0, v83, v123 op_sel:[1,0,0] op_sel_hi:[0,0,0] cbsz:4"
    (line, d, a, b, c, s, wide), = _scaled("\t" + one + " ; a comment\n")
    assert wide and d & b and not d & a and not c and s == {("v", 83), ("v", 123)} and len(b) == 8
    two = "v_mfma_scale_f32_32x32x64_f8f6f4 a[0:15], v[0:3], v[4:7], a[0:15], v8, v9 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
    (line, d, a, b, c, s, wide), = _scaled(two + "\n")
    assert not wide and d == c and len(d) == 16 and s == {("v", 8), ("v", 9)}


@pytest.mark.parametrize("src", ["k_attn.hip", "k_rows.hip", "k_mx4.hip", "k_mx4_tile.hip"])
def test_results_lie_in_no_operand(src, tmp_path):
    out = tmp_path / "k.s"
    subprocess.run([build.HIPCC, *build.COMMON, "-x", "hip", "-S", "--cuda-device-only", os.path.join(build.CSRC, src), "-o", str(out)],
                   check=True, capture_output=True, timeout=600)
    n = 0
    for line, d, a, b, c, s, wide in _scaled(out.read_text()):
        n += 1
        assert not d & s, line
        for x in (a, b):
            # (4-bit operands are read in one pass: a result may take the place of one)
            assert not d & x or (not wide and d == x), line
    assert n > 0
