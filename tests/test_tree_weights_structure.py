"""Structure of the attention of drafted tokens as it is built (CPU only: hipcc -S for gfx950): what a weight's rounding to bf16
left of it is one v_dot2 instruction, whose factors (-1, 0) and (0, -1) have to stay in registers.  As a constant the first is
written as -1.0, which the instruction reads as another pair."""
import os
import re
import subprocess

import pytest

from paper_2609_24270_amd import build
from tests.test_kernel_structure import CSRC


def differences(asm):
    """The operands of every v_dot2 instruction on bf16."""
    return [m.group(1) for m in re.finditer(r"^\s*v_dot2c?_f32_bf16\S*\s+([^;\n]*)", asm, re.M)]


def constants(asm):
    return [ops for ops in differences(asm) if not all(re.match(r"^-?[vs](\d+|\[)", x.strip().split()[0]) for x in ops.split(","))]


def test_factors_of_the_differences_are_in_registers(tmp_path):
    out = tmp_path / "attn_tree.s"
    r = subprocess.run([build.hipcc(), *build.COMMON, *build.DEVICE_ONLY, *build.EXTRA["attn_tree.hip"], "--cuda-device-only", "-S",
                        os.path.join(CSRC, "attn_tree.hip"), "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    asm = out.read_text()
    assert len(differences(asm)) >= 6 * 16  # six kernels, the weights of a block
    assert not constants(asm), constants(asm)[:2]


@pytest.mark.parametrize("line,bad", [("\tv_dot2c_f32_bf16_e32 v0, -1.0, v3", True), ("\tv_dot2c_f32_bf16_e32 v1, 0xbf800000, v3", True),
                                      ("\tv_dot2c_f32_bf16_e32 v1, s4, v3", False), ("\tv_dot2_f32_bf16 v1, v2, s3, v4", False)])
def test_the_check_finds_constants(line, bad):
    assert bool(constants(line + "\n")) == bad
