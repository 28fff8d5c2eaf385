"""Loads that go straight to LDS (CPU only: the sources and hipcc -S for gfx950).

Such a load takes its LDS address from M0, and the scalar write of M0 needs one
wait state before it: issued at once, the load may still see the address before.
The compiler keeps to that for its own loads but does not look into inline asm,
so there the instruction between the two stands in the text, and M0, which the
text writes, is declared.
"""
import os
import re

import pytest

from tests.test_kernel_structure import CSRC, asm_of

SOURCES = ["attn_prefill.hip", "gemm.hip", "gemm_skinny.hip", "mla_decode.hip"]


def instructions(asm: str):
    """Every instruction in order (the labels between them left out)."""
    out = []
    for line in asm.splitlines():
        s = line.split(";")[0].strip()
        if s and not s.startswith(".") and not s.endswith(":"):
            out.append(s)
    return out


def too_early(insts):
    """The loads to LDS that come right behind a write of M0."""
    return [(a, b) for a, b in zip(insts, insts[1:])
            if re.match(r"(buffer|global)_load_\S+ .*\blds\b|global_load_lds", b) and re.match(r"s_\w+ m0,", a)]


def test_the_check_itself():
    load = "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"
    assert too_early(["s_mov_b32 m0, s1", load]) == [("s_mov_b32 m0, s1", load)]
    assert not too_early(["s_mov_b32 m0, s1", "s_nop 0", load, load])
    assert not too_early(["s_mov_b32 m0, s1", "buffer_load_dwordx4 v[0:3], v1, s[4:7], 0 offen"])


@pytest.mark.parametrize("src", SOURCES)
def test_a_wait_state_behind_every_write_of_m0(src, tmp_path):
    insts = instructions(asm_of(src, tmp_path))
    assert any(re.search(r"\blds\b", i) for i in insts)
    assert not too_early(insts), (len(too_early(insts)), too_early(insts)[:2])


@pytest.mark.parametrize("src", SOURCES)
def test_asm_that_writes_m0_says_so(src):
    with open(os.path.join(CSRC, src)) as f:
        blocks = [b for b in re.findall(r"asm volatile\((.*?)\);", f.read(), re.S) if re.search(r"\bm0,", b)]
    assert blocks
    for b in blocks:
        assert re.search(r':[^:]*"m0"[^:]*$', b), b
