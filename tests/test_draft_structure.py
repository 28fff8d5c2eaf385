"""Structure of the kernels of drafted tokens as they are built (CPU only: the source and hipcc -S for gfx950).

Their attention loads pages straight to LDS, with the address in M0, by inline asm that the compiler
does not look into; reads its arguments again in every phase, so that they do not take the registers
that the loops need; and takes other lanes' values by lane number, for which those lanes must be on.
"""
import os
import re
import subprocess

import pytest

from paper_2609_24270_amd import build
from tests.test_kernel_structure import CSRC, function_body
from tests.test_lds_loads import instructions, too_early

SOURCES = ["attn_tree.hip", "draft_verify.hip", "rotary.hip"]


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    out = {}
    for src in SOURCES:
        path = tmp_path_factory.mktemp("asm") / (src + ".s")
        cmd = [build.hipcc(), *build.COMMON, *build.DEVICE_ONLY, *build.EXTRA.get(src, []), "--cuda-device-only", "-S",
               os.path.join(CSRC, src), "-o", str(path)]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        out[src] = path.read_text()
    return out


def test_a_wait_state_behind_every_write_of_m0(built):
    insts = instructions(built["attn_tree.hip"])
    assert sum(bool(re.search(r"^buffer_load_dwordx4 .*\blds\b", i)) for i in insts) >= 4
    assert not too_early(insts), too_early(insts)[:2]


def test_asm_that_writes_m0_says_so():
    with open(os.path.join(CSRC, "attn_tree.hip")) as f:
        blocks = [b for b in re.findall(r"asm volatile\((.*?)\);", f.read(), re.S) if re.search(r"\bm0,", b)]
    assert blocks
    for b in blocks:
        assert re.search(r':[^:]*"m0"[^:]*$', b), b


@pytest.mark.parametrize("src", SOURCES)
def test_no_registers_in_memory_and_no_packed_fp32(built, src):
    asm = built[src]
    sizes = re.findall(r"\.private_segment_fixed_size:\s*(\d+)", asm)
    assert sizes and set(sizes) == {"0"}
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm)
    assert not re.search(r"\bs_(store|atomic|buffer_store|scratch_store)", asm)


@pytest.mark.parametrize("form,lds", [("Li4ELi2ELi1ELi0E", 64), ("Li4ELi2ELi1ELi2E", 64), ("Li4ELi2ELi2ELi0E", 64), ("Li4ELi2ELi2ELi2E", 64),
                                      ("Li8ELi4ELi2ELi0E", 128), ("Li8ELi4ELi2ELi2E", 128)])
def test_the_loop_waits_for_no_more_than_its_tiles(built, form, lds):
    asm = built["attn_tree.hip"]
    name = f"attn_tree_kernelI{form}"
    body = function_body(asm, name)
    # (the tiles, and a little for the workgroup's vote on infinities)
    size = int(re.search(r"\.amdhsa_kernel \S*" + name + r".*?\.amdhsa_group_segment_fixed_size (\d+)", asm, re.S).group(1))
    assert lds * 1024 <= size <= lds * 1024 + 512
    text = "\n".join(body)
    assert "v_mfma_f32_16x16x32_bf16" in text and "ds_read_b64_tr_b16" in text
    # the main loop's stretches without a branch: a block's 64 products (32 of one block of rows) are two halves, and between
    # the first and the last of each nothing waits for all loads on their way
    runs, now = [], []
    for l in body:
        if re.match(r"^\.LBB", l):
            runs.append(now)
            now = []
        now.append(l)
    half = 16 * int(form[10])
    full = [r for r in runs + [now] if sum("v_mfma" in l for l in r) >= half]
    assert len(full) >= 2
    for r in full[:2]:
        at = [i for i, l in enumerate(r) if "v_mfma" in l]
        assert not any(re.search(r"s_waitcnt.*vmcnt\(0\)", l) for l in r[at[0]:at[-1]])
