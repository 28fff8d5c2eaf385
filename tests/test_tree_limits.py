"""The attention of drafted tokens joins pieces with a wave for two heads of a token, 256 threads a workgroup: with one head the largest
call whose threads fit 32 bits has 2^26 - 4 tokens (CPU only: what the calls would need is asked for)."""
import ctypes

import pytest

import paper_2609_24270_amd as asym
from tests.test_draft_oracles import code


@pytest.mark.parametrize("T,Hq,fits", [((1 << 26) - 4, 1, True), ((1 << 26) - 3, 1, False), ((1 << 26) - 1, 1, False), ((1 << 25) - 1, 2, True),
                                       (1 << 25, 2, False), ((1 << 26) // 3, 3, True), ((1 << 24) - 1, 4, True), (1 << 24, 4, False)])
def test_rows_of_the_joining_launch(T, Hq, fits):
    n = ctypes.c_size_t()
    assert code("asym_attn_tree_paged_workspace", 1, Hq, 1, T, 64, 0, ctypes.byref(n)) == (asym.OK if fits else asym.EUNSUPPORTED)
