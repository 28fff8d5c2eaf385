"""Outputs whose rows lie on each other (a broadcast tensor's) are refused by the rotary calls, since several rows would be written
to one place (CPU only; the addresses are never read).  Inputs may be broadcast."""
import pytest

import paper_2609_24270_amd as asym
from tests.test_draft_oracles import APPEND, ROPE, code


@pytest.mark.parametrize("change", [dict(yt=0), dict(yh=0), dict(yt=56), dict(yh=56), dict(yt=64, yh=64), dict(yt=0, yh=0), dict(T=3, H=1, yt=0),
                                    dict(T=1, H=2, yh=8)])
def test_rope(change):
    assert code("asym_rope_bf16", *{**ROPE, **change}.values()) == asym.EINVAL
    assert "rows of y" in asym.last_error()


@pytest.mark.parametrize("change", [dict(qot=0), dict(qoh=0), dict(qot=120), dict(qoh=64), dict(qot=128), dict(T=1, qoh=0)])
def test_append(change):
    assert code("asym_kv_append_bf16", *{**APPEND, **change}.values()) == asym.EINVAL
    assert "rows of q_out" in asym.last_error()

