"""kv_keep has up to 1024 threads a request, and the threads of a launch are counted in 32 bits: calls past that are refused
(CPU only; the addresses are never read)."""
import pytest

import paper_2609_24270_amd as asym
from tests.test_draft_oracles import KEEP, code


@pytest.mark.parametrize("change", [
    dict(n=1 << 22, H=1, page=1 << 18), dict(n=(1 << 24) - 1, H=1, page=1 << 18), dict(n=1 << 23, H=1, page=1 << 18, vp=None),
    dict(n=1 << 22, H=3, page=1 << 17), dict(n=(1 << 24) - 1, H=1, page=1 << 17)])
def test_launches_of_2_to_the_32_threads_are_refused(change):
    args = {**KEEP, **change}
    words = args["page"] // 512 * args["H"] * (2 if args["vp"] else 1)
    assert args["n"] * min(-(-words // 64) * 64, 1024) >= 1 << 32 and args["n"] * args["H"] < 1 << 24
    assert code("asym_kv_keep", *args.values()) == asym.EUNSUPPORTED
    assert asym.last_error().startswith("kv keep: too many requests")
