"""The operators of a drafting step on streams with half of the chip's CUs: the same bits as on the whole chip."""
import pytest
import torch

import paper_2609_24270_amd as asym
from paper_2609_24270_amd import workloads
from tests.test_gpu_drafts import Drafts, cache
from tests.test_gpu_tree import Case, dev, i32, offsets  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stream(dev):
    topo = asym.probe_topology(0, asym.PROBE_IDENTITY | asym.PROBE_MASKMAP)
    s = asym.stream_create(topo, workloads.random_mask_bits(4, 1, 128)[0])
    yield s
    s.synchronize()
    asym.stream_destroy(s)


@pytest.mark.parametrize("new,lens,Hq,H,room", [([1] * 9, [300 * i + 5 for i in range(9)], 8, 2, 0), ([8], [777], 32, 8, 0), ([8, 20], [777, 500], 8, 2, 2000),
                                                ([40, 64], [500, 900], 8, 2, 9000), ([70, 60], [800, 333], 8, 2, 5760)])
def test_attention(dev, stream, new, lens, Hq, H, room):
    c = Case(dev, new, lens, Hq, H, seed=3, room=room)
    ref, lse = c.run(), c.lse
    torch.cuda.synchronize()
    o, again = torch.empty_like(ref), torch.empty_like(lse)
    args = [c.q, c.kp, c.vp, i32(c.kt, dev), i32(c.vt, dev), i32(c.cu, dev), i32(c.lens, dev)]
    torch.cuda.synchronize()
    asym.attn_tree_paged(*args, mask=c.mask, o=o, lse=again, stream=stream)
    stream.synchronize()
    assert torch.equal(o, ref) and torch.equal(again, lse)


@pytest.mark.parametrize("V", [5000, 40000])
def test_verification(dev, stream, V):
    d = Drafts([6, 9, 1, 20], V, seed=5, width=8, noise=2.0)
    torch.cuda.synchronize()
    args = [d.target.to(dev), d.draft.to(dev), i32(d.tokens, dev), i32(sum(d.parents, []), dev), i32(d.cu, dev), d.accept.to(dev), d.final.to(dev)]
    torch.cuda.synchronize()
    r = asym.draft_verify(*args, stream=stream)
    stream.synchronize()
    assert tuple(x.tolist() for x in r) == d.want()


def test_appends_and_keeping(dev, stream):
    g = torch.Generator().manual_seed(4)
    qkv = torch.randn((4500, 8, 128), generator=g).to(torch.bfloat16).to(dev)
    freq, table = asym.rope_freq(128)[0].to(dev), torch.arange(2 * 2 * 80, dtype=torch.int32, device=dev).view(2, 2, 80)
    cu, start = i32([0, 2100, 4500], dev), i32([3, 40], dev)

    def run(s):
        pools = [torch.zeros((320, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
        torch.cuda.synchronize()
        turned = asym.kv_append(qkv[:, 4:6], qkv[:, 6:], *pools, table, table, cu, start, q=qkv[:, :4], freq=freq, stream=s)
        back = asym.rope(qkv[:, :4], torch.arange(4500, dtype=torch.int32, device=dev), freq, backward=True, stream=s)
        _, state = cache(dev, [100, 60, 33], 4, 5, 2, 64)
        more = [i32([2, 0, 1], dev), i32([0, 10, 30, 45], dev), i32([0, 3, 4] + [-1] * 7 + [0, 5] + [-1] * 18 + list(range(15)), dev), i32([3, 2, 15], dev)]
        torch.cuda.synchronize()
        asym.kv_keep(*state, *more, stream=s)
        torch.cuda.synchronize()
        return [turned, back, *pools, *state]

    for a, b in zip(run(None), run(stream)):
        assert torch.equal(a, b)
