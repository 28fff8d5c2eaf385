"""Prompt attention in the form of long prompts (256-row tiles), through the C ABI.

A call takes that form by its sizes (`wide`).  What it computes for a row does not depend on
the form: the same 32 rows share a wave, and every block of keys is taken in the same order.  So each
sequence of a wide batch has the bits of that sequence in a call of its own that takes
128-row tiles, which tests/test_gpu_prefill.py compares with the oracle element by element.  A
sequence that would be cut along its keys there, and sampled rows of the others, are compared
with the oracle here, within the same derived bound.
"""
import pytest
import torch

import paper_2609_24270_amd as asym
from tests.test_gpu_prefill import SCALE, check, dev, i32, inputs, offsets  # noqa: F401 (dev: a fixture)

pytestmark = pytest.mark.gpu


def wide(B, Tq, Hq, Hkv):
    rows = Tq * (Hq // Hkv)
    return rows // 256 * Hkv >= 512 and rows > 128 * B


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0))


def alone(q, k, v, cu_q, cu_k, b, causal=True, lse=None):
    """Sequence b in a call of its own (128-row tiles): its rows of O; None if it would be cut."""
    rows, keys = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
    Lq, Lk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
    assert not wide(1, Lq, q.shape[1], k.shape[1])
    if asym._prefill_workspace(1, q.shape[1], k.shape[1], Lq, Lk):
        return None
    return asym.attn_prefill(q[rows], k[keys], v[keys], i32([0, Lq], q.device), i32([0, Lk], q.device), lse=lse, causal=causal)


WIDE = [  # query lengths, key lengths, H_q, H_kv: group sizes that divide 256 and that do not, every rule for the heads' places
    ([1300, 0, 1, 23, 700, 33, 257, 1300, 500], [1300, 40, 1, 2000, 700, 700, 257, 2100, 180], 32, 8),
    ([1700, 4, 1700], [1777, 900, 1700], 40, 8),        # 5 heads a group: a tile is 51.2 tokens
    ([1000, 31, 1000], [1000, 31, 1111], 72, 24),       # 3 heads a group, 24 key/value heads
    ([1500, 1300, 129], [1500, 1364, 129], 48, 3),      # 3 key/value heads
    ([2000, 40, 2100], [2000, 40, 2100], 32, 1),
    ([4000, 200, 4000], [4000, 327, 3900], 16, 16),     # (rows of the last one see nothing)
    # more sequences than a wave looks at once, most of them a tile and a bit
    ([61 + b % 7 for b in range(66)] + [5, 0], [61 + b % 7 + b % 5 * 9 for b in range(66)] + [70, 3], 32, 8)]


@pytest.mark.parametrize("lq,lk,Hq,Hkv", WIDE)
@pytest.mark.parametrize("causal", [True, False])
def test_a_wide_batch_is_its_sequences(dev, lq, lk, Hq, Hkv, causal):
    cu_q, cu_k = offsets(lq), offsets(lk)
    assert wide(len(lq), cu_q[-1], Hq, Hkv)
    q, k, v = inputs(dev, cu_q[-1], cu_k[-1], Hq, Hkv, seed=Hq + len(lq))
    lse = torch.full((cu_q[-1], Hq), 7.0, device=dev)
    o = asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev), lse=lse, causal=causal)
    compared = 0
    for b, n in enumerate(lq):
        rows, keys = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        if n == 0:
            continue
        l1 = torch.empty((n, Hq), device=dev)
        one = alone(q, k, v, cu_q, cu_k, b, causal, l1)
        if one is None:
            check(q[rows], k[keys], v[keys], [0, n], [0, lk[b]], SCALE, causal, o[rows], lse[rows])
            continue
        assert torch.equal(o[rows], one) and torch.equal(lse[rows], l1), b
        compared += n
    assert 2 * compared > cu_q[-1]
    # the oracle on single rows, over the keys that each sees
    for b, n in enumerate(lq):
        for i in sorted({0, n // 3, n - 1}) if n > 1 else []:
            r, left = cu_q[b] + i, (i + lk[b] - n + 1 if causal else lk[b])
            if left <= 0:
                assert not o[r].any() and torch.all(lse[r] == -float("inf"))
                continue
            ks = slice(cu_k[b], cu_k[b] + left)
            check(q[r:r + 1], k[ks], v[ks], [0, 1], [0, left], SCALE, causal, o[r:r + 1], lse[r:r + 1])
    for mapping in ("oblivious_grouped", "oblivious_rowmajor", "aware"):
        assert torch.equal(o, asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev), causal=causal, mapping=mapping))


def test_thousands_of_one_token_sequences(dev):
    # as many rows as a wide call has, but one token (a row of four heads) in each tile: 128-row tiles
    n, Hq, Hkv = 4200, 32, 8
    assert not wide(n, n, Hq, Hkv)
    lk = [1 + (7 * b) % 90 for b in range(n)]
    lk[1700] = 900
    cu_q, cu_k = offsets([1] * n), offsets(lk)
    q, k, v = inputs(dev, n, cu_k[-1], Hq, Hkv, seed=1)
    o = asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev))
    for a in range(0, n, 700):
        assert asym._prefill_workspace(700, Hq, Hkv, 700, cu_k[a + 700] - cu_k[a]) == 0
        keys = slice(cu_k[a], cu_k[a + 700])
        part = asym.attn_prefill(q[a:a + 700], k[keys], v[keys], i32(offsets([1] * 700), dev), i32(offsets(lk[a:a + 700]), dev))
        assert torch.equal(o[a:a + 700], part)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_cannot_reach_it(dev, bad):
    lq, lk = [1100, 1300, 800, 1300], [1100, 1427, 800, 1300]
    cu_q, cu_k = offsets(lq), offsets(lk)
    q, k, v = inputs(dev, cu_q[-1], cu_k[-1], 32, 8, seed=21)
    assert wide(len(lq), cu_q[-1], 32, 8)
    run = lambda k, v: asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev))
    clean = run(k, v)
    at = [(0, 63, 0), (0, 700, 3), (1, 127 + 65, 7), (1, 1426, 2), (2, 0, 1), (2, 511, 6), (3, 1023, 4), (3, 1024, 5)]
    v2, k2 = v.clone(), k.clone()
    hit = torch.zeros(clean.shape, dtype=torch.bool, device=dev)
    seen, near = (torch.zeros(clean.shape[:2], dtype=torch.bool, device=dev) for _ in range(2))
    for b, j, h in at:
        first = cu_q[b] + max(j - (lk[b] - lq[b]), 0)  # the first row that sees key j
        v2[cu_k[b] + j, h, 11] = v2[cu_k[b] + j, h, 120] = bad
        k2[cu_k[b] + j, h] = bad
        hit[first:cu_q[b + 1], 4 * h:4 * h + 4, 11] = hit[first:cu_q[b + 1], 4 * h:4 * h + 4, 120] = True
        seen[first:cu_q[b + 1], 4 * h:4 * h + 4] = True
        near[cu_q[b] + (first - cu_q[b]) // 8 * 8:first, 4 * h:4 * h + 4] = True  # in a wave (8 tokens of 4 heads) with it
    got = run(k, v2)
    assert torch.equal(got[~hit], clean[~hit])
    x = got[hit].float()
    assert torch.all(torch.isnan(x)) if bad != bad else torch.all(x == bad)
    for b in range(len(lq)):
        assert same(got[cu_q[b]:cu_q[b + 1]], alone(q, k, v2, cu_q, cu_k, b))
    # A wave raises its rows' maxima together, so what one of them sees may change how its
    # neighbours are rounded, and nothing else: both are within the bound of the exact result,
    # whose A is at most max |v| (and the fp32 part less than 2^-10 of it).
    got = run(k2, v)
    assert torch.equal(got[~seen & ~near], clean[~seen & ~near])
    a, c = got[near & ~seen].float(), clean[near & ~seen].float()
    assert a.numel() and torch.all((a - c).abs() <= 2 * (2.0 ** -8 * (1 + 2.0 ** -8) + 2.0 ** -10) * (v.float().abs().max() + c.abs()))


def test_opposite_infinities(dev):
    # of both signs in one block and in two, in a wide tile's edge blocks and before them
    lq = [1500, 1300, 1400]
    cu = offsets(lq)
    q, k, v = inputs(dev, cu[-1], cu[-1], 32, 8, seed=22)
    assert wide(len(lq), cu[-1], 32, 8)
    inf = float("inf")
    v[cu[1] + 70, 2, 3], v[cu[1] + 100, 2, 3], v[cu[1] + 200, 2, 9], v[cu[1] + 900, 2, 9] = inf, -inf, -inf, inf
    o = asym.attn_prefill(q, k, v, i32(cu, dev)).float()
    mine = o[cu[1]:cu[2], 8:12]
    assert torch.all(torch.isfinite(mine[:70])) and torch.all(mine[70:100, :, 3] == inf) and torch.all(torch.isnan(mine[100:, :, 3]))
    assert torch.all(torch.isfinite(mine[:200, :, 9])) and torch.all(mine[200:900, :, 9] == -inf)
    assert torch.all(torch.isnan(mine[900:, :, 9]))
    mine[..., 3] = mine[..., 9] = 0
    assert torch.all(torch.isfinite(o))


def test_strided_views_and_rows_outside(dev):
    g = torch.Generator().manual_seed(23)
    T, Hq, Hkv = 4300, 32, 8
    qkv = torch.randn((T, Hq + 2 * Hkv, 128), generator=g).to(torch.bfloat16).to(dev)
    lq = [1300, 0, 1450, 1460]
    cu = offsets(lq, first=7)
    qkv[:7], qkv[cu[-1]:] = float("nan"), float("inf")
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    assert wide(len(lq), T, Hq, Hkv)
    o = torch.full((T, Hq, 128), 7.0, dtype=torch.bfloat16, device=dev)
    lse = torch.full((T, Hq), 7.0, device=dev)
    asym.attn_prefill(q, k, v, i32(cu, dev), o=o, lse=lse)
    assert torch.all(o[:7] == 7) and torch.all(o[cu[-1]:] == 7) and torch.all(lse[:7] == 7) and torch.all(lse[cu[-1]:] == 7)
    for b in (0, 2, 3):
        assert torch.equal(o[cu[b]:cu[b + 1]], alone(q, k, v, cu, cu, b))
    # head-major storage gives the same bits
    qh, kh, vh = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))
    assert torch.equal(o, asym.attn_prefill(qh, kh, vh, i32(cu, dev), o=torch.full_like(o, 7.0)))


def test_one_key_value_head_read_by_all(dev):
    # broadcast heads (a stride of 0) are the heads of their copy
    cu = i32(offsets([1500, 2700]), dev)
    q, k, v = inputs(dev, 4200, 4200, 32, 1, seed=24)
    ke, ve = k.expand(4200, 8, 128), v.expand(4200, 8, 128)
    a = asym.attn_prefill(q, ke, ve, cu)
    assert torch.equal(a, asym.attn_prefill(q, ke.contiguous(), ve.contiguous(), cu))


def test_offsets_that_say_too_much_are_held(dev):
    q, k, v = inputs(dev, 4100, 4000, 32, 8, seed=25)
    o = torch.full((4100, 32, 128), 7.0, dtype=torch.bfloat16, device=dev)
    asym.attn_prefill(q, k, v, i32([-9, 4100, 2000000000, 20], dev), i32([-3, 2 ** 31 - 1, 50, 7], dev), o=o)
    assert torch.equal(o, asym.attn_prefill(q, k, v, i32([0, 4100], dev), i32([0, 4000], dev)))


def test_captured_and_replayed_on_another_stream(dev):
    T = 4200
    cu = i32(offsets([1300, 1400, 1500]), dev)
    q, k, v = inputs(dev, T, T, 32, 8, seed=26)
    o, lse = torch.empty_like(q), torch.empty((T, 32), device=dev)
    asym.attn_prefill(q, k, v, cu, o=o, lse=lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        asym.attn_prefill(q, k, v, cu, o=o, lse=lse)
    side = torch.cuda.Stream()
    for seed in (1, 2, 3):
        q2, k2, v2 = inputs(dev, T, T, 32, 8, seed=seed)
        q.copy_(q2), k.copy_(k2), v.copy_(v2)
        cu.copy_(i32(offsets([1300 - seed, 1400 + 64 * seed, 1500 - 63 * seed]), dev))
        o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        ref = asym.attn_prefill(q2, k2, v2, cu)  # beside it
        torch.cuda.synchronize()
        assert torch.equal(o, ref)
