"""GPU parity of prompt attention over packed sequences, through the C ABI.

Against the float64 oracle, element by element.  The bound (derived, not fitted): the
probabilities are rounded to bf16 before the second product, at most 2^-8 of each, so
2^-8 A in the output (A = sum_j w_j |v_j|), and the output once more, 2^-8 |O|; what is
computed in fp32 adds a relative error to each weight of at most 2^-24 times
(131 N for a score's 128 products and its scaling, twice for numerator and maximum; 8
for the exponential's argument and value) and to the two sums of 2^-24 each per key,
together A * 2^-23 * (264 N + 16 + keys).
"""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import prompt
from tests.checks import bf16_bits_to_f64

pytestmark = pytest.mark.gpu

SCALE = 128 ** -0.5


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    asym.load_library()
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


def f64(t):
    return bf16_bits_to_f64(t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16))


def offsets(lens, first=0):
    return (np.cumsum([0] + list(lens)) + first).tolist()


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def inputs(dev, Tq, Tk, Hq, Hkv, seed, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    mk = lambda *s: (torch.randn(s, generator=g) * sigma).to(torch.bfloat16).to(dev)
    return mk(Tq, Hq, 128), mk(Tk, Hkv, 128), mk(Tk, Hkv, 128)


def check(q, k, v, cu_q, cu_k, scale, causal, o, lse, rows=None):
    R, Rl, A, N = prompt.prompt_attention(f64(q), f64(k), f64(v), cu_q, cu_k, scale, causal)
    got, gl = f64(o), lse.double().cpu().numpy()
    keys = max([b - a for a, b in zip(cu_k, cu_k[1:])] + [1])
    inside = ~np.isnan(Rl)
    assert inside.any()
    eps32 = 2.0 ** -23 * (264 * N + 16 + keys)
    bound = 2.0 ** -8 * (1 + 2.0 ** -8) * (A + np.abs(R)) + A * eps32[..., None] + 1e-37
    assert np.all(np.isfinite(got[inside]))
    worst = float(np.max((np.abs(got - R) / bound)[inside]))
    assert worst <= 1, worst
    empty = inside & (Rl == -np.inf)
    assert np.all(got[empty] == 0) and np.all(gl[empty] == -np.inf)
    some = inside & ~empty
    assert np.all(np.abs(gl[some] - Rl[some]) <= 2.0 ** -23 * (132 * N + 16 + keys + np.abs(Rl))[some])


CASES = [  # query lengths, key lengths, H_q, H_kv
    ([1], [1], 1, 1), ([1], [300], 4, 1), ([64], [64], 4, 4), ([65], [65], 8, 2), ([32, 31], [32, 31], 16, 1),
    ([7, 0, 33], [7, 0, 33], 6, 2), ([5, 3], [2, 9], 4, 2), ([0], [5], 4, 2), ([4], [0], 4, 2), ([129], [129], 1, 1),
    ([200, 1, 17], [200, 90, 17], 10, 2), ([40], [170], 3, 3), ([3, 50, 1, 2], [70, 50, 1, 65], 35, 5),
    ([20], [20], 32, 1), ([130, 2], [193, 2], 8, 8), ([1] * 70, [3] * 70, 8, 2), ([9] * 20, [9] * 20, 40, 8),
    ([2], [130], 8, 16 // 2)]


@pytest.mark.parametrize("lq,lk,Hq,Hkv", CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_against_oracle(dev, lq, lk, Hq, Hkv, causal):
    cu_q, cu_k = offsets(lq), offsets(lk)
    q, k, v = inputs(dev, max(cu_q[-1], 1), max(cu_k[-1], 1), Hq, Hkv, seed=sum(lq) + 7 * Hq)
    if cu_q[-1] == 0:
        o = torch.full((1, Hq, 128), 3.0, dtype=torch.bfloat16, device=dev)
        lse = torch.full((1, Hq), 3.0, device=dev)
        asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev), o=o, lse=lse, causal=causal)
        assert torch.all(o == 3.0) and torch.all(lse == 3.0)
        return
    lse = torch.empty((q.shape[0], Hq), device=dev)
    o = asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev), lse=lse, causal=causal)
    check(q, k, v, cu_q, cu_k, SCALE, causal, o, lse)


@pytest.mark.parametrize("scale,sigma", [(0.0, 1.0), (-0.11, 1.0), (3.0, 1.0), (SCALE, 8.0), (1e-30, 1.0)])
def test_scales(dev, scale, sigma):
    cu = offsets([70, 9])
    q, k, v = inputs(dev, 79, 79, 6, 2, seed=5, sigma=sigma)
    lse = torch.empty((79, 6), device=dev)
    o = asym.attn_prefill(q, k, v, i32(cu, dev), lse=lse, scale=scale)
    check(q, k, v, cu, cu, scale, True, o, lse)


def test_strided_views_and_rows_outside(dev):
    # a fused projection's output; sequences that start behind row 0 and end before the last
    g = torch.Generator().manual_seed(11)
    qkv = torch.randn((150, 8 + 2 + 2, 128), generator=g).to(torch.bfloat16).to(dev)
    cu = offsets([60, 0, 71], first=5)
    qkv[:5] = float("nan")
    qkv[136:] = float("inf")
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    o = torch.full((150, 8, 128), 7.0, dtype=torch.bfloat16, device=dev)
    lse = torch.full((150, 8), 7.0, device=dev)
    asym.attn_prefill(q, k, v, i32(cu, dev), o=o, lse=lse)
    assert torch.all(o[:5] == 7) and torch.all(o[136:] == 7) and torch.all(lse[:5] == 7) and torch.all(lse[136:] == 7)
    sub = slice(5, 136)
    check(q[sub], k[sub], v[sub], offsets([60, 0, 71]), offsets([60, 0, 71]), SCALE, True, o[sub], lse[sub])
    # head-major storage gives the same bits
    qh, kh, vh = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))
    o2 = torch.full_like(o, 7.0)
    asym.attn_prefill(qh, kh, vh, i32(cu, dev), o=o2)
    assert torch.equal(o, o2)


@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (8, 8), (6, 3), (16, 16)])
def test_mappings_give_the_same_bits(dev, Hq, Hkv):
    cu = i32(offsets([100, 3, 210]), dev)
    q, k, v = inputs(dev, 313, 313, Hq, Hkv, seed=3)
    a = asym.attn_prefill(q, k, v, cu)
    for mapping in ("oblivious_grouped", "oblivious_rowmajor"):
        assert torch.equal(a, asym.attn_prefill(q, k, v, cu, mapping=mapping))


@pytest.mark.parametrize("at,G", [(37, 1), (63, 4), (64, 4), (90, 2), (0, 4)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_cannot_reach_it(dev, at, G, bad):
    n = 130
    cu = offsets([n])
    q, k, v = inputs(dev, n, n, G, 1, seed=at)
    clean = asym.attn_prefill(q, k, v, i32(cu, dev))
    v2 = v.clone()
    v2[at, 0, 5] = bad
    v2[at, 0, 100] = bad
    got = asym.attn_prefill(q, k, v2, i32(cu, dev))
    mask = torch.zeros((n, 1, 128), dtype=torch.bool, device=dev)
    mask[at:, :, 5] = mask[at:, :, 100] = True
    mask = mask.expand_as(got)
    assert torch.equal(got[~mask], clean[~mask])
    hit = got[mask].float()
    assert torch.all(torch.isnan(hit)) if bad != bad else torch.all(hit == bad)
    k2 = k.clone()
    k2[at] = bad
    got = asym.attn_prefill(q, k2, v, i32(cu, dev))
    assert torch.equal(got[:at], clean[:at])


def test_opposite_infinities_in_one_block(dev):
    n = 40
    q, k, v = inputs(dev, n, n, 2, 1, seed=1)
    v[10, 0, 0], v[20, 0, 0], v[30, 0, 1] = float("inf"), -float("inf"), -float("inf")
    o = asym.attn_prefill(q, k, v, i32([0, n], dev)).float()
    assert torch.all(torch.isfinite(o[:10])) and torch.all(o[10:20, :, 0] == float("inf"))
    assert torch.all(torch.isnan(o[20:, :, 0])) and torch.all(o[30:, :, 1] == -float("inf"))
    assert torch.all(torch.isfinite(o[:30, :, 1])) and torch.all(torch.isfinite(o[:, :, 2:]))


def test_scores_of_the_lowest_value(dev):
    # keys that push scores to the lowest bf16, and keys of zero weight beside them
    n = 96
    q, k, v = inputs(dev, n, n, 2, 1, seed=2)
    q[:] = 1.0
    k[:] = 0.0
    k[::3] = torch.finfo(torch.bfloat16).min / 256
    o = asym.attn_prefill(q, k, v, i32([0, n], dev), causal=False).float()
    w = torch.ones(n, device=dev)
    w[::3] = 0
    ref = (w[:, None] * v[:, 0].float()).sum(0) / w.sum()
    assert torch.allclose(o, ref.expand_as(o), rtol=2 ** -6, atol=2 ** -8)


def test_long_prompt_sampled(dev):
    lens, pre = [2600, 700], [0, 1500]
    cu_q, cu_k = offsets(lens), offsets([a + b for a, b in zip(lens, pre)])
    q, k, v = inputs(dev, cu_q[-1], cu_k[-1], 8, 2, seed=8)
    lse = torch.empty((cu_q[-1], 8), device=dev)
    o = asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev), lse=lse)
    for b, i in [(0, 0), (0, 63), (0, 64), (0, 1300), (0, 2599), (1, 0), (1, 699), (1, 350)]:
        r, n = cu_q[b] + i, i + pre[b] + 1  # the row alone, over the keys that it sees
        ks = slice(cu_k[b], cu_k[b] + n)
        check(q[r:r + 1], k[ks], v[ks], [0, 1], [0, n], SCALE, True, o[r:r + 1], lse[r:r + 1])


def test_offsets_that_say_too_much_are_held(dev):
    q, k, v = inputs(dev, 50, 50, 4, 2, seed=4)
    o = torch.full((50, 4, 128), 7.0, dtype=torch.bfloat16, device=dev)
    asym.attn_prefill(q, k, v, i32([-9, 50, 2000000000, 20], dev), i32([0, 90, 50, 7], dev), o=o)
    assert torch.equal(o, asym.attn_prefill(q, k, v, i32([0, 50], dev)))


def test_captured_and_replayed(dev):
    cu = i32(offsets([100, 29]), dev)
    q, k, v = inputs(dev, 129, 129, 8, 2, seed=6)
    o, lse = torch.empty_like(q), torch.empty((129, 8), device=dev)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        asym.attn_prefill(q, k, v, cu, o=o, lse=lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        asym.attn_prefill(q, k, v, cu, o=o, lse=lse)
    for seed in (7, 8, 9):
        q2, k2, v2 = inputs(dev, 129, 129, 8, 2, seed=seed)
        q.copy_(q2), k.copy_(k2), v.copy_(v2)
        cu.copy_(i32(offsets([100 - seed, 29 + seed]), dev))
        o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, asym.attn_prefill(q2, k2, v2, cu))


def test_on_another_stream(dev):
    cu = i32(offsets([300, 29]), dev)
    q, k, v = inputs(dev, 329, 329, 8, 2, seed=6)
    ref = asym.attn_prefill(q, k, v, cu)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    o = asym.attn_prefill(q, k, v, cu, stream=s)
    s.synchronize()
    assert torch.equal(o, ref)


def test_refusals(dev):
    q, k, v = inputs(dev, 8, 8, 4, 2, seed=0)
    cu = i32([0, 8], dev)
    with pytest.raises(TypeError):
        asym.attn_prefill(q.float(), k, v, cu)
    with pytest.raises(TypeError):
        asym.attn_prefill(q, k, v, cu.long())
    with pytest.raises(ValueError):
        asym.attn_prefill(q, k, v[:7], cu)
    with pytest.raises(ValueError):
        asym.attn_prefill(q[..., ::2], k, v, cu)
    with pytest.raises(ValueError):
        asym.attn_prefill(q, k, v, cu, i32([0, 4, 8], dev))
    with pytest.raises(ValueError):
        asym.attn_prefill(q, k, v.cpu(), cu)
    with pytest.raises(ValueError):
        asym.attn_prefill(q, k, v, cu, o=torch.empty((8, 4, 128), device=dev))
    with pytest.raises(asym.AsymError):  # 3 heads over 2
        asym.attn_prefill(q[:, :3], k, v, cu)
    with pytest.raises(asym.AsymError):
        asym.attn_prefill(q, k, v, cu, scale=float("nan"))
    with pytest.raises(asym.AsymError):  # every token's keys at one address
        asym.attn_prefill(q, k[:1].expand(8, 2, 128), v, cu)
    big = torch.zeros(8 * 4 * 128 + 1, dtype=torch.bfloat16, device=dev)
    with pytest.raises(asym.AsymError):  # 2-byte aligned
        asym.attn_prefill(big[1:].view(8, 4, 128), k, v, cu)


# Few rows over many keys: tiles cut along the keys and joined.  Joining adds to the bound of
# the sums (module docstring) two roundings for each piece's weight and product, an exponential
# (8) and one addition a piece: fewer than the keys that the bound counts.
CUT = [  # query lengths, key lengths, H_q, H_kv
    ([1], [700], 4, 1), ([3], [2500], 32, 8), ([40, 1, 9], [600, 2000, 9], 8, 2), ([2], [20000], 2, 1),
    ([1, 0, 2, 1], [513, 700, 0, 64], 5, 5), ([130], [1000], 3, 1), ([300], [300], 4, 2), ([700, 2], [40, 900], 2, 2),
    ([5] * 30, [90] * 29 + [1500], 4, 4), ([1] * 70, [11] * 70, 4, 2), ([2] * 70, [11] * 66 + [900, 5, 700, 1], 2, 1)]


@pytest.mark.parametrize("lq,lk,Hq,Hkv", CUT)
@pytest.mark.parametrize("causal", [True, False])
def test_few_rows_over_many_keys(dev, lq, lk, Hq, Hkv, causal):
    cu_q, cu_k = offsets(lq), offsets(lk)
    Tk = max(cu_k[-1], 8192)  # (rows behind the last sequence: any batch with room for a long one may be cut)
    assert asym._prefill_workspace(len(lq), Hq, Hkv, cu_q[-1], Tk) > 0
    q, k, v = inputs(dev, cu_q[-1], Tk, Hq, Hkv, seed=sum(lk) + Hq)
    lse = torch.empty((q.shape[0], Hq), device=dev)
    o = asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev), lse=lse, causal=causal)
    check(q, k, v, cu_q, cu_k, SCALE, causal, o, lse)
    for mapping in ("oblivious_grouped", "oblivious_rowmajor"):
        assert torch.equal(o, asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev), causal=causal, mapping=mapping))


def test_cut_rows_outside_are_left_and_unseen_values_do_not_reach(dev):
    cu_q, cu_k = offsets([5, 0, 9], first=2), offsets([800, 3, 1500], first=7)
    q, k, v = inputs(dev, 30, 2400, 8, 2, seed=4)
    o = torch.full((30, 8, 128), 7.0, dtype=torch.bfloat16, device=dev)
    lse = torch.full((30, 8), 7.0, device=dev)
    asym.attn_prefill(q, k, v, i32(cu_q, dev), i32(cu_k, dev), o=o, lse=lse)
    assert torch.all(o[:2] == 7) and torch.all(o[16:] == 7) and torch.all(lse[:2] == 7) and torch.all(lse[16:] == 7)
    # the last key of a sequence is seen by its last token alone
    k2, v2 = k.clone(), v.clone()
    for bad in (float("nan"), float("inf")):
        k2[:7] = v2[:7] = k2[2310:] = v2[2310:] = bad
        v2[806, 1, 3] = v2[2309, 0, 9] = bad
        got = asym.attn_prefill(q, k2, v2, i32(cu_q, dev), i32(cu_k, dev), o=torch.full_like(o, 7.0))
        hit = torch.zeros_like(o, dtype=torch.bool)
        hit[6, 4:, 3] = hit[15, :4, 9] = True
        assert torch.equal(got[~hit], o[~hit])
        assert not torch.any(torch.isfinite(got[hit].float()))


def test_cut_call_on_a_library_stream(dev):
    cu_q, cu_k = i32(offsets([4, 2]), dev), i32(offsets([900, 1700]), dev)
    q, k, v = inputs(dev, 6, 2600, 8, 2, seed=9)
    ref = asym.attn_prefill(q, k, v, cu_q, cu_k)
    torch.cuda.synchronize()
    s = asym.stream_create()
    outs = [asym.attn_prefill(q, k, v, cu_q, cu_k, stream=s) for _ in range(3)]
    here = [asym.attn_prefill(q, k, v, cu_q, cu_k) for _ in range(3)]  # beside them, on torch's own
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs + here)
    asym.stream_destroy(s)


def test_cut_offsets_that_say_too_much_are_held(dev):
    q, k, v = inputs(dev, 6, 9000, 8, 2, seed=2)
    want = asym.attn_prefill(q, k, v, i32([0, 6], dev), i32([0, 9000], dev))
    assert torch.equal(want, asym.attn_prefill(q, k, v, i32([-5, 100000], dev), i32([-7, 2 ** 31 - 1], dev)))


@pytest.mark.parametrize("Hkv", [1, 4])
def test_no_keys_at_all(dev, Hkv):
    q = torch.randn((5, 8, 128), device=dev).to(torch.bfloat16)
    kv = torch.empty((0, Hkv, 128), dtype=torch.bfloat16, device=dev)
    lse = torch.empty((5, 8), device=dev)
    o = asym.attn_prefill(q, kv, kv, i32([0, 5], dev), i32([0, 0], dev), lse=lse)
    assert torch.all(o == 0) and torch.all(lse == -float("inf"))


def test_cut_call_captured(dev):
    cu_q, cu_k = i32(offsets([4, 2]), dev), i32(offsets([900, 1700]), dev)
    q, k, v = inputs(dev, 6, 2600, 8, 2, seed=9)
    want = [asym.attn_prefill(q * s, k, v, cu_q, cu_k) for s in (1, -1, 2)]
    held, o1, o2 = q.clone(), torch.empty_like(q), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        asym.attn_prefill(held, k, v, cu_q, cu_k, o=o1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asym.attn_prefill(held, k, v, cu_q, cu_k, o=o1)
        asym.attn_prefill(-held, k, v, cu_q, cu_k, o=o2)
    for s, w in zip((1, -1, 2), want):
        held.copy_(q * s)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o1, w)
        assert torch.equal(o2, asym.attn_prefill(q * -s, k, v, cu_q, cu_k))
