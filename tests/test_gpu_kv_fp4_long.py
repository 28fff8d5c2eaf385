"""Decode attention over the 4-bit cache where a wave walks many pages and where the cache
is past what the memory-side cache holds (read non-temporally), through the C ABI: against float64
attention over the values that the pages hold, within tests/test_gpu_kv_fp4.py's derived bound."""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import kv_fp4
from tests.test_gpu_kv_fp4 import SCALE, attend, bf16_bits_to_f64, bits, clean_cache, dev, i32, poison_behind  # noqa: F401

pytestmark = pytest.mark.gpu


def compare(o, lse, q, kp, vp, kt, vt, lens):
    R, L, bo, bl = attend(q, kp, vp, kt, vt, lens, SCALE)
    got, gl = bf16_bits_to_f64(bits(o)), lse.double().cpu().numpy()
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - R) <= bo), float(np.max(np.abs(got - R) / bo))
    some = ~np.isinf(L)
    assert np.all(gl[~some] == -np.inf) and np.all(got[~some] == 0)
    assert np.all(np.abs(gl[some] - L[some]) <= bl[some])


# A wave holds the numbers of 64 pages at a time: shares that end before, at and behind the
# next 64, that begin inside a head, and that hold the ends of two.
@pytest.mark.parametrize("pages", [63, 64, 65, 128, 129, 200])
@pytest.mark.parametrize("lens,Hq,Hkv", [
    ([32 * 200], 4, 1), ([32 * 129 - 5, 0, 32 * 66 + 1, 17], 3, 1), ([32 * 65, 32 * 70 - 31], 4, 2), ([1, 32 * 257 + 9], 2, 1)])
def test_shares_of_many_pages(dev, pages, lens, Hq, Hkv):
    pph = -(-max(lens) // 32) + 1
    (kp, vp), kt, vt = clean_cache(len(lens), Hkv, pph, seed=pages + len(lens))
    poison_behind(kp, kt, lens, False)
    poison_behind(vp, vt, lens, True)
    g = torch.Generator().manual_seed(pages)
    q = torch.randn((len(lens), Hq, 128), generator=g).to(torch.bfloat16).to(dev)
    lse = torch.empty(q.shape[:2], device=dev)
    o = asym.attn_decode_paged_fp4(q, torch.tensor(kp, device=dev), torch.tensor(vp, device=dev), i32(kt, dev), i32(vt, dev),
                                   i32(lens, dev), lse=lse, split_tokens=32 * pages)
    compare(o, lse, q, kp, vp, kt, vt, lens)


def big_cache(dev, lens, H, pph, seed):
    """Random pools on the GPU with a page for every 32 tokens of the lengths, and -1 behind them."""
    g = torch.Generator(device=dev).manual_seed(seed)
    n = [-(-x // 32) for x in lens]
    pages = sum(n) * H + 3
    pools = []
    for _ in range(2):
        p = torch.randint(0, 256, (pages, 2176), generator=g, device=dev, dtype=torch.uint8)
        p[:, 2048:] = p[:, 2048:] % 4 + 123
        pools.append(p)
    tables = []
    have = (torch.arange(pph, device=dev) < torch.tensor(n, device=dev)[:, None, None]).expand(len(lens), H, pph)
    for _ in range(2):
        t = torch.full((len(lens), H, pph), -1, dtype=torch.int32, device=dev)
        t[have] = torch.randperm(pages, generator=g, device=dev)[:sum(n) * H].to(torch.int32)
        tables.append(t)
    return pools, tables


def sampled(o, lse, q, pools, tables, lens, picks):
    """The requests and key/value heads of `picks`, each as a call of its own for the oracle."""
    G = q.shape[1] // tables[0].shape[1]
    for b, h in picks:
        rows = slice(h * G, (h + 1) * G)
        n = -(-lens[b] // 32)
        small, local = [], np.arange(max(n, 1), dtype=np.int32).reshape(1, 1, -1)
        for pool, table in zip(pools, tables):
            small.append(pool[table[b, h, :max(n, 1)].clamp(min=0).long()].cpu().numpy())
        compare(o[b:b + 1, rows], lse[b:b + 1, rows], q[b:b + 1, rows].contiguous(), *small, local, local, [lens[b]])


def test_long_contexts_past_the_memory_side_cache(dev):
    # 40 requests, 8 key/value heads, up to 18000 tokens: 2048 shares of about 70 pages each
    B, H, Hq, S = 40, 8, 32, 18000
    g = np.random.default_rng(3)
    lens = [int(x) for x in g.integers(S - 4500, S + 1, B)]
    lens[0], lens[7], lens[20], lens[39] = S, 0, 33, 9000
    pools, tables = big_cache(dev, lens, H, -(-S // 32), seed=3)
    assert 2 * pools[0].numel() >= 256 << 20 and 2 * B * H * -(-S // 32) * 2176 >= 256 << 20  # what decides the loads' kind
    assert sum(-(-x // 32) for x in lens) * H > 64 * asym.attn_decode_paged_fp4_plan(B, Hq, H, S)["tasks"]
    q = torch.randn((B, Hq, 128), device=dev).to(torch.bfloat16)
    lse = torch.empty((B, Hq), device=dev)
    o = asym.attn_decode_paged_fp4(q, *pools, *tables, i32(lens, dev), S=S, lse=lse)
    sampled(o, lse, q, pools, tables, lens, [(0, 0), (0, 7), (1, 3), (6, 7), (7, 0), (8, 0), (20, 5), (25, 2), (39, 0), (39, 7)])
    again = asym.attn_decode_paged_fp4(q, *pools, *tables, i32(lens, dev), S=S)
    assert torch.equal(o, again)


def test_many_short_requests_past_the_memory_side_cache(dev):
    # a wave a (request, head), whole
    B, H, Hq, S = 280, 8, 16, 1000
    g = np.random.default_rng(4)
    lens = [int(x) for x in g.integers(S - 100, S + 1, B)]
    lens[0], lens[1], lens[2], lens[-1] = 0, 1, 32, S
    pools, tables = big_cache(dev, lens, H, 33, seed=4)
    assert 2 * pools[0].numel() >= 256 << 20
    assert asym.attn_decode_paged_fp4_plan(B, Hq, H, S)["workspace_bytes"] == 0
    q = torch.randn((B, Hq, 128), device=dev).to(torch.bfloat16)
    lse = torch.empty((B, Hq), device=dev)
    o = asym.attn_decode_paged_fp4(q, *pools, *tables, i32(lens, dev), S=S, lse=lse)
    sampled(o, lse, q, pools, tables, lens, [(0, 0), (1, 1), (2, 7), (3, 0), (100, 4), (279, 7), (279, 0)])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite_reaches_its_head_only(dev, bad):
    lens = [70, 64, 1]
    (kp, vp), kt, vt = clean_cache(3, 2, 3, seed=5)
    q = torch.randn((3, 8, 128), device=dev).to(torch.bfloat16)
    args = (torch.tensor(kp, device=dev), torch.tensor(vp, device=dev), i32(kt, dev), i32(vt, dev), i32(lens, dev))
    clean = asym.attn_decode_paged_fp4(q, *args)
    q2 = q.clone()
    q2[1, 5, 77] = bad  # infinite scores of either sign, or NaN: no softmax
    got = asym.attn_decode_paged_fp4(q2, *args)
    mask = torch.zeros_like(got, dtype=torch.bool)
    mask[1, 5] = True
    assert torch.all(torch.isnan(got[mask]))
    # (the heads of a key/value head raise their maxima together, which may change their rounding)
    group = torch.zeros_like(mask)
    group[1, 4:] = True
    assert torch.equal(got[~group], clean[~group])
    R, _, bo, _ = attend(q, kp, vp, kt, vt, lens, 128 ** -0.5)
    other = (group & ~mask).cpu().numpy()
    assert np.all(np.abs(bf16_bits_to_f64(bits(got)) - R)[other] <= bo[other])


def test_sizes_past_32_bits_are_refused(dev):
    q = torch.zeros((1, 1, 128), dtype=torch.bfloat16, device=dev)
    pool, table = torch.zeros((1, 2176), dtype=torch.uint8, device=dev), i32([[[0]]], dev)
    for kw in (dict(S=(1 << 32) + 32), dict(split_tokens=(1 << 32) + 32)):
        with pytest.raises(ValueError):
            asym.attn_decode_paged_fp4(q, pool, pool, table, table, i32([1], dev), **kw)
