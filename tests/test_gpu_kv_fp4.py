"""GPU parity of the 4-bit paged cache: writing and reading tokens, and decode attention over
it, through the C ABI.

Pages are compared bit by bit with the oracle's.  Decode attention is compared element by
element with float64 attention over the values that the pages hold.  Its bound (derived):
probabilities times a power of two are rounded to bf16 (2^-8 A, A = sum_j w_j |v_j|), the
output once more (2^-8 |O|); q goes in as two 4-bit-mantissa parts, off by at most 2^-22 of
the row's largest magnitude per value: scale * 2^-22 max|q| sum_d |k_d| =: E in a score;
fp32 sums as in prompt attention: A (2 E + 2^-23 (264 N + 16 + keys)).
"""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import kv_fp4, prompt
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


def bits(t):
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def offsets(lens, first=0):
    return (np.cumsum([0] + list(lens)) + first).tolist()


def make_cache(dev, B, H, pph, seed, spare=3):
    """Pools of random bytes (scales about one, some of them NaN) and a random table."""
    g = np.random.default_rng(seed)
    n = B * H * pph + spare
    pools = []
    for _ in range(2):
        p = g.integers(0, 256, (n, 2176)).astype(np.uint8)
        p[:, 2048:] = g.choice([120, 126, 127, 128, 255], (n, 128))
        pools.append(p)
    table = g.permutation(n)[:B * H * pph].reshape(B, H, pph).astype(np.int32)
    vtable = g.permutation(n)[:B * H * pph].reshape(B, H, pph).astype(np.int32)
    return pools, table, vtable


def special(k):
    """Some blocks of extreme values."""
    flat = k.view(-1, 32)
    fi = torch.finfo(torch.bfloat16)
    for i, x in enumerate([0.0, -0.0, fi.max, fi.min, fi.tiny, 2.0 ** -133, 2.0 ** -124, float("nan"), float("inf"), -float("inf")]):
        flat[(7 * i) % flat.shape[0], i % 32] = x
    flat[1 % flat.shape[0]] = 0.0
    flat[2 % flat.shape[0]] = 2.0 ** -130
    return k


@pytest.mark.parametrize("new,start,H,pph", [
    ([1], [0], 1, 1), ([1], [31], 2, 1), ([32], [0], 1, 1), ([33], [31], 2, 2), ([5, 0, 70], [30, 9, 1], 2, 3),
    ([1, 1, 1, 1], [0, 17, 40, 95], 3, 3), ([3, 3], [94, -1], 2, 3), ([40], [60], 1, 3), ([1] * 66, list(range(66)), 1, 3),
    ([2, 2], [96, 2000000000], 1, 3), ([90, 7], [3, 62], 8, 4)])
def test_written_pages_are_the_oracles(dev, new, start, H, pph):
    B, T = len(new), sum(new)
    (kp, vp), kt, vt = make_cache(dev, B, H, pph, seed=T + 31 * H)
    g = torch.Generator().manual_seed(T)
    k = special(torch.randn((T, H, 128), generator=g).to(torch.bfloat16)).to(dev)
    v = special(torch.randn((T, H, 128), generator=g).to(torch.bfloat16).flip(0)).to(dev)
    kd, vd = torch.tensor(kp, device=dev), torch.tensor(vp, device=dev)
    ktd, vtd, cu, st = i32(kt, dev), i32(vt, dev), i32(offsets(new), dev), i32(start, dev)
    asym.kv_write_fp4(k, v, kd, vd, ktd, vtd, cu, st)
    cut = offsets(new)
    for x, pool, table, values in ((bits(k), kp, kt, False), (bits(v), vp, vt, True)):
        codes, scales = kv_fp4.quantise(x.reshape(-1, 128))
        codes, scales = codes.reshape(T, H, 128), scales.reshape(T, H, 4)
        for b in range(B):
            for i in range(new[b]):
                pos = start[b] + i
                if start[b] < 0 or pos >= 32 * pph:
                    continue
                for h in range(H):
                    kv_fp4.put(pool[table[b, h, pos // 32]], pos % 32, codes[cut[b] + i, h], scales[cut[b] + i, h], values)
    assert np.array_equal(kd.cpu().numpy(), kp) and np.array_equal(vd.cpu().numpy(), vp)
    # and read back: exactly what the pages say; rows without a place stay
    ko = torch.full((T, H, 128), 9.0, dtype=torch.bfloat16, device=dev)
    vo = torch.full_like(ko, 9.0)
    asym.kv_read_fp4(kd, vd, ktd, vtd, cu, st, ko, vo)
    for out, pool, table, values in ((ko, kp, kt, False), (vo, vp, vt, True)):
        got, ref = bf16_bits_to_f64(bits(out)), np.full((T, H, 128), 9.0)
        for b in range(B):
            for i in range(new[b]):
                pos = start[b] + i
                if start[b] >= 0 and pos < 32 * pph:
                    for h in range(H):
                        ref[cut[b] + i, h] = kv_fp4.page_values(pool[table[b, h, pos // 32]], values)[pos % 32]
        assert np.array_equal(got, ref, equal_nan=True)


def test_every_bf16_value_is_quantised_as_the_oracle_does(dev):
    x = np.arange(65536, dtype=np.uint32).astype(np.uint16).reshape(512, 128)  # blocks of neighbouring patterns
    alone = np.zeros((2048, 128), np.uint16)                                   # and values beside a larger one
    rng = np.random.default_rng(0)
    alone[:, ::32] = rng.integers(0, 0x7F80, (2048, 4))
    for b in range(4):
        alone[:, 32 * b + 1:32 * b + 32] = np.minimum(alone[:, 32 * b:32 * b + 1], 0x7F00) - rng.integers(0, 900, (2048, 31))
    alone &= 0x7FFF
    x = np.concatenate([x, alone])
    T = x.shape[0]
    t = torch.tensor(x.view(np.int16)).view(torch.bfloat16).view(T, 1, 128).to(dev)
    pph = T // 32
    pools = [torch.zeros((pph, 2176), dtype=torch.uint8, device=dev) for _ in range(2)]
    table = torch.arange(pph, dtype=torch.int32, device=dev).view(1, 1, pph)
    asym.kv_write_fp4(t, t, pools[0], pools[1], table, table, i32([0, T], dev), i32([0], dev))
    codes, scales = kv_fp4.quantise(x)
    for values in (False, True):
        p = pools[values].cpu().numpy()
        for i in range(pph):
            c, s = kv_fp4.get(p[i], values)
            assert np.array_equal(c, codes[32 * i:32 * i + 32]) and np.array_equal(s, scales[32 * i:32 * i + 32])


def test_strided_tokens_and_rows_outside(dev):
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((50, 8, 128), generator=g).to(torch.bfloat16).to(dev)
    k, v = qkv[:, 4:6], qkv[:, 6:8]
    table = i32(np.arange(8).reshape(2, 2, 2), dev)
    cu, st = i32([4, 20, 45], dev), i32([3, 30], dev)
    a = [torch.zeros((8, 2176), dtype=torch.uint8, device=dev) for _ in range(2)]
    b = [torch.zeros((8, 2176), dtype=torch.uint8, device=dev) for _ in range(2)]
    asym.kv_write_fp4(k, v, *a, table, table, cu, st)
    asym.kv_write_fp4(k.contiguous(), v.contiguous(), *b, table, table, cu, st)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ko = torch.full((50, 2, 128), 5.0, dtype=torch.bfloat16, device=dev)
    vo = ko.clone()
    asym.kv_read_fp4(*a, table, table, cu, st, ko, vo)
    assert torch.all(ko[:4] == 5) and torch.all(ko[45:] == 5) and torch.all(vo[:4] == 5) and torch.all(vo[45:] == 5)
    assert float((ko[4:45] - k[4:45]).abs().max()) < 1.0


def test_entries_outside_the_pool(dev):
    k = torch.randn((64, 1, 128), device=dev).to(torch.bfloat16)
    pools = [torch.full((3, 2176), 7, dtype=torch.uint8, device=dev) for _ in range(2)]
    table = i32([[[1, -1]]], dev)
    table2 = i32([[[3, 2]]], dev)
    asym.kv_write_fp4(k, k, *pools, table, table2, i32([0, 64], dev), i32([0], dev))
    assert torch.all(pools[0][[0, 2]] == 7) and torch.all(pools[1][:2] == 7)
    ko, vo = torch.ones_like(k), torch.ones_like(k)
    asym.kv_read_fp4(*pools, table, table2, i32([0, 64], dev), i32([0], dev), ko, vo)
    assert torch.all(ko[32:] == 0) and torch.all(vo[:32] == 0) and bool(ko[:32].any()) and bool(vo[32:].any())
    # in attention: keys of zeros (every such token weighs alike) and values of zeros
    q = torch.randn((1, 2, 128), device=dev).to(torch.bfloat16)
    o = asym.attn_decode_paged_fp4(q, *pools, i32([[[-1, 99]]], dev), i32([[[2, 2000000000]]], dev), i32([64], dev))
    ref = vo[32:, 0].float().sum(0) / 64
    assert torch.allclose(o[0].float(), ref.expand(2, 128), rtol=2 ** -6, atol=2 ** -7)


def attend(q, kp, vp, kt, vt, lens, scale):
    """float64 attention over the values that the pages hold: (O, lse, bound of |error|, of lse's)."""
    B, Hq, _ = q.shape
    H = kt.shape[1]
    G = Hq // H
    qf = bf16_bits_to_f64(bits(q))
    O, L, bo, bl = np.zeros(q.shape), np.zeros((B, Hq)), np.zeros(q.shape), np.zeros((B, Hq))
    for b in range(B):
        n = lens[b]
        pages = -(-n // 32)
        k, v = np.zeros((max(n, 1), H, 128)), np.zeros((max(n, 1), H, 128))
        for h in range(H):
            if n:
                k[:, h] = np.concatenate([kv_fp4.page_values(kp[kt[b, h, j]], False) for j in range(pages)])[:n]
                v[:, h] = np.concatenate([kv_fp4.page_values(vp[vt[b, h, j]], True) for j in range(pages)])[:n]
        o, lse, A, N = prompt.prompt_attention(qf[b:b + 1], k[:n], v[:n], [0, 1], [0, n], scale, False)
        O[b], L[b] = o[0], lse[0]
        with np.errstate(invalid="ignore"):
            most = np.abs(k).sum(-1).max(0) if n else np.zeros(H)
        E = abs(scale) * 2.0 ** -22 * np.abs(qf[b]).max(-1) * np.repeat(most, G)
        eps = 2 * E + 2.0 ** -23 * (264 * N[0] + 16 + n)
        bo[b] = 2.0 ** -8 * (1 + 2.0 ** -8) * (A[0] + np.abs(O[b])) + A[0] * eps[:, None] + 1e-37
        bl[b] = E + 2.0 ** -23 * (132 * N[0] + 16 + n + np.abs(np.where(np.isinf(L[b]), 0, L[b])))
    return O, L, bo, bl


def clean_cache(B, H, pph, seed):
    g = np.random.default_rng(seed)
    n = B * H * pph + 2
    pools = []
    for _ in range(2):
        p = g.integers(0, 256, (n, 2176)).astype(np.uint8)
        p[:, 2048:] = g.choice([123, 124, 125, 126], (n, 128))
        pools.append(p)
    return pools, g.permutation(n)[:n - 2].reshape(B, H, pph).astype(np.int32), \
        g.permutation(n)[:n - 2].reshape(B, H, pph).astype(np.int32)


def poison_behind(pool, table, lens, values):
    """NaN scales and any codes where no token of the lengths is."""
    _, _, sc = kv_fp4.places(values)
    for b in range(table.shape[0]):
        for h in range(table.shape[1]):
            for j in range(table.shape[2]):
                for t in range(32):
                    if 32 * j + t >= lens[b]:
                        pool[table[b, h, j]][sc[t]] = 255


@pytest.mark.parametrize("lens,Hq,Hkv,pph,split", [
    ([1], 1, 1, 1, 0), ([31, 32, 33], 4, 2, 2, 0), ([0, 5, 0, 64], 8, 2, 2, 32), ([100, 7, 65], 16, 1, 4, 32),
    ([300, 1, 0, 257], 5, 1, 10, 64), ([96], 3, 3, 3, 96), ([500, 20], 12, 4, 16, 0), ([1000], 32, 8, 32, 128),
    ([40] * 70, 2, 1, 2, 0), ([2049, 64], 7, 1, 65, 2048), ([640], 14, 2, 20, 32),
    # batches of more requests than a wave looks at once, requests without tokens between them
    ([0, 33, 64] * 100 + [0] * 300 + [50, 0, 0], 2, 2, 2, 0), ([70] + [0] * 520 + [45], 4, 2, 3, 32),
    ([3, 0, 40, 65] * 512, 1, 1, 3, 0), ([0] * 5, 4, 2, 2, 0), ([5000, 1, 0, 4097], 3, 1, 157, 0)])
def test_decode_against_oracle(dev, lens, Hq, Hkv, pph, split):
    B = len(lens)
    (kp, vp), kt, vt = clean_cache(B, Hkv, pph, seed=sum(lens) + Hq)
    poison_behind(kp, kt, lens, False)
    poison_behind(vp, vt, lens, True)
    g = torch.Generator().manual_seed(Hq)
    q = torch.randn((B, Hq, 128), generator=g).to(torch.bfloat16).to(dev)
    lse = torch.empty((B, Hq), device=dev)
    args = (torch.tensor(kp, device=dev), torch.tensor(vp, device=dev), i32(kt, dev), i32(vt, dev), i32(lens, dev))
    o = asym.attn_decode_paged_fp4(q, *args, lse=lse, split_tokens=split)
    R, L, bo, bl = attend(q, kp, vp, kt, vt, lens, SCALE)
    got, gl = bf16_bits_to_f64(bits(o)), lse.double().cpu().numpy()
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - R) <= bo), float(np.max(np.abs(got - R) / bo))
    some = ~np.isinf(L)
    assert np.all(gl[~some] == -np.inf) and np.all(got[~some] == 0)
    assert np.all(np.abs(gl[some] - L[some]) <= bl[some])


@pytest.mark.parametrize("scale,sigma", [(0.0, 1), (-0.2, 1), (2.0, 1), (SCALE, 2.0 ** 60), (SCALE, 2.0 ** -100)])
def test_decode_scales(dev, scale, sigma):
    lens = [70, 33]
    (kp, vp), kt, vt = clean_cache(2, 2, 3, seed=4)
    if sigma > 1:
        kp[:, 2048:] -= 60
    g = torch.Generator().manual_seed(4)
    q = (torch.randn((2, 8, 128), generator=g) * sigma).to(torch.bfloat16)
    q[0, 0, 1:] *= 2.0 ** -9  # values far below the row's largest
    q[1, 1] = 0
    q = q.to(dev)
    o = asym.attn_decode_paged_fp4(q, torch.tensor(kp, device=dev), torch.tensor(vp, device=dev), i32(kt, dev), i32(vt, dev),
                                   i32(lens, dev), scale=scale)
    R, L, bo, bl = attend(q, kp, vp, kt, vt, lens, scale)
    assert np.all(np.abs(bf16_bits_to_f64(bits(o)) - R) <= bo)


def test_nan_blocks_reach_their_request_only(dev):
    lens = [64, 64]
    (kp, vp), kt, vt = clean_cache(2, 1, 2, seed=9)
    q = torch.randn((2, 4, 128), device=dev).to(torch.bfloat16)
    run = lambda: asym.attn_decode_paged_fp4(q, torch.tensor(kp, device=dev), torch.tensor(vp, device=dev), i32(kt, dev),
                                             i32(vt, dev), i32(lens, dev))
    clean = run()
    kv_fp4.put(vp[vt[0, 0, 1]], 3, np.zeros(128, np.uint8), np.array([125, 255, 125, 125], np.uint8), True)
    got = run()
    assert torch.all(torch.isnan(got[0, :, 32:64])) and not torch.isnan(got[0, :, :32]).any()
    assert not torch.isnan(got[0, :, 64:]).any() and torch.equal(got[1], clean[1])
    kv_fp4.put(kp[kt[0, 0, 0]], 20, np.zeros(128, np.uint8), np.array([125, 125, 125, 255], np.uint8), False)
    got = run()
    assert torch.all(torch.isnan(got[0])) and torch.equal(got[1], clean[1])


def test_pages_past_four_gigabytes(dev):
    n = 2_000_000  # 4.35 GB a pool
    (kp, vp), kt, vt = clean_cache(1, 2, 2, seed=12)
    far = np.array([5, 1, 0, 2, 4, 3]) + n - 6
    pools = [torch.empty((n, 2176), dtype=torch.uint8, device=dev) for _ in range(2)]
    for pool, small in zip(pools, (kp, vp)):
        pool[torch.tensor(far, device=dev)] = torch.tensor(small, device=dev)
    q = torch.randn((1, 4, 128), device=dev).to(torch.bfloat16)
    a = asym.attn_decode_paged_fp4(q, *pools, i32(far[kt], dev), i32(far[vt], dev), i32([60], dev))
    small = (torch.tensor(kp, device=dev), torch.tensor(vp, device=dev))
    b = asym.attn_decode_paged_fp4(q, *small, i32(kt, dev), i32(vt, dev), i32([60], dev))
    assert torch.equal(a, b)
    k = torch.randn((3, 2, 128), device=dev).to(torch.bfloat16)
    asym.kv_write_fp4(k, k, *pools, i32(far[kt], dev), i32(far[vt], dev), i32([0, 3], dev), i32([31], dev))
    asym.kv_write_fp4(k, k, *small, i32(kt, dev), i32(vt, dev), i32([0, 3], dev), i32([31], dev))
    for pool, s in zip(pools, small):
        assert torch.equal(pool[torch.tensor(far, device=dev)], s)
    out = [torch.empty_like(k) for _ in range(4)]
    asym.kv_read_fp4(*pools, i32(far[kt], dev), i32(far[vt], dev), i32([0, 3], dev), i32([31], dev), out[0], out[1])
    asym.kv_read_fp4(*small, i32(kt, dev), i32(vt, dev), i32([0, 3], dev), i32([31], dev), out[2], out[3])
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])


def test_captured_decode_step(dev):
    """Write and attend in two graphs that are replayed at once on two streams."""
    B, H, pph = 5, 2, 40
    graphs, states = [], []
    for i in range(2):
        (kp, vp), kt, vt = clean_cache(B, H, pph, seed=20 + i)
        st = dict(kp=torch.tensor(kp, device=dev), vp=torch.tensor(vp, device=dev), kt=i32(kt, dev), vt=i32(vt, dev),
                  k=torch.zeros((B, H, 128), dtype=torch.bfloat16, device=dev), lens=i32([0] * B, dev), start=i32([0] * B, dev),
                  cu=i32(list(range(B + 1)), dev), q=torch.zeros((B, 8, 128), dtype=torch.bfloat16, device=dev))

        def step(s):
            asym.kv_write_fp4(s["k"], s["k"], s["kp"], s["vp"], s["kt"], s["vt"], s["cu"], s["start"])
            return asym.attn_decode_paged_fp4(s["q"], s["kp"], s["vp"], s["kt"], s["vt"], s["lens"], split_tokens=64)
        step(st)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st["out"] = step(st)
        graphs.append(g)
        states.append((st, step))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for n in (3, 700, 1200):
        for st, _ in states:
            st["q"].normal_(), st["k"].normal_()
            st["start"].copy_(i32([n - 1, n, n + 1, 0, n // 2], dev))
            st["lens"].copy_(st["start"] + 1)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for st, step in states:
            got = st["out"].clone()
            assert torch.equal(got, step(st))


def test_refusals(dev):
    q = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device=dev)
    pool = torch.zeros((4, 2176), dtype=torch.uint8, device=dev)
    t = i32(np.zeros((2, 2, 1)), dev)
    lens = i32([1, 1], dev)
    with pytest.raises(TypeError):
        asym.attn_decode_paged_fp4(q.float(), pool, pool, t, t, lens)
    with pytest.raises(TypeError):
        asym.attn_decode_paged_fp4(q, pool.float(), pool, t, t, lens)
    with pytest.raises(TypeError):
        asym.attn_decode_paged_fp4(q, pool, pool, t.long(), t, lens)
    with pytest.raises(ValueError):
        asym.attn_decode_paged_fp4(q, pool[:, :2160], pool, t, t, lens)
    with pytest.raises(ValueError):
        asym.attn_decode_paged_fp4(q[:1], pool, pool, t, t, lens)
    with pytest.raises(ValueError):
        asym.attn_decode_paged_fp4(q, pool, pool, t, t, lens[:1])
    with pytest.raises(ValueError):
        asym.attn_decode_paged_fp4(q, pool, pool, t, t, lens.cpu())
    with pytest.raises(asym.AsymError):
        asym.attn_decode_paged_fp4(q, pool, pool, t, t, lens, S=33)
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=dev)
    with pytest.raises(ValueError):
        asym.kv_write_fp4(k[:, :1], k[:, :1], pool, pool, t, t, i32([0, 1, 2], dev), lens)
    with pytest.raises(ValueError):
        asym.kv_write_fp4(k, k, pool, pool, t, t, i32([0, 1], dev), lens)
    with pytest.raises(ValueError):
        asym.kv_read_fp4(pool, pool, t, t, i32([0, 1, 2], dev), lens, k.transpose(0, 1), k)
    with pytest.raises(TypeError):
        asym.kv_read_fp4(pool, pool, t, t, i32([0, 1, 2], dev), lens, k.float(), k)
