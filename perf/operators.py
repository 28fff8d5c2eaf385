"""The serving operators that are timed: prompt attention, the 4-bit paged cache with the attention that reads it, and the
cache's pages.  `run` computes each in its plain form (elementary torch operations in 32 bits), or, where `own` is set, by the
framework's entry points.

Sizes are those of an 8B-class decoder (32 query heads of 128, 8 or 32 key/value heads) and of its tensor-parallel shards, the
same that the products and the decode attention are timed at.

The 4-bit page (2176 bytes, 32 tokens of one head), as both forms read and write it.  A block of 32 channels of a token has the
scale X = 2^(s - 127), s = max(exponent field of the largest magnitude, 4) - 2, and 4-bit values (1 sign, 2 exponent and 1
mantissa bits: 0, 0.5, 1, 1.5, 2, 3, 4, 6), rounded to nearest even and saturated; a block that holds an infinity or a NaN has
s = 255 and zeros.  Token t, channel c, block b = c / 32:
  keys:   value in nibble c % 2 of byte 64 t + c / 2, scale in byte 2048 + 2 (t % 16 + 16 b) + t / 16;
  values: with q = t % 16 / 4 and j = t % 4 + 4 (t / 16), value in nibble j % 2 of byte
          1024 (c / 64) + 16 (c % 16 + 16 q) + 4 (c / 16 % 4) + j / 2, scale in byte 2048 + 32 q + 4 j + b.
"""
import math

import torch

own = False

DEV = "cuda:0"
D = 128
PT = 32           # tokens of a page
PAGE = 2176       # bytes of a 4-bit page


# ---- cases ---------------------------------------------------------------------------------------------------------------


def _prefill(B, T, P, Hq, Hkv):
    return {"op": "prefill", "B": B, "T": T, "P": P, "Hq": Hq, "Hkv": Hkv}


def _cache(B, T, start, Hkv):
    return {"op": "cache", "B": B, "T": T, "start": start, "Hkv": Hkv}


def _decode(B, Hq, Hkv, S):
    return {"op": "decode", "B": B, "Hq": Hq, "Hkv": Hkv, "S": S}


def _pages(op, R, H, S):
    return {"op": op, "R": R, "H": H, "S": S}


def listed():
    return [
        # three short prompts of a shard with two key/value heads: launch and latency
        dict(_prefill(3, 140, 0, 8, 2), name="prefill_short"),
        # a scheduler's step: eight chunks of different lengths, each behind a cached prefix of its own
        dict(_prefill(8, 8191, 4096, 32, 8), name="prefill_chunks"),
        # one long prompt, queries, keys and values lying in the fused projection's output
        dict(_prefill(1, 16384, 0, 32, 8), name="prefill_long"),
        # a decode step's tokens into the 4-bit cache, and the pages that they fell into read back
        dict(_cache(32, 32, 3000, 8), name="cache_append"),
        # prompts into the 4-bit cache, and read back as a chunk behind them needs them
        dict(_cache(6, 16381, 500, 8), name="cache_prompt"),
        # one request of a few hundred tokens
        dict(_decode(1, 32, 8, 777), name="decode_fp4_one"),
        # a decode step of 16 requests of up to 8000 tokens
        dict(_decode(16, 32, 8, 8000), name="decode_fp4_batch"),
        # long contexts at full batch
        dict(_decode(64, 32, 8, 32768), name="decode_fp4_long"),
        # four beams of a short request forked, then every row's next token gets its place
        dict(_pages("fork", 8, 8, 700), name="fork_beams"),
        # 256 samples forked from 256 prompts
        dict(_pages("fork", 512, 8, 4000), name="fork_batch"),
        # some of a few requests end, and the cache is packed
        dict(_pages("compact", 12, 8, 900), name="compact_few"),
        # a third of 256 requests end, and the cache is packed
        dict(_pages("compact", 256, 8, 4000), name="compact_batch"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("prefill", "prefill", "decode", "decode", "cache", "fork", "compact"))
    Hkv = rng.choice((1, 2, 4, 8, 8))
    G = rng.choice((1, 2, 3, 4, 4, 5, 8, 16))
    if op == "prefill":
        B = _log(rng, 1, 48)
        T = max(B, _log(rng, 16, 16384))
        P = rng.choice((0, _log(rng, 1, 8192)))
        G = min(G, 32 // Hkv)
        while T * (T // B + P) * Hkv * G > 14000 ** 2 * 32:  # no more than the longest prompt's work
            T, P = max(B, T // 2), P // 2
        return _prefill(B, T, P, Hkv * G, Hkv)
    if op == "cache":
        B = _log(rng, 1, 256)
        return _cache(B, max(B, _log(rng, 1, 16384)), _log(rng, 1, 4000), Hkv)
    if op == "decode":
        B = _log(rng, 1, 64)
        return _decode(B, Hkv * G, Hkv, _log(rng, 1, min(32768, (64 * 32768 * 8) // (B * Hkv))))
    R = _log(rng, 4, 512 if op == "fork" else 256)
    H = rng.choice((1, 2, 4, 8))
    return _pages(op, R, H, _log(rng, 40, 4000))


def _lengths(case):
    """New tokens and cached tokens of each sequence: the same for every seed, so that a case's work is one number."""
    B, T = case["B"], case["T"]
    g = torch.Generator(device="cpu").manual_seed(7)
    u = torch.rand(B, generator=g, dtype=torch.float64) * 0.8 + 0.2
    cut = (torch.cumsum(u, 0) / u.sum() * (T - B)).long().tolist()
    new = [1 + c - (cut[i - 1] if i else 0) for i, c in enumerate(cut)]
    new[-1] += T - sum(new)
    top = case["P"] if case["op"] == "prefill" else case["start"]
    old = [int(top * float(x)) for x in torch.rand(B, generator=g, dtype=torch.float64)]
    if B == 1:
        old = [top]
    return new, old


def _decode_lengths(case):
    """From a quarter of the longest on; the first request is the longest."""
    g = torch.Generator(device="cpu").manual_seed(9)
    u = torch.rand(case["B"], generator=g, dtype=torch.float64) * 0.75 + 0.25
    lens = [max(1, int(case["S"] * float(x))) for x in u]
    lens[0] = case["S"]
    return lens


# ---- inputs --------------------------------------------------------------------------------------------------------------


def _normal(g, shape):
    return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)


def _offsets(lens):
    return torch.cumsum(torch.tensor([0] + lens), 0).to(device=DEV, dtype=torch.int32)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _tables(g, lens, H, pph, spare):
    """A page of the pool for every 32 tokens of each (request, head), in random order; -1 where there is none."""
    n = [-(-x // PT) for x in lens]
    need = sum(n) * H
    perm = torch.randperm(need + spare, generator=g, device=DEV)[:need].to(torch.int32)
    have = torch.arange(pph, device=DEV)[None, None, :] < torch.tensor(n, device=DEV)[:, None, None]
    have = have.expand(len(lens), H, pph)
    table = torch.full((len(lens), H, pph), -1, dtype=torch.int32, device=DEV)
    table[have] = perm
    return table, need + spare


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op = case["op"]
    if op == "prefill":
        new, old = _lengths(case)
        Hq, Hkv, T = case["Hq"], case["Hkv"], case["T"]
        both = [a + b for a, b in zip(new, old)]
        st = {"op": op, "new": new, "both": both, "cu_q": _offsets(new), "cu_k": _offsets(both), "scale": 1 / math.sqrt(D)}
        if case["P"]:
            st["q"] = _normal(g, (T, Hq, D))
            st["k"], st["v"] = _normal(g, (sum(both), Hkv, D)), _normal(g, (sum(both), Hkv, D))
        else:  # the fused projection's output, seen as its three parts
            qkv = _normal(g, (T, (Hq + 2 * Hkv), D))
            st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        st["o"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=DEV)
        return st
    if op == "cache":
        new, old = _lengths(case)
        H, T = case["Hkv"], case["T"]
        lens = [a + b for a, b in zip(new, old)]
        pph = -(-max(lens) // PT) + 1
        table, pages = _tables(g, lens, H, pph, 7)
        # what the pages hold already: any 4-bit values, scales about one
        pools = [torch.randint(0, 256, (pages, PAGE), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        for p in pools:
            p[:, 2048:] = p[:, 2048:] % 4 + 124
        back = [x // PT * PT for x in old]  # read back from the start of the first page that is written
        n_back = [a - b for a, b in zip(lens, back)]
        return {"op": op, "k": _normal(g, (T, H, D)), "v": _normal(g, (T, H, D)), "k_pool": pools[0], "v_pool": pools[1],
                "table": table, "cu": _offsets(new), "start": _i32(old), "cu_back": _offsets(n_back), "start_back": _i32(back),
                "k_back": torch.empty((sum(n_back), H, D), dtype=torch.bfloat16, device=DEV),
                "v_back": torch.empty((sum(n_back), H, D), dtype=torch.bfloat16, device=DEV)}
    if op == "decode":
        lens = _decode_lengths(case)
        Hq, H, B = case["Hq"], case["Hkv"], case["B"]
        table, pages = _tables(g, lens, H, -(-case["S"] // PT), 5)
        pools = [torch.empty((pages, PAGE), dtype=torch.uint8, device=DEV) for _ in range(2)]
        for i, p in enumerate(pools):
            for a in range(0, pages, 1 << 15):  # N(0, 1) keys and values, quantised
                n = min(1 << 15, pages - a)
                p[a:a + n] = _pack(torch.randn((n, PT, D), generator=g, device=DEV).to(torch.bfloat16), i == 1)
        return {"op": op, "q": _normal(g, (B, Hq, D)), "k_pool": pools[0], "v_pool": pools[1], "table": table, "lens": _i32(lens),
                "S": case["S"], "scale": 1 / math.sqrt(D), "o": torch.empty((B, Hq, D), dtype=torch.bfloat16, device=DEV),
                "lse": torch.empty((B, Hq), dtype=torch.float32, device=DEV)}
    # the pages of a cache of 16-bit keys and values
    R, H, S = case["R"], case["H"], case["S"]
    pph = -(-S // PT) + 1
    gl = torch.Generator(device="cpu").manual_seed(13)  # the lengths of a case are the same for every seed
    lens = torch.randint(max(1, S // 4), S + 1, (R,), generator=gl).tolist()
    active = R // 2 if op == "fork" else R
    lens[active:] = [0] * (R - active)
    table, total = _tables(g, lens, H, pph, 0)
    total += 2 * R * H + 8
    for r in range(1, active, 2):  # every second request shares the first half of its neighbour's whole pages
        n = min(lens[r - 1], lens[r]) // PT // 2
        table[r, :, :n] = table[r - 1, :, :n]
    perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table[table >= 0] = perm[table[table >= 0].long()]
    refs = torch.bincount(table[table >= 0].long(), minlength=total).to(torch.int32)
    st = {"op": op, "table0": table, "lens0": _i32(lens), "refs0": refs, "status": torch.zeros(2, dtype=torch.int32, device=DEV),
          "k_pool": _normal(g, (total, PT, D)), "v_pool": _normal(g, (total, PT, D))}
    for name in ("table", "lens", "refs"):
        st[name] = st[name + "0"].clone()
    if op == "fork":
        n = R - active
        st["src"] = torch.randint(0, active, (n,), generator=g, device=DEV, dtype=torch.int32)
        st["dst"] = (active + torch.randperm(n, generator=g, device=DEV)).to(torch.int32)
        st["req"] = torch.arange(R, device=DEV, dtype=torch.int32)
        after = st["lens0"].clone()
        after[st["dst"].long()] = after[st["src"].long()]
        st["after"] = after + 1
    else:
        st["req"] = torch.randperm(R, generator=g, device=DEV)[:max(1, R // 3)].to(torch.int32)
    return st


# ---- the plain forms -----------------------------------------------------------------------------------------------------


def _attend(q, k, v, seen, scale):
    """q [H, M, D], k and v [H, N, D] in 32 bits, seen [M, N]: (O [H, M, D], lse [H, M])."""
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(s - m)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return o, (m + torch.log(total))[..., 0]


def _plain_prefill(st):
    q, k, v, o, lse = st["q"], st["k"], st["v"], st["o"], st["lse"]
    Hkv = k.shape[1]
    G = q.shape[1] // Hkv
    a = b = 0
    for n, m in zip(st["new"], st["both"]):
        for h in range(Hkv):
            kh, vh = k[b:b + m, h].float()[None], v[b:b + m, h].float()[None]
            for r in range(0, n, 2048):
                e = min(n, r + 2048)
                top = m - n + e  # no row of this part sees a later key
                seen = torch.arange(top, device=q.device)[None, :] <= torch.arange(m - n + r, top, device=q.device)[:, None]
                qh = q[a + r:a + e, h * G:(h + 1) * G].float().transpose(0, 1).contiguous()
                oh, lh = _attend(qh, kh[:, :top], vh[:, :top], seen, st["scale"])
                o[a + r:a + e, h * G:(h + 1) * G] = oh.transpose(0, 1).to(torch.bfloat16)
                lse[a + r:a + e, h * G:(h + 1) * G] = lh.transpose(0, 1)
        a, b = a + n, b + m
    return o, lse


def _quantise(x):
    """x [..., 128] bf16 -> (codes uint8 [..., 128], scale bytes uint8 [..., 4])."""
    blocks = x.float().reshape(*x.shape[:-1], 4, 32)
    bad = ~torch.isfinite(blocks).all(-1)
    top = torch.where(torch.isfinite(blocks), blocks, torch.zeros_like(blocks)).abs().amax(-1)
    field = (top.view(torch.int32) >> 23).clamp(min=4) - 2
    y = blocks.abs() * torch.exp2((127 - field).float())[..., None]
    code = (y > 0.25).to(torch.uint8)
    for edge, closed in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code = code + ((y >= edge) if closed else (y > edge)).to(torch.uint8)
    code = torch.where(torch.signbit(blocks), code + 8, code)
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    return code.reshape(x.shape), torch.where(bad, torch.full_like(field, 255), field).to(torch.uint8)


def _value(codes, scales):
    """codes [..., 128] and scale bytes [..., 4] -> fp32 [..., 128]."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0] * 2, device=codes.device)
    grid[8:] *= -1
    x = torch.exp2(scales.float() - 127)
    x = torch.where(scales == 255, torch.full_like(x, math.nan), x)
    return (grid[codes.long()].reshape(*codes.shape[:-1], 4, 32) * x[..., None]).reshape(codes.shape)


def _pack(x, values):
    """x [n, 32, 128] bf16 -> pages [n, 2176]."""
    n = x.shape[0]
    codes, scales = _quantise(x)
    if values:  # [tb, q, t3, c / 64, c / 16 % 4, c % 16] -> [c / 64, q, c % 16, c / 16 % 4, tb, t3]
        codes = codes.view(n, 2, 4, 4, 2, 4, 16).permute(0, 4, 2, 6, 5, 1, 3)
        scales = scales.view(n, 2, 4, 4, 4).permute(0, 2, 1, 3, 4)
    else:
        scales = scales.view(n, 2, 16, 4).permute(0, 3, 2, 1)
    c = codes.reshape(n, 2048, 2)
    return torch.cat([c[..., 0] | (c[..., 1] << 4), scales.reshape(n, 128)], 1)


def _unpack(pages, values):
    """pages [n, 2176] -> fp32 [n, 32, 128]."""
    n = pages.shape[0]
    c = torch.stack([pages[:, :2048] & 15, pages[:, :2048] >> 4], -1)
    s = pages[:, 2048:]
    if values:
        c = c.reshape(n, 2, 4, 16, 4, 2, 4).permute(0, 5, 2, 6, 1, 4, 3).reshape(n, PT, D)
        s = s.reshape(n, 4, 2, 4, 4).permute(0, 2, 1, 3, 4).reshape(n, PT, 4)
    else:
        c = c.reshape(n, PT, D)
        s = s.reshape(n, 4, 16, 2).permute(0, 3, 2, 1).reshape(n, PT, 4)
    return _value(c, s)


def _places(table, cu, start, T):
    """The page [T, H] and the token's place in it [T] of T packed tokens."""
    i = torch.arange(T, device=cu.device)
    b = torch.searchsorted(cu[1:].contiguous(), i.to(torch.int32), right=True)
    pos = start[b].long() + i - cu[b].long()
    return table[b, :, pos // PT].long(), pos % PT


def _plain_cache(st):
    table, T = st["table"], st["k"].shape[0]
    page, t = _places(table, st["cu"], st["start"], T)
    c = torch.arange(D, device=t.device)
    blk = torch.arange(4, device=t.device)
    base = (page * PAGE)[..., None]
    for x, pool, values in ((st["k"], st["k_pool"], False), (st["v"], st["v_pool"], True)):
        codes, scales = _quantise(x)
        flat = pool.view(-1)
        if not values:
            at = base + (64 * t[:, None] + c[None, ::2] // 2)[:, None]
            flat[at] = codes[..., ::2] | (codes[..., 1::2] << 4)
            flat[base + 2048 + (2 * (t % 16)[:, None] + 32 * blk + (t // 16)[:, None])[:, None]] = scales
        else:
            q, j = t % 16 // 4, t % 4 + 4 * (t // 16)
            at = base + ((1024 * (c // 64) + 16 * (c % 16) + 4 * (c // 16 % 4))[None] + (256 * q + j // 2)[:, None])[:, None]
            for half in (0, 1):  # a byte holds two tokens
                m = j % 2 == half
                keep = flat[at[m]] & (0xF0 if half == 0 else 0x0F)
                flat[at[m]] = keep | (codes[m] << (4 * half))
            flat[base + 2048 + ((32 * q + 4 * j)[:, None] + blk)[:, None]] = scales
    n = st["k_back"].shape[0]
    page, t = _places(table, st["cu_back"], st["start_back"], n)
    at = torch.arange(n, device=t.device)
    for h in range(table.shape[1]):
        for pool, out, values in ((st["k_pool"], st["k_back"], False), (st["v_pool"], st["v_back"], True)):
            for a in range(0, n, 4096):
                e = min(n, a + 4096)
                out[a:e, h] = _unpack(pool[page[a:e, h]], values)[at[:e - a], t[a:e]].to(torch.bfloat16)
    return st["k_back"], st["v_back"]


def _plain_decode(st):
    q, table, lens, S = st["q"], st["table"], st["lens"], st["S"]
    B, Hq, _ = q.shape
    H = table.shape[1]
    for b in range(B):
        page = table[b].clamp(min=0).long().reshape(-1)
        k = _unpack(st["k_pool"][page], False).view(H, -1, D)[:, :S]
        v = _unpack(st["v_pool"][page], True).view(H, -1, D)[:, :S]
        seen = torch.arange(S, device=q.device) < lens[b]
        v = torch.where(seen[:, None], v, torch.zeros_like(v))
        o, lse = _attend(q[b].float().view(H, Hq // H, D), k, v, seen[None], st["scale"])
        st["o"][b] = o.reshape(Hq, D).to(torch.bfloat16)
        st["lse"][b] = lse.reshape(Hq)
    return st["o"], st["lse"]


def _release(table, lens, refs, rows):
    """Takes the references of these rows' entries away."""
    pph = table.shape[2]
    have = torch.arange(pph, device=table.device)[None, None, :] < ((lens[rows] + PT - 1) // PT)[:, None, None]
    e = table[rows]
    refs.index_add_(0, e.clamp(min=0).reshape(-1).long(), -(have.expand_as(e).reshape(-1).to(torch.int32)))


def _plain_fork(st):
    """The rows dst[i] become forks of the rows src[i]: whole pages are shared, a part page is copied into the lowest free
    page (i by i, head by head); then every row of req gets places up to its new length."""
    table, lens, refs = st["table"], st["lens"], st["refs"]
    R, H, pph = table.shape
    src, dst = st["src"].long(), st["dst"].long()
    new, n_new = table[src].clone(), lens[src].clone()
    col = torch.arange(pph, device=table.device)
    last = (n_new // PT).long()
    part = n_new % PT != 0
    free = torch.nonzero(refs == 0)[:, 0]
    rank = (torch.cumsum(part.long(), 0) - 1)[:, None] * H + torch.arange(H, device=table.device)
    rank, at, hd = rank[part], last[part], torch.arange(H, device=table.device)[None]
    i = torch.arange(len(src), device=table.device)[part][:, None]
    old, got = new[i, hd, at[:, None]].long(), free[rank]
    whole = (col[None] < last[:, None])[:, None].expand_as(new)
    refs.index_add_(0, new.clamp(min=0).reshape(-1).long(), whole.reshape(-1).to(torch.int32))
    new[i, hd, at[:, None]] = got.to(torch.int32)
    refs[got] = 1
    _release(table, lens, refs, dst)
    for pool in (st["k_pool"], st["v_pool"]):
        pool[got.reshape(-1)] = pool[old.reshape(-1)]
    table[dst] = torch.where((col[None] < ((n_new + PT - 1) // PT)[:, None])[:, None], new, torch.full_like(new, -1))
    lens[dst] = n_new
    taken = got.numel()
    # the next token's places, request by request, head by head
    req = st["req"].long()
    had, want = (lens[req] + PT - 1) // PT, (st["after"] + PT - 1) // PT
    free = torch.nonzero(refs == 0)[:, 0]
    add = ((col[None] >= had[:, None]) & (col[None] < want[:, None]))[:, None].expand(len(req), H, pph)
    n = int(add.sum())
    rows = table[req]
    rows[add] = free[:n].to(torch.int32)
    refs[free[:n]] = 1
    table[req] = rows
    lens[req] = st["after"]
    st["status"].copy_(torch.tensor([n, 0], dtype=torch.int32))
    return table, lens, refs, st["k_pool"], st["v_pool"], st["status"]


def _plain_compact(st):
    """The rows of req end; then the live pages at or above the number of live pages move, in order, into the free ones below."""
    table, lens, refs = st["table"], st["lens"], st["refs"]
    req = st["req"].long()
    _release(table, lens, refs, req)
    table[req] = -1
    lens[req] = 0
    live = refs > 0
    n = int(live.sum())
    holes = torch.nonzero(~live[:n])[:, 0]
    moved = n + torch.nonzero(live[n:])[:, 0]
    where = torch.arange(len(refs), device=refs.device)
    where[moved] = holes
    for pool in (st["k_pool"], st["v_pool"]):
        pool[holes] = pool[moved]
    refs[holes] = refs[moved]
    refs[moved] = 0
    table.copy_(torch.where(table >= 0, where[table.clamp(min=0).long()].to(torch.int32), table))
    st["status"].copy_(torch.tensor([len(holes), n], dtype=torch.int32))
    return table, lens, refs, st["k_pool"], st["v_pool"], st["status"]


def run(state):
    op = state["op"]
    if op in ("fork", "compact"):  # from the same tables at every pass
        for name in ("table", "lens", "refs"):
            state[name].copy_(state[name + "0"])
    if not own:
        return {"prefill": _plain_prefill, "cache": _plain_cache, "decode": _plain_decode, "fork": _plain_fork,
                "compact": _plain_compact}[op](state)
    import paper_2609_24270_amd as asym
    s = state
    if op == "prefill":
        asym.attn_prefill(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], o=s["o"], lse=s["lse"], scale=s["scale"])
        return s["o"], s["lse"]
    if op == "cache":
        asym.kv_write_fp4(s["k"], s["v"], s["k_pool"], s["v_pool"], s["table"], s["table"], s["cu"], s["start"])
        return asym.kv_read_fp4(s["k_pool"], s["v_pool"], s["table"], s["table"], s["cu_back"], s["start_back"], s["k_back"],
                                s["v_back"])
    if op == "decode":
        asym.attn_decode_paged_fp4(s["q"], s["k_pool"], s["v_pool"], s["table"], s["table"], s["lens"], S=s["S"], o=s["o"],
                                   lse=s["lse"], scale=s["scale"])
        return s["o"], s["lse"]
    if op == "fork":
        asym.kv_fork(s["k_pool"], s["v_pool"], s["table"], s["lens"], s["refs"], s["src"], s["dst"], s["status"])
        asym.kv_extend(s["table"], s["lens"], s["refs"], s["req"], s["after"], s["status"])
    else:
        asym.kv_free(s["table"], s["lens"], s["refs"], s["req"])
        asym.kv_compact(s["k_pool"], s["v_pool"], s["table"], s["lens"], s["refs"], s["status"])
    return s["table"], s["lens"], s["refs"], s["k_pool"], s["v_pool"], s["status"]


# ---- work ----------------------------------------------------------------------------------------------------------------


def work(case):
    op = case["op"]
    if op == "prefill":
        new, old = _lengths(case)
        Hq, Hkv, T = case["Hq"], case["Hkv"], case["T"]
        pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(new, old))
        rows = 2 * T * Hq + 2 * (T + sum(old)) * Hkv
        return {"bytes": rows * D * 2 + 4 * T * Hq, "flops": 4 * D * pairs * Hq}
    if op == "cache":
        new, old = _lengths(case)
        back = sum(n + p % PT for n, p in zip(new, old))
        H = case["Hkv"]
        # tokens in and their 68 bytes out; 68 bytes in and the tokens back out; keys and values
        return {"bytes": 2 * H * (256 + 68) * (case["T"] + back), "flops": 0}
    if op == "decode":
        tokens = sum(_decode_lengths(case))
        return {"bytes": tokens * case["Hkv"] * 2 * 68 + case["B"] * case["Hq"] * (4 * D + 4), "flops": 4 * D * tokens * case["Hq"]}
    R, H, S = case["R"], case["H"], case["S"]
    pph = -(-S // PT) + 1
    page = 2 * 2 * PT * D * 2  # a page of keys and one of values, read and written
    if op == "fork":
        n = R - R // 2
        pages = int(n * H * 31 / 32)  # part pages
        return {"bytes": pages * page + n * H * pph * 4 * 2, "flops": 0}
    live = R * H * (5 * S / 8 / PT) * 0.875  # mean length 5/8 S; an eighth of the pages is shared
    left = live * 2 / 3
    moved = left * (1 - left / (live + 2 * R * H))  # live pages lie evenly over the pool
    return {"bytes": int(moved * page) + 2 * R * H * pph * 4, "flops": 0}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------


def exact(case, seed):
    op = case["op"]
    if op == "prefill":
        return _exact_prefill(prepare(case, seed))
    if op == "cache":
        return _exact_cache(prepare(case, seed))
    if op == "decode":
        return _exact_decode(prepare(case, seed))
    return None  # whole numbers, and pages moved as they are


def _soft(scores, values):
    """Softmax of scores [M, N] over values [N, D] in 64 bits; log-sum-exp beside it."""
    lse = torch.logsumexp(scores, -1)
    w = torch.exp(scores - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    return w @ values, lse


def _exact_prefill(st):
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    T, Hq, _ = q.shape
    G = Hq // k.shape[1]
    out, lse = torch.zeros_like(q), torch.full((T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    cq, ck = st["cu_q"].tolist(), st["cu_k"].tolist()
    for b in range(len(cq) - 1):
        L = ck[b + 1] - ck[b]
        for h in range(Hq):
            kt, vh = k[ck[b]:ck[b + 1], h // G].t().contiguous(), v[ck[b]:ck[b + 1], h // G].contiguous()
            for r in range(cq[b], cq[b + 1], 4096):
                e = min(cq[b + 1], r + 4096)
                s = st["scale"] * (q[r:e, h] @ kt)
                left = L - (cq[b + 1] - torch.arange(r, e, device=q.device)) + 1  # keys that a row sees
                s.masked_fill_(torch.arange(L, device=q.device)[None] >= left[:, None], -math.inf)
                out[r:e, h], lse[r:e, h] = _soft(s, vh)
    return out, lse


def _exact_number(code, byte):
    """What a 4-bit code and its scale byte stand for, in 64 bits."""
    e, m = (code >> 1) & 3, (code & 1).double()
    mag = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e.double() - 1))
    x = torch.where(byte == 255, torch.full_like(mag, math.nan), torch.exp2(byte.double() - 127))
    return torch.where(code >= 8, -mag, mag) * x


def _exact_at(pool, page, t, values):
    """The numbers of tokens t [n] of pages page [n], looked up value by value: [n, 128] in 64 bits."""
    c = torch.arange(D, device=t.device)[None]
    t = t[:, None]
    if values:
        q, j = (t & 15) >> 2, (t & 3) | ((t >> 4) << 2)
        byte, odd = ((c >> 6) << 10) + (((c & 15) + 16 * q) << 4) + (((c >> 4) & 3) << 2) + (j >> 1), (j & 1).expand(-1, D)
        sb = 2048 + 32 * q + 4 * j + (c >> 5)
    else:
        byte, odd = 64 * t + (c >> 1), (c & 1).expand(t.shape[0], D)
        sb = 2048 + 2 * ((t & 15) + 16 * (c >> 5)) + (t >> 4)
    rows = pool[page]
    b = torch.gather(rows, 1, byte)
    return _exact_number(torch.where(odd == 1, b >> 4, b & 15).long(), torch.gather(rows, 1, sb).long())


def _exact_cache(st):
    outs = []
    cu, start, cb, sb = (st[x].tolist() for x in ("cu", "start", "cu_back", "start_back"))
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    for x, pool, values in ((st["k"], st["k_pool"], False), (st["v"], st["v_pool"], True)):
        # the nearest 4-bit value of each; of two as near, the one with an even code
        y = x.double().view(-1, 32)
        top = y.abs().amax(1)
        X = torch.exp2((torch.floor(torch.log2(top)).clamp(min=-123) - 2))
        d = (y.abs()[..., None] / X[:, None, None] - grid).abs() + torch.tensor([0, 1e-9] * 4, dtype=torch.float64, device=DEV)
        near = (torch.copysign(grid[d.argmin(-1)], y) * X[:, None]).view(x.shape)
        out = torch.empty(st["k_back"].shape, dtype=torch.float64, device=DEV)
        for b in range(len(start)):
            old = start[b] - sb[b]  # tokens of the first page that were there before
            a = cb[b]
            if old:
                for h in range(x.shape[1]):
                    page = st["table"][b, h, sb[b] // PT].long()
                    out[a:a + old, h] = _exact_at(pool, page.expand(old), torch.arange(old, device=DEV), values)
            out[a + old:cb[b + 1]] = near[cu[b]:cu[b + 1]]
        outs.append(out)
    return tuple(outs)


def _exact_decode(st):
    q, table, lens = st["q"].double(), st["table"], st["lens"].tolist()
    B, Hq, _ = q.shape
    H = table.shape[1]
    out, lse = torch.zeros_like(q), torch.full((B, Hq), -math.inf, dtype=torch.float64, device=q.device)
    for b in range(B):
        t = torch.arange(lens[b], device=q.device)
        for h in range(H):
            page = table[b, h, :].long()[t // PT]
            if not lens[b]:
                continue
            k, v = torch.empty((lens[b], D), dtype=torch.float64, device=q.device), None
            v = torch.empty_like(k)
            for a in range(0, lens[b], 8192):
                part = slice(a, min(lens[b], a + 8192))
                k[part] = _exact_at(st["k_pool"], page[part], t[part] % PT, False)
                v[part] = _exact_at(st["v_pool"], page[part], t[part] % PT, True)
            rows = slice(h * Hq // H, (h + 1) * Hq // H)
            out[b, rows], lse[b, rows] = _soft(st["scale"] * (q[b, rows] @ k.t().contiguous()), v)
    return out, lse
