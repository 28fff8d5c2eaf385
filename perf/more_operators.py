"""The operators of a speculative decoding step over the 16-bit paged cache: rotary positions, appending to the cache with the
rotation on the way, attention of a tree of drafted tokens, the drafts' verification, and keeping the accepted ones.  `run`
computes each in its plain form (elementary torch operations in 32 or 64 bits), or, where `own` is set, by the framework's entry
points.

Sizes are those of an 8B-class decoder (32 query heads of 128, 8 key/value heads), of its tensor-parallel shards, and of latent
attention's 64 rotary channels.  A page holds 32 tokens of one head, [32][128] bf16.  A request's drafted tokens are the nodes of a
tree: node 0 is the root (the token that was accepted last), a node's parent comes before it, and the nodes are the last tokens of
the request in the cache.
"""
import math

import torch

own = False

DEV = "cuda:0"
D = 128
PT = 32           # tokens of a page


# ---- cases ---------------------------------------------------------------------------------------------------------------


def _rope(T, H, width, rot, layout, back, far):
    return {"op": "rope", "T": T, "H": H, "width": width, "rot": rot, "layout": layout, "back": back, "far": far}


def _append(B, T, start, Hq, Hkv, rot, layout):
    return {"op": "append", "B": B, "T": T, "start": start, "Hq": Hq, "Hkv": Hkv, "rot": rot, "layout": layout}


def _tree(B, T, S, Hq, Hkv, shape):
    return {"op": "tree", "B": B, "T": T, "S": S, "Hq": Hq, "Hkv": Hkv, "shape": shape}


def _verify(B, T, V, shape, draft, dtype):
    return {"op": "verify", "B": B, "T": T, "V": V, "shape": shape, "draft": draft, "dtype": dtype}


def _keep(B, T, H, S):
    return {"op": "keep", "B": B, "T": T, "H": H, "S": S}


def listed():
    return [
        # a decode step of latent attention: the 64 rotary channels of 128 query heads, far into a long context
        dict(_rope(64, 128, 64, 64, "interleaved", False, 131072), name="rope_latent"),
        # the gradient through the rotation of a long prompt's queries
        dict(_rope(16384, 32, 128, 128, "half", True, 16384), name="rope_grad"),
        # one token of each of 32 requests, projected at once: rotated and put into the cache
        dict(_append(32, 32, 3000, 32, 8, 128, "half"), name="append_step"),
        # a scheduler's step of prompt chunks, half of each head's channels rotated
        dict(_append(6, 16381, 500, 32, 8, 64, "half"), name="append_prompt"),
        # one request that verifies a tree of eight nodes
        dict(_tree(1, 8, 777, 32, 8, "tree"), name="tree_one"),
        # plain decoding, a token a request, lengths of their own
        dict(_tree(64, 64, 8000, 32, 8, "chain"), name="tree_single"),
        # 32 requests with trees of 24 nodes on the average
        dict(_tree(32, 768, 8000, 32, 8, "tree"), name="tree_batch"),
        # 64 drafted nodes each behind long contexts
        dict(_tree(8, 512, 32768, 32, 8, "tree"), name="tree_long"),
        # 16 chains of four drafted tokens, a small vocabulary
        dict(_verify(16, 80, 32000, "chain", True, "float32"), name="verify_chain"),
        # 64 trees of 31 drafted tokens on the average, a large vocabulary
        dict(_verify(64, 2048, 128000, "tree", True, "float32"), name="verify_tree"),
        # a few requests keep the accepted path of their trees
        dict(_keep(8, 64, 8, 900), name="keep_few"),
        # a full batch of them
        dict(_keep(256, 8192, 8, 4000), name="keep_batch"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rope", "append", "tree", "tree", "tree", "verify", "verify", "keep"))
    layout = rng.choice(("half", "interleaved"))
    Hkv = rng.choice((1, 2, 4, 8, 8))
    G = rng.choice((1, 2, 3, 4, 4, 5, 8, 16))
    shape = rng.choice(("chain", "tree", "tree"))
    if op == "rope":
        width = rng.choice((64, 64, 128, 128, 128, 256))
        rot = rng.choice((width, width, width // 2, width // 4, width - 24))
        H = rng.choice((1, 2, 8, 16, 32, 128))
        T = _log(rng, 1, min(16384, 16384 * 32 * 128 // (H * width)))
        return _rope(T, H, width, rot, layout, rng.random() < 0.4, _log(rng, 100, 1000000))
    if op == "append":
        B = _log(rng, 1, 256)
        T = max(B, _log(rng, 1, 16384))
        return _append(B, T, _log(rng, 1, 4000), Hkv * min(G, 32 // Hkv), Hkv, rng.choice((128, 128, 64, 32, 104)), layout)
    if op == "tree":
        B, n = _log(rng, 1, 64), _log(rng, 1, 64)
        S = _log(rng, 2 * n + 1, min(32768, 8 * 32768 * 8 // (B * Hkv)))
        G = min(G, 32 // Hkv)
        while B * n * S * Hkv * G > 8 * 64 * 32768 * 32:  # no more than the longest trees' work
            n = max(1, n // 2)
        return _tree(B, B * n, S, Hkv * G, Hkv, shape)
    if op == "verify":
        B, n, V = _log(rng, 1, 64), _log(rng, 2, 32), _log(rng, 1000, 128000)
        return _verify(B, B * n, V, shape, rng.random() < 0.7, rng.choice(("float32", "float32", "bfloat16")))
    B = _log(rng, 1, 256)
    return _keep(B, B * _log(rng, 2, 32), Hkv, _log(rng, 100, 4000))


def _gen(case):
    """What is the same for every seed, so that a case's work is one number."""
    return torch.Generator(device="cpu").manual_seed(7 + case["B"] + case["T"])


def _new(case, g):
    """New tokens (nodes) of each request: from half the mean to one and a half, T in all."""
    B, T = case["B"], case["T"]
    u = torch.rand(B, generator=g, dtype=torch.float64) + 0.5
    cut = (torch.cumsum(u, 0) / u.sum() * (T - B)).long()
    new = torch.diff(cut, prepend=torch.zeros(1, dtype=torch.long)) + 1
    new[-1] += T - int(new.sum())
    return new.tolist()


def _old(case, g, top, new):
    """Tokens of each request in the cache before them: from a quarter of the most on; the first request has the most."""
    u = torch.rand(case["B"], generator=g, dtype=torch.float64) * 0.75 + 0.25
    u[0] = 1
    return [max(0, int(top * float(x)) - n) for x, n in zip(u, new)]


def _parents(case, new, g):
    """Each node's parent in its request: a chain, or a tree in which a node has two or three children."""
    out = []
    for n in new:
        w = 1 if case["shape"] == "chain" else 1 + int(torch.randint(1, 3, (1,), generator=g))
        out += [[(i - 1) // w if i else -1 for i in range(n)]]
    return out


def _kept(new, g):
    """A path of each request's tree: the root, then on the average every fourth node."""
    out = []
    for n in new:
        take = torch.rand(n, generator=g) < 0.25
        take[0] = True
        out.append(torch.nonzero(take)[:, 0].tolist())
    return out


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


def _pool(g, pages):
    pool = torch.empty((pages, PT, D), dtype=torch.bfloat16, device=DEV)
    for a in range(0, pages, 1 << 15):
        pool[a:a + (1 << 15)] = _normal(g, (min(1 << 15, pages - a), PT, D))
    return pool


def _freq(rot):
    """Frequencies of a context stretched eightfold: slow channels turn eight times slower, fast ones as ever."""
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    turns = 8192 * f / (2 * math.pi)
    keep = ((turns - 1) / (4 - 1)).clamp(0, 1)
    return (f * (keep + (1 - keep) / 8)).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op = case["op"]
    if op == "rope":
        T, H, W = case["T"], case["H"], case["width"]
        if W == 64:  # the last channels of a wider query
            x = _normal(g, (T, H, 576))[..., 512:]
        else:
            x = _normal(g, (T, H, W))
        pos = torch.randint(0, case["far"], (T,), generator=g, device=DEV, dtype=torch.int32)
        return {"op": op, "x": x, "pos": pos, "freq": _freq(case["rot"]), "layout": case["layout"], "back": case["back"],
                "amp": 1.2, "out": torch.empty((T, H, W), dtype=torch.bfloat16, device=DEV)}
    gl = _gen(case)
    new = _new(case, gl)
    if op == "append":
        Hq, H, T = case["Hq"], case["Hkv"], case["T"]
        old = _old(case, gl, case["start"], [0] * len(new))
        lens = [a + b for a, b in zip(new, old)]
        table, pages = _tables(g, lens, H, -(-max(lens) // PT) + 1, 5)
        qkv = _normal(g, (T, Hq + 2 * H, D))  # the fused projection's output, seen as its three parts
        return {"op": op, "q": qkv[:, :Hq], "k": qkv[:, Hq:Hq + H], "v": qkv[:, Hq + H:], "table": table,
                "k_pool": _pool(g, pages), "v_pool": _pool(g, pages), "cu": _offsets(new), "start": _i32(old),
                "freq": _freq(case["rot"]), "layout": case["layout"], "amp": 1.1,
                "q_out": torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV)}
    if op == "tree":
        Hq, H, T, S = case["Hq"], case["Hkv"], case["T"], case["S"]
        old = _old(case, gl, S, new)
        lens = [a + b for a, b in zip(new, old)]
        table, pages = _tables(g, lens, H, -(-S // PT), 5)
        parents = _parents(case, new, gl)
        words = -(-max(new) // 64)
        mask = torch.zeros((T, words * 64), dtype=torch.bool)
        row = 0
        for par in parents:
            for i, p in enumerate(par):
                if i:
                    mask[row + i] = mask[row + p]
                mask[row + i, i] = True
            row += len(par)
        bit = torch.ones(64, dtype=torch.int64) << torch.arange(64)
        mask = (mask.view(T, words, 64) * bit).sum(-1)  # (a sum of distinct bits: the sign bit is one of them)
        return {"op": op, "q": _normal(g, (T, Hq, D)), "k_pool": _pool(g, pages), "v_pool": _pool(g, pages), "table": table,
                "cu": _offsets(new), "lens": _i32(lens), "mask": None if case["shape"] == "chain" else mask.to(DEV), "S": S,
                "most": max(new), "parents": parents, "scale": 1 / math.sqrt(D),
                "o": torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV),
                "lse": torch.empty((T, Hq), dtype=torch.float32, device=DEV)}
    if op == "verify":
        B, T, V = case["B"], case["T"], case["V"]
        dtype = getattr(torch, case["dtype"])
        parents = _parents(case, new, gl)
        cu = _offsets(new)
        first = torch.repeat_interleave(cu[:-1].long(), torch.tensor(new, device=DEV))
        parent = _i32(sum(parents, []))
        z = torch.randn((T, V), generator=g, device=DEV).mul_(2.5)
        target = torch.softmax(z, 1).to(dtype)
        draft = torch.softmax(z.add_(torch.randn((T, V), generator=g, device=DEV), alpha=0.8), 1).to(dtype)  # a model that nearly agrees
        del z
        at = first + parent.clamp(min=0).long()
        # each node's token drawn from what its parent's row of the draft says
        u = torch.rand((T, 1), generator=g, device=DEV)
        tokens = torch.empty(T, dtype=torch.int32, device=DEV)
        for a in range(0, T, 256):
            cum = torch.cumsum(draft[at[a:a + 256]].float(), 1)
            tokens[a:a + 256] = torch.searchsorted(cum, u[a:a + 256] * cum[:, -1:])[:, 0].clamp(max=V - 1).to(torch.int32)
        return {"op": op, "target": target, "draft": draft if case["draft"] else None, "tokens": tokens,
                "parents": None if case["shape"] == "chain" else parent, "cu": cu, "most": max(new),
                "accept": torch.rand(T, generator=g, device=DEV), "final": torch.rand(B, generator=g, device=DEV),
                "path": torch.empty(T, dtype=torch.int32, device=DEV), "count": torch.empty(B, dtype=torch.int32, device=DEV),
                "token": torch.empty(B, dtype=torch.int32, device=DEV)}
    B, H, S = case["B"], case["H"], case["S"]
    old = _old(case, gl, S, new)
    lens = [a + b for a, b in zip(new, old)]
    kept = _kept(new, gl)
    table, pages = _tables(g, lens, H, -(-max(lens) // PT), 9)
    rows = torch.randperm(B, generator=g, device=DEV)
    path = [p + [-1] * (n - len(p)) for p, n in zip(kept, new)]
    table0, lens0 = torch.empty_like(table), torch.empty(B, dtype=torch.int32, device=DEV)
    table0[rows], lens0[rows] = table, _i32(lens)
    refs0 = torch.bincount(table[table >= 0].long(), minlength=pages).to(torch.int32)
    return {"op": op, "table0": table0, "lens0": lens0, "refs0": refs0, "table": table0.clone(), "lens": lens0.clone(),
            "refs": refs0.clone(), "k_pool": _pool(g, pages), "v_pool": _pool(g, pages), "rows": rows.to(torch.int32),
            "cu": _offsets(new), "path": _i32(sum(path, [])), "count": _i32([len(p) for p in kept])}


# ---- the plain forms -----------------------------------------------------------------------------------------------------


def _turn(x, pos, freq, layout, amp, back):
    """x [T, H, W], the first 2 * len(freq) channels turned by pos * freq, in 32 bits."""
    angle = pos.double()[:, None] * freq  # (in 64: far positions)
    cos, sin = (torch.cos(angle) * amp).float()[:, None], (torch.sin(angle) * amp).float()[:, None]
    if back:
        sin = -sin
    y, r = x.float(), 2 * freq.shape[0]
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if layout == "interleaved" else (y[..., :r // 2], y[..., r // 2:r])
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, d], -1).flatten(-2) if layout == "interleaved" else torch.cat([c, d], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_rope(st):
    return st["out"].copy_(_turn(st["x"], st["pos"], st["freq"], st["layout"], st["amp"], st["back"]))


def _places(cu, start, T):
    """Each packed token's request and its position in it."""
    i = torch.arange(T, device=cu.device)
    b = torch.searchsorted(cu[1:].contiguous(), i.to(torch.int32), right=True)
    return b, start[b].long() + i - cu[b].long()


def _plain_append(st):
    b, pos = _places(st["cu"], st["start"], st["k"].shape[0])
    turn = st["freq"], st["layout"], st["amp"], False
    page, t = st["table"][b, :, pos // PT].long(), (pos % PT)[:, None]
    st["k_pool"][page, t] = _turn(st["k"], pos, *turn)
    st["v_pool"][page, t] = st["v"]
    st["q_out"].copy_(_turn(st["q"], pos, *turn))
    return st["q_out"], st["k_pool"], st["v_pool"]


def _plain_tree(st):
    q, table, cu, lens, S, n = st["q"], st["table"], st["cu"].long(), st["lens"].long(), st["S"], st["most"]
    B, H, _ = table.shape
    T, Hq, _ = q.shape
    G = Hq // H
    j = torch.arange(n, device=q.device)
    count = cu[1:] - cu[:-1]
    base = lens - count
    at = (cu[:-1, None] + j).clamp(max=T - 1)  # (rows past a request's last are computed and dropped)
    qp = q[at].float().view(B, n, H, G, D).transpose(1, 2).reshape(B, H, n * G, D)
    page = table.clamp(min=0).long()
    k = st["k_pool"][page].view(B, H, -1, D)[:, :, :S].float()
    t = torch.arange(S, device=q.device)
    node = t[None] - base[:, None]  # [B, S]: which node a position holds
    if st["mask"] is None:
        seen = node[:, None] <= j[:, None]
    else:
        word = (node.clamp(0, n - 1) // 64)[:, None].expand(B, n, S)
        bit = torch.gather(st["mask"][at], 2, word) >> (node.clamp(min=0) % 64)[:, None] & 1
        seen = (node < 0)[:, None] | ((bit == 1) & (node < count[:, None])[:, None])
    seen = seen & (t[None] < lens[:, None])[:, None]
    s = torch.matmul(qp, k.transpose(2, 3).contiguous()).mul_(st["scale"])
    del k
    s.view(B, H, n, G, S).masked_fill_(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    v = st["v_pool"][page].view(B, H, -1, D)[:, :, :S].float()
    v = torch.where((t[None] < lens[:, None])[:, None, :, None], v, torch.zeros_like(v))
    o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (m + torch.log(total)).view(B, H, n, G).transpose(1, 2).reshape(B, n, Hq)
    o = o.view(B, H, n, G, D).transpose(1, 2).reshape(B, n, Hq, D)
    i = torch.arange(T, device=q.device)
    b = torch.searchsorted(cu[1:].contiguous(), i, right=True)
    st["o"].copy_(o[b, i - cu[b]])
    st["lse"].copy_(lse[b, i - cu[b]])
    return st["o"], st["lse"]


def _plain_verify(st):
    """The nodes of all requests in order; in 64 bits, since the outputs are choices."""
    P, Q, tokens, cu = st["target"], st["draft"], st["tokens"].long(), st["cu"].long()
    T, V = P.shape
    first, n = cu[:-1], cu[1:] - cu[:-1]
    B = first.shape[0]
    b = torch.arange(B, device=P.device)
    zero, one = torch.zeros(B, dtype=torch.float64, device=P.device), torch.ones(B, dtype=torch.float64, device=P.device)
    cur, c, m, kept = torch.zeros_like(first), zero, one, torch.ones_like(first)
    path = torch.full((B, st["most"]), -1, dtype=torch.int32, device=P.device)
    path[:, 0] = 0
    dead = torch.zeros((B, V), dtype=torch.bool, device=P.device)
    for i in range(1, st["most"]):
        at = (first + i).clamp(max=T - 1)
        t = tokens[at]
        tried = (n > i) & (cur == (i - 1 if st["parents"] is None else st["parents"][at]))
        row = first + cur
        p = P[row, t].double()
        if Q is not None:
            q = Q[row, t].double()
            left = (p - c * q).clamp(min=0)
            took = tried & (st["accept"][at].double() * q * m < left)
        else:
            took = tried & ~dead[b, t] & (st["accept"][at].double() * m < p)
        lost = tried & ~took
        if Q is not None:
            c = torch.where(lost, c + m, c)
            m = torch.where(lost, (P[row].double() - c[:, None] * Q[row].double()).clamp(min=0).sum(1), m)
        else:
            m = torch.where(lost & ~dead[b, t], m - p, m)
            dead[b, t] |= lost
            dead &= ~took[:, None]
        c, m, cur = torch.where(took, zero, c), torch.where(took, one, m), torch.where(took, i, cur)
        place = kept.clamp(max=st["most"] - 1)
        path[b, place] = torch.where(took, i, path[b, place]).to(torch.int32)
        kept = kept + took
    row = first + cur
    p = P[row].double()
    left = (p - c[:, None] * Q[row].double()).clamp(min=0) if Q is not None else torch.where(dead, torch.zeros_like(p), p)
    left = torch.where((left.sum(1) > 0)[:, None], left, p)
    cum = torch.cumsum(left, 1)
    token = (cum <= (st["final"].double() * cum[:, -1])[:, None]).sum(1)
    j = torch.arange(T, device=P.device)
    of = torch.searchsorted(cu[1:].contiguous(), j, right=True)
    st["path"].copy_(path[of, j - cu[of]])
    st["count"].copy_(kept)
    st["token"].copy_(token)
    return st["path"], st["count"], st["token"]


def _plain_keep(st):
    table, lens, refs = st["table"], st["lens"], st["refs"]
    rows, cu, path = st["rows"].long(), st["cu"].long(), st["path"].long()
    i = torch.arange(path.shape[0], device=path.device)
    b = torch.searchsorted(cu[1:].contiguous(), i, right=True)
    j = i - cu[b]
    base = lens[rows].long() - (cu[1:] - cu[:-1])
    to = base[b] + j
    src = torch.where(j < st["count"][b], base[b] + path, to)  # (a token that is not kept stays where it is)
    head = torch.arange(table.shape[1], device=path.device)[None]
    where = [table[rows[b][:, None], head, x[:, None] // PT].long() * PT + x[:, None] % PT for x in (to, src)]
    for pool in (st["k_pool"], st["v_pool"]):
        flat = pool.view(-1, D)
        flat[where[0]] = flat[where[1]]
    now = base + st["count"]
    col = torch.arange(table.shape[2], device=path.device)
    e = table[rows]
    gone = (col >= (now[:, None] + PT - 1) // PT) & (col < (lens[rows].long()[:, None] + PT - 1) // PT)
    gone = gone[:, None].expand_as(e)
    refs.index_add_(0, e.clamp(min=0).reshape(-1).long(), -gone.reshape(-1).to(torch.int32))
    table[rows] = torch.where(gone, torch.full_like(e, -1), e)
    lens[rows] = now.to(torch.int32)
    return st["k_pool"], st["v_pool"], table, lens, refs


def run(state):
    s, op = state, state["op"]
    if op == "keep":  # from the same tables at every pass
        for name in ("table", "lens", "refs"):
            s[name].copy_(s[name + "0"])
    if not own:
        return {"rope": _plain_rope, "append": _plain_append, "tree": _plain_tree, "verify": _plain_verify, "keep": _plain_keep}[op](s)
    import paper_2609_24270_amd as asym
    if op == "rope":
        return asym.rope(s["x"], s["pos"], s["freq"], out=s["out"], layout=s["layout"], amplitude=s["amp"], backward=s["back"])
    if op == "append":
        asym.kv_append(s["k"], s["v"], s["k_pool"], s["v_pool"], s["table"], s["table"], s["cu"], s["start"], q=s["q"],
                       q_out=s["q_out"], freq=s["freq"], layout=s["layout"], amplitude=s["amp"])
        return s["q_out"], s["k_pool"], s["v_pool"]
    if op == "tree":
        asym.attn_tree_paged(s["q"], s["k_pool"], s["v_pool"], s["table"], s["table"], s["cu"], s["lens"], mask=s["mask"],
                             S=s["S"], o=s["o"], lse=s["lse"], scale=s["scale"])
        return s["o"], s["lse"]
    if op == "verify":
        return asym.draft_verify(s["target"], s["draft"], s["tokens"], s["parents"], s["cu"], s["accept"], s["final"],
                                 path=s["path"], count=s["count"], token=s["token"])
    asym.kv_keep(s["k_pool"], s["v_pool"], s["table"], s["lens"], s["refs"], s["rows"], s["cu"], s["path"], s["count"])
    return s["k_pool"], s["v_pool"], s["table"], s["lens"], s["refs"]


# ---- work ----------------------------------------------------------------------------------------------------------------


def work(case):
    op, T = case["op"], case["T"]
    if op == "rope":
        return {"bytes": T * (4 * case["H"] * case["width"] + 4), "flops": 3 * T * case["H"] * case["rot"]}
    g = _gen(case)
    new = _new(case, g)
    if op == "append":
        heads = case["Hq"] + 2 * case["Hkv"]
        return {"bytes": T * heads * D * 4, "flops": 3 * T * (case["Hq"] + case["Hkv"]) * case["rot"]}
    if op == "tree":
        old = _old(case, g, case["S"], new)
        pairs = 0
        for n, o, par in zip(new, old, _parents(case, new, g)):
            depth = []
            for p in par:
                depth.append(1 if p < 0 else depth[p] + 1)
            pairs += n * o + sum(depth)
        kv = (sum(new) + sum(old)) * case["Hkv"] * 2 * D * 2
        return {"bytes": kv + T * case["Hq"] * (4 * D + 4), "flops": 4 * D * pairs * case["Hq"]}
    if op == "verify":
        # at least the row that the last token is drawn from, and what each node says
        row = case["V"] * (4 if case["dtype"] == "float32" else 2) * (2 if case["draft"] else 1)
        return {"bytes": case["B"] * (row + 12) + 20 * T, "flops": 0}
    old = _old(case, g, case["S"], new)
    moved = sum(sum(i != p for i, p in enumerate(path)) for path in _kept(new, g))
    return {"bytes": moved * case["H"] * 2 * 2 * D * 2 + 4 * case["B"] * case["H"] * 2 + 8 * T + 4 * sum(new + old) // PT // 8,
            "flops": 0}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------


def exact(case, seed):
    op = case["op"]
    if op == "rope":
        st = prepare(case, seed)
        return _exact_turn(st["x"].double(), st["pos"], st["freq"], st["layout"], st["amp"], st["back"])
    if op == "append":
        return _exact_append(prepare(case, seed))
    if op == "tree":
        return _exact_tree(prepare(case, seed))
    return None  # choices, and tokens moved as they are


def _exact_turn(x, pos, freq, layout, amp, back):
    """Pairs as complex numbers, times amp * exp(i angle)."""
    r = 2 * freq.shape[0]
    angle = pos.double()[:, None] * freq * (-1 if back else 1)
    w = torch.polar(torch.full_like(angle, amp), angle)[:, None]
    out = x.clone()
    if layout == "interleaved":
        out[..., :r] = torch.view_as_real(torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2)) * w).flatten(-2)
    else:
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * w
        out[..., :r // 2], out[..., r // 2:r] = z.real, z.imag
    return out


def _exact_append(st):
    k_pool, v_pool = st["k_pool"].double(), st["v_pool"].double()
    q_out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    cu, start = st["cu"].tolist(), st["start"].tolist()
    for b in range(len(start)):
        rows = slice(cu[b], cu[b + 1])
        pos = torch.arange(start[b], start[b] + cu[b + 1] - cu[b], device=DEV)
        turn = pos, st["freq"], st["layout"], st["amp"], False
        q_out[rows] = _exact_turn(st["q"][rows].double(), *turn)
        k, v = _exact_turn(st["k"][rows].double(), *turn), st["v"][rows].double()
        for h in range(k.shape[1]):
            page = st["table"][b, h].long()[pos // PT]
            k_pool[page, pos % PT], v_pool[page, pos % PT] = k[:, h], v[:, h]
    return q_out, k_pool, v_pool


def _exact_tree(st):
    """Request by request and head by head, on dense keys; what a node sees found by walking to the root."""
    q, table, lens, cu = st["q"].double(), st["table"], st["lens"].tolist(), st["cu"].tolist()
    T, Hq, _ = q.shape
    H = table.shape[1]
    G = Hq // H
    out, lse = torch.zeros_like(q), torch.full((T, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, par in enumerate(st["parents"]):
        n, L = len(par), lens[b]
        see = torch.zeros((n, L), dtype=torch.bool)
        see[:, :L - n] = True
        for i in range(n):
            a = i
            while a >= 0:
                see[i, L - n + a] = True
                a = par[a]
        see = see.to(DEV)[:, None]
        rows = slice(cu[b], cu[b + 1])
        for h in range(H):
            page = table[b, h, :-(-L // PT)].long()
            k, v = (st[x][page].view(-1, D)[:L].double() for x in ("k_pool", "v_pool"))
            s = (q[rows, h * G:(h + 1) * G].reshape(n * G, D) @ k.t().contiguous()).view(n, G, L) * st["scale"]
            s = torch.where(see, s, torch.full_like(s, -math.inf))
            z = torch.logsumexp(s, -1)
            lse[rows, h * G:(h + 1) * G] = z
            out[rows, h * G:(h + 1) * G] = (torch.exp(s - z[..., None]).view(n * G, L) @ v).view(n, G, D)
    return out, lse
