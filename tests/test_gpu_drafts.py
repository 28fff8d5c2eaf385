"""GPU parity of the verification of drafted tokens and of keeping them, and a whole step of drafting, through the C ABI.

Choices are compared with the oracle's as they are: both are computed in 64 bits, and the random numbers
here keep away from borders by more than 10^-12 (checked where they are made).
"""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import drafts, kv_pages, prompt
from tests.checks import bf16_bits_to_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    asym.load_library()
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


def f64(t):
    return bf16_bits_to_f64(t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16))


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def offsets(lens, first=0):
    return (np.cumsum([0] + list(lens)) + first).tolist()


class Drafts:
    def __init__(self, new, V, seed, dtype=torch.float32, chain=False, noise=0.7, peak=2.0, width=3):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.new, self.V, self.cu, self.dtype = new, V, offsets(new), dtype
        T = self.T = self.cu[-1]
        z = torch.randn((T, V), generator=g) * peak
        self.target = torch.softmax(z, 1).to(dtype)
        self.draft = torch.softmax(z + torch.randn((T, V), generator=g) * noise, 1).to(dtype)
        self.parents = [[-1] + [i - 1 if chain else int(rng.integers(max(0, (i - 1) // width), i)) for i in range(1, n)] if n else [] for n in new]
        self.chain = chain
        self.tokens = []
        for b, par in enumerate(self.parents):
            for i, p in enumerate(par):
                row = self.draft[self.cu[b] + max(p, 0)].double().numpy()
                self.tokens.append(int(rng.choice(V, p=row / row.sum())) if i else -7)
        # (multiples of 2^-24 as fp32 gives them; exact in both)
        self.accept = torch.rand(T, generator=g)
        self.final = torch.rand(len(new), generator=g)

    def want(self, draft=True):
        path, count, token = [-1] * self.T, [], []
        n64 = lambda t: t.double().numpy()
        for b, n in enumerate(self.new):
            if n == 0:
                count.append(0), token.append(-1)
                continue
            rows = slice(self.cu[b], self.cu[b + 1])
            p, t = drafts.verify(n64(self.target[rows]), n64(self.draft[rows]) if draft else None, self.tokens[rows], self.parents[b],
                                 n64(self.accept[rows]).tolist(), float(self.final[b]))
            path[self.cu[b]:self.cu[b] + len(p)] = p
            count.append(len(p)), token.append(t)
        return path, count, token

    def run(self, dev, draft=True, **kw):
        par = None if self.chain else i32(sum(self.parents, []), dev)
        r = asym.draft_verify(self.target.to(dev), self.draft.to(dev) if draft else None, i32(self.tokens, dev), par, i32(self.cu, dev),
                              self.accept.to(dev), self.final.to(dev), **kw)
        return tuple(x.tolist() for x in r)


@pytest.mark.parametrize("new,V", [([1], 1), ([1], 5), ([4], 7), ([2, 0, 5], 100), ([8, 1, 3], 2047), ([12], 2048), ([6, 6], 2049), ([30], 50001),
                                   ([5, 9, 2, 7], 8193), ([70, 3], 1000), ([140], 64), ([3] * 70, 333), ([9] * 5, 40000)])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("chain", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_against_oracle(dev, new, V, draft, chain, dtype):
    d = Drafts(new, V, seed=sum(new) + V, dtype=dtype, chain=chain)
    assert d.run(dev, draft) == d.want(draft)


@pytest.mark.parametrize("seed", range(12))
def test_many_siblings(dev, seed):
    # drafts that are far from the target, and wide trees: several rejections at a node, more than the launches that
    # sum in parallel, and nothing left of what the target has
    d = Drafts([24, 17, 40, 2], [50, 500, 3000, 10000][seed % 4], seed=seed, noise=3.0, peak=1.0 + seed % 3, width=12)
    assert d.run(dev) == d.want()
    assert d.run(dev, False) == d.want(False)


@pytest.mark.parametrize("new,V", [([24, 17, 40, 2], 16385), ([30], 20000), ([24, 17, 40, 2, 9], 70000), ([20, 5], 140000), ([7] * 20, 33000)])
@pytest.mark.parametrize("noise", [1.0, 3.0])
def test_many_siblings_of_a_large_vocabulary(dev, new, V, noise):
    # rows that are summed by launches of their own, fewer than some request's rejections
    d = Drafts(new, V, seed=V, noise=noise, peak=2.0, width=12)
    assert d.run(dev) == d.want()
    assert d.run(dev, False) == d.want(False)


def test_borders(dev):
    # powers of two: every sum exact, every comparison a tie or not at all
    V = 4
    p = torch.tensor([[0.5, 0.25, 0.125, 0.125], [0.25, 0.25, 0.25, 0.25], [0, 0, 1, 0]])
    q = torch.tensor([[0.25, 0.5, 0.125, 0.125], [1.0, 0, 0, 0], [0.25] * 4])
    def run(tokens, accept, final, draft=True, parents=(-1, 0, 1)):
        r = asym.draft_verify(p.to(dev), q.to(dev) if draft else None, i32(tokens, dev), i32(parents, dev), i32([0, 3], dev),
                              torch.tensor(accept, device=dev), torch.tensor([final], device=dev))
        return [x.tolist() for x in r]
    assert run([0, 1, 9], [0, 0.5, 0], 0.0) == [[0, -1, -1], [1], [0]]                     # 0.5 * 0.5 < 0.25 is false: a tie rejects
    assert run([0, 1, 0], [0, 0.25, 0.125], 0.0) == [[0, 1, 2], [3], [2]]                  # leading zeros are not drawn
    assert run([0, 1, 0], [0, 0.25, 0.25], 0.25) == [[0, 1, -1], [2], [1]]                 # row 1 less (1, 0, 0, 0): 1/4 each; 1/4 > 3/16
    assert run([0, 9, 0], [0, 0.0, 0.0], 0.5) == [[0, -1, -1], [1], [1]]                    # token 9 is passed over; 0.5 > 0.5 is false
    assert run([0, -1, 0], [0, 0.0, 0.0], 0.4375) == [[0, -1, -1], [1], [0]]
    assert run([0, 1, 1], [0, 0.5, 0.0], 0.5, False, (-1, 0, 0)) == [[0, -1, -1], [1], [0]]  # rejected once: no second chance
    assert run([0, 1, 0], [0, 0.5, 0.5], 0.5, False, (-1, 0, 0)) == [[0, 2, -1], [2], [2]]   # m = 3/4: 0.375 < 0.5
    assert run([0, 1, 0], [0, 0.0, 0.0], 0.5, True, (-1, 5, 2)) == [[0, -1, -1], [1], [1]]   # parents that do not come before
    assert run([0, 1, 0], [0, 0.0, 0.0], 0.5, True, (-1, -1, 1)) == [[0, -1, -1], [1], [1]]
    assert run([0, 1, 0], [0, float("nan"), 0.0], float("nan"), True, (-1, 0, 1))[0] == [0, -1, -1]


def test_what_is_no_probability_counts_as_0(dev):
    p = torch.tensor([[float("nan"), -1.0, 0.5, float("inf")], [0, 0, 0, 0]])
    for draft in (None, torch.full((2, 4), 0.25)):
        r = asym.draft_verify(p.to(dev), None if draft is None else draft.to(dev), i32([0, 2], dev), None, i32([0, 2], dev),
                              torch.tensor([0.0, 0.25], device=dev), torch.tensor([0.5], device=dev))
        assert [x.tolist() for x in r] == [[0, 1], [2], [-1]]  # behind node 1 the target says nothing
        r = asym.draft_verify(p.to(dev), None if draft is None else draft.to(dev), i32([0, 3], dev), None, i32([0, 2], dev),
                              torch.tensor([0.0, 0.0], device=dev), torch.tensor([0.5], device=dev))
        assert [x.tolist() for x in r] == [[0, -1], [1], [2]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_alignment_and_rows_outside(dev, dtype):
    d = Drafts([5, 0, 8], 1001, seed=3, dtype=dtype)
    path, count, token = d.want()
    wide = torch.full((d.T + 4, 1200), float("nan"), dtype=dtype, device=dev)
    wide[2:2 + d.T, 3:1004] = d.target.to(dev)
    other = torch.full((d.T + 4, 1003), float("nan"), dtype=dtype, device=dev)
    other[2:2 + d.T, 1:1002] = d.draft.to(dev)
    pad = lambda x, v: torch.nn.functional.pad(x, (2, 2), value=v)
    out = torch.full((d.T + 4,), 77, dtype=torch.int32, device=dev)
    r = asym.draft_verify(wide[:, 3:1004], other[:, 1:1002], pad(i32(d.tokens, dev), 5), pad(i32(sum(d.parents, []), dev), 0),
                          i32(offsets(d.new, 2), dev), pad(d.accept.to(dev), 0.0), d.final.to(dev), path=out)
    assert r[0] is out and out[2:-2].tolist() == path and r[1].tolist() == count and r[2].tolist() == token
    assert out[:2].tolist() == out[-2:].tolist() == [77, 77]


def test_offsets_that_say_too_much_are_held(dev):
    d = Drafts([6], 300, seed=4)
    want = d.run(dev)
    d.cu = [-5, 1000]
    assert d.run(dev) == want


@pytest.mark.parametrize("V", [5000, 70000])
def test_streams_and_graphs(dev, V):
    a, b = Drafts([6, 9, 1], V, seed=5, width=8, noise=2.0), Drafts([6, 9, 1], V, seed=6, width=8, noise=2.0)
    s = asym.stream_create()
    torch.cuda.synchronize()
    assert a.run(dev, stream=None) == a.want()
    ta, tb = ([x.to(dev) for x in (d.target, d.draft)] + [i32(d.tokens, dev), i32(sum(d.parents, []), dev), i32(d.cu, dev),
                                                         d.accept.to(dev), d.final.to(dev)] for d in (a, b))
    torch.cuda.synchronize()
    r = asym.draft_verify(*ta, stream=s)
    s.synchronize()
    assert tuple(x.tolist() for x in r) == a.want()
    asym.stream_destroy(s)
    held = [x.clone() for x in ta]
    outs = [torch.empty_like(x) for x in r]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asym.draft_verify(*held, path=outs[0], count=outs[1], token=outs[2])
    for src, d in ((ta, a), (tb, b), (ta, a), (tb, b)):
        for h, x in zip(held, src):
            h.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert tuple(x.tolist() for x in outs) == d.want()


def test_verify_refusals(dev):
    d = Drafts([3], 10, seed=0)
    args = [d.target.to(dev), d.draft.to(dev), i32(d.tokens, dev), i32(d.parents[0], dev), i32(d.cu, dev), d.accept.to(dev), d.final.to(dev)]
    for at, x, kind in ((0, args[0].half(), TypeError), (1, args[1].bfloat16(), TypeError), (1, args[1][:, :9], ValueError),
                        (0, args[0][:2], ValueError), (2, args[2].long(), TypeError), (2, args[2][:2], ValueError), (3, args[3][:2], ValueError),
                        (4, args[4].cpu(), ValueError), (5, args[5].double(), TypeError), (6, args[5], ValueError),
                        (0, args[0].t().contiguous().t(), ValueError), (0, args[0][:1].expand(3, 10), asym.AsymError)):
        bad = list(args)
        bad[at] = x
        with pytest.raises(kind):
            asym.draft_verify(*bad)
    with pytest.raises(ValueError):
        asym.draft_verify(*args, token=i32([1, 2], dev))
    empty = asym.draft_verify(args[0][:0], args[1][:0], args[2][:0], args[3][:0], i32([0, 0], dev), args[5][:0], args[6])
    assert [x.tolist() for x in empty] == [[], [0], [-1]]


# -- keeping ---------------------------------------------------------------------------

def cache(dev, lens, H, pph, seed, width=16, dtype=torch.int32):
    """A kv_pages.Cache of random rows, and the same on the GPU."""
    rng = np.random.default_rng(seed)
    R = len(lens)
    total = R * H * pph + 5
    table = np.full((R, H, pph), -1, np.int32)
    perm, at = rng.permutation(total), 0
    for r, n in enumerate(lens):
        for h in range(H):
            for c in range(-(-n // 32)):
                table[r, h, c] = perm[at]
                at += 1
    refs = np.zeros(total, np.int32)
    np.add.at(refs, table[table >= 0], 1)
    pools = [rng.integers(0, 1 << 30, (total, 32, width)).astype(np.int32) for _ in range(2)]
    return kv_pages.Cache(table, np.array(lens, np.int32), refs, pools), [torch.tensor(x, device=dev) for x in (*pools, table, np.array(lens, np.int32), refs)]


def same(c, state):
    for want, got in zip((*c.pools, c.table, c.lens, c.refs), state):
        assert np.array_equal(want, got.cpu().numpy())


@pytest.mark.parametrize("lens,H,new,width", [([1], 1, [1], 4), ([70], 2, [8], 4), ([64, 33, 100], 3, [5, 33, 40], 16), ([40] * 9, 1, [7] * 9, 64),
                                             ([31, 32, 0, 65], 2, [31, 1, 0, 65], 8), ([300, 10], 8, [70, 10], 64), ([50], 40, [20], 64)])
@pytest.mark.parametrize("seed", range(3))
def test_keep_against_oracle(dev, lens, H, new, width, seed):
    c, state = cache(dev, lens, H, max(1, -(-max(lens) // 32)) + 1, seed, width)
    rng = np.random.default_rng(seed + 50)
    rows = rng.permutation(len(lens)).astype(np.int32)
    n = [new[r] for r in rows]
    cu = offsets(n)
    path, count = np.full(cu[-1], -1, np.int32), []
    for i, m in enumerate(n):
        mine = np.nonzero(rng.random(m) < [0.4, 1.0, 0.1][seed])[0]
        path[cu[i]:cu[i] + len(mine)] = mine
        count.append(len(mine))
    drafts.keep(c, rows, cu, path, count)
    asym.kv_keep(*state, i32(rows, dev), i32(cu, dev), i32(path, dev), i32(count, dev))
    same(c, state)


def test_keep_leaves_out_what_makes_no_sense(dev):
    lens = [70, 70, 70, 70, 5, 70, 70, 70]
    c, state = cache(dev, lens, 2, 4, 1)
    rows = [0, 1, 2, 3, 4, 0, 99, -1, 5, 6, 7]
    paths = [[0, 2], [2, 1], [1, 1], [0, 8], [0], [0], [0], [0], [-1, 2], [3], [3, 4]]
    cu, path, count = [0], [], []
    for i, p in enumerate(paths):
        path += p + [-1] * (8 - len(p))
        cu.append(cu[-1] + 8)
        count.append(len(p))
    count[9], count[10] = 9, -2
    drafts.keep(c, rows, cu, path, count)
    assert c.lens.tolist() == [64, 70, 70, 70, 5, 70, 70, 70]
    asym.kv_keep(*state, i32(rows, dev), i32(cu, dev), i32(path, dev), i32(count, dev))
    same(c, state)
    # entries without a page, one pool, offsets that say too much
    state[2][1, 0, 2] = -1
    c.table[1, 0, 2] = -1
    c.pools = c.pools[:1]
    drafts.keep(c, [1], [0, 8], [1, 3, 5, 7], [4])
    asym.kv_keep(state[0], None, *state[2:], i32([1], dev), i32([-1, 8], dev), i32([1, 3, 5, 7, 0, 0, 0, 0], dev), i32([4], dev))
    same(c, [state[0], *state[2:]])


def test_keep_writes_to_no_page_of_another_row(dev):
    # row 3 has row 0's pages, drafted tokens and all, row 4 those of row 1 up to its last 32 tokens; row 2 shares what it does not write to
    c, state = cache(dev, [90, 96, 70, 0, 0, 0], 2, 4, 3)
    for to, of, pages in ((3, 0, 2), (4, 1, 2), (5, 2, 1)):
        c.table[to, :, :pages] = c.table[of, :, :pages]
        np.add.at(c.refs, c.table[to, :, :pages], 1)
        c.lens[to] = 32 * pages
    for x, y in zip(state[2:], (c.table, c.lens, c.refs)):
        x.copy_(torch.tensor(y))
    rows, cu, path, count = [0, 1, 2], [0, 40, 60, 80], [-1] * 80, [3, 2, 4]
    path[:3], path[40:42], path[60:64] = [0, 12, 39], [0, 19], [1, 5, 6, 19]
    before = [x.copy() for x in c.pools]
    drafts.keep(c, rows, cu, path, count)
    # (row 0: 50 tokens and 3 of 40, the moved ones in page 1, which is row 3's too; row 1: 76 and 2 of 20, in page 2; row 2: 50 and 4)
    assert c.lens.tolist() == [90, 78, 54, 64, 64, 32] and not np.array_equal(before[0], c.pools[0])
    asym.kv_keep(*state, i32(rows, dev), i32(cu, dev), i32(path, dev), i32(count, dev))
    same(c, state)


def test_keep_captured_and_on_another_stream(dev):
    c, state = cache(dev, [100, 60, 33], 4, 5, 2, 64)
    first = [x.clone() for x in state]
    args = [i32([2, 0, 1], dev), i32([0, 10, 30, 45], dev), i32([0, 3, 4] + [-1] * 7 + [0, 5] + [-1] * 18 + list(range(15)), dev), i32([3, 2, 15], dev)]
    drafts.keep(c, [2, 0, 1], args[1].tolist(), args[2].tolist(), [3, 2, 15])
    s = asym.stream_create()
    torch.cuda.synchronize()
    asym.kv_keep(*state, *args, stream=s)
    s.synchronize()
    same(c, state)
    asym.stream_destroy(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asym.kv_keep(*state, *args)
    for _ in range(3):
        for x, y in zip(state, first):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        same(c, state)


def test_keep_refusals(dev):
    _, s = cache(dev, [40], 1, 2, 0)
    args = [i32([0], dev), i32([0, 4], dev), i32([0, 1, 2, 3], dev), i32([2], dev)]
    for bad, kind in ((lambda: asym.kv_keep(s[0][:, :16], s[1], *s[2:], *args), ValueError), (lambda: asym.kv_keep(*s, args[0], args[0], *args[2:]), ValueError),
                      (lambda: asym.kv_keep(*s, *args[:3], args[1]), ValueError), (lambda: asym.kv_keep(*s, *args[:2], args[2].long(), args[3]), TypeError),
                      (lambda: asym.kv_keep(s[0], s[0], *s[2:], *args), asym.AsymError),
                      (lambda: asym.kv_keep(*[x[..., :3].contiguous() for x in s[:2]], *s[2:], *args), asym.AsymError)):
        with pytest.raises(kind):
            bad()


# -- a step as a program runs it -----------------------------------------------------------

def test_drafting_steps(dev):
    """Prompts appended, then steps of: a tree drafted, its tokens appended (turned by their depth), attended to, verified
    and kept.  The cache is compared with a dense one that only ever held the tokens that were kept."""
    H, Hq, R, pph, V = 2, 8, 3, 6, 64
    total = R * H * pph + 10
    g = torch.Generator().manual_seed(0)
    rng = np.random.default_rng(0)
    freq, amp = asym.rope_freq(128, scaling="parts", factor=4)
    freq = freq.to(dev)
    pools = [torch.zeros((total, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    table = torch.full((R, H, pph), -1, dtype=torch.int32, device=dev)
    lens, refs, status = i32([0] * R, dev), i32([0] * total, dev), i32([0, 0], dev)
    rows = i32(list(range(R)), dev)
    dense = [[], [], []]  # per row: (k unturned, v, position) of each token kept

    def qkv(T):
        x = torch.randn((T, Hq + 2 * H, 128), generator=g).to(torch.bfloat16).to(dev)
        return x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]

    n = [50, 31, 64]
    cu = offsets(n)
    q, k, v = qkv(cu[-1])
    asym.kv_extend(table, lens, refs, rows, i32(n, dev), status)
    asym.kv_append(k, v, *pools, table, table, i32(cu, dev), i32([0] * R, dev), freq=freq, amplitude=amp)
    for r in range(R):
        dense[r] = [(k[cu[r] + i], v[cu[r] + i], i) for i in range(n[r])]
    for step in range(4):
        sizes = [int(x) for x in rng.integers(3, 14, R)]
        cu = offsets(sizes)
        T = cu[-1]
        parents = [[-1] + [int(rng.integers(0, i)) for i in range(1, m)] for m in sizes]
        trees = [asym.draft_tree(p) for p in parents]
        mask = torch.cat([t[0] for t in trees]).to(dev)
        base = [len(d) for d in dense]
        assert lens.tolist() == base
        pos = sum([[b + d for d in t[1]] for b, t in zip(base, trees)], [])
        q, k, v = qkv(T)
        asym.kv_extend(table, lens, refs, rows, i32([b + m for b, m in zip(base, sizes)], dev), status)
        turned = asym.kv_append(k, v, *pools, table, table, i32(cu, dev), i32(base, dev), q=q, freq=freq, positions=i32(pos, dev), amplitude=amp)
        o = asym.attn_tree_paged(turned, *pools, table, table, i32(cu, dev), lens, mask=mask)
        # against attention over the tokens kept and the node's own branch, one node at a time
        for r in range(R):
            for i in (0, sizes[r] - 1):
                branch = []
                a = i
                while a >= 0:
                    branch.insert(0, a)
                    a = parents[r][a]
                own = [(k[cu[r] + j], v[cu[r] + j], base[r] + d) for d, j in enumerate(branch)]
                kk, vv, pp = zip(*(dense[r] + own))
                kd = asym.rope(torch.stack(kk), i32(list(pp), dev), freq, amplitude=amp)
                qd = asym.rope(q[cu[r] + i][None], i32([pp[-1]], dev), freq, amplitude=amp)
                R64, _, A, N = prompt.prompt_attention(f64(qd), f64(kd), f64(torch.stack(vv)), [0, 1], [0, len(kk)], 128 ** -0.5)
                bound = 2.0 ** -8 * (1 + 2.0 ** -8) * (A + np.abs(R64)) + A * (2.0 ** -23 * (264 * N + 16 + len(kk)))[..., None]
                assert np.all(np.abs(f64(o[cu[r] + i][None]) - R64) <= bound)
        z = torch.randn((T, V), generator=g) * 2
        target, draft = torch.softmax(z, 1).to(dev), torch.softmax(z + 0.5 * torch.randn((T, V), generator=g), 1).to(dev)
        tokens = i32(rng.integers(0, V, T), dev)
        path, count, token = asym.draft_verify(target, draft, tokens, i32(sum(parents, []), dev), i32(cu, dev),
                                               torch.rand(T, generator=g).to(dev) * 0.5, torch.rand(R, generator=g).to(dev))
        asym.kv_keep(*pools, table, lens, refs, rows, i32(cu, dev), path, count)
        for r in range(R):
            kept = path[cu[r]:cu[r] + int(count[r])].tolist()
            assert kept[0] == 0 and all(parents[r][b] == a for a, b in zip(kept, kept[1:]))
            dense[r] += [(k[cu[r] + j], v[cu[r] + j], base[r] + d) for d, j in enumerate(kept)]
        assert lens.tolist() == [len(d) for d in dense]
        assert int(refs.sum()) == int((table >= 0).sum()) == sum(-(-len(d) // 32) * H for d in dense)
    # what the cache holds is what was kept
    for r in range(R):
        kk, vv, pp = zip(*dense[r])
        kd = asym.rope(torch.stack(kk), i32(list(pp), dev), freq, amplitude=amp)
        for h in range(H):
            page = table[r, h].long()
            at = torch.arange(len(kk), device=dev)
            assert torch.equal(pools[0][page[at // 32], at % 32], kd[:, h])
            assert torch.equal(pools[1][page[at // 32], at % 32], torch.stack(vv)[:, h])
