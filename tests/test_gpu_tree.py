"""GPU parity of the attention of drafted tokens over the 16-bit paged cache, through the C ABI.

Against the float64 oracle, element by element, over the values that the pages hold.  The bound is
prompt attention's, derived: probabilities rounded to bf16, 2^-8 A (A = sum_j w_j |v_j|), the output once
more, 2^-8 |O|; fp32 scores, exponentials and sums, A * 2^-23 * (264 N + 16 + keys); the weights and
additions by which pieces and waves are joined are fewer than the keys that this counts.
"""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import drafts
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


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def offsets(lens, first=0):
    return (np.cumsum([0] + list(lens)) + first).tolist()


class Case:
    """Requests of `new` nodes that are the last of `lens` tokens, in random pages, and tables with room for `room` more."""

    def __init__(self, dev, new, lens, Hq, H, seed=0, sigma=1.0, tree=True, pph=None, spare=3, room=0):
        self.new, self.lens, self.Hq, self.H, self.dev = new, lens, Hq, H, dev
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.pph = pph or max(1, -(-max(lens + [1]) // 32))
        n = len(new) * H * self.pph + spare
        mk = lambda *s: (torch.randn(s, generator=g) * sigma).to(torch.bfloat16).to(dev)
        self.kp, self.vp = mk(n, 32, 128), mk(n, 32, 128)
        self.kt, self.vt = (rng.permutation(n)[:len(new) * H * self.pph].reshape(len(new), H, self.pph).astype(np.int32) for _ in range(2))
        self.kt, self.vt = (np.pad(t, ((0, 0), (0, 0), (0, room)), constant_values=-1) for t in (self.kt, self.vt))
        self.cu = offsets(new)
        self.T = self.cu[-1]
        self.q = mk(max(self.T, 1), Hq, 128)[:self.T]
        words = max(1, -(-max(new + [1]) // 64))
        self.parents = [[-1] + [int(rng.integers(max(0, i - 4), i)) for i in range(1, m)] if m else [] for m in new]
        self.sees, masks = [], []
        for m, par in zip(new, self.parents):
            mask, _ = asym.draft_tree(par)
            masks.append(torch.nn.functional.pad(mask, (0, words - mask.shape[1])))
            if tree:
                self.sees.append([{j for j in range(m) if int(mask[i, j // 64]) >> (j % 64) & 1} for i in range(m)])
            else:
                self.sees.append([set(range(i + 1)) for i in range(m)])
        self.mask = torch.cat(masks).to(dev) if tree else None

    def run(self, **kw):
        args = dict(mask=self.mask, **kw)
        self.lse = torch.full((self.T, self.Hq), 3.0, device=self.dev)
        if kw.get("lse", 0) is None:
            self.lse = None
        else:
            args["lse"] = self.lse
        return asym.attn_tree_paged(self.q, self.kp, self.vp, i32(self.kt, self.dev), i32(self.vt, self.dev), i32(self.cu, self.dev),
                                    i32(self.lens, self.dev), **args)

    def dense(self, b):
        L = self.lens[b]
        take = lambda pool, t: f64(pool[torch.tensor(t[b, :, :self.pph].astype(np.int64)).to(self.dev)]).transpose(0, 1, 2, 3).reshape(
            self.H, -1, 128)[:, :L].transpose(1, 0, 2)
        return take(self.kp, self.kt), take(self.vp, self.vt)

    def check(self, o, scale=SCALE, only=None):
        got, gl = f64(o), self.lse.double().cpu().numpy()
        q = f64(self.q)
        for b in range(len(self.new)) if only is None else only:
            rows = slice(self.cu[b], self.cu[b + 1])
            if not self.new[b]:
                continue
            k, v = self.dense(b)
            R, Rl, A, N = drafts.tree_attention(q[rows], k, v, self.sees[b], self.lens[b] - self.new[b], scale)
            keys = max(self.lens[b], 1)
            eps32 = 2.0 ** -23 * (264 * N + 16 + keys)
            bound = 2.0 ** -8 * (1 + 2.0 ** -8) * (A + np.abs(R)) + A * eps32[..., None] + 1e-37
            assert np.all(np.isfinite(got[rows]))
            worst = float(np.max(np.abs(got[rows] - R) / bound))
            assert worst <= 1, (b, worst)
            some = Rl > -np.inf
            assert np.all(got[rows][~some] == 0) and np.all(gl[rows][~some] == -np.inf)
            assert np.all(np.abs(gl[rows][some] - Rl[some]) <= 2.0 ** -23 * (132 * N + 16 + keys + np.abs(Rl))[some])


CASES = [  # nodes, tokens with them, H_q, H_kv
    ([1], [1], 1, 1), ([1], [300], 4, 1), ([1], [32], 8, 8), ([1], [33], 8, 2), ([8], [777], 32, 8), ([3, 0, 7], [40, 5, 7], 6, 2),
    ([5, 3], [3, 65], 4, 2), ([2], [0], 4, 2), ([64], [64], 4, 1), ([65], [97], 2, 1), ([31, 33, 1], [64, 64, 1], 8, 4),
    ([129], [200], 3, 3), ([20], [31], 5, 1), ([1] * 70, [3] * 70, 8, 2), ([2] * 67, list(range(2, 136, 2)), 4, 1),
    ([17, 16, 15], [500, 16, 1000], 16, 1), ([40], [130], 35, 5), ([9] * 5, [9, 100, 33, 31, 32], 40, 8), ([1, 60, 4], [2000, 61, 3], 8, 2),
    ([200], [190], 4, 2), ([6] * 20, [200 + 37 * i for i in range(20)], 10, 2), ([1] * 3, [5000, 1, 3100], 1, 1)]


# A call with little room for its number of requests and heads gives every segment a workgroup of its own, one with more
# cuts them, and one with much more, if its requests have more than 40 rows in the mean, has 128 rows a workgroup and not 64.
ROOM = [0, 2000, 9000]


@pytest.mark.parametrize("new,lens,Hq,H", CASES)
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("room", ROOM)
def test_against_oracle(dev, new, lens, Hq, H, tree, room):
    c = Case(dev, new, lens, Hq, H, seed=sum(lens) + Hq, tree=tree, room=room)
    c.check(c.run())


def test_many_rows_of_a_segment_each(dev):
    c = Case(dev, [50] * 40, [50 + 6 * i for i in range(40)], 32, 8, seed=13, room=80)
    assert asym._tree_workspace(40, 32, 8, 2000, c.kt.shape[2] * 32, 0) == 0
    c.check(c.run(), only=[0, 1, 31, 39])


@pytest.mark.parametrize("B,room", [(300, 0), (4096, 0), (4500, 0), (300, 700), (4500, 300)])
def test_very_many_requests(dev, B, room):
    new = [i % 3 if i % 7 else 0 for i in range(B)]
    new[-1], new[B // 2] = 2, 40
    c = Case(dev, new, [max(n, 7 * i % 60) for i, n in enumerate(new)], 2, 1, seed=B, room=room)
    assert (asym._tree_workspace(B, 2, 1, c.T, c.kt.shape[2] * 32, 0) == 0) == (room == 0)
    o = torch.full_like(c.q, 7.0)
    c.check(c.run(o=o), only=[0, 1, 2, 63, 64, 65, B // 2 - 1, B // 2, B // 2 + 1, B - 2, B - 1] + list(range(3, B, B // 17)))
    assert not torch.any(torch.all(o.flatten(1) == 7, dim=1))  # every row is written


def test_which_calls_are_cut(dev):
    assert asym._tree_workspace(64, 32, 8, 64 * 32, 2000, 0) == 0 < asym._tree_workspace(8, 32, 8, 8 * 32, 2000, 0)
    assert asym._tree_workspace(1, 8, 1, 1, 384, 0) == 0 < asym._tree_workspace(1, 8, 1, 1, 385, 0)


@pytest.mark.parametrize("split", [32, 64, 96, 4096])
def test_shares_of_any_length(dev, split):
    c = Case(dev, [7, 1, 30], [900, 40, 333], 8, 2, seed=split)
    c.check(c.run(split_tokens=split))


# Sizes at which a workgroup has eight waves: more than 192 rows a request in the mean, and room in the tables for
# 180 x 256 pages of units, of which the lengths need not make use, and too much for a workgroup a segment.
MANY_ROWS = [([70, 0, 129, 60], [1000, 5, 700, 64], 8, 2, 2880), ([17, 16, 15, 33], [500, 16, 1000, 90], 16, 1, 5120),
             ([200, 257], [190, 600], 3, 3, 5120), ([300], [2100], 4, 1, 15360), ([50] * 70, [50 + 13 * i for i in range(70)], 8, 2, 190)]


def many_rows(dev, new, lens, Hq, H, room, **kw):
    c = Case(dev, new, lens, Hq, H, seed=sum(lens), room=room - max(1, -(-max(lens) // 32)), **kw)
    G = Hq // H
    assert c.kt.shape[2] == room and c.T * G > 192 * len(new) and (c.T * G // 256 + len(new)) * H * room >= 180 * 256
    assert asym._tree_workspace(len(new), Hq, H, c.T, room * 32, 0) > 0
    return c


@pytest.mark.parametrize("split", [0, 96])
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("new,lens,Hq,H,room", MANY_ROWS)
def test_many_rows_against_oracle(dev, new, lens, Hq, H, room, tree, split):
    c = many_rows(dev, new, lens, Hq, H, room, tree=tree)
    c.check(c.run(split_tokens=split), only=[b for b in range(len(new)) if b < 2 or b % 31 < 2 or b == len(new) - 1])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_many_rows_do_not_see_what_they_should_not(dev, bad):
    n, lens = 130, [475, 300]
    c = many_rows(dev, [n, 100], lens, 4, 2, 11520)
    ref = c.run()
    k0, v0 = c.kp.clone(), c.vp.clone()
    for b in range(2):
        for h in range(2):
            for pool, t in ((c.kp, c.kt), (c.vp, c.vt)):
                pool[int(t[b, h, lens[b] // 32]), lens[b] % 32:] = bad
    assert torch.equal(c.run(), ref)
    c.kp.copy_(k0)
    j = 5
    at = 475 - n + j
    c.vp[int(c.vt[0, 1, at // 32]), at % 32, 100] = bad
    got = c.run()
    hit = torch.zeros_like(ref, dtype=torch.bool)
    for i in range(n):
        if j in c.sees[0][i]:
            hit[i, 2:, 100] = True
    assert hit.any() and torch.equal(got[~hit], ref[~hit])
    assert torch.all(torch.isnan(got[hit]) if bad != bad else got[hit] == bad)
    c.vp.copy_(v0)


def test_many_rows_captured_and_replayed(dev):
    c = many_rows(dev, [70, 60], [800, 333], 8, 2, 5760)
    args = [c.kp, c.vp, i32(c.kt, dev), i32(c.vt, dev), i32(c.cu, dev), i32(c.lens, dev)]
    eager = lambda q, lens: asym.attn_tree_paged(q, *args[:5], lens, mask=c.mask)
    held, lens, o = c.q.clone(), args[5].clone(), torch.empty_like(c.q)
    eager(held, lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asym.attn_tree_paged(held, *args[:5], lens, mask=c.mask, o=o)
    for s, new in ((1, [800, 333]), (-1, [700, 60]), (2, [71, 320])):
        held.copy_(c.q * s), lens.copy_(i32(new, dev))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager(c.q * s, i32(new, dev)))


@pytest.mark.parametrize("G", [1, 5])
def test_rows_of_very_many_pieces(dev, G):
    # (joined by a workgroup each)
    c = Case(dev, [2], [9000], G, 1, seed=12)
    c.check(c.run(split_tokens=32))
    c.check(c.run())


@pytest.mark.parametrize("B", [3, 130])
@pytest.mark.parametrize("split", [0, 32])
@pytest.mark.parametrize("room", ROOM)
def test_offsets_that_fall_write_nothing(dev, B, split, room):
    c = Case(dev, [4] * B, [70] * B, 4, 2, seed=B, room=room)
    ref = c.run(split_tokens=split)
    good, c.cu = c.cu, list(c.cu)
    c.cu[-2] = c.cu[-3] - 1
    o = torch.full_like(c.q, 7.0)
    c.run(o=o, split_tokens=split)
    assert torch.all(o == 7) and torch.all(c.lse == 3)
    c.cu = good
    assert torch.equal(c.run(split_tokens=split), ref)


@pytest.mark.parametrize("scale,sigma", [(0.0, 1.0), (-0.11, 1.0), (3.0, 1.0), (SCALE, 8.0), (1e-30, 1.0)])
def test_scales(dev, scale, sigma):
    c = Case(dev, [9, 2], [70, 300], 6, 2, seed=5, sigma=sigma)
    c.check(c.run(scale=scale), scale)


@pytest.mark.parametrize("room", ROOM)
def test_masks_that_are_not_trees(dev, room):
    # any bits: nodes that see later ones, only others, or nothing (behind no token at all)
    c = Case(dev, [70, 40], [70, 41], 4, 2, seed=3, room=room)
    bits = torch.rand((110, 128), generator=torch.Generator().manual_seed(1)) < 0.4
    bits[5] = bits[64] = bits[80] = False
    c.sees = [[{j for j in range(128) if bits[i, j]} for i in range(70)], [{j for j in range(128) if bits[70 + i, j]} for i in range(40)]]
    weight = torch.ones(64, dtype=torch.int64) << torch.arange(64)
    c.mask = (bits.view(110, 2, 64) * weight).sum(-1).to(dev)
    o = c.run()
    c.check(o)
    assert torch.all(o[5] == 0) and torch.all(o[64] == 0) and torch.all(c.lse[5] == -float("inf"))
    # nodes behind the mask's words are not seen
    c.mask = c.mask[:, :1].contiguous()
    c.sees = [[{j for j in s if j < 64} for s in x] for x in c.sees]
    c.check(c.run())


def test_split_and_unsplit_agree_with_prompt_attention(dev):
    # a chain behind a prefix is what prompt attention computes on the dense keys
    c = Case(dev, [33, 5], [400, 900], 8, 2, seed=8, tree=False)
    o = c.run()
    k, v = (torch.cat([torch.tensor(c.dense(b)[x]).to(torch.bfloat16) for b in range(2)]).to(dev) for x in (0, 1))
    p = asym.attn_prefill(c.q, k, v, i32(c.cu, dev), i32([0, 400, 1300], dev))
    # both are within the module's bound of the same values: twice its bf16 part, 2 * 2^-8 (A + |O|), A and O below 4 here
    assert float((o.float() - p.float()).abs().max()) <= 2 * 2.0 ** -8 * 8


@pytest.mark.parametrize("room", ROOM)
def test_strides_and_rows_outside(dev, room):
    c = Case(dev, [6, 0, 9], [50, 3, 100], 8, 2, seed=9, room=room)
    ref, lse = c.run(), c.lse
    wide = torch.full((c.T + 7, 14, 128), float("nan"), dtype=torch.bfloat16, device=dev)
    wide[4:4 + c.T, 3:11] = c.q
    mask = torch.zeros((c.T + 7, 1), dtype=torch.int64, device=dev)
    mask[4:4 + c.T] = c.mask
    o, l2 = torch.full((c.T + 7, 8, 128), 7.0, dtype=torch.bfloat16, device=dev), torch.full((c.T + 7, 8), 7.0, device=dev)
    asym.attn_tree_paged(wide[:, 3:11], c.kp, c.vp, i32(c.kt, dev), i32(c.vt, dev), i32(offsets(c.new, 4), dev), i32(c.lens, dev),
                         mask=mask, o=o, lse=l2)
    assert torch.equal(o[4:4 + c.T], ref) and torch.equal(l2[4:4 + c.T], lse)
    assert torch.all(o[:4] == 7) and torch.all(o[4 + c.T:] == 7) and torch.all(l2[:4] == 7) and torch.all(l2[4 + c.T:] == 7)


@pytest.mark.parametrize("G,n", [(1, 3), (4, 12), (4, 40)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("room", ROOM)
def test_what_a_node_does_not_see_cannot_reach_it(dev, G, n, bad, room):
    c = Case(dev, [n, 2], [75, 40], 2 * G, 2, seed=n + G, room=room)
    ref = c.run()
    # behind the requests' tokens, in other pages, and in no node's sight
    k0, v0 = c.kp.clone(), c.vp.clone()
    for b in range(2):
        L = c.lens[b]
        for h in range(2):
            for pool, t in ((c.kp, c.kt), (c.vp, c.vt)):
                page = int(t[b, h, L // 32]) if L // 32 < c.pph else -1
                if page >= 0:
                    pool[page, L % 32:] = bad
                for extra in range(L // 32 + 1, c.pph):
                    pool[int(t[b, h, extra])] = bad
    assert torch.equal(c.run(), ref)
    # a node's own value: only those that see it
    c.kp.copy_(k0), c.vp.copy_(v0)
    j = n - 2
    at = 75 - n + j
    c.vp[int(c.vt[0, 1, at // 32]), at % 32, 17] = bad
    got = c.run()
    hit = torch.zeros_like(ref, dtype=torch.bool)
    for i in range(n):
        if j in c.sees[0][i]:
            hit[i, G:, 17] = True
    assert hit.any() and torch.equal(got[~hit], ref[~hit])
    assert torch.all(torch.isnan(got[hit]) if bad != bad else got[hit] == bad)
    # a node's own key
    c.vp.copy_(v0)
    c.kp[int(c.kt[0, 0, at // 32]), at % 32, 5] = float("nan")
    got = c.run()
    hit.zero_()
    for i in range(n):
        if j in c.sees[0][i]:
            hit[i, :G] = True
    assert torch.equal(got[~hit], ref[~hit]) and torch.all(torch.isnan(got[hit]))


def test_scores_of_the_lowest_value(dev):
    # every score the type's lowest value, or an infinity below every other
    c = Case(dev, [2], [40], 1, 1, seed=1)
    lowest = torch.finfo(torch.bfloat16).min
    c.q.zero_()
    c.q[:, 0, 0] = 1
    c.kp.zero_()
    c.kp[..., 0] = lowest
    o = c.run(scale=1.0)
    c.check(o, 1.0)
    c.kp[int(c.kt[0, 0, 0]), 3, 0] = -float("inf")  # weight 0
    k, v = c.dense(0)
    keep = [t for t in range(40) if t != 3]
    got = f64(c.run(scale=1.0))
    want = [v[[t for t in keep if t < 38 or t - 38 in c.sees[0][i]], 0].mean(0) for i in range(2)]
    assert np.all(np.abs(got[:, 0] - np.array(want)) <= 2.0 ** -7 * 4)


@pytest.mark.parametrize("room", ROOM)
def test_entries_outside_the_pool_read_zeros(dev, room):
    c = Case(dev, [4], [100], 4, 1, seed=2, room=room)
    c.kp[int(c.kt[0, 0, 1])] = 0
    c.vp[int(c.vt[0, 0, 2])] = 0
    ref = c.run()
    c.kt[0, 0, 1], c.vt[0, 0, 2] = -1, c.kp.shape[0]
    assert torch.equal(c.run(), ref)


def test_lengths_that_say_too_much_are_held(dev):
    c = Case(dev, [3, 2], [64, 64], 4, 2, seed=4)
    ref = c.run()
    c.lens = [100000, 2 ** 31 - 1]
    assert torch.equal(c.run(S=64), ref)
    c.lens, c.cu = [64, 64], [-3, 3, 1000]
    assert torch.equal(c.run(), ref)
    c.lens, c.cu = [-5, 64], [0, 3, 5]
    o = c.run()
    assert torch.all(o[:3] == 0) and torch.equal(o[3:], ref[3:])


def test_long_context_sampled(dev):
    new, lens = [24, 1, 64], [20000, 33000, 12345]
    c = Case(dev, new, lens, 32, 8, seed=6)
    c.check(c.run(), only=[1])
    # of the others some rows
    o = c.run()
    for b, keep in ((0, [0, 11, 23]), (2, [0, 40, 63])):
        k, v = c.dense(b)
        q = f64(c.q[c.cu[b]:c.cu[b + 1]])[keep]
        R, _, A, N = drafts.tree_attention(q, k, v, [c.sees[b][i] for i in keep], lens[b] - new[b], SCALE)
        eps32 = 2.0 ** -23 * (264 * N + 16 + lens[b])
        got = f64(o[c.cu[b]:c.cu[b + 1]])[keep]
        assert np.all(np.abs(got - R) <= 2.0 ** -8 * (1 + 2.0 ** -8) * (A + np.abs(R)) + A * eps32[..., None])


def test_pages_past_4_gib(dev):
    n = (1 << 19) + 10
    c = Case(dev, [3], [40], 4, 1, seed=7)
    ref = c.run()
    big = [torch.empty((n, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    table = np.array([[[n - 1, n - 5]]], np.int32)
    for pool, old, t in ((big[0], c.kp, c.kt), (big[1], c.vp, c.vt)):
        for i in range(2):
            pool[int(table[0, 0, i])] = old[int(t[0, 0, i])]
    c.kp, c.vp = big
    c.kt = c.vt = table
    assert torch.equal(c.run(), ref)


@pytest.mark.parametrize("room", ROOM)
def test_streams_and_runs_give_the_same_bits(dev, room):
    c = Case(dev, [12, 3, 1] + ([2] * 300 if not room else []), [800, 333, 2100] + ([9] * 300 if not room else []), 8, 2, seed=10, room=room)
    ref = c.run()
    torch.cuda.synchronize()
    s = asym.stream_create()
    args = (c.kp, c.vp, i32(c.kt, dev), i32(c.vt, dev), i32(c.cu, dev), i32(c.lens, dev))
    torch.cuda.synchronize()
    outs = [asym.attn_tree_paged(c.q, *args, mask=c.mask, stream=s) for _ in range(3)]
    here = [asym.attn_tree_paged(c.q, *args, mask=c.mask) for _ in range(3)]
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs + here)
    asym.stream_destroy(s)


@pytest.mark.parametrize("lens,other", [([800, 333], [700, 40]), ([200, 133], [100, 0])])
def test_captured_and_replayed(dev, lens, other):
    c = Case(dev, [12, 3], lens, 8, 2, seed=11)
    args = [c.kp, c.vp, i32(c.kt, dev), i32(c.vt, dev), i32(c.cu, dev), i32(c.lens, dev)]
    eager = lambda q, lens: asym.attn_tree_paged(q, *args[:5], lens, mask=c.mask)
    held, lens, o = c.q.clone(), args[5].clone(), torch.empty_like(c.q)
    o2 = torch.empty_like(c.q)
    eager(held, lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asym.attn_tree_paged(held, *args[:5], lens, mask=c.mask, o=o)
        asym.attn_tree_paged(-held, *args[:5], lens, mask=c.mask, o=o2)
    for s, new in ((1, c.lens), (-1, other), (2, [12, 3])):
        held.copy_(c.q * s), lens.copy_(i32(new, dev))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager(c.q * s, i32(new, dev))) and torch.equal(o2, eager(c.q * -s, i32(new, dev)))


def test_refusals(dev):
    c = Case(dev, [3], [40], 4, 2, seed=0)
    args = dict(q=c.q, k_pool=c.kp, v_pool=c.vp, k_pages=i32(c.kt, dev), v_pages=i32(c.vt, dev), cu=i32(c.cu, dev), lens=i32(c.lens, dev),
                mask=c.mask)
    for change, kind in ((dict(q=c.q.float()), TypeError), (dict(q=c.q[..., ::2]), ValueError), (dict(k_pool=c.kp.float()), TypeError),
                         (dict(v_pool=c.vp[:-1]), ValueError), (dict(k_pages=i32(c.kt, dev).long()), TypeError),
                         (dict(v_pages=i32(c.vt, dev)[:, :1]), ValueError), (dict(cu=i32([0, 1, 3], dev)), ValueError),
                         (dict(lens=i32([4, 4], dev)), ValueError), (dict(mask=c.mask.int()), TypeError), (dict(mask=c.mask[:2]), ValueError),
                         (dict(mask=c.mask.cpu()), ValueError), (dict(S=65), asym.AsymError), (dict(S=0), asym.AsymError),
                         (dict(q=c.q[:, :3]), asym.AsymError), (dict(scale=float("inf")), asym.AsymError),
                         (dict(split_tokens=40), asym.AsymError), (dict(o=torch.empty((3, 4, 128), device=dev)), ValueError)):
        with pytest.raises(kind):
            asym.attn_tree_paged(**{**args, **change})
