"""GPU parity of the attention of drafted tokens where a workgroup's segments are long, in every form of it: page numbers are held 64
blocks (of two pages) at a time and handed on, and caches of 256 MiB and more are read non-temporally.

Some rows of each request against the float64 oracle, within the bound of the weights' tests: E = A * (2^-16 + 2^-23 * (264 N + 16 +
keys)) before the output's rounding, 2^-8 |R| + (1 + 2^-8) E behind it.
"""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import drafts
from tests.test_gpu_tree import SCALE, dev, f64, i32, offsets  # noqa: F401

pytestmark = pytest.mark.gpu


class Long:
    """Requests of `new` nodes, the last of `lens` tokens, in random pages of pools made on the GPU; tables of `pages` columns."""

    def __init__(self, dev, new, lens, Hq, H, seed, tree=True, pages=0):
        self.new, self.lens, self.Hq, self.H, self.dev = new, lens, Hq, H, dev
        g = torch.Generator(device=dev).manual_seed(seed)
        rng = np.random.default_rng(seed)
        have = -(-max(lens) // 32)
        self.pages = max(pages, have)
        n = len(new) * H * have + 3
        self.kp, self.vp = (torch.empty((n, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2))
        for pool, sigma in ((self.kp, 0.25), (self.vp, 1.0)):
            for a in range(0, n, 1 << 14):
                part = pool[a:a + (1 << 14)]
                part.copy_(torch.randn(part.shape, generator=g, device=dev) * sigma)
        self.kt, self.vt = (rng.permutation(n)[:len(new) * H * have].reshape(len(new), H, have).astype(np.int32) for _ in range(2))
        self.cu = offsets(new)
        self.T = self.cu[-1]
        self.q = torch.randn((self.T, Hq, 128), generator=g, device=dev).to(torch.bfloat16)
        words = max(1, -(-max(new) // 64))
        self.sees, masks = [], []
        for m in new:
            mask, _ = asym.draft_tree([-1] + [int(rng.integers(max(0, i - 4), i)) for i in range(1, m)])
            masks.append(torch.nn.functional.pad(mask, (0, words - mask.shape[1])))
            self.sees.append([{j for j in range(m) if not tree and j <= i or tree and int(mask[i, j // 64]) >> (j % 64) & 1} for i in range(m)])
        self.mask = torch.cat(masks).to(dev) if tree else None

    def kv_bytes(self):
        """What the pools hold, at least what the tables could name of them (see the plan's rule of 256 MiB)."""
        return min(2 * len(self.new) * self.H * self.pages, 2 * self.kp.shape[0]) * 8192

    def run(self, split=0):
        wide = [i32(np.pad(t, ((0, 0), (0, 0), (0, self.pages - t.shape[2])), constant_values=-1), self.dev) for t in (self.kt, self.vt)]
        self.lse = torch.empty((self.T, self.Hq), device=self.dev)
        return asym.attn_tree_paged(self.q, self.kp, self.vp, *wide, i32(self.cu, self.dev), i32(self.lens, self.dev), mask=self.mask, lse=self.lse,
                                    split_tokens=split)

    def check(self, o, requests=None, heads=None):
        G = self.Hq // self.H
        for b in range(len(self.new)) if requests is None else requests:
            L, n = self.lens[b], self.new[b]
            nodes = sorted({0, n // 2, n - 1})
            for h in range(self.H) if heads is None else heads:
                mine = slice(h * G, (h + 1) * G)
                k, v = (f64(pool[torch.tensor(t[b, h, :-(-L // 32)].astype(np.int64), device=self.dev)]).reshape(-1, 1, 128)[:L]
                        for pool, t in ((self.kp, self.kt), (self.vp, self.vt)))
                at = [self.cu[b] + i for i in nodes]
                R, Rl, A, N = drafts.tree_attention(f64(self.q[at][:, mine]), k, v, [self.sees[b][i] for i in nodes], L - n, SCALE)
                eps32 = 2.0 ** -23 * (264 * N + 16 + L)
                E = A * (2.0 ** -16 + eps32)[..., None]
                worst = float(np.max(np.abs(f64(o[at][:, mine]) - R) / (2.0 ** -8 * np.abs(R) + (1 + 2.0 ** -8) * E)))
                assert worst <= 1, (b, h, worst)
                lse = self.lse[at][:, mine].double().cpu().numpy()
                assert np.all(np.abs(lse - Rl) <= 2.0 ** -23 * (132 * N + 16 + L + np.abs(Rl)))


# A request's rows and what its tables have room for decide the form: one block of rows a wave, two, eight waves
FORMS = {"one": (3, 4, 0), "two": (50, 1, 17000), "eight": (200, 1, 46080)}


def form(name, dev, L, seed, tree=True, more=()):
    n, G, pages = FORMS[name]
    c = Long(dev, [n] * (1 + len(more)), [L, *more], G, 1, seed, tree, pages)
    mean, wide = n * G, (n * G // 128 + 1) * c.pages
    assert name == ("one" if mean <= 40 else "eight" if mean > 192 and (n * G // 256 + 1) * c.pages >= 180 * 256 else "two" if wide > 16384 else "")
    return c


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("base", [63 * 64, 64 * 64 - 1, 64 * 64, 64 * 64 + 33, 65 * 64, 66 * 64 + 7, 127 * 64 + 63, 128 * 64, 129 * 64 + 31])
def test_whole_blocks_end_beside_a_change_of_page_numbers(dev, base, name, tree):
    c = form(name, dev, base + FORMS[name][0], base, tree)
    c.check(c.run(split=16384))


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("split", [4064, 4096, 4128, 8192, 16384])
def test_long_shares(dev, name, split):
    c = form(name, dev, 20011, split, more=[9001, 300])
    c.check(c.run(split=split))


@pytest.mark.parametrize("new,lens,Hq,pages,heads", [
    ([1] * 64, [129 * 32 - 37 * i for i in range(64)], 32, 129, [0, 7]),          # whole segments, one block of rows, past 64 blocks
    ([4] * 16, [8192 - 300 * i for i in range(16)], 32, 256, [3]),                # cut, one block of rows
    ([48] * 64, [4000 - 50 * i for i in range(64)], 32, 125, [1]),                # whole segments, two blocks
    ([24] * 32, [8000 - 200 * i for i in range(32)], 32, 250, [5]),               # cut, two blocks
    ([70, 60], [70000, 66001], 32, 2188, [0, 6])])                                # eight waves, over 128 pages a share
def test_caches_that_are_read_non_temporally(dev, new, lens, Hq, pages, heads):
    c = Long(dev, new, lens, Hq, 8, seed=len(new), pages=pages)
    assert c.kv_bytes() >= 256 << 20
    whole = asym._tree_workspace(len(new), Hq, 8, c.T, pages * 32, 0) == 0
    assert whole == (len(new) == 64)
    c.check(c.run(), requests=sorted({0, 1, len(new) - 1}), heads=heads)
    if not whole:
        c.check(c.run(split=8192), requests=[0], heads=heads)
