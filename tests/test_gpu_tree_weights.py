"""GPU parity of the weights in the attention of drafted tokens: the output is rounded to bf16, the weights are not.

A weight enters the products as the sum of two bf16 values, which lose 2^-8 of 2^-8 of it.  So, with A = sum_j w_j |v_j| and
the fp32 steps' share as in the module beside (2^-23 * (264 N + 16 + keys) of A), an output computed as O' is within
E = A * (2^-16 + fp32) of the oracle's R, and its rounding within 2^-8 |O'| of O': 2^-8 |R| + (1 + 2^-8) E.
Weights of one bf16 value would be off by up to 2^-8 A.
"""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import drafts
from tests.test_gpu_tree import SCALE, Case, dev, f64, i32, many_rows  # noqa: F401

pytestmark = pytest.mark.gpu


def check(c, o, only=None):
    got, q = f64(o), f64(c.q)
    for b in range(len(c.new)) if only is None else only:
        rows = slice(c.cu[b], c.cu[b + 1])
        if not c.new[b]:
            continue
        k, v = c.dense(b)
        R, _, A, N = drafts.tree_attention(q[rows], k, v, c.sees[b], c.lens[b] - c.new[b], SCALE)
        E = A * (2.0 ** -16 + 2.0 ** -23 * (264 * N + 16 + c.lens[b]))[..., None]
        assert np.all(np.isfinite(got[rows]))
        worst = float(np.max(np.abs(got[rows] - R) / (2.0 ** -8 * np.abs(R) + (1 + 2.0 ** -8) * E + 1e-37)))
        assert worst <= 1, (b, worst)


# One token a request, trees in one block of rows and in two, whole segments, cut ones, forced shares (keys of a 16th, so that
# N, and with it the fp32 steps' share, is small)
@pytest.mark.parametrize("new,lens,Hq,H,room,split", [
    ([1], [300], 4, 1, 0, 0), ([1] * 20, [37 * i + 1 for i in range(20)], 8, 2, 0, 0), ([8], [777], 32, 8, 0, 0), ([8], [777], 32, 8, 2000, 0),
    ([5, 30], [90, 800], 8, 2, 0, 64), ([40, 64], [500, 900], 8, 2, 9000, 0), ([40, 64], [500, 900], 8, 2, 9000, 96)])
@pytest.mark.parametrize("tree", [True, False])
def test_weights_are_not_rounded_to_bf16(dev, new, lens, Hq, H, room, split, tree):
    c = Case(dev, new, lens, Hq, H, seed=sum(lens), tree=tree, room=room)
    c.kp /= 16
    check(c, c.run(split_tokens=split))


@pytest.mark.parametrize("split", [0, 96])
def test_weights_of_many_rows_are_not_rounded_to_bf16(dev, split):
    c = many_rows(dev, [70, 60], [800, 333], 8, 2, 5760)
    c.kp /= 16
    check(c, c.run(split_tokens=split))


def infinities(c, n0, G):
    """Infinities and NaN among values that every node sees, far enough before the nodes to lie in whole blocks: the channel that
    holds one has it in every row of the head's group, the rest is as it was."""
    ref = c.run()
    assert c.lens[0] - c.new[0] >= 256  # (two whole blocks or more)
    nan, inf = float("nan"), float("inf")
    for values in ([(3, inf)], [(70, -inf)], [(130, nan)], [(3, inf), (131, inf)], [(3, inf), (4, -inf)], [(64, -inf), (65, nan)]):
        v0 = c.vp.clone()
        for at, x in values:
            c.vp[int(c.vt[0, 1, at // 32]), at % 32, 77] = x
        got = c.run()
        hit = torch.zeros_like(ref, dtype=torch.bool)
        hit[:n0, G:2 * G, 77] = True
        assert torch.equal(got[~hit], ref[~hit])
        kinds = {x for _, x in values}
        if len(kinds) == 1 and values[0][1] == values[0][1]:
            assert torch.all(got[hit] == values[0][1])
        else:
            assert torch.all(torch.isnan(got[hit]))
        c.vp.copy_(v0)
    # a key that is NaN: everything of its head's group
    c.kp[int(c.kt[0, 0, 2]), 5, 9] = nan
    got = c.run()
    hit = torch.zeros_like(ref, dtype=torch.bool)
    hit[:n0, :G] = True
    assert torch.all(torch.isnan(got[hit])) and torch.equal(got[~hit], ref[~hit])


@pytest.mark.parametrize("n,G,room,split", [(1, 4, 0, 0), (5, 2, 0, 0), (8, 4, 2000, 0), (8, 4, 0, 64), (40, 4, 0, 0), (64, 4, 9000, 0)])
def test_infinities_that_are_seen(dev, n, G, room, split):
    c = Case(dev, [n, 3], [600, 40], 2 * G, 2, seed=n, room=room)
    if split:
        run = c.run
        c.run = lambda: run(split_tokens=split)
    infinities(c, n, G)


def test_infinities_that_are_seen_by_many_rows(dev):
    infinities(many_rows(dev, [130, 100], [700, 300], 4, 2, 11520), 130, 2)
