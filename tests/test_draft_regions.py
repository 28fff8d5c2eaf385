"""Verification of drafted tokens in the oracle, on the CPU: the exact distribution of what it gives, and how far the random numbers of the
GPU tests keep from its borders."""
import numpy as np
import pytest
import torch

from oracle import drafts
from tests.test_gpu_drafts import Drafts


def upper(f):
    """The share of [0, 1) in which f holds, which holds below some number and not above it (bisection to 2^-53)."""
    lo, hi = 0.0, 1.0
    for _ in range(54):
        mid = (lo + hi) / 2
        lo, hi = (mid, hi) if f(mid) else (lo, mid)
    return lo if not f(lo) else hi


P = [0.1, 0.2, 0.3, 0.4]


@pytest.mark.parametrize("p,q", [(P, P[::-1]), (P, P), (P, [0.25] * 4), ([0.5, 0, 0.5, 0], [0.1, 0.4, 0.2, 0.3]), ([0.97, 0.01, 0.01, 0.01], [0.01, 0.97, 0.01, 0.01])])
@pytest.mark.parametrize("siblings", [1, 2, 3])
def test_the_first_token_has_the_targets_distribution(p, q, siblings):
    """Siblings drawn from q behind the root: the probability of the first token behind it, kept or drawn, summed over the regions of
    all random numbers (each a product of intervals, whose ends are found by bisection), is the target's."""
    n = siblings + 1
    target, draft = np.array([p] * n), np.array([q] * n)
    seen = np.zeros(4)
    for drawn in np.ndindex(*[4] * siblings):
        weight = float(np.prod([q[t] for t in drawn]))
        if weight == 0:
            continue
        run = lambda u, last: drafts.verify(target, draft, [0, *drawn], [-1] + [0] * siblings, [0.0, *u], last, margin=0)
        u = [1.0] * siblings  # (1: never below)
        for i, t in enumerate(drawn):
            a = upper(lambda x: run(u[:i] + [x] + u[i + 1:], 0.5)[0] == [0, i + 1])
            seen[t] += weight * a
            weight *= 1 - a
            if weight == 0:
                break
        below = 0.0
        for t in range(4):  # the last token's intervals, in order
            end = upper(lambda x: run(u, x)[1] <= t) if t < 3 else 1.0
            seen[t] += weight * (end - below)
            below = end
    # at most 4^3 draws of 7 ends each, of 2^-52, and as many roundings
    assert np.all(np.abs(seen - p) <= 64 * 7 * 2.0 ** -51)


def test_a_number_beside_a_border_is_told():
    p, q = np.array([[0.5, 0.3, 0.2], [0.2, 0.3, 0.5]]), np.array([[0.2, 0.6, 0.2], [1.0, 0, 0]])
    run = lambda u, last: drafts.verify(p, q, [0, 1], [-1, 0], [0, u], last)
    assert run(0.49, 0.1)[0] == [0, 1] and run(0.51, 0.1)[0] == [0]
    for u, last in ((0.5 + 1e-13, 0.1), (0.49, 0.5 - 1e-13), (0.49, 0.2 + 1e-14)):
        with pytest.raises(drafts.Border):
            run(u, last)
    with pytest.raises(drafts.Border):
        drafts.verify(p, None, [0, 1], [-1, 0], [0, 0.3 - 1e-14], 0.1)


def test_random_numbers_of_the_gpu_tests_keep_from_borders():
    # (the oracle raises Border otherwise; the same inputs as there)
    for dtype in (torch.float32, torch.bfloat16):
        for chain in (True, False):
            for new, V in [([2, 0, 5], 100), ([8, 1, 3], 2047), ([5, 9, 2, 7], 8193), ([70, 3], 1000), ([140], 64), ([3] * 70, 333), ([9] * 5, 40000)]:
                d = Drafts(new, V, seed=sum(new) + V, dtype=dtype, chain=chain)
                d.want(), d.want(False)
    for seed in range(12):
        d = Drafts([24, 17, 40, 2], [50, 500, 3000, 10000][seed % 4], seed=seed, noise=3.0, peak=1.0 + seed % 3, width=12)
        d.want(), d.want(False)
