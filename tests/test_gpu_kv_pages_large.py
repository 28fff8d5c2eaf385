"""Page operations in pools of more than 16384 pages and in calls of more than 1024 requests,
which take the launches of many workgroups (a smaller call is one workgroup's): whole
numbers, equal to the oracle's.  The pool is counted in segments of 4096 pages."""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from tests.test_gpu_kv_fp4 import i32
from tests.test_gpu_kv_pages import Pair, dev  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

SEG, SMALL_PAGES, SMALL_REQUESTS = 4096, 16384, 1024


def scatter(p, g, rows, most, first=()):
    """Gives rows of random lengths pages from all over the pool, `first` of them first."""
    free = g.permutation(np.flatnonzero(p.o.refs == 0))
    free = np.concatenate([np.array(first, int), free[~np.isin(free, first)]])
    at = 0
    for r in rows:
        n = int(g.integers(1, most + 1))
        for h in range(p.o.H):
            for c in range(-(-n // 32)):
                p.o.table[r, h, c], p.o.refs[free[at]] = free[at], 1
                at += 1
        p.o.lens[r] = n
    p.put()


def borders(pool):
    return [x for s in range(0, pool + 1, SEG) for x in (s - 1, s) if 0 <= x < pool] + [pool - 1]


@pytest.mark.parametrize("seed,pool,R,H,pph,pools,words", [
    (0, 20001, 60, 4, 20, 2, 8), (1, SMALL_PAGES + 1, 40, 8, 9, 1, 8), (2, 24576, 50, 3, 30, 2, 544), (3, 41000, 1100, 2, 6, 2, 4)])
def test_a_long_run(dev, seed, pool, R, H, pph, pools, words):
    g = np.random.default_rng(seed)
    p = Pair(dev, R, H, pph, pool, words=words, pools=pools, seed=seed)
    scatter(p, g, range(0, R, 2), 32 * pph, first=sorted(set(borders(pool)))[::2])
    for _ in range(4):
        n = int(g.integers(R // 2, R))
        rows = g.permutation(R)[:n].tolist()
        p.extend(rows, [int(p.o.lens[r]) + int(g.integers(0, 40)) for r in rows])
        p.fork(g.integers(0, R, n).tolist(), g.permutation(R)[:n].tolist())
        p.free(g.permutation(R)[:max(1, n // 3)].tolist())
        p.compact()
    p.compact()                                # nothing left to move
    p.extend([], [])
    p.fork([], [])


@pytest.mark.parametrize("pool", [3000, 17000])  # (the requests alone make a call large, and with the pool)
def test_many_requests(dev, pool):
    R = 1400
    g = np.random.default_rng(pool)
    p = Pair(dev, R, 1, 3, pool, seed=6)
    assert R > SMALL_REQUESTS
    rows = g.permutation(R).tolist()
    p.extend(rows, [int(x) for x in g.integers(0, 40, R)])  # (some need nothing)
    # rows twice, far apart and side by side, outside the table, shorter, beyond the table
    rows = g.integers(-3, R + 3, 1500).tolist() + [5, 5, 9, 5]
    p.extend(rows, [int(x) for x in g.integers(0, 100, len(rows))])
    src, dst = g.integers(-2, R + 2, 1300).tolist(), g.integers(-2, R + 2, 1300).tolist()
    src[7], dst[7] = 11, 11                    # onto itself, before another request for it
    dst[1200] = 11
    p.fork(src, dst)
    p.fork(list(range(R)), list(range(1, R)) + [0])  # every row moves on by one
    p.free(g.integers(-2, R + 2, 1300).tolist())
    p.compact()


def test_too_few_pages(dev):
    pool = SMALL_PAGES + 3000
    p = Pair(dev, 90, 8, 80, pool, words=4, seed=8)
    p.extend(list(range(30)), [2500] * 30)     # 30 * 8 * 79 pages: 424 are left
    p.extend(list(range(30, 40)), [2500] * 10)
    assert p.status.tolist() == [0, 10 * 8 * 79 - 424]
    p.fork([0] * 10, list(range(30, 40)))      # a part page for each of 8 heads
    p.extend([0, 1, 2], [2560] * 3)
    p.fork([5] * 42, list(range(40, 82)))      # 320 are left
    assert p.status.tolist() == [0, 16]
    p.fork([5] * 40, list(range(40, 80)))      # and all of them taken
    assert p.status.tolist() == [320, 0] and p.o.refs.min() == 1
    p.extend([85], [1])
    assert p.status.tolist() == [0, 8]
    p.extend([79], [2510])                     # (needs no page)
    p.fork([2], [85])                          # (none either)
    p.free([5, 41])
    p.extend([85, 3], [2560, 2560])
    p.compact()


def test_empty_and_full_pools(dev):
    pool = 5 * SEG
    p = Pair(dev, 4, 1, pool, pool, words=4, seed=9)
    p.compact()                                # no page in use
    assert p.status.tolist() == [0, 0]
    p.extend([2], [32 * pool])                 # all of them, in order
    p.compact()
    assert p.status.tolist() == [0, pool]
    p.extend([0], [1])
    assert p.status.tolist() == [0, 1]
    p.fork([2], [1])                           # whole pages: none is taken
    p.free([2, 1])
    p.extend([3, 0], [32 * (pool - 1), 32])
    p.free([3])                                # the last page alone is left: into the first
    p.compact()
    assert p.status.tolist() == [1, 1] and p.o.table[0, 0, 0] == 0


def test_more_segments_than_a_workgroup_has_threads(dev):
    pool = 257 * SEG + 5
    g = np.random.default_rng(10)
    p = Pair(dev, 30, 2, 40, pool, words=4, seed=10)
    scatter(p, g, range(0, 30, 2), 1200, first=[0, pool - 1, pool - 5, pool - 6, 256 * SEG, 256 * SEG - 1, SEG])
    p.extend(list(range(30)), [1280] * 30)
    p.fork([0, 2, 4], [1, 3, 5])
    p.free(list(range(0, 30, 3)))
    p.compact()
    p.extend([0, 3, 6], [700, 800, 900])


def test_captured(dev):
    pool = 18000
    p = Pair(dev, 60, 4, 10, pool, seed=11)
    g = np.random.default_rng(11)
    scatter(p, g, range(0, 30), 320)
    start = [t.clone() for t in (p.table, p.lens, p.refs, *p.pools)]
    src, dst = i32(list(range(20)), dev), i32(list(range(30, 50)), dev)
    rows, lens, ended = i32(list(range(60)), dev), i32([320] * 60, dev), i32([1, 2, 40], dev)

    def step():
        asym.kv_fork(*p.pools, p.table, p.lens, p.refs, src, dst, p.status)
        asym.kv_extend(p.table, p.lens, p.refs, rows, lens, p.status)
        asym.kv_free(p.table, p.lens, p.refs, ended)
        asym.kv_compact(*p.pools, p.table, p.lens, p.refs, p.status)

    def reset():
        for t, x in zip((p.table, p.lens, p.refs, *p.pools), start):
            t.copy_(x)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3):
        g = np.random.default_rng(seed)
        reset()
        src.copy_(i32(g.integers(0, 60, 20).tolist(), dev)), dst.copy_(i32(g.permutation(60)[:20].tolist(), dev))
        lens.copy_(i32(g.integers(0, 321, 60).tolist(), dev))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (p.table, p.lens, p.refs, *p.pools)]
        reset()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (p.table, p.lens, p.refs, *p.pools)):
            assert torch.equal(a, b)
