"""GPU parity of a paged cache's page operations (whole numbers: equal to the oracle's), and the
serving loop that they make with prompt attention and the 4-bit cache, through the C ABI."""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import kv_pages
from tests.test_gpu_kv_fp4 import attend, bf16_bits_to_f64, bits, i32, offsets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    asym.load_library()
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


class Pair:
    """A cache on the GPU and the oracle's."""

    def __init__(self, dev, R, H, pph, pool, words=8, pools=2, seed=0):
        g = np.random.default_rng(seed)
        self.dev = dev
        data = [g.integers(0, 1 << 30, (pool, words)).astype(np.int32) for _ in range(pools)]
        self.o = kv_pages.Cache(np.full((R, H, pph), -1, np.int32), np.zeros(R, np.int32), np.zeros(pool, np.int32), data)
        self.table, self.lens, self.refs = (torch.tensor(x, device=dev) for x in (self.o.table, self.o.lens, self.o.refs))
        self.pools = [torch.tensor(p, device=dev) for p in self.o.pools] + [None] * (2 - pools)
        self.status = torch.full((2,), -7, dtype=torch.int32, device=dev)

    def put(self):
        """The oracle's state onto the GPU."""
        for t, x in ((self.table, self.o.table), (self.lens, self.o.lens), (self.refs, self.o.refs)):
            t.copy_(torch.tensor(x))

    def same(self, status=None):
        assert np.array_equal(self.table.cpu().numpy(), self.o.table)
        assert np.array_equal(self.lens.cpu().numpy(), self.o.lens)
        assert np.array_equal(self.refs.cpu().numpy(), self.o.refs)
        for t, p in zip(self.pools, self.o.pools):
            assert np.array_equal(t.cpu().numpy(), p)
        if status is not None:
            assert tuple(self.status.tolist()) == status

    def extend(self, rows, lens):
        asym.kv_extend(self.table, self.lens, self.refs, i32(rows, self.dev), i32(lens, self.dev), self.status)
        self.same(self.o.extend(rows, lens))

    def fork(self, src, dst):
        asym.kv_fork(*self.pools, self.table, self.lens, self.refs, i32(src, self.dev), i32(dst, self.dev), self.status)
        self.same(self.o.fork(src, dst))

    def free(self, rows):
        asym.kv_free(self.table, self.lens, self.refs, i32(rows, self.dev))
        self.o.free(rows)
        self.same()

    def compact(self):
        asym.kv_compact(*self.pools, self.table, self.lens, self.refs, self.status)
        self.same(self.o.compact())


def test_extend(dev):
    p = Pair(dev, 6, 2, 4, 40)
    p.extend([0, 3, 5], [1, 32, 33])
    p.extend([0, 3, 5], [32, 33, 40])          # one of them needs a page
    p.extend([5, 5, 0, 9, -1, 3], [128, 60, 20, 50, 50, 129])  # twice, shorter, outside, beyond the table
    p.extend([], [])
    p.extend([1, 2, 4], [128, 128, 128])
    p.extend([0, 1, 2, 3, 4], [128] * 5)       # too few free pages: nothing changes
    assert p.status.tolist()[1] > 0
    p.extend([0], [128])


def test_fork(dev):
    p = Pair(dev, 8, 3, 3, 60, seed=1)
    p.extend([0, 1, 2], [70, 64, 5])
    p.fork([0, 0, 1, 2], [3, 4, 5, 6])
    p.fork([0, 1], [1, 0])                     # rows change places
    p.fork([3, 4, 5], [4, 5, 3])
    p.fork([2, 2, 0, 9, 0, -1], [2, 7, 7, 1, 8, 4])  # onto itself, a target twice, outside the table
    p.fork([7], [0])                           # (an empty row or not: as the oracle says)
    p.fork([], [])
    p.fork([0] * 4 + [1] * 3, [7, 6, 5, 4, 3, 2, 0])


def test_fork_without_room(dev):
    p = Pair(dev, 4, 2, 2, 9, seed=2)
    p.extend([0], [50])
    p.fork([0, 0], [1, 2])
    p.fork([0, 1, 2], [3, 2, 1])               # two pages are free, six are needed
    assert p.status.tolist() == [0, 5]
    p.free([2])
    p.fork([0], [3])


def test_one_pool_and_no_status(dev):
    p = Pair(dev, 4, 1, 3, 20, pools=1, seed=3)
    p.extend([0, 1], [40, 80])
    p.fork([0], [2])
    p.free([0, 1])
    p.compact()
    asym.kv_extend(p.table, p.lens, p.refs, i32([3], dev), i32([96], dev))
    p.o.extend([3], [96])
    p.same()


def test_free_and_compact(dev):
    p = Pair(dev, 10, 2, 4, 100, words=544, seed=4)
    p.extend(list(range(10)), [100, 3, 64, 128, 1, 90, 33, 50, 20, 10])
    p.fork([0, 3], [1, 2])
    p.free([0, 4, 4, 7, -3, 11, 8])
    p.compact()
    p.compact()                                # nothing left to move
    p.extend([0, 4], [128, 100])
    p.free(list(range(10)))
    p.compact()                                # an empty cache
    assert p.status.tolist() == [0, 0]


def test_compact_a_full_pool(dev):
    p = Pair(dev, 2, 1, 8, 12, seed=5)
    p.extend([0, 1], [256, 128])
    p.compact()
    p.free([0])
    p.compact()
    assert p.status.tolist() == [4, 4]


@pytest.mark.parametrize("seed,pool,R,H,pph", [(0, 300, 12, 2, 6), (1, 9000, 40, 8, 5), (2, 4096, 30, 3, 9), (3, 12289, 300, 1, 12)])
def test_a_long_run(dev, seed, pool, R, H, pph):
    g = np.random.default_rng(seed)
    p = Pair(dev, R, H, pph, pool, seed=seed)
    # pages scattered over the pool, in every segment of the scan
    for r in range(0, R, 2):
        n = int(g.integers(1, 32 * pph + 1))
        for h in range(H):
            for c in range(-(-n // 32)):
                free = np.flatnonzero(p.o.refs == 0)
                e = int(g.choice(free))
                p.o.table[r, h, c], p.o.refs[e] = e, 1
        p.o.lens[r] = n
    p.put()
    for _ in range(6):
        n = int(g.integers(1, R))
        rows = g.permutation(R)[:n].tolist()
        p.extend(rows, [int(p.o.lens[r]) + int(g.integers(0, 40)) for r in rows])
        p.fork(g.integers(0, R, n).tolist(), g.permutation(R)[:n].tolist())
        p.free(g.permutation(R)[:max(1, n // 3)].tolist())
        p.compact()


def test_many_requests(dev):
    # more requests than a workgroup has threads
    p = Pair(dev, 700, 1, 2, 2000, seed=6)
    p.extend(list(range(700)), [1 + r % 64 for r in range(700)])
    p.fork(list(range(300)), list(range(400, 700)))
    p.free(list(range(0, 700, 2)))
    p.compact()


def test_captured(dev):
    p = Pair(dev, 8, 2, 4, 64, seed=7)
    p.extend([0, 1, 2], [40, 60, 80])
    start = [t.clone() for t in (p.table, p.lens, p.refs, *p.pools)]
    src, dst, rows, lens = i32([0, 1], dev), i32([4, 5], dev), i32([0, 4, 5], dev), i32([65, 66, 67], dev)
    ended = i32([1, 2], dev)

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
    g = torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(g):
        step()
    for s, d in (([0, 1], [4, 5]), ([2, 2], [4, 5]), ([1, 0], [3, 6])):
        reset()
        src.copy_(i32(s, dev)), dst.copy_(i32(d, dev))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (p.table, p.lens, p.refs, *p.pools)]
        reset()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (p.table, p.lens, p.refs, *p.pools)):
            assert torch.equal(a, b)


def test_refusals(dev):
    p = Pair(dev, 4, 1, 2, 8)
    rows, one = i32([0, 1], dev), i32([5], dev)
    with pytest.raises(ValueError):
        asym.kv_extend(p.table, p.lens, p.refs, rows, one)
    with pytest.raises(TypeError):
        asym.kv_extend(p.table, p.lens, p.refs, rows.long(), rows)
    with pytest.raises(ValueError):
        asym.kv_extend(p.table, p.lens[:3], p.refs, rows, rows)
    with pytest.raises(ValueError):
        asym.kv_extend(p.table, p.lens, p.refs, rows, rows, status=one)
    with pytest.raises(ValueError):
        asym.kv_extend(p.table.cpu(), p.lens, p.refs, rows, rows)
    with pytest.raises(ValueError):
        asym.kv_fork(p.pools[0][:4], None, p.table, p.lens, p.refs, rows, rows)
    with pytest.raises(ValueError):
        asym.kv_fork(p.pools[0], p.pools[1].float(), p.table, p.lens, p.refs, rows, rows)
    with pytest.raises(ValueError):
        asym.kv_compact(p.pools[0].t(), None, p.table, p.lens, p.refs)
    with pytest.raises(asym.AsymError):  # one pool twice
        asym.kv_compact(p.pools[0], p.pools[0], p.table, p.lens, p.refs)
    with pytest.raises(asym.AsymError):  # pages of 12 bytes
        q = torch.zeros((8, 3), dtype=torch.int32, device=dev)
        asym.kv_compact(q, None, p.table, p.lens, p.refs)


def test_serving_loop(dev):
    """Prompts run and written, rows forked, grown and decoded, some ended, the cache compacted and decoded again."""
    H, Hq, R, pph = 2, 8, 6, 6
    pool = 80
    pools = [torch.full((pool, asym.FP4_PAGE_BYTES), 255, dtype=torch.uint8, device=dev) for _ in range(2)]
    table = torch.full((R, H, pph), -1, dtype=torch.int32, device=dev)
    lens, refs = torch.zeros(R, dtype=torch.int32, device=dev), torch.zeros(pool, dtype=torch.int32, device=dev)
    status = torch.zeros(2, dtype=torch.int32, device=dev)
    g = torch.Generator().manual_seed(0)
    mk = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).to(dev)

    # prompts of rows 0 .. 2
    n = [70, 33, 64]
    T = sum(n)
    cu = i32(offsets(n), dev)
    asym.kv_extend(table, lens, refs, i32([0, 1, 2], dev), i32(n, dev), status)
    assert status.tolist() == [(3 + 2 + 2) * H, 0]
    qkv = mk(T, Hq + 2 * H, 128)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    first = asym.attn_prefill(q, k, v, cu)
    asym.kv_write_fp4(k, v, *pools, table[:3], table[:3], cu, i32([0, 0, 0], dev))

    # a chunk behind the first prompt: the cached prefix, then its own keys
    c = 20
    chunk = mk(c, Hq + 2 * H, 128)
    kk, vv = (torch.empty((n[0] + c, H, 128), dtype=torch.bfloat16, device=dev) for _ in range(2))
    asym.kv_read_fp4(*pools, table[:1], table[:1], i32([0, n[0]], dev), i32([0], dev), kk, vv)
    kk[n[0]:], vv[n[0]:] = chunk[:, Hq:Hq + H], chunk[:, Hq + H:]
    out = asym.attn_prefill(chunk[:, :Hq], kk, vv, i32([0, c], dev), i32([0, n[0] + c], dev))
    # its last row is a decode step over the same keys once they are in the cache (4-bit: only near)
    asym.kv_extend(table, lens, refs, i32([0], dev), i32([n[0] + c], dev), status)
    asym.kv_write_fp4(chunk[:, Hq:Hq + H], chunk[:, Hq + H:], *pools, table[:1], table[:1], i32([0, c], dev), i32([n[0]], dev))
    step = asym.attn_decode_paged_fp4(chunk[-1:, :Hq].contiguous(), *pools, table[:1], table[:1], lens[:1])
    near = (step.float() - out[-1:].float()).norm() / out[-1:].float().norm()
    assert torch.isfinite(first.float()).all() and near < 0.3

    # rows 3 .. 5 fork from 0, 1, 1; every row decodes three tokens
    asym.kv_fork(*pools, table, lens, refs, i32([0, 1, 1], dev), i32([3, 4, 5], dev), status)
    every, ones = i32(list(range(R)), dev), i32(list(range(R + 1)), dev)
    for _ in range(3):
        start = lens.clone()
        asym.kv_extend(table, lens, refs, every, start + 1, status)
        new = mk(R, Hq + 2 * H, 128)
        asym.kv_write_fp4(new[:, Hq:Hq + H], new[:, Hq + H:], *pools, table, table, ones, start)
        qs = new[:, :Hq].contiguous()
        o = asym.attn_decode_paged_fp4(qs, *pools, table, table, lens)
        R_, L, bo, bl = attend(qs, pools[0].cpu().numpy(), pools[1].cpu().numpy(), table.cpu().numpy(), table.cpu().numpy(),
                               lens.tolist(), 128 ** -0.5)
        assert np.all(np.abs(bf16_bits_to_f64(bits(o)) - R_) <= bo)
    assert lens.tolist() == [93, 36, 67, 93, 36, 36]

    # rows 0 and 4 end; the rest answers the same after compaction
    asym.kv_free(table, lens, refs, i32([0, 4], dev))
    before = asym.attn_decode_paged_fp4(qs, *pools, table, table, lens)
    asym.kv_compact(*pools, table, lens, refs, status)
    after = asym.attn_decode_paged_fp4(qs, *pools, table, table, lens)
    assert torch.equal(before, after) and torch.all(after[0] == 0) and torch.all(after[4] == 0)
    used = table[table >= 0]
    assert int(used.max()) < status.tolist()[1] == int((refs > 0).sum())
    asym.kv_free(table, lens, refs, every)
    assert not refs.any() and not lens.any() and torch.all(table == -1)
