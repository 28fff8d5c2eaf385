"""GPU parity of rotary positions, alone and on the way into the 16-bit paged cache, through the C ABI.

Against the float64 oracle, element by element.  The bound (derived): the angle's turns are
rounded to fp32 within [-1/2, 1/2], 2^-26 of a turn, 2^-23.3 radians; cosine and sine add 2 ulp, 2^-22;
their product with the amplitude, the two products and the sum 2^-24 each: together
2^-20 A (|a| + |b|); and the output's rounding to bf16, 2^-8 of it.  What is copied is the same bits.
"""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import rope
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


def normal(dev, seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(dev)


def check(x, y, pos, freq, layout, amp=1.0, backward=False):
    R, scale = rope.rope(f64(x), pos, freq.tolist(), layout, amp, backward)
    err = np.abs(f64(y) - R)
    assert np.all(err <= 2.0 ** -8 * (np.abs(R) + 2.0 ** -20 * scale) * (scale > 0) + 2.0 ** -20 * scale), err.max()


@pytest.mark.parametrize("T,H,D,rotary", [
    (1, 1, 8, 8), (1, 1, 8, 0), (1, 5, 128, 128), (3, 2, 64, 64), (7, 1, 128, 64), (40, 3, 64, 40), (5, 4, 128, 104), (33, 1, 16, 16),
    (9, 2, 128, 2), (2, 130, 64, 64), (65, 8, 128, 128), (4, 3, 256, 232), (6, 2, 24, 24), (3, 1, 1024, 1024), (2, 2, 1016, 1010),
    (300, 1, 8, 6), (1, 33, 1024, 512)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("backward", [False, True])
def test_against_oracle(dev, T, H, D, rotary, layout, backward):
    x = normal(dev, T + D, T, H, D)
    pos = torch.randint(0, 5000, (T,), generator=torch.Generator().manual_seed(T)).tolist()
    freq, _ = asym.rope_freq(rotary)
    y = asym.rope(x, i32(pos, dev), freq.to(dev), layout=layout, amplitude=1.25, backward=backward)
    check(x, y, pos, freq, layout, 1.25, backward)
    assert torch.equal(y[..., rotary:], x[..., rotary:])


def test_far_and_negative_positions(dev):
    pos = [0, 1, -1, 131071, 1000003, 2 ** 31 - 1, -2 ** 31, -77777]
    x = normal(dev, 1, len(pos), 2, 128)
    freq, _ = asym.rope_freq(128, 500000.0, "parts", 8)
    for layout in ("half", "interleaved"):
        y = asym.rope(x, i32(pos, dev), freq.to(dev), layout=layout)
        check(x, y, pos, freq, layout)
        assert torch.equal(y[0], x[0])  # position 0 turns nothing


def test_the_gradient_against_differences(dev):
    # the map is linear: <g, rope(x + d) - rope(x)> = <backward(g), d>, within both sides' bounds
    T, H, D = 5, 3, 64
    x, g = normal(dev, 3, T, H, D), normal(dev, 4, T, H, D)
    pos, (freq, _) = [3, 1000, 7, 0, 65535], asym.rope_freq(48)
    for layout in ("half", "interleaved"):
        y = f64(asym.rope(x, i32(pos, dev), freq.to(dev), layout=layout, amplitude=0.75))
        back = f64(asym.rope(g, i32(pos, dev), freq.to(dev), layout=layout, amplitude=0.75, backward=True))
        left, right = (f64(g) * y).sum(), (back * f64(x)).sum()
        _, sx = rope.rope(f64(x), pos, freq.tolist(), layout, 0.75)
        _, sg = rope.rope(f64(g), pos, freq.tolist(), layout, 0.75)
        slack = (np.abs(f64(g)) * (2.0 ** -8 * np.abs(y) * 1.01 + 2.0 ** -20 * sx)).sum() \
            + (np.abs(f64(x)) * (2.0 ** -8 * np.abs(back) * 1.01 + 2.0 ** -20 * sg)).sum()
        assert abs(left - right) <= slack


def test_views_in_place_and_what_lies_beside(dev):
    wide = normal(dev, 5, 20, 6, 576)
    pos, (freq, _) = list(range(100, 120)), asym.rope_freq(64)
    ref = asym.rope(wide[:, 1:4, 512:].contiguous(), i32(pos, dev), freq.to(dev), layout="interleaved")
    got = wide.clone()
    view = got[:, 1:4, 512:]
    assert asym.rope(view, i32(pos, dev), freq.to(dev), out=view, layout="interleaved") is view
    assert torch.equal(got[:, 1:4, 512:], ref)
    assert torch.equal(got[:, 0], wide[:, 0]) and torch.equal(got[:, 4:], wide[:, 4:]) and torch.equal(got[..., :512], wide[..., :512])


def test_infinities_stay_in_their_pair(dev):
    x = normal(dev, 6, 2, 1, 64)
    x[0, 0, 3], x[1, 0, 40] = float("nan"), float("inf")
    freq, _ = asym.rope_freq(64)
    y = asym.rope(x, i32([5, 6], dev), freq.to(dev))
    bad = ~torch.isfinite(y.float())
    assert bad[0, 0].nonzero()[:, 0].tolist() == [3, 35] and bad[1, 0].nonzero()[:, 0].tolist() == [8, 40]


# -- appending ------------------------------------------------------------------------

def append_oracle(k, v, kp, vp, kt, vt, cu, start, pos, freq, layout, amp, q=None):
    """What the pools hold, element by element: the kernel's own rows of K (from rope, checked apart) and V."""
    T = k.shape[0]
    where = [-1] * T
    for b in range(len(start)):
        for i in range(max(cu[b], 0), min(cu[b + 1], T)):
            if start[b] >= 0:
                where[i] = start[b] + i - cu[b]
    at = [p if pos is None else pos[i] for i, p in enumerate(where)]
    turn = lambda x: asym.rope(x.contiguous(), i32([min(p, 2 ** 31 - 1) for p in at], x.device), freq, layout=layout,
                               amplitude=amp) if freq is not None else x
    kr = turn(k)
    for b in range(len(start)):
        for i in range(max(cu[b], 0), min(cu[b + 1], T)):
            p = where[i]
            if p < 0 or p >= 32 * kt.shape[2]:
                continue
            for h in range(kt.shape[1]):
                for rows, pool, table in ((kr, kp, kt), (v, vp, vt)):
                    page = int(table[b, h, p // 32])
                    if 0 <= page < pool.shape[0]:
                        pool[page, p % 32] = rows[i, h]
    return where, at, None if q is None else turn(q)


@pytest.mark.parametrize("new,start,Hq,H,pph", [
    ([1], [0], 0, 1, 1), ([1], [31], 4, 2, 1), ([33], [31], 3, 1, 3), ([5, 0, 70], [30, 9, 1], 8, 2, 3),
    ([1, 1, 1, 1], [0, 17, 40, 95], 6, 3, 3), ([3, 3], [94, -1], 4, 2, 3), ([40], [60], 1, 1, 3), ([1] * 66, list(range(66)), 2, 1, 3),
    ([2, 2], [96, 2000000000], 4, 2, 3), ([90, 7], [3, 62], 32, 8, 4), ([4], [2 ** 31 - 2], 2, 1, 2)])
@pytest.mark.parametrize("rotary,layout,given", [(128, "half", False), (64, "interleaved", True), (104, "half", False), (6, "interleaved", True),
                                                 (0, "half", False)])
def test_appended_pages(dev, new, start, Hq, H, pph, rotary, layout, given):
    B, T = len(new), sum(new)
    rng = np.random.default_rng(T + H)
    n = B * H * pph + 3
    kp, vp = normal(dev, 1, n, 32, 128), normal(dev, 2, n, 32, 128)
    kt, vt = (rng.permutation(n)[:B * H * pph].reshape(B, H, pph).astype(np.int32) for _ in range(2))
    kt[0, 0, 0], vt[-1, -1, -1] = -1, n  # no pages of the pool
    qkv = normal(dev, 3, T, Hq + 2 * H, 128)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    freq = asym.rope_freq(rotary)[0].to(dev) if rotary else None
    pos = rng.integers(0, 9000, T).tolist() if given else None
    cu = offsets(new)
    ek, ev = kp.clone(), vp.clone()
    where, at, qr = append_oracle(k, v, ek, ev, kt, vt, cu, start, pos, freq, layout, 1.5, q if Hq else None)
    out = torch.full((T, Hq, 128), 9.0, dtype=torch.bfloat16, device=dev) if Hq else None
    r = asym.kv_append(k, v, kp, vp, i32(kt, dev), i32(vt, dev), i32(cu, dev), i32(start, dev), q=q if Hq else None, q_out=out, freq=freq,
                       positions=None if pos is None else i32(pos, dev), layout=layout, amplitude=1.5)
    assert torch.equal(kp, ek) and torch.equal(vp, ev)
    assert r is out
    for i in range(T if Hq else 0):
        if where[i] < 0:
            assert bool((out[i] == 9).all())
        elif at[i] < 2 ** 31 or freq is None:
            assert torch.equal(out[i], qr[i])
        else:  # (places that rope's positions do not reach)
            check(q[i:i + 1], out[i:i + 1], [at[i]], freq.cpu(), layout, 1.5)


def test_append_in_place_rows_outside_and_new_output(dev):
    q, k, v = (normal(dev, s, 12, h, 128) for s, h in ((1, 4), (2, 2), (3, 2)))
    table = i32(np.arange(8).reshape(2, 2, 2), dev)
    cu, start = i32([2, 5, 9], dev), i32([30, 0], dev)
    freq = asym.rope_freq(128)[0].to(dev)
    pools = [torch.zeros((8, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    new = asym.kv_append(k, v, *pools, table, table, cu, start, q=q, freq=freq)
    held = q.clone()
    asym.kv_append(k, v, *pools, table, table, cu, start, q=held, q_out=held, freq=freq)
    assert torch.equal(held[2:9], new[2:9]) and torch.equal(held[:2], q[:2]) and torch.equal(held[9:], q[9:])
    assert torch.equal(held[2:9], asym.rope(q[2:9], i32([30, 31, 32, 0, 1, 2, 3], dev), freq))
    # offsets that say too much are held
    again = [torch.zeros_like(p) for p in pools]
    asym.kv_append(k, v, *again, table[:1], table[:1], i32([-4, 100], dev), i32([7], dev), freq=freq)
    assert torch.equal(again[1][table[0, 1, 0]][7:19], v[:, 1])


def test_long_rows_of_a_large_pool(dev):
    # pages past 4 GiB of the pool
    n = (1 << 19) + 40
    pools = [torch.empty((n, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    k, v = normal(dev, 1, 3, 1, 128), normal(dev, 2, 3, 1, 128)
    table = i32([[[n - 1, n - 7]]], dev)
    asym.kv_append(k, v, *pools, table, table, i32([0, 3], dev), i32([31], dev))
    assert torch.equal(pools[0][n - 1, 31], k[0, 0]) and torch.equal(pools[1][n - 7, :2], v[1:, 0])


def test_streams_and_graphs(dev):
    q, k, v = (normal(dev, s, 40, h, 128) for s, h in ((1, 8), (2, 2), (3, 2)))
    table = i32(np.arange(12).reshape(2, 2, 3), dev)
    cu, start = i32([0, 25, 40], dev), i32([3, 50], dev)
    freq = asym.rope_freq(128)[0].to(dev)
    want = []
    for s in (1.0, -1.0, 2.0):
        pools = [torch.zeros((12, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
        want.append((asym.kv_append(k * s, v * s, *pools, table, table, cu, start, q=q * s, freq=freq), *pools,
                     asym.rope(q * s, start.repeat(20), freq)))
    torch.cuda.synchronize()
    side = asym.stream_create()
    pools = [torch.zeros((12, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    torch.cuda.synchronize()
    got = asym.kv_append(k, v, *pools, table, table, cu, start, q=q, freq=freq, stream=side)
    side.synchronize()
    assert torch.equal(got, want[0][0]) and torch.equal(pools[0], want[0][1])
    asym.stream_destroy(side)
    hq, hk, hv, out, turned, pos = q.clone(), k.clone(), v.clone(), torch.empty_like(q), torch.empty_like(q), start.repeat(20)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asym.kv_append(hk, hv, *pools, table, table, cu, start, q=hq, q_out=out, freq=freq)
        asym.rope(hq, pos, freq, out=turned)
    for s, w in zip((1.0, -1.0, 2.0), want):
        hq.copy_(q * s), hk.copy_(k * s), hv.copy_(v * s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, *pools, turned), w))


def test_refusals(dev):
    x, pos, freq = normal(dev, 1, 4, 2, 64), i32([0, 1, 2, 3], dev), asym.rope_freq(64)[0].to(dev)
    for bad, kind in ((lambda: asym.rope(x.float(), pos, freq), TypeError), (lambda: asym.rope(x, pos.long(), freq), TypeError),
                      (lambda: asym.rope(x, pos, freq.float()), TypeError), (lambda: asym.rope(x, pos[:3], freq), ValueError),
                      (lambda: asym.rope(x[..., ::2], pos, freq), ValueError), (lambda: asym.rope(x, pos, freq, out=x[:3]), ValueError),
                      (lambda: asym.rope(x, pos.cpu(), freq), ValueError), (lambda: asym.rope(x, pos, freq[None]), ValueError),
                      (lambda: asym.rope(x, pos, freq, layout="other"), KeyError),
                      (lambda: asym.rope(x, pos, asym.rope_freq(66)[0].to(dev)), asym.AsymError),
                      (lambda: asym.rope(x[..., :60].contiguous(), pos, freq[:8]), asym.AsymError)):
        with pytest.raises(kind):
            bad()
    k, table, cu, start = normal(dev, 2, 4, 2, 128), i32([[[0], [1]]], dev), i32([0, 4], dev), i32([0], dev)
    pools = [torch.zeros((2, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    for bad, kind in ((lambda: asym.kv_append(k, k[:3], *pools, table, table, cu, start), ValueError),
                      (lambda: asym.kv_append(k, k, *pools, table[:, :1], table[:, :1], cu, start), ValueError),
                      (lambda: asym.kv_append(k, k, *pools, table, table, cu[:1], start), ValueError),
                      (lambda: asym.kv_append(k, k, *pools, table, table, cu, start, q=k[:3]), ValueError),
                      (lambda: asym.kv_append(k, k, *pools, table, table, cu, start, q_out=k), ValueError),
                      (lambda: asym.kv_append(k, k, *pools, table, table, cu, start, positions=start), ValueError),
                      (lambda: asym.kv_append(k, k, pools[0].float(), pools[1], table, table, cu, start), TypeError),
                      (lambda: asym.kv_append(k, k, *[p[:, :16] for p in pools], table, table, cu, start), ValueError)):
        with pytest.raises(kind):
            bad()
