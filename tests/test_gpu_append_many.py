"""GPU parity of appends of many tokens, where a thread has two: places against indexing, keys and queries against asym.rope (compared
with the oracle in the module of its tests), bit by bit."""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from tests.test_gpu_rotary import dev, i32, offsets  # noqa: F401

pytestmark = pytest.mark.gpu


def lengths(T, seed):
    """Requests of 0 to 40 tokens, their borders anywhere in a workgroup's tokens, T in all."""
    rng = np.random.default_rng(seed)
    out = []
    while sum(out) < T:
        out.append(int(min(rng.choice([0, 1, 2, 3, 5, 7, 8, 40]), T - sum(out))))
    return out


# heads: few (four tokens a workgroup, twice), as many as fit one, more (workgroups that share a token); runs of 8, 4 and 1 channels
@pytest.mark.parametrize("T", [4095, 4096, 4097, 4999])
@pytest.mark.parametrize("Hq,H,rotary,layout", [(0, 1, 128, "half"), (4, 2, 104, "half"), (1, 1, 6, "interleaved"), (32, 8, 64, "interleaved"),
                                                (31, 8, 104, "interleaved"), (96, 8, 128, "half"), (12, 4, 6, "half"), (3, 1, 0, "half")])
def test_many_tokens(dev, T, Hq, H, rotary, layout):
    new = lengths(T, T + H)
    B, pph = len(new), 4
    rng = np.random.default_rng(T)
    start = rng.integers(0, 80, B)
    start[::17] = -1              # left out
    start[5::29] = 32 * pph - 3   # past the table
    n = B * H * pph + 3
    g = torch.Generator(device=dev).manual_seed(T + Hq)
    normal = lambda *s: torch.randn(s, generator=g, device=dev).to(torch.bfloat16)
    kp, vp, qkv = normal(n, 32, 128), normal(n, 32, 128), normal(T, Hq + 2 * H, 128)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    kt, vt = (rng.permutation(n)[:B * H * pph].reshape(B, H, pph).astype(np.int32) for _ in range(2))
    kt[1::13, 0, 1] = -1          # no pages of the pool
    vt[2::13, -1, 0] = n
    cu = offsets(new)
    owner = np.repeat(np.arange(B), new)
    at = start[owner] + np.arange(T) - np.array(cu)[owner]
    in_request = start[owner] >= 0
    freq = asym.rope_freq(rotary)[0].to(dev) if rotary else None
    turn = lambda x: asym.rope(x.contiguous(), i32(np.maximum(at, 0), dev), freq, layout=layout, amplitude=1.5) if rotary else x
    ek, ev = kp.clone(), vp.clone()
    for rows, pool, table in ((turn(k), ek, kt), (v, ev, vt)):
        for h in range(H):
            page = table[owner, h, np.minimum(np.maximum(at, 0) // 32, pph - 1)]
            ok = in_request & (at < 32 * pph) & (page >= 0) & (page < n)
            pool[torch.tensor(page[ok].astype(np.int64), device=dev), torch.tensor(at[ok] % 32, device=dev)] = rows[torch.tensor(ok, device=dev), h]
    out = torch.full((T, Hq, 128), 9.0, dtype=torch.bfloat16, device=dev) if Hq else None
    want = None
    if Hq:
        some = torch.tensor(in_request, device=dev)[:, None, None]
        want = torch.where(some, turn(q), out)
    asym.kv_append(k, v, kp, vp, i32(kt, dev), i32(vt, dev), i32(cu, dev), i32(start, dev), q=q if Hq else None, q_out=out, freq=freq,
                   layout=layout, amplitude=1.5)
    assert torch.equal(kp, ek) and torch.equal(vp, ev)
    assert out is None or torch.equal(out, want)


def test_many_tokens_in_place_and_captured(dev):
    T, H, Hq = 4099, 2, 4
    qkv = torch.randn((T, Hq + 2 * H, 128), generator=torch.Generator(device=dev).manual_seed(1), device=dev).to(torch.bfloat16)
    freq = asym.rope_freq(128)[0].to(dev)
    table = i32(np.arange(3 * H * 64).reshape(3, H, 64), dev)
    cu, start = i32([2, 1500, 3000, T - 1], dev), i32([0, 7, 31], dev)
    pools = [torch.zeros((3 * H * 64, 32, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    ref = asym.kv_append(qkv[:, Hq:Hq + H], qkv[:, Hq + H:], *pools, table, table, cu, start, q=qkv[:, :Hq], freq=freq)
    held, again = qkv.clone(), [torch.zeros_like(p) for p in pools]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asym.kv_append(held[:, Hq:Hq + H], held[:, Hq + H:], *again, table, table, cu, start, q=held[:, :Hq], q_out=held[:, :Hq], freq=freq)
    for _ in range(3):
        held.copy_(qkv)
        for p in again:
            p.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[2:T - 1, :Hq], ref[2:T - 1]) and torch.equal(held[:2], qkv[:2]) and torch.equal(held[T - 1:], qkv[T - 1:])
        assert torch.equal(held[:, Hq:], qkv[:, Hq:]) and all(torch.equal(a, b) for a, b in zip(again, pools))
