"""Pins of the rotary and drafted-token oracles, the host helpers, and the new calls' refusals, on the CPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import drafts, kv_pages, rope

P = 1 << 20  # an address that is never read: the calls are refused, or have nothing to do


def code(name, *args):
    return getattr(asym.load_library(), name)(*args)


# -- oracles --------------------------------------------------------------------

def test_rope_oracle_pins():
    x = np.zeros((1, 1, 6))
    x[0, 0] = [1, 2, 3, 4, 5, 6]
    quarter = [math.pi / 2, math.pi]
    y, _ = rope.rope(x, [1], quarter, "half")  # pairs (1, 3) and (2, 4)
    assert np.allclose(y[0, 0], [-3, -2, 1, -4, 5, 6])
    y, _ = rope.rope(x, [1], quarter, "interleaved", amplitude=2.0)  # pairs (1, 2) and (3, 4)
    assert np.allclose(y[0, 0], [-4, 2, -6, -8, 5, 6])
    z, _ = rope.rope(y, [1], quarter, "interleaved", amplitude=0.5, backward=True)
    assert np.allclose(z, x)


def test_rope_gradient_is_that_of_differences():
    rng = np.random.default_rng(0)
    x, g, f = rng.normal(size=(3, 2, 8)), rng.normal(size=(3, 2, 8)), [0.3, 0.01, 2.0]
    back, _ = rope.rope(g, [5, 0, 100], f, "half", 1.3, True)
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = 1e-3
        up, down = (rope.rope(x + s * d, [5, 0, 100], f, "half", 1.3)[0] for s in (1, -1))
        assert abs(((up - down) * g).sum() / 2e-3 - back[i]) < 1e-9


def test_tree_attention_oracle_pins():
    q, k = np.zeros((2, 1, 2)), np.zeros((3, 1, 2))
    v = np.array([[[1.0, 0]], [[0, 3.0]], [[5.0, 7.0]]])
    O, lse, _, _ = drafts.tree_attention(q, k, v, [{0}, {1}], 1, 1.0)
    assert np.allclose(O[:, 0], [[0.5, 1.5], [3, 3.5]]) and np.allclose(lse, math.log(2))
    O, lse, _, _ = drafts.tree_attention(q, k, v, [set(), {0, 1}], 0, 1.0)
    assert np.all(O[0] == 0) and lse[0, 0] == -np.inf and np.allclose(O[1, 0], [0.5, 1.5])
    O, _, _, _ = drafts.tree_attention(q, k, v, [{0}, {1}], -1, 1.0)  # node 0 is not there
    assert np.all(O[0] == 0) and np.allclose(O[1, 0], [1, 0])


def test_verify_oracle_pins():
    p = np.array([[0.5, 0.25, 0.25], [0.25, 0.5, 0.25]])
    q = np.array([[0.25, 0.5, 0.25], [1.0, 0, 0]])
    # token 1: p / q = 1/2; u below it accepts, and the last token comes from the second row
    assert drafts.verify(p, q, [9, 1], [-1, 0], [0, 0.49], 0.3) == ([0, 1], 1)
    assert drafts.verify(p, q, [9, 1], [-1, 0], [0, 0.5], 0.9) == ([0], 0)  # what is left: token 0 alone
    assert drafts.verify(p, None, [9, 1], [-1, 0], [0, 0.24], 0.0) == ([0, 1], 0)
    assert drafts.verify(p, None, [9, 1], [-1, 0], [0, 0.25], 0.7) == ([0], 2)  # tokens 0 and 2, two to one
    # the second sibling: r = (1, 0, 0) after the first, which its own token 2 has no part of
    three = np.concatenate([p, p[:1]])
    assert drafts.verify(three, np.concatenate([q, q[:1]]), [9, 1, 2], [-1, 0, 0], [0, 0.9, 0.0], 0.1) == ([0], 0)
    assert drafts.verify(np.zeros((1, 4)), None, [0], [-1], [0], 0.5) == ([0], -1)


def test_verified_tokens_have_the_targets_distribution():
    """Two drafted siblings over four tokens: the frequency of the first token behind the root, kept or drawn, against
    the target's.  60000 trials: each frequency within 5 of its standard deviations, 5 * 0.5 / sqrt(60000)."""
    rng = np.random.default_rng(1)
    p = np.array([0.1, 0.2, 0.3, 0.4])
    q = np.array([0.4, 0.3, 0.2, 0.1])
    t, d = np.stack([p] * 3), np.stack([q] * 3)
    seen = np.zeros(4)
    trials = 60000
    draws = rng.choice(4, size=(trials, 2), p=q)
    u = rng.random((trials, 4))
    for i in range(trials):
        tokens = [0, int(draws[i, 0]), int(draws[i, 1])]
        path, last = drafts.verify(t, d, tokens, [-1, 0, 0], [0, u[i, 0], u[i, 1]], u[i, 2])
        seen[tokens[path[1]] if len(path) > 1 else last] += 1
    assert np.all(np.abs(seen / trials - p) <= 5 * 0.5 / math.sqrt(trials))


def test_keep_oracle_pins():
    c = kv_pages.Cache(np.arange(4).reshape(1, 1, 4), [70], [1, 1, 1, 0], (np.arange(4 * 32).reshape(4, 32, 1).copy(),))
    drafts.keep(c, [0], [0, 8], [0, 3, 7, -1, -1, -1, -1, -1], [3])
    assert c.lens[0] == 65 and c.pools[0].reshape(-1)[62:65].tolist() == [62, 65, 69] and c.refs.tolist() == [1, 1, 1, 0]
    drafts.keep(c, [0], [0, 5], [1, -1, -1, -1, -1], [1])
    assert c.lens[0] == 61 and c.table[0, 0].tolist() == [0, 1, -1, 3] and c.refs.tolist() == [1, 1, 0, 0]
    before = c.pools[0].copy()
    drafts.keep(c, [0, 0], [0, 2, 4], [1, 0, 0, 1], [2, 2])  # falls; the row is named before
    assert c.lens[0] == 61 and np.array_equal(c.pools[0], before)


# -- host helpers -----------------------------------------------------------------

def test_frequencies():
    f, a = asym.rope_freq(8, 10000.0)
    assert a == 1.0 and f.dtype is torch.float64 and torch.allclose(f, torch.tensor([1, 0.1, 0.01, 0.001], dtype=torch.float64))
    assert torch.equal(asym.rope_freq(8, scaling="linear", factor=4)[0], f / 4)
    g, _ = asym.rope_freq(8, scaling="base", factor=16)
    assert g[0] == 1 and abs(g[3] * 16 - f[3]) < 1e-15  # the slowest turns 16 times slower
    h, a = asym.rope_freq(128, scaling="parts", factor=8, original=4096, fast=32, slow=1)
    whole, _ = asym.rope_freq(128)
    turns = 4096 * whole / (2 * math.pi)
    assert torch.equal(h[turns > 32], whole[turns > 32]) and torch.equal(h[turns < 1], whole[turns < 1] / 8)
    between = (turns <= 32) & (turns >= 1)
    assert torch.all(h[between] <= whole[between]) and torch.all(h[between] >= whole[between] / 8)
    assert abs(a - (1 + 0.1 * math.log(8))) < 1e-15
    assert asym.rope_freq(0)[0].numel() == 0
    for bad in (dict(rotary=7), dict(rotary=-2), dict(rotary=8, factor=0.5), dict(rotary=8, scaling="x"), dict(rotary=2, scaling="base"),
                dict(rotary=8, base=0.0), dict(rotary=8, fast=1.0, slow=1.0)):
        with pytest.raises(ValueError):
            asym.rope_freq(**bad)


def test_draft_tree():
    mask, depth = asym.draft_tree([-1, 0, 0, 1, 3])
    assert mask[:, 0].tolist() == [1, 3, 5, 11, 27] and depth == [0, 1, 1, 2, 3]
    mask, depth = asym.draft_tree([-1] + list(range(129)))  # a chain of 130
    assert mask.shape == (130, 3) and depth[-1] == 129
    assert mask[63].tolist() == [-1, 0, 0] and mask[64].tolist() == [-1, 1, 0] and mask[129].tolist() == [-1, -1, 3]
    assert asym.draft_tree([])[0].shape == (0, 1)
    for bad in ([-1, 1], [-1, -1], [-1, 0, 5]):
        with pytest.raises(ValueError):
            asym.draft_tree(bad)


# -- refusals -----------------------------------------------------------------------

ROPE = dict(T=2, H=3, D=64, rotary=32, x=P, xt=192, xh=64, y=P, yt=192, yh=64, pos=P, freq=P, layout=0, amp=1.0, back=0, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(T=-1), asym.EINVAL), (dict(H=0), asym.EINVAL), (dict(D=60), asym.EUNSUPPORTED), (dict(D=1032), asym.EUNSUPPORTED),
    (dict(D=0), asym.EUNSUPPORTED), (dict(rotary=31), asym.EINVAL), (dict(rotary=66), asym.EINVAL), (dict(rotary=-2), asym.EINVAL),
    (dict(layout=2), asym.EINVAL), (dict(amp=float("inf")), asym.EINVAL), (dict(freq=None), asym.EINVAL), (dict(freq=P + 4), asym.EINVAL),
    (dict(x=None), asym.EINVAL), (dict(y=P + 8), asym.EINVAL), (dict(pos=None), asym.EINVAL), (dict(pos=P + 2), asym.EINVAL),
    (dict(xt=100), asym.EINVAL), (dict(yh=-64), asym.EINVAL), (dict(H=1 << 21), asym.EUNSUPPORTED),
    (dict(T=1 << 24, H=64), asym.EUNSUPPORTED), (dict(T=0, x=None, y=None, pos=None), asym.OK)])
def test_rope_refusals(change, want):
    assert code("asym_rope_bf16", *{**ROPE, **change}.values()) == want


APPEND = dict(B=1, Hq=4, H=2, T=8, q=P, qt=512, qh=128, qo=P, qot=512, qoh=128, k=P, kt=256, kh=128, v=P, vt=256, vh=128, kp=P, vp=P,
              pool=4, kt_=P, vt_=P, pph=2, cu=P, start=P, pos=None, rotary=128, freq=P, layout=0, amp=1.0, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), asym.EINVAL), (dict(H=0), asym.EINVAL), (dict(Hq=-1), asym.EINVAL), (dict(T=-5), asym.EINVAL), (dict(pph=0), asym.EINVAL),
    (dict(pool=0), asym.EINVAL), (dict(pool=1 << 31), asym.EINVAL), (dict(pph=1 << 26), asym.EUNSUPPORTED), (dict(rotary=130), asym.EINVAL),
    (dict(rotary=3), asym.EINVAL), (dict(layout=-1), asym.EINVAL), (dict(freq=None), asym.EINVAL), (dict(kp=None), asym.EINVAL),
    (dict(cu=None), asym.EINVAL), (dict(q=None), asym.EINVAL), (dict(qo=None), asym.EINVAL), (dict(kp=P + 8), asym.EINVAL),
    (dict(qo=P + 2), asym.EINVAL), (dict(start=P + 2), asym.EINVAL), (dict(pos=P + 1), asym.EINVAL), (dict(kt=260), asym.EINVAL),
    (dict(qoh=-8), asym.EINVAL), (dict(T=2 ** 31 - 1), asym.EUNSUPPORTED), (dict(H=1 << 20), asym.EUNSUPPORTED),
    (dict(B=0), asym.OK), (dict(T=0), asym.OK)])
def test_append_refusals(change, want):
    assert code("asym_kv_append_bf16", *{**APPEND, **change}.values()) == want


TREE = dict(B=2, Hq=8, H=2, T=6, S=64, D=128, q=P, qt=1024, qh=128, kp=P, vp=P, pool=4, kt=P, vt=P, pph=2, cu=P, lens=P, mask=P, words=1,
            o=P, lse=None, scale=1.0, split=64, ws=None, wsb=0, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), asym.EINVAL), (dict(T=-1), asym.EINVAL), (dict(S=0), asym.EINVAL), (dict(S=65), asym.EINVAL), (dict(Hq=7), asym.EINVAL),
    (dict(D=64), asym.EUNSUPPORTED), (dict(split=33), asym.EINVAL), (dict(split=(1 << 20) + 32), asym.EINVAL), (dict(split=-32), asym.EINVAL),
    (dict(pool=0), asym.EINVAL), (dict(q=None), asym.EINVAL), (dict(lens=None), asym.EINVAL), (dict(o=P + 4), asym.EINVAL),
    (dict(lens=P + 1), asym.EINVAL), (dict(mask=P + 4), asym.EINVAL), (dict(words=0), asym.EINVAL), (dict(qt=1028), asym.EINVAL),
    (dict(qh=-128), asym.EINVAL), (dict(scale=float("nan")), asym.EINVAL), (dict(), asym.EINVAL), (dict(ws=P, wsb=16), asym.EINVAL),
    (dict(ws=P + 4, wsb=1 << 30), asym.EINVAL), (dict(B=1 << 20, S=1 << 30, pph=1 << 25), asym.EUNSUPPORTED),
    (dict(T=1 << 26), asym.EUNSUPPORTED), (dict(B=0), asym.OK), (dict(T=0), asym.OK)])
def test_tree_refusals(change, want):
    assert code("asym_attn_tree_paged_bf16", *{**TREE, **change}.values()) == want
    if want != asym.OK:
        assert asym.last_error().startswith("tree attention: ")


VERIFY = dict(B=2, T=6, V=100, bf16=0, target=P, trow=100, draft=P, drow=100, tokens=P, parents=P, cu=P, accept=P, final=P, path=P, count=P,
              token=P, ws=P, wsb=1 << 20, stream=None)
LONG = dict(V=20000, trow=20000, drow=20000)  # (shorter vocabularies need no workspace)


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), asym.EINVAL), (dict(T=-1), asym.EINVAL), (dict(V=0), asym.EINVAL), (dict(V=(1 << 30) + 1), asym.EUNSUPPORTED),
    (dict(trow=99), asym.EINVAL), (dict(drow=99), asym.EINVAL), (dict(target=None), asym.EINVAL), (dict(tokens=None), asym.EINVAL),
    (dict(final=None), asym.EINVAL), (dict(path=None), asym.EINVAL), (dict(target=P + 2), asym.EINVAL), (dict(bf16=1, draft=P + 1), asym.EINVAL),
    (dict(parents=P + 2), asym.EINVAL), (dict(LONG, ws=None), asym.EINVAL), (dict(LONG, wsb=8), asym.EINVAL), (dict(LONG, ws=P + 8), asym.EINVAL),
    (dict(B=1 << 22), asym.EUNSUPPORTED), (dict(B=0), asym.OK)])
def test_verify_refusals(change, want):
    assert code("asym_draft_verify", *{**VERIFY, **change}.values()) == want


KEEP = dict(R=4, H=2, pph=3, table=P, lens=P, refs=P, kp=P, vp=P + 64, page=8192, pool=100, n=5, rows=P, T=20, cu=P, path=P, count=P, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(R=0), asym.EINVAL), (dict(n=-1), asym.EINVAL), (dict(table=None), asym.EINVAL), (dict(kp=None), asym.EINVAL), (dict(vp=P), asym.EINVAL),
    (dict(page=2176), asym.EUNSUPPORTED), (dict(page=24), asym.EINVAL), (dict(T=-1), asym.EINVAL), (dict(rows=None), asym.EINVAL),
    (dict(cu=P + 1), asym.EINVAL), (dict(path=None), asym.EINVAL), (dict(count=None), asym.EINVAL), (dict(pool=0), asym.EINVAL),
    (dict(n=1 << 24), asym.EUNSUPPORTED), (dict(n=0, rows=None), asym.OK)])
def test_keep_refusals(change, want):
    assert code("asym_kv_keep", *{**KEEP, **change}.values()) == want


def test_workspaces():
    n = ctypes.c_size_t()
    assert code("asym_attn_tree_paged_workspace", 2, 8, 2, 6, 6400, 0, ctypes.byref(n)) == asym.OK and n.value > 0
    assert code("asym_attn_tree_paged_workspace", 2, 8, 2, 6, 64, 32, ctypes.byref(n)) == asym.OK and n.value > 0
    assert code("asym_attn_tree_paged_workspace", 2, 8, 2, 6, 64, 0, ctypes.byref(n)) == asym.OK and n.value == 0  # one launch
    assert code("asym_attn_tree_paged_workspace", 2, 8, 2, 6, 64, 0, None) == asym.EINVAL
    assert code("asym_attn_tree_paged_workspace", 2, 8, 3, 6, 64, 0, ctypes.byref(n)) == asym.EINVAL
    assert code("asym_attn_tree_paged_workspace", 0, 8, 2, 6, 64, 0, ctypes.byref(n)) == asym.OK and n.value == 0
    assert code("asym_draft_verify_workspace", 2, 6, 16385, ctypes.byref(n)) == asym.OK and n.value > 0
    assert code("asym_draft_verify_workspace", 2, 6, 16384, ctypes.byref(n)) == asym.OK and n.value == 0  # one launch
    assert code("asym_draft_verify_workspace", 2, 6, 1000, None) == asym.EINVAL


@pytest.mark.parametrize("big", [1 << 31, (1 << 32) + 64])
def test_sizes_past_32_bits_are_refused(big):
    for call in (lambda: asym._tree_workspace(1, 8, 8, 4, big, 0), lambda: asym._verify_workspace(1, big, 100)):
        with pytest.raises(ValueError, match="2\\^31"):
            call()
