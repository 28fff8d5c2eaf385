"""Pins of the 4-bit cache's and the pages' oracles, and the new calls' refusals, on the CPU."""
import ctypes
import itertools

import numpy as np
import pytest

import paper_2609_24270_amd as asym
from oracle import kv_fp4, kv_pages, prompt


def bf16(x):
    u = np.atleast_1d(np.asarray(x, dtype=np.float32)).view(np.uint32)
    assert np.all(u & 0xFFFF == 0), "not a bf16 value"
    return (u >> 16).astype(np.uint16)


def row(first, rest=0.0):
    x = np.full(128, rest, np.float32)
    x[:len(first)] = first
    return bf16(x)[None]


def test_every_code_of_a_block_is_kept():
    # a block whose largest value is 6: the scale is 1, and the grid's own values come back
    codes, scales = kv_fp4.quantise(row([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6]))
    assert codes[0, :16].tolist() == list(range(16)) and scales[0, 0] == 127
    assert kv_fp4.value(codes, scales)[0, :8].tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6]


def test_ties_go_to_the_even_code_and_large_values_saturate():
    codes, _ = kv_fp4.quantise(row([7.96875, .25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.03125, 6.5]))
    assert codes[0, :10].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 7, 7]


def test_scales_of_extreme_blocks():
    big = 2.0 ** 127 * 1.9921875
    for x, s in [(big, 252), (2.0 ** -126, 2), (2.0 ** -133, 2), (0.0, 2), (8.0, 128), (1.0, 125), (2.0 ** -122, 3)]:
        codes, scales = kv_fp4.quantise(row([x]))
        assert scales[0, 0] == s, x
        assert np.all(np.isfinite(kv_fp4.value(codes, scales)))
    for x in (np.inf, -np.inf, np.nan):
        u = row([1.0, 2.0])
        u[0, 3] = np.array([x], np.float32).view(np.uint32)[0] >> 16
        codes, scales = kv_fp4.quantise(u)
        assert scales[0].tolist() == [255, 2, 2, 2] and not codes[0, :32].any()
        assert np.isnan(kv_fp4.value(codes, scales)[0, :32]).all()


@pytest.mark.parametrize("values", [False, True])
def test_a_page_has_one_place_for_everything(values):
    byte, nib, sc = kv_fp4.places(values)
    used = set(zip(byte.ravel().tolist(), nib.ravel().tolist()))
    assert used == set(itertools.product(range(2048), range(2)))
    assert set(sc.ravel().tolist()) == set(range(2048, 2176))
    rng = np.random.default_rng(1)
    page = np.zeros(2176, np.uint8)
    codes, scales = rng.integers(0, 16, (32, 128)).astype(np.uint8), rng.integers(0, 255, (32, 4)).astype(np.uint8)
    for t in rng.permutation(32):
        kv_fp4.put(page, t, codes[t], scales[t], values)
    c, s = kv_fp4.get(page, values)
    assert np.array_equal(c, codes) and np.array_equal(s, scales)


def test_value_error_bound():
    # of values in [X / 4, 6 X] (X the scale) the format keeps all but a quarter step: at most 1/6 relative above X / 2
    x = np.random.default_rng(2).standard_normal((64, 128)).astype(np.float32)
    u = (x.view(np.uint32) >> 16).astype(np.uint16)
    x = (u.astype(np.uint32) << 16).view(np.float32).astype(float)
    codes, scales = kv_fp4.quantise(u)
    X = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=1)
    err = np.abs(kv_fp4.value(codes, scales) - x)
    assert np.all(err <= np.where(np.abs(x) > 6 * X, 2 * X, np.where(np.abs(x) > 4 * X, X, np.where(
        np.abs(x) > 2 * X, X / 2, X / 4))))


def test_prompt_oracle_pins():
    q = np.zeros((3, 1, 2))
    v = np.array([[[1., 2.]], [[3., 4.]], [[5., 9.]]])
    O, lse, A, N = prompt.prompt_attention(q, np.ones_like(v), v, [0, 3], [0, 3], 1.0)
    assert np.allclose(O[:, 0], [[1, 2], [2, 3], [3, 5]]) and np.allclose(lse[:, 0], np.log([1, 2, 3]))
    O, lse, _, _ = prompt.prompt_attention(q, np.ones((1, 1, 2)), v[:1], [0, 3], [0, 1], 1.0)  # two rows see nothing
    assert np.all(O[:2] == 0) and np.all(lse[:2] == -np.inf) and np.allclose(O[2, 0], [1, 2])
    v[2] = np.nan
    O, _, _, _ = prompt.prompt_attention(q, np.ones_like(v), v, [0, 3], [0, 3], 1.0)
    assert np.all(np.isfinite(O[:2])) and np.all(np.isnan(O[2]))


def test_pages_oracle_pins():
    c = kv_pages.Cache(np.full((4, 1, 4), -1), np.zeros(4, int), np.zeros(10, int), [np.arange(10)])
    assert c.extend([0, 2, 0], [40, 32, 90]) == (3, 0)            # the second request for row 0 is left out
    assert c.table[0, 0].tolist() == [0, 1, -1, -1] and c.table[2, 0, 0] == 2 and c.lens.tolist() == [40, 0, 32, 0]
    assert c.fork([0, 2], [1, 3]) == (1, 0)                       # page 0 shared, page 1 copied to 3; page 2 shared
    assert c.table[1, 0].tolist() == [0, 3, -1, -1] and c.refs[:4].tolist() == [2, 1, 2, 1]
    assert c.pools[0][3] == 1
    c.free([0])
    assert c.refs[:4].tolist() == [1, 0, 2, 1]
    assert c.compact() == (1, 3)                                  # page 3 into 1
    assert c.table[1, 0].tolist() == [0, 1, -1, -1] and c.refs[:4].tolist() == [1, 1, 2, 0]
    assert c.extend([0], [999]) == (0, 0) and c.extend([0, 2], [128, 128]) == (7, 0)
    assert c.extend([1], [100]) == (0, 2)                         # too few: nothing changes
    assert c.lens[1] == 40


# ---- refusals, before anything touches a device ----------------------------------------------------------------------

P = 4096  # an aligned address that no refused call reads


def code(name, *args):
    return getattr(asym.load_library(), name)(*args)


PREFILL = dict(B=1, Hq=4, Hkv=2, D=128, Tq=8, Tk=8, q=P, qt=512, qh=128, k=P, kt=256, kh=128, v=P, vt=256, vh=128, o=P,
               lse=None, cu_q=P, cu_k=P, scale=1.0, causal=1, mapping=0, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), asym.EINVAL), (dict(Tq=-1), asym.EINVAL), (dict(Hq=0), asym.EINVAL), (dict(Hq=5), asym.EINVAL),
    (dict(D=64), asym.EUNSUPPORTED), (dict(mapping=3), asym.EINVAL), (dict(scale=float("inf")), asym.EINVAL),
    (dict(q=None), asym.EINVAL), (dict(k=None), asym.EINVAL), (dict(o=None), asym.EINVAL), (dict(cu_q=None), asym.EINVAL),
    (dict(q=P + 2), asym.EINVAL), (dict(o=P + 8), asym.EINVAL), (dict(lse=P + 2), asym.EINVAL), (dict(cu_k=P + 1), asym.EINVAL),
    (dict(qt=516), asym.EINVAL), (dict(kh=-128), asym.EINVAL), (dict(kt=0), asym.EUNSUPPORTED), (dict(vt=120), asym.EUNSUPPORTED),
    (dict(kt=1 << 24), asym.EUNSUPPORTED), (dict(Tq=2 ** 31 - 1, Hq=512, Hkv=8), asym.EUNSUPPORTED),
    (dict(Tk=4096), asym.EINVAL), (dict(Tk=4096, ws=P, ws_bytes=4096), asym.EINVAL),
    (dict(Tk=4096, ws=P + 8, ws_bytes=1 << 30), asym.EINVAL)])
def test_prefill_refusals(change, want):
    assert code("asym_attn_prefill_bf16", *{**PREFILL, **change}.values()) == want
    assert asym.last_error().startswith("prefill: ")


def test_prefill_workspace():
    import ctypes
    n = ctypes.c_size_t(7)
    sizes = lambda *a: (code("asym_attn_prefill_workspace", *a, ctypes.byref(n)), n.value)
    # a piece is 128 rows of 130 values; few rows over many keys are cut, everything else is not
    assert sizes(1, 4, 2, 8, 4096) == (asym.OK, (1 + 512 // 2) * 2 * 128 * 130 * 4)
    assert sizes(1, 4, 2, 8, 8) == sizes(64, 32, 8, 64, 1 << 20) == sizes(1, 32, 8, 16384, 16384) == (asym.OK, 0)
    assert sizes(0, 4, 2, 8, 4096) == sizes(1, 4, 2, 0, 4096) == (asym.OK, 0)
    for bad in ((-1, 4, 2, 8, 8), (1, 5, 2, 8, 8), (1, 4, 0, 8, 8), (1, 4, 2, -1, 8), (1, 4, 2, 8, -1)):
        assert sizes(*bad)[0] == asym.EINVAL
    assert code("asym_attn_prefill_workspace", 1, 4, 2, 8, 8, None) == asym.EINVAL


def test_empty_calls_do_nothing():
    assert code("asym_attn_prefill_bf16", *{**PREFILL, "B": 0, "q": None}.values()) == asym.OK
    assert code("asym_attn_prefill_bf16", *{**PREFILL, "Tq": 0}.values()) == asym.OK
    assert code("asym_kv_write_fp4", *{**WRITE, "T": 0}.values()) == asym.OK
    assert code("asym_kv_read_fp4", *{**READ, "B": 0}.values()) == asym.OK
    assert code("asym_attn_decode_paged_fp4", *{**DECODE, "B": 0}.values()) == asym.OK
    assert code("asym_kv_free", 1, 1, 1, P, P, P, 4, 0, None, None) == asym.OK


WRITE = dict(B=1, H=2, T=8, k=P, kt=256, kh=128, v=P, vt=256, vh=128, kp=P, vp=P, pool=4, kt_=P, vt_=P, pph=2, cu=P, start=P,
             stream=None)
READ = dict(B=1, H=2, T=8, kp=P, vp=P, pool=4, kt_=P, vt_=P, pph=2, cu=P, start=P, k=P, v=P, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), asym.EINVAL), (dict(H=0), asym.EINVAL), (dict(T=-5), asym.EINVAL), (dict(pph=0), asym.EINVAL),
    (dict(pool=0), asym.EINVAL), (dict(pool=1 << 31), asym.EINVAL), (dict(pph=1 << 26), asym.EUNSUPPORTED),
    (dict(kp=None), asym.EINVAL), (dict(cu=None), asym.EINVAL), (dict(kp=P + 8), asym.EINVAL), (dict(start=P + 2), asym.EINVAL),
    (dict(k=None), asym.EINVAL), (dict(v=P + 2), asym.EINVAL), (dict(T=2 ** 31 - 1, H=64), asym.EUNSUPPORTED)])
def test_cache_refusals(change, want):
    assert code("asym_kv_write_fp4", *{**WRITE, **change}.values()) == want
    assert code("asym_kv_read_fp4", *{**READ, **change}.values()) == want


@pytest.mark.parametrize("change", [dict(kt=260), dict(vh=-8)])
def test_write_strides(change):
    assert code("asym_kv_write_fp4", *{**WRITE, **change}.values()) == asym.EINVAL


DECODE = dict(B=2, Hq=8, Hkv=2, S=64, D=128, q=P, kp=P, vp=P, pool=4, kt=P, vt=P, pph=2, lens=P, o=P, lse=None, scale=1.0,
              split=64, ws=None, wsb=0, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(B=-1), asym.EINVAL), (dict(S=0), asym.EINVAL), (dict(S=65), asym.EINVAL), (dict(Hq=7), asym.EINVAL),
    (dict(Hq=34), asym.EUNSUPPORTED), (dict(D=64), asym.EUNSUPPORTED), (dict(split=33), asym.EINVAL),
    (dict(split=(1 << 20) + 32), asym.EINVAL), (dict(split=-32), asym.EINVAL), (dict(pool=0), asym.EINVAL), (dict(q=None), asym.EINVAL),
    (dict(lens=None), asym.EINVAL), (dict(o=P + 4), asym.EINVAL), (dict(lens=P + 1), asym.EINVAL),
    (dict(scale=float("nan")), asym.EINVAL), (dict(split=32), asym.EINVAL), (dict(split=32, ws=P, wsb=16), asym.EINVAL),
    (dict(split=32, ws=P + 4, wsb=1 << 20), asym.EINVAL), (dict(B=1 << 20, S=1 << 30, pph=1 << 25), asym.EUNSUPPORTED)])
def test_decode_refusals(change, want):
    assert code("asym_attn_decode_paged_fp4", *{**DECODE, **change}.values()) == want
    assert asym.last_error().startswith("fp4 attention: ")


def test_decode_plan():
    p = asym.attn_decode_paged_fp4_plan(16, 32, 8, 8000)
    assert p["tasks"] == 2048 and p["split_tokens"] == -(-16 * 8 * 250 // 2048) * 32
    assert p["workspace_bytes"] >= 2048 * 2 * 4 * 130 * 4 + 16 * 8 * 8
    assert p["n_splits"] == 126  # 250 pages in shares of two, which need not begin where they do
    one = asym.attn_decode_paged_fp4_plan(1, 8, 8, 32)
    assert one["tasks"] == 8 and one["n_splits"] == 1
    assert asym.attn_decode_paged_fp4_plan(1, 8, 8, 320, split_tokens=96)["tasks"] == 27
    short = asym.attn_decode_paged_fp4_plan(256, 32, 8, 300)  # a wave a head
    assert short["tasks"] == 2048 and short["n_splits"] == 1 and short["workspace_bytes"] == 0
    with pytest.raises(asym.AsymError):
        asym.attn_decode_paged_fp4_plan(1, 8, 8, 0)
    assert code("asym_attn_decode_paged_fp4_plan", 1, 8, 8, 32, 128, 0, None) == asym.EINVAL


def ws_bytes(op, **kw):
    n = ctypes.c_size_t()
    a = dict(R=4, H=2, pph=3, pool=100, n=5)
    a.update(kw)
    rc = code("asym_kv_pages_workspace", op, *a.values(), ctypes.byref(n))
    return rc, n.value


def test_pages_refusals():
    lib = asym.load_library()
    for op in (asym.KV_EXTEND, asym.KV_FORK, asym.KV_COMPACT):
        rc, n = ws_bytes(op)
        assert rc == asym.OK and n >= 400
        for bad in (dict(R=0), dict(H=0), dict(pph=0), dict(pool=0), dict(n=-1), dict(pool=1 << 31)):
            assert ws_bytes(op, **bad)[0] == asym.EINVAL
    assert ws_bytes(7)[0] == asym.EINVAL
    big = 1 << 20
    ext = dict(R=4, H=2, pph=3, table=P, lens=P, refs=P, pool=100, n=5, rows=P, new=P, status=P, ws=P, wsb=big, stream=None)
    for change, want in [(dict(R=0), -1), (dict(n=-1), -1), (dict(table=None), -1), (dict(lens=P + 2), -1), (dict(rows=None), -1),
                         (dict(new=P + 1), -1), (dict(status=P + 2), -1), (dict(ws=None), -1), (dict(wsb=100), -1),
                         (dict(ws=P + 4), -1), (dict(pool=0), -1), (dict(pph=1 << 26), -3), (dict(n=1 << 24), -3),
                         (dict(R=1 << 10, H=1 << 6, pph=1 << 15), -3), (dict(R=2, H=1 << 16, pph=1 << 20), -3)]:
        assert lib.asym_kv_extend(*{**ext, **change}.values()) == want, change
    fork = dict(R=4, H=2, pph=3, table=P, lens=P, refs=P, kp=P, vp=P + 64, page=2176, pool=100, n=5, src=P, dst=P, status=None,
                ws=P, wsb=big, stream=None)
    for change in (dict(kp=None), dict(kp=P + 8), dict(vp=P), dict(page=0), dict(page=24), dict(src=None), dict(dst=P + 2),
                   dict(wsb=0)):
        assert lib.asym_kv_fork(*{**fork, **change}.values()) == -1, change
    assert lib.asym_kv_free(4, 2, 3, P, P, P, 100, 2, None, None) == -1
    assert lib.asym_kv_free(4, 2, 3, P, P, None, 100, 2, P, None) == -1
    comp = dict(R=4, H=2, pph=3, table=P, refs=P, kp=P, vp=None, page=8192, pool=100, status=None, ws=P, wsb=big, stream=None)
    for change in (dict(refs=None), dict(kp=None), dict(vp=P), dict(page=8), dict(status=P + 1), dict(ws=None), dict(wsb=64)):
        assert lib.asym_kv_compact(*{**comp, **change}.values()) == -1, change


@pytest.mark.parametrize("big", [1 << 31, (1 << 32) + 64])
def test_sizes_past_32_bits_are_refused(big):
    # (the C ABI's sizes are 32-bit integers: 2^32 + 64 would arrive as 64)
    for call in (lambda: asym.attn_decode_paged_fp4_plan(1, 8, 8, big), lambda: asym.attn_decode_paged_fp4_plan(big, 8, 8, 64),
                 lambda: asym.attn_decode_paged_fp4_plan(1, 8, 8, 640, split_tokens=big),
                 lambda: asym._fp4_plan_workspace(1, 8, 8, big, 0), lambda: asym._prefill_workspace(1, 8, 8, 64, big),
                 lambda: asym._pages_workspace(asym.KV_EXTEND, big, 1, 1, 100, 5), lambda: asym._sizes(1, big)):
        for _ in range(2):  # (nothing is kept of a refused call)
            with pytest.raises(ValueError, match="2\\^31"):
                call()
