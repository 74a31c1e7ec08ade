"""The paged cache and its attention without a GPU: pins of the oracle, refusals of the ABI and of the binding."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2309_15531_amd import binding as B
from tests.test_abi_cpu import A16, ODD, ctx  # noqa: F401  (the fixture)

F16, BF16, F32, MX4 = B.TYPE_F16, B.TYPE_BF16, B.TYPE_F32, B.TYPE_MX4
BYTE = ctypes.c_void_p(0x1001)


# ------------------------------------------------------------------------------------------ the oracle
def test_a_position_by_hand():
    """Key 0, 1, 2, .. 6 in a block of scale 2^0 (its largest is in [4, 8)), value twice that: the same codes at twice the scale."""
    cache = np.zeros((1, 1, 1, 34 * 64), np.uint8)
    k = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -1])[None, None]
    co.store(cache, k, 2 * k, [21])                             # 21: second half, g = 1, i = 1 + 4
    r = cache[0, 0, 0]
    assert r[21 * 32:21 * 32 + 5].tolist() == [0x10, 0x32, 0x54, 0x76, 0x0A] and r[:21 * 32].max() == 0
    values = r[1024:2048].reshape(4, 16, 8, 2)
    assert values[1, 0, 5].tolist() == [0x10, 0x32] and values[1, 1, 5].tolist() == [0x54, 0x76] and values[1, 2, 5].tolist() == [0x0A, 0]
    assert np.count_nonzero(values) == 5
    assert r[2048:2112].reshape(32, 2)[21].tolist() == [127, 127] and r[2112:].reshape(4, 2, 8)[1, :, 5].tolist() == [128, 127]
    assert all(np.array_equal(a, b) for a, b in zip(co.load(cache, [21, -1, 32], 9), (np.concatenate([m * k, 0 * k, 0 * k]) for m in (1, 2))))


@pytest.mark.parametrize("dim", [1, 33, 64, 80, 128, 200, 256])
def test_every_position_has_bytes_of_its_own(dim):
    cache = np.full((2, 2, 2, 34 * co.filled(dim)), 0xEE, np.uint8)
    r = np.random.default_rng(dim)
    k, v = r.standard_normal((2, 128, 2, dim))
    order = r.permutation(128)
    co.store(cache, k, v, order)
    whole = [co.codes(k[t, h], v[t, h]) for t in (0, 127) for h in (0, 1)]
    a, b = co.load(cache, order, dim)
    for (kc, ks, vc, vs), (t, h) in zip(whole, ((0, 0), (0, 1), (127, 0), (127, 1))):
        assert np.array_equal(a[t, h], (co.mo.VALUES[kc].reshape(-1, 32) * np.exp2(ks - 127.0)[:, None]).reshape(-1)[:dim])
        assert np.array_equal(b[t, h], (co.mo.VALUES[vc].reshape(-1, 32) * np.exp2(vs - 127.0)[:, None]).reshape(-1)[:dim])
    assert (np.abs(a - k) <= np.abs(k).max() / 4).all() and (np.abs(b - v) <= np.abs(v).max() / 4).all()


def test_scales_are_held_and_a_position_that_is_not_finite_is_marked():
    k = np.zeros((3, 1, 64))
    k[0, 0, 0], k[0, 0, 32] = 1e30, 1e-30
    k[1, 0, :] = 1.0
    v = k.copy()
    v[1, 0, 40] = np.inf
    cache = np.zeros((1, 1, 1, 34 * 64), np.uint8)
    co.store(cache, k, v, [0, 1, 2])
    a, b = co.load(cache, [0, 1, 2], 64)
    assert a[0, 0, 0] == 49152 and a[0, 0, 32] == 0 and np.isnan(a[1]).all() and (b[1] == 0).all() and (a[2] == 0).all()


def test_attention_by_hand():
    """Two positions with scores 0 and log 3: weights 1/4 and 3/4."""
    cache = np.zeros((3, 1, 1, 34 * 64), np.uint8)
    k, v = np.zeros((3, 1, 2)), np.zeros((3, 1, 2))
    k[1, 0, 0], v[0, 0, 1], v[1, 0, 0], v[2] = 1.0, 4.0, 4.0, np.nan
    co.store(cache, k, v, [64, 65, 66])
    q = np.full((4, 2, 2), 0.0)
    q[:, 0, 0] = np.log(3.0)
    table = np.array([[2], [0], [-1]])
    y, w, _ = co.attention(q, cache, table, [1, 2, 2, 3], [2, 0, 5], 2, 1.0)
    assert np.isnan(y[[0, 3]]).all() and np.allclose(y[1], [[3, 1], [2, 2]]) and np.array_equal(y[2], np.zeros((2, 2))) and np.allclose(w[1], y[1])
    y, _, _ = co.attention(q, cache, table, [0, 2, 2, 2], [3, 0, 0], 2, 1.0)
    assert np.allclose(y[0, 0], [3, 1]) and np.isnan(y[1]).all()          # the row of position 1 does not see the NaN of position 2
    y, _, _ = co.attention(q, cache, table, [0, 1, 1, 1], [2, 0, 0], 2, 1.0, window=1)
    assert np.allclose(y[0, 0], [4, 0])


def test_reserve_and_trim_by_hand():
    table = np.full((3, 3), 9, np.int32)
    r = co.reserve([31, 0, 32], [2, 0, 33], 32, table, [5, 6, 7, 8], 4, 40)
    assert r["table"].tolist() == [[9, 8, 9], [9, 9, 9], [9, 7, 6]] and r["offsets"] == [0, 2, 2, 35] and r["left"] == 1 and r["lacking"] == 0
    assert r["slots"][:4] == [9 * 32 + 31, 8 * 32, 7 * 32, 7 * 32 + 1] and r["slots"][34] == 6 * 32 and r["slots"][35:] == [-1] * 5
    assert r["positions"][:3] == [31, 32, 32] and r["lengths"] == [33, 0, 65]
    r = co.reserve([31, 0, 32], [2, 0, 33], 32, table, [5, 6, 7, 8], 2, 40)
    assert r["lacking"] == 1 and r["lengths"] == [31, 0, 32] and r["slots"] == [-1] * 40 and r["left"] == 2 and (r["table"] == 9).all()
    for held, added, tokens in (([31, 0, 64], [2, 0, 33], 40), ([31, 0, 32], [2, 0, 33], 34), ([31, -1, 32], [2, 0, 33], 40)):
        assert co.reserve(held, added, 32, table, [5, 6, 7, 8], 4, tokens)["lacking"] == -1
    t = co.trim([33, 0, 65], [32, 5, 0], 32, np.array([[9, 8, 9], [9, 9, 9], [4, 7, 6]]), [5, 0, 0, 0, 0, 0], 1)
    assert t["free"] == [5, 8, 4, 7, 6, 0] and t["lengths"] == [32, 0, 0] and t["left"] == 5


# ------------------------------------------------------------------------------------------ refusals
def test_sizes(ctx):
    lib = B.load_library()
    for pages, page, heads, dim in ((1, 32, 1, 1), (3, 64, 2, 65), (7, 256, 8, 128), (2, 32, 3, 129)):
        assert lib.adadim_mx4_cache_bytes(pages, page, heads, dim) == np.prod(B.mx4_cache_shape(pages, page, heads, dim))
    for bad in ((0, 32, 1, 64), (1, 16, 1, 64), (1, 48, 1, 64), (1, 32, 0, 64), (1, 32, 1, 257), (1, 32, 1, 0), (-1, 32, 1, 64)):
        assert lib.adadim_mx4_cache_bytes(*bad) == 0


@pytest.mark.parametrize("name", ["adadim_cache_reserve", "adadim_cache_trim"])
def test_page_refusals(ctx, name):
    reserve = name == "adadim_cache_reserve"

    def call(held=A16, change=A16, n=4, page=64, table=A16, width=8, free=A16, pool=9, count=A16, lengths=A16, left=A16, **more):
        if not reserve:
            return ctx.raw(name, held, change, n, page, table, width, free, pool, count, lengths, left)
        m = {"offsets": A16, "slots": A16, "positions": A16, "tokens": 5, "lacking": A16, **more}
        return ctx.raw(name, held, change, n, page, table, width, free, pool, count, lengths, m["offsets"], m["slots"], m["positions"], m["tokens"], left,
                       m["lacking"])
    for bad in ({"n": 0}, {"n": 4097}, {"page": 16}, {"page": 96}, {"page": 1 << 17}, {"width": 0}, {"pool": 0}, {"width": 1 << 25}, {"pool": 1 << 25}, {"n": 4096, "width": 1 << 19}):
        assert call(**bad) == B.EINVAL, bad
        assert name in ctx.last_error()
    pointers = ["held", "change", "table", "free", "count", "lengths", "left"]
    if reserve:
        assert call(tokens=-1) == B.EINVAL and call(tokens=(1 << 20) + 1) == B.EINVAL
        pointers += ["offsets", "slots", "positions", "lacking"]
    for p in pointers:
        assert call(**{p: None}) == B.ENULL, p
        assert call(**{p: BYTE}) == B.EALIGN, p


@pytest.mark.parametrize("name", ["adadim_mx4_cache_store", "adadim_mx4_cache_load"])
def test_row_refusals(ctx, name):
    def call(K=A16, V=A16, type=F16, tokens=4, ldk=128, ldv=128, slots=A16, cache=A16, pages=3, page=64, heads=2, dim=64):
        if name.endswith("store"):
            return ctx.raw(name, K, V, type, tokens, ldk, ldv, slots, cache, pages, page, heads, dim)
        return ctx.raw(name, slots, tokens, cache, pages, page, heads, dim, K, V, type, ldk, ldv)
    for bad in ({"type": MX4}, {"tokens": -1}, {"tokens": (1 << 20) + 1}, {"ldk": 127}, {"ldv": 127}, {"pages": 0}, {"pages": 1 << 25}, {"page": 33},
                {"heads": 0}, {"heads": 1025, "ldk": 1 << 20, "ldv": 1 << 20}, {"dim": 0}, {"dim": 257, "ldk": 514, "ldv": 514},
                {"tokens": 1 << 20, "heads": 512, "dim": 1, "ldk": 512, "ldv": 512}):
        assert call(**bad) == B.EINVAL, bad
    for p in ("K", "V", "slots", "cache"):
        assert call(**{p: None}) == B.ENULL and call(**{p: BYTE}) == B.EALIGN, p
    assert call(cache=ODD) == B.EALIGN
    assert call(tokens=0, K=None, V=None, slots=None, cache=None) == B.OK


def test_attention_refusals(ctx):
    def call(Q=A16, type=F16, tokens=4, ldq=512, q_heads=8, cache=A16, pages=3, page=64, heads=2, dim=64, table=A16, width=5, n=2, offsets=A16, lengths=A16,
             Y=A16, y_type=F16, ldy=512, scale=0.125, causal=1, window=0):
        return ctx.raw("adadim_mx4_attention", Q, type, tokens, ldq, q_heads, cache, pages, page, heads, dim, table, width, n, offsets, lengths, Y, y_type,
                       ldy, ctypes.c_float(scale), causal, window, 0, 0)
    for bad in ({"type": F32}, {"type": MX4}, {"y_type": MX4}, {"tokens": -1}, {"tokens": (1 << 20) + 1}, {"ldq": 511}, {"ldy": 511}, {"q_heads": 7},
                {"q_heads": 0}, {"pages": 0}, {"pages": 1 << 25}, {"page": 16}, {"heads": 0}, {"dim": 0}, {"dim": 257}, {"width": 0}, {"width": 1 << 25},
                {"n": 0}, {"n": 4097}, {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"causal": 2}, {"window": -1},
                {"tokens": 1 << 20, "q_heads": 1024, "heads": 1024, "ldq": 1 << 16, "ldy": 1 << 16},
                {"tokens": 1 << 20, "q_heads": 192, "heads": 192, "ldq": 12288, "ldy": 12288}):
        assert call(**bad) == B.EINVAL, bad
    for p in ("Q", "cache", "table", "offsets", "lengths", "Y"):
        assert call(**{p: None}) == B.ENULL and call(**{p: BYTE}) == B.EALIGN, p
    assert call(cache=ODD) == B.EALIGN
    assert call(tokens=0, Q=None, cache=None, table=None, offsets=None, lengths=None, Y=None) == B.OK


def test_binding_refuses_host_tensors(ctx):
    """(What it refuses of device tensors is in the GPU tests: a host tensor is refused before its shape is looked at.)"""
    cache = torch.zeros(B.mx4_cache_shape(2, 64, 2, 64), dtype=torch.uint8)
    rows, ints = torch.zeros((3, 128)), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError):
        ctx.adadim_mx4_cache_store(rows, rows, ints, cache)
    with pytest.raises(TypeError):
        ctx.adadim_mx4_cache_load(ints, cache, rows, rows)
    with pytest.raises(TypeError):
        ctx.adadim_mx4_attention(rows.half(), cache, ints[None], ints[:2], ints[:1], rows.half(), 64)
    with pytest.raises(TypeError):
        ctx.adadim_cache_trim(ints, ints, 64, ints[:, None], ints, ints[:1], ints, ints[:1])
    with pytest.raises(TypeError):
        ctx.adadim_cache_reserve(ints, ints, 64, ints[:, None], ints, ints[:1], ints, torch.zeros(4, dtype=torch.int32), ints, ints, ints[:1], ints[:1])
