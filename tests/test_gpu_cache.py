"""The paged cache of keys and values in mx4 and the attention over it against the oracle, through the C ABI.

Whole numbers, codes and scales are equal bit for bit.  Tolerance of the attention, with y = sum_j w_j v_j, A = sum_j w_j |v_j| and n positions:
  scores     D products exact in fp32's range, summed in fp32 (2 D 2^-24 of the sum of magnitudes S for sums that may truncate), then the
             product with scale log2(e) and the difference to the maximum, two roundings of at most 2 S: 4 x 2^-24 S.  As an error of the exponent of
             2 it is 1.443 times that and comes back by log 2.  So w_j is off by (2 D + 4) 2^-24 S, and its normalized value by twice that
  2^x        2^-22 of itself, and as much again from the raised maxima's factors (each at least 2^7: fewer than 37 of them): 2^-16 at the most
  fp16       half a step of 11 bits, 2^-11; below 2^-14 half of 2^-24, which is 2^-33 of the row's largest p (that is at least 2^8), and the
             row's sum is at least the largest: n 2^-33 max |v|
  sums       n terms in fp32 for the numerator and for the sum: 4 n 2^-24
  result     half a unit of its type, and of fp16's smallest subnormal
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2309_15531_amd import binding as B
from test_gpu_mx4 import TINY, TYPES, UNIT, Guarded, host, pitched

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


def rng(*seed):
    return np.random.default_rng([37, *seed])


def ints(a):
    return torch.as_tensor(np.asarray(a, dtype=np.int32)).cuda()


def rounded(a, dtype):
    """a as the type holds it, in fp64."""
    return torch.as_tensor(a).to(TYPES[dtype]).double().numpy()


# ------------------------------------------------------------------------------------------ pages
def reserve(ctx, held, added, page, table, free, count, tokens):
    n = len(held)
    t, out = ints(table), {k: Guarded((m,), torch.int32) for k, m in (("lengths", n), ("offsets", n + 1), ("slots", tokens), ("positions", tokens), ("left", 1),
                                                                      ("lacking", 1))}
    ctx.adadim_cache_reserve(ints(held), ints(added), page, t, ints(free), ints([count]), *(out[k].t for k in ("lengths", "offsets", "slots", "positions", "left",
                                                                                                            "lacking")))
    r = {k: v.check().tolist() for k, v in out.items()}
    return {**r, "table": t.cpu().numpy(), "left": r["left"][0], "lacking": r["lacking"][0]}


def same(got, want):
    assert got.keys() == want.keys()
    for k in want:
        assert np.array_equal(np.asarray(got[k]), np.asarray(want[k])), k


@pytest.mark.parametrize("n,page,most,tokens", [(1, 32, 1, 1), (1, 64, 300, 300), (5, 32, 40, 200), (63, 64, 1, 63), (64, 128, 3, 200), (300, 32, 70, 20000),
                                                (1024, 64, 1, 1024), (1025, 64, 2, 4096), (1500, 32, 5, 4097), (4096, 64, 1, 5000), (3, 256, 0, 0),
                                                (7, 32, 5000, 40000)])
def test_reserve_is_the_oracles(ctx, n, page, most, tokens):
    r = rng(1, n, page)
    held = r.integers(0, 5 * page, n) * (r.random(n) < 0.8)
    held[r.random(n) < 0.2] //= page
    held[r.random(n) < 0.3] //= page
    held = held // 1
    held[: n // 3] = held[: n // 3] // page * page                # on a page's edge
    added = r.integers(0, most + 1, n) if most > 1 else np.full(n, most)
    width = int((held + added).max() + page - 1) // page + 1
    pool = int(sum(-(-(h + a) // page) for h, a in zip(held, added))) + 5
    ids = r.permutation(pool + 9)
    table = np.full((n, width), -7, np.int32)
    at = 0
    for s in range(n):
        k = -(-int(held[s]) // page)
        table[s, :k] = ids[at:at + k]
        at += k
    free = np.append(ids[at:], [-5] * 4)
    free = free[:pool] if len(free) >= pool else np.append(free, [-5] * (pool - len(free)))
    count = min(len(ids) - at, pool)
    assert added.sum() <= tokens
    same(reserve(ctx, held, added, page, table, free, count, tokens), co.reserve(held.tolist(), added.tolist(), page, table, free, count, tokens))


@pytest.mark.parametrize("held,added,count,tokens", [
    ([31, 0, 32], [2, 0, 33], 2, 40), ([31, 0, 32], [2, 0, 33], 0, 40), ([31, 0, 96], [2, 0, 33], 4, 40), ([31, 0, 32], [2, 0, 33], 4, 34),
    ([31, -1, 32], [2, 0, 33], 4, 40), ([31, 0, 32], [2, -5, 33], 4, 40), ([31, 0, 32], [2, 2 ** 31 - 1, 2 ** 31 - 1], 4, 40),
    ([31, 2 ** 31 - 1, 32], [2, 1, 3], 4, 40), ([31, 0, 32], [2, 0, 33], 2, 5000), ([31, 0, 32], [2, 0, 33], -3, 40)])
def test_reserve_takes_all_or_nothing(ctx, held, added, count, tokens):
    table = np.arange(12).reshape(3, 4).astype(np.int32)
    got = reserve(ctx, held, added, 32, table, [20, 21, 22, 23, 24], count, tokens)
    want = co.reserve(held, added, 32, table, [20, 21, 22, 23, 24], max(count, 0), tokens)
    assert want["lacking"] != 0
    same(got, want)


@pytest.mark.parametrize("n,page,long", [(1, 32, 1), (1, 32, 3000), (5, 64, 700), (64, 64, 3000), (300, 32, 5000), (300, 32, 9000), (1500, 32, 50), (4096, 64, 300)])
def test_trim_is_the_oracles(ctx, n, page, long):
    r = rng(2, n, page)
    held = r.integers(0, long + 1, n)
    kept = np.where(r.random(n) < 0.3, 0, held - r.integers(-3, 6, n))
    width = -(-long // page)
    pages = [-(-int(h) // page) for h in held]
    pool = sum(pages) + 6
    ids = r.permutation(pool)
    table = np.full((n, width), -7, np.int32)
    at = 0
    for s in range(n):
        table[s, :pages[s]] = ids[at:at + pages[s]]
        at += pages[s]
    free = np.append(ids[at:], [-5] * at)
    for alias in (False, True):
        h, f, c = ints(held), ints(free), ints([pool - at])
        lengths, left = (h, c) if alias else (torch.empty_like(h), torch.empty_like(c))
        ctx.adadim_cache_trim(h, ints(kept), page, ints(table), f, c, lengths, left)
        want = co.trim(held.tolist(), kept.tolist(), page, table, free, pool - at)
        assert f.tolist() == want["free"] and lengths.tolist() == want["lengths"] and left.tolist() == [want["left"]]


def test_trim_drops_what_the_pool_has_no_room_for(ctx):
    table = np.arange(30).reshape(3, 10).astype(np.int32)
    f, c = torch.full((7,), -5, dtype=torch.int32, device="cuda"), ints([2])
    guard = f.clone()
    lengths, left = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    ctx.adadim_cache_trim(ints([320, 5, 2 ** 31 - 1]), ints([250, -9, 2 ** 31 - 1]), 32, ints(table), f[:4], c, lengths, left)
    want = co.trim([320, 5, 2 ** 31 - 1], [250, -9, 2 ** 31 - 1], 32, table, [-5] * 4, 2)
    assert f[:4].tolist() == want["free"] and f[4:].tolist() == guard[4:].tolist() and lengths.tolist() == want["lengths"] and left.tolist() == [4]


@pytest.mark.parametrize("tokens", [100, 9000])
def test_lengths_and_count_in_place(ctx, tokens):
    """A batch that grows step by step with one array of lengths and one count, and gives all back."""
    r = rng(3, tokens)
    n, page, width, pool = 9, 32, 60, 400
    lengths, count, table = ints([0] * n), ints([pool]), ints(np.full((n, width), -1))
    free = ints(r.permutation(pool))
    want_table, want_free, want_count, held = np.full((n, width), -1, np.int32), free.tolist(), pool, [0] * n
    offsets, slots, positions, lacking = (torch.empty(k, dtype=torch.int32, device="cuda") for k in (n + 1, tokens, tokens, 1))
    for step in range(6):
        added = r.integers(0, 90 if step else 300, n).tolist()
        if sum(added) > tokens:
            added = [a * tokens // sum(added) for a in added]
        ctx.adadim_cache_reserve(lengths, ints(added), page, table, free, count, lengths, offsets, slots, positions, count, lacking)
        want = co.reserve(held, added, page, want_table, want_free, want_count, tokens)
        assert lacking.item() == 0 and slots.tolist() == want["slots"] and positions.tolist() == want["positions"] and offsets.tolist() == want["offsets"]
        want_table, want_count, held = want["table"], want["left"], want["lengths"]
        assert np.array_equal(table.cpu().numpy(), want_table) and count.item() == want_count and lengths.tolist() == held
        kept = [max(0, h - int(x)) for h, x in zip(held, r.integers(0, 40, n))]
        ctx.adadim_cache_trim(lengths, ints(kept), page, table, free, count, lengths, count)
        want = co.trim(held, kept, page, want_table, want_free, want_count)
        want_free, want_count, held = want["free"], want["left"], want["lengths"]
        assert lengths.tolist() == held and count.item() == want_count and free.tolist() == want_free
    ctx.adadim_cache_trim(lengths, ints([0] * n), page, table, free, count, lengths, count)
    assert count.item() == pool and sorted(free.tolist()) == list(range(pool))


# ------------------------------------------------------------------------------------------ store, load
@pytest.mark.parametrize("x", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 1, 32), (5, 2, 64, 32), (33, 3, 80, 64), (40, 1, 33, 32), (70, 2, 128, 128), (9, 5, 100, 64),
                                                   (37, 2, 256, 32), (21, 1, 200, 64), (8300, 1, 64, 256), (1100, 8, 128, 64), (300, 32, 40, 32)])
def test_store_and_load_are_the_oracles(ctx, tokens, heads, dim, page, x):
    r = rng(4, tokens, heads, dim)
    pages = -(-tokens // page) + 2
    slots = r.permutation(pages * page)[:tokens] if tokens < 200 else (np.arange(tokens) + 7)
    slots[r.random(tokens) < 0.05] = -1
    if tokens > 2:
        slots[2] = pages * page
    k, v = (r.standard_normal((tokens, heads * dim)) * np.exp2(r.integers(-30, 14, (tokens, 1))) for _ in range(2))
    k[r.random(k.shape) < 0.05] = 0.0
    kd, vd = pitched(k, TYPES[x], 3), pitched(v, TYPES[x], 0)
    if tokens > 4:
        kd[1, 0], vd[3, heads * dim - 1] = float("nan"), float("-inf")
    cache = Guarded(B.mx4_cache_shape(pages, page, heads, dim), torch.uint8)
    cache.t.fill_(0xEE)
    ctx.adadim_mx4_cache_store(kd, vd, ints(slots), cache.t)
    want = np.full(cache.t.shape, 0xEE, np.uint8)
    some = np.arange(tokens) if tokens < 400 else r.choice(tokens, 300, replace=False)
    ka, va = (host(t).astype(np.float64).reshape(tokens, heads, dim) for t in (kd, vd))
    if tokens < 400:
        co.store(want, ka, va, slots)
        assert np.array_equal(cache.check().cpu().numpy(), want)
    else:
        co.store(want, ka[some], va[some], slots[some])
    for y in ("f32", x):
        yk, yv = pitched(np.zeros((len(some), heads * dim)), TYPES[y], 5), pitched(np.zeros((len(some), heads * dim)), TYPES[y], 1)
        yk.fill_(7.0)
        yv.fill_(7.0)
        ctx.adadim_mx4_cache_load(ints(slots[some]), cache.t, yk, yv)
        for got, ref in zip((yk, yv), co.load(want, slots[some], dim)):
            assert np.array_equal(host(got).astype(np.float64).reshape(ref.shape), ref, equal_nan=True)
    cache.check()


def test_positions_beside_the_stored_ones_stay(ctx):
    r = rng(5)
    for dim in (64, 128, 256):
        cache = torch.from_numpy(r.integers(0, 256, B.mx4_cache_shape(3, 32, 2, dim)).astype(np.uint8)).cuda()
        want = cache.cpu().numpy().copy()
        for slots in ([5], [40, 41, 63], [95]):
            k, v = r.standard_normal((2, len(slots), 2 * dim)).astype(np.float32)
            ctx.adadim_mx4_cache_store(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), ints(slots), cache)
            co.store(want, k.reshape(-1, 2, dim), v.reshape(-1, 2, dim), slots)
            assert np.array_equal(cache.cpu().numpy(), want)


# ------------------------------------------------------------------------------------------ attention
def make_cache(r, pages, page, heads, dim, garbage=True):
    """A cache whose bytes are any at all but for the scales of the values' magnitudes, as store leaves them; the rest of a pool may hold what it likes."""
    shape = B.mx4_cache_shape(pages, page, heads, dim)
    full = co.filled(dim)
    c = r.integers(0, 256, shape).astype(np.uint8)
    c[..., 32 * full:] = r.integers(123, 129, (*shape[:3], 2 * full))
    return c


def zero_fill(c, dim):
    """Elements beyond dim as store leaves them: codes and scales of zeros."""
    full = co.filled(dim)
    if dim == full:
        return
    e = np.arange(full)
    keep = e < dim
    k = c[..., :16 * full].reshape(*c.shape[:3], 32, full // 2)
    nib = np.stack([k & 15, k >> 4], -1).reshape(*c.shape[:3], 32, full) * keep
    c[..., :16 * full] = (nib[..., 0::2] | nib[..., 1::2] << 4).reshape(*c.shape[:3], -1)
    unit = full // 16
    v = c[..., 16 * full:32 * full].reshape(*c.shape[:3], 4, 16, 8, unit // 2)
    nib = np.stack([v & 15, v >> 4], -1).reshape(*c.shape[:3], 4, 16, 8, unit)
    nib = nib * keep.reshape(16, unit)[:, None, :]
    c[..., 16 * full:32 * full] = (nib[..., 0::2] | nib[..., 1::2] << 4).reshape(*c.shape[:3], -1)


def batch(r, lengths, page, pages, width):
    table = np.full((len(lengths), width), -1, np.int32)
    ids = r.permutation(pages)
    at = 0
    for s, n in enumerate(lengths):
        k = -(-n // page)
        table[s, :k] = ids[at:at + k]
        at += k
    return table


def poison(c, table, lengths, page, dim):
    """What lies behind a sequence's last position: NaN and infinite scales, any codes."""
    full = co.filled(dim)
    used = np.zeros((c.shape[0], page), bool)
    for s, n in enumerate(lengths):
        for j in range(n):
            if 0 <= table[s, j // page] < c.shape[0]:
                used[table[s, j // page], j % page] = True
    for p in range(c.shape[0]):
        for b in range(page // 32):
            for t in np.flatnonzero(~used[p, 32 * b:32 * b + 32]):
                g, i = co.place(int(t))
                c[p, :, b, 32 * full:33 * full].reshape(-1, 32, full // 32)[:, t] = 255
                c[p, :, b, 33 * full:].reshape(-1, 4, full // 32, 8)[:, g, :, i] = 255 if t % 2 else 250


def check(got, want, weight, slack, dim, n, vmax, y):
    e = 2.0 ** -24
    rel = 2 * (2 * dim + 4) * e * slack + 2.0 ** -16 + 2.0 ** -11 + 4 * n * e
    tol = weight * rel + n * 2.0 ** -33 * vmax
    tol = tol * (1 + UNIT[y]) + np.abs(want) * UNIT[y] + TINY[y]
    bad = ~(np.abs(got - want) <= tol) & ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], (np.abs(got - want) / tol)[bad][:5])


def run_attention(ctx, seed, added, lengths, heads, group, dim, page, x, y, causal=True, window=0, hints=(0, 0), pad=(0, 0), spare=0, scale=None, change=None):
    """One call against the oracle; spare: rows of Q and Y behind the last sequence's, which must stay."""
    r = rng(6, seed, *added[:4])
    width = max(-(-n // page) for n in lengths) + 1
    pages = sum(-(-n // page) for n in lengths) + 2
    table = batch(r, lengths, page, pages, width)
    c = make_cache(r, pages, page, heads, dim)
    zero_fill(c, dim)
    if change:
        change(c, table)
    poison(c, table, lengths, page, dim)
    tokens, hq = sum(added) + spare, heads * group
    q = rounded(r.standard_normal((tokens, hq, dim)) * 0.7, x)
    offsets = np.concatenate([[0], np.cumsum(added)])
    qd = pitched(q.reshape(tokens, -1), TYPES[x], pad[0])
    yd = pitched(np.full((tokens, hq * dim), 5.0), TYPES[y], pad[1], fill=9.0)
    before = qd.clone()
    s = dim ** -0.5 if scale is None else scale
    ctx.adadim_mx4_attention(qd, torch.from_numpy(c).cuda(), ints(table), ints(offsets), ints(lengths), yd, dim, scale=scale, causal=causal, window=window,
                             max_new=hints[0], max_length=hints[1])
    got = host(yd).astype(np.float64).reshape(tokens, hq, dim)
    want, weight, slack = co.attention(q, c, table, offsets, lengths, dim, float(np.float32(s)), causal, window)
    if spare:
        assert (got[tokens - spare:] == 5.0).all()
        got, want, weight, slack = (a[:tokens - spare] for a in (got, want, weight, slack))
    if pad[1]:
        assert (yd.as_strided((tokens - 1, pad[1]), (yd.stride(0), 1), yd.storage_offset() + hq * dim) == 9.0).all()
    assert torch.equal(qd, before)
    check(got, want, weight, slack, dim, max(lengths), 6 * 2.0, y)
    return got, want


CASES = [
    # added, lengths, heads, group, dim, page
    ([1], [1], 1, 1, 64, 32), ([1], [31], 2, 1, 128, 32), ([1], [32], 1, 3, 128, 64), ([1], [33], 1, 16, 256, 32), ([1, 1, 1], [700, 1, 95], 2, 7, 128, 64),
    ([1, 1], [1500, 640], 1, 8, 80, 256), ([1], [2300], 1, 17, 64, 32), ([3, 0, 2], [300, 77, 2], 2, 5, 96, 32), ([4], [515], 1, 8, 128, 128),
    ([5, 2], [200, 330], 1, 9, 128, 32), ([7], [1100], 2, 9, 64, 32), ([2], [129], 3, 8, 256, 64), ([9, 1, 30], [9, 260, 150], 2, 4, 128, 32),
    ([70], [70], 1, 4, 64, 64), ([33, 40], [200, 40], 2, 2, 200, 32), ([129], [400], 1, 2, 128, 64), ([1, 90], [500, 90], 1, 6, 33, 32), ([3], [40], 1, 100, 128, 32),
]


@pytest.mark.parametrize("x", ["f16", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_is_the_oracles(ctx, case, x):
    added, lengths, heads, group, dim, page = CASES[case]
    most = max(added)
    print("case", case, x, CASES[case], flush=True)
    run_attention(ctx, case, added, lengths, heads, group, dim, page, x, x, hints=(most, max(lengths)), pad=(case % 3, 2 * (case % 2)), spare=case % 2)


@pytest.mark.parametrize("hints", [(0, 0), (1, 1), (2, 64), (3, 100000), (8, 700), (1000, 40)])
def test_hints_pick_the_form_and_not_the_result(ctx, hints):
    """Every form of one batch, shares of its positions among them: one token, a few, many; lengths beyond what the host announced."""
    for dim in (64, 128, 256):
        run_attention(ctx, 100, [1, 6, 20], [700, 333, 1200], 2, 4, dim, 32, "f16", "f32", hints=hints)


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("causal,window", [(True, 1), (True, 40), (False, 0), (False, 33)])
def test_masks(ctx, case, causal, window):
    added, lengths, heads, group, dim, page = CASES[case]
    run_attention(ctx, 200 + case, added, lengths, heads, group, dim, page, "f16", "f32", causal, window, hints=(max(added), max(lengths)))


@pytest.mark.parametrize("dim,added,lengths,window", [(64, [1, 2, 1], [4200, 130, 2500], 0), (128, [1, 1, 1, 0, 1], [2100, 33, 5000, 400, 2], 0),
                                                      (128, [3, 9], [6000, 2500], 2200), (256, [1, 1], [2600, 4400], 0), (100, [7, 1], [40, 3000], 0),
                                                      (128, [120, 90], [4000, 5000], 0)])
def test_long_and_short_sequences_in_shares(ctx, dim, added, lengths, window):
    """Shares of the same length over sequences of unlike ones, more for the longer; and many rows in shares."""
    run_attention(ctx, 500 + dim, added, lengths, 1, 3, dim, 64, "f16", "f32", window=window, hints=(max(added), max(lengths)))
    run_attention(ctx, 501 + dim, added, lengths, 1, 3, dim, 64, "bf16", "bf16", window=window, hints=(1, 0))


@pytest.mark.parametrize("most", [1, 20, 1000])
def test_rows_that_see_nothing_are_zeros(ctx, most):
    """No positions, fewer than rows, pages that are not there, and sequences without rows."""
    def gone(c, table):
        table[2, :] = -1
        table[3, 0] = len(c)
        table[4, 1] = -5
    got, want = run_attention(ctx, 300, [2, 5, 3, 1, 40, 0], [0, 2, 70, 20, 100, 50], 2, 2, 64, 32, "bf16", "bf16", hints=(most, 100), change=gone)
    assert (got[:2] == 0).all() and (got[2:5] == 0).all() and (got[5:7] != 0).any() and (got[7:11] == 0).all() and (got[11:] != 0).any()


@pytest.mark.parametrize("dim,added", [(64, [1, 1, 1]), (128, [5, 9, 30]), (256, [1, 40, 2])])
def test_a_position_that_is_not_finite_reaches_whom_it_is_seen_by(ctx, dim, added):
    lengths = [50, 64, 45]

    def mark(c, table):
        for s, pos in ((0, 49), (1, 40), (2, 44), (2, 3)):
            co.store(c[table[s, pos // 32]:][:1], np.full((1, 1, dim), np.nan if s else 1.0), np.full((1, 1, dim), 1.0 if s else np.inf), [pos % 32])
    for window in (0, 20):
        got, want = run_attention(ctx, 400, added, lengths, 1, 2, dim, 32, "f16", "f32", window=window, hints=(max(added), 64), change=mark)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got).any() and (max(added) == 1 or not np.isnan(got).all())


def test_one_score_far_above_the_others(ctx):
    """A weight of nearly 1 beside thousands that together still count, a maximum that rises from record to record, and scales that are large and small."""
    r = rng(7)
    dim, page, n = 128, 64, 3000
    pages = -(-n // page)
    table = batch(r, [n], page, pages, pages)
    for kind in ("sink", "rising", "scales"):
        k, v = r.standard_normal((n, 1, dim)) * 0.05, r.standard_normal((n, 1, dim))
        k[:, 0, 0] = 0.0
        if kind == "sink":
            k[0, 0, 0], k[2000, 0, 0] = 16.0, 15.0
            v[0] = v[2000] = 0.0
        elif kind == "rising":
            k[:, 0, 0] = np.arange(n) // 32 * 4.0
        else:
            v *= np.exp2(r.integers(-20, 12, (1, 1, dim // 32))).repeat(32, -1)
        c = np.zeros(B.mx4_cache_shape(pages, page, 1, dim), np.uint8)
        co.store(c, k, v, table[0][np.arange(n) // page] * page + np.arange(n) % page)
        for added, group in ((1, 1), (20, 2), (70, 1)):
            q = rounded(r.standard_normal((added, group, dim)) * 0.3, "f16")
            q[..., 0] = 1.0
            yd = torch.empty((added, group * dim), dtype=torch.float32, device="cuda")
            ctx.adadim_mx4_attention(torch.from_numpy(q.reshape(added, -1)).half().cuda(), torch.from_numpy(c).cuda(), ints(table), ints([0, added]), ints([n]), yd, dim,
                                     scale=1.0, max_new=added)
            want, weight, slack = co.attention(q, c, table, [0, added], [n], dim, 1.0)
            vmax = np.abs(co.load(c, np.arange(pages * page), dim)[1]).max((0, 1))
            check(host(yd).astype(np.float64).reshape(want.shape), want, weight, slack, dim, n, vmax, "f32")


def test_offsets_and_lengths_outside_are_taken_as_the_nearer_end(ctx):
    r = rng(8)
    dim, page, heads = 64, 32, 2
    c = make_cache(r, 6, page, heads, dim)
    table = r.permutation(6).reshape(2, 3).astype(np.int32)
    q = rounded(r.standard_normal((7, 4, dim)), "bf16")
    for offsets, lengths in (([-4, 3, 99], [40, 10 ** 9]), ([2, 1, 5], [40, 90]), ([7, 7, 7], [5, 5]), ([0, 0, 7], [-3, 96]), ([1, 2, 6], [96, 96])):
        yd = torch.full((7, 4 * dim), 5.0, dtype=torch.float32, device="cuda")
        ctx.adadim_mx4_attention(torch.from_numpy(q.reshape(7, -1)).bfloat16().cuda(), torch.from_numpy(c).cuda(), ints(table), ints(offsets), ints(lengths), yd, dim)
        want, weight, slack = co.attention(q, c, table, offsets, lengths, dim, dim ** -0.5)
        got = host(yd).astype(np.float64).reshape(want.shape)
        none = np.isnan(want)
        assert (got[none] == 5.0).all()
        keep = ~none.any((1, 2))
        check(got[keep], want[keep], weight[keep], slack[keep], dim, 96, 12.0, "f32")


@pytest.mark.parametrize("added", [3, 300])
def test_a_cache_beyond_32_bits(ctx, added):
    """Pages on both sides of 4 GB: 70000 pages of 64 positions, 8 heads of 128."""
    r = rng(12, added)
    dim, page, heads, group, n, pages = 128, 64, 8, 1, 330, 70000
    cache = torch.empty(B.mx4_cache_shape(pages, page, heads, dim), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 ** 32 + 2 ** 29
    table = np.array([[69999, 0, 65000, 30839, 61681, 61682]], np.int32)
    k, v = r.standard_normal((2, n, heads * dim)).astype(np.float32)
    slots = table[0][np.arange(n) // page] * page + np.arange(n) % page
    ctx.adadim_mx4_cache_store(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), ints(slots), cache)
    small = np.zeros(B.mx4_cache_shape(6, page, heads, dim), np.uint8)
    co.store(small, k.reshape(n, heads, dim), v.reshape(n, heads, dim), np.arange(n))
    got = [torch.empty((n, heads * dim), device="cuda") for _ in range(2)]
    ctx.adadim_mx4_cache_load(ints(slots), cache, *got)
    assert all(np.array_equal(host(g).reshape(n, heads, dim), w) for g, w in zip(got, co.load(small, np.arange(n), dim)))
    q = rounded(r.standard_normal((added, heads * group, dim)), "f16")
    y = torch.empty((added, heads * group * dim), dtype=torch.float32, device="cuda")
    ctx.adadim_mx4_attention(torch.from_numpy(q.reshape(added, -1)).half().cuda(), cache, ints(table), ints([0, added]), ints([n]), y, dim, max_new=added)
    want, weight, slack = co.attention(q[-3:], small, np.arange(6)[None], [0, 3], [n], dim, dim ** -0.5)
    check(host(y).astype(np.float64).reshape(added, heads * group, dim)[-3:], want, weight, slack, dim, n, 8.0, "f32")


def test_same_bits_every_run(ctx):
    r = rng(9)
    dim, page, heads, group, n = 128, 64, 4, 8, 9000
    pages = -(-n // page)
    c = torch.from_numpy(make_cache(r, pages, page, heads, dim)).cuda()
    table = ints(r.permutation(pages)[None])
    for added in (1, 4, 50):
        q = torch.from_numpy(r.standard_normal((added, heads * group * dim))).half().cuda()
        ys = [torch.empty_like(q) for _ in range(6)]
        for y in ys:
            ctx.adadim_mx4_attention(q, c, table, ints([0, added]), ints([n]), y, dim, max_new=added, max_length=n)
        assert all(torch.equal(y, ys[0]) for y in ys) and torch.isfinite(ys[0]).all()


def test_the_binding_refuses_shapes(ctx):
    cache = torch.zeros(B.mx4_cache_shape(2, 64, 2, 64), dtype=torch.uint8, device="cuda")
    rows, n3 = torch.zeros((3, 128), device="cuda"), ints([0, 1, 2])
    for bad in ((rows, rows[:2], n3, cache), (rows, rows.half(), n3, cache), (rows[:, :127], rows[:, :127], n3, cache), (rows, rows, n3[:2], cache),
                (rows, rows, n3, cache[..., :100]), (rows, rows, n3, cache[0])):
        with pytest.raises(ValueError):
            ctx.adadim_mx4_cache_store(*bad)
        with pytest.raises(ValueError):
            ctx.adadim_mx4_cache_load(bad[2], bad[3], *bad[:2])
    q = rows.half()
    good = dict(Q=q, cache=cache, table=n3[None], offsets=n3[:2], lengths=n3[:1], Y=torch.empty_like(q), dim=64)
    ctx.adadim_mx4_attention(**good)
    for bad in ({"Y": q[:2]}, {"dim": 128}, {"dim": 300}, {"offsets": n3}, {"lengths": n3}, {"table": n3}, {"cache": cache[:, :, :, :50]}):
        with pytest.raises(ValueError):
            ctx.adadim_mx4_attention(**{**good, **bad})
    with pytest.raises(TypeError):
        ctx.adadim_mx4_attention(**{**good, "Q": q.long()})
    for bad in ({"Q": rows}, {"scale": 0.0}, {"window": -1}):
        with pytest.raises(B.AdaDimError):
            ctx.adadim_mx4_attention(**{**good, **bad})
    with pytest.raises(ValueError):
        ctx.adadim_cache_trim(n3, n3[:2], 64, n3[:, None], n3, n3[:1], n3, n3[:1])
