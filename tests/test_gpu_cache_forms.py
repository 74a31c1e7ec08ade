"""Attention over the mx4 cache: that each form takes the batches in which it can go wrong, and batches of many sequences, against the oracle."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2309_15531_amd import binding as B
from test_gpu_cache import batch, check, host, ints, rng, rounded, run_attention

pytestmark = pytest.mark.gpu

FEW, TILES, JOIN = "mx4_attend_few", "mx4_attend_tiles", "mx4_attend_join"


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


def launched(ctx, call):
    """The attention kernels that a call launches, and what it returns."""
    ctx.adadim_profile(True)
    out = call()
    names = {n for n in ctx.adadim_profile_read() if n.startswith("mx4_attend")}
    ctx.adadim_profile(False)
    return names, out


@pytest.mark.parametrize("dim", [64, 100, 128, 256])
@pytest.mark.parametrize("new,length,form", [(0, 0, {FEW}), (1, 1, {FEW}), (64, 700, {FEW}), (65, 1200, {TILES, JOIN}), (90, 40, {TILES}), (97, 100000, {TILES, JOIN})])
def test_one_batch_by_every_form(ctx, dim, new, length, form):
    """360 rows of a sequence beside 24 and 4, lengths beyond what the host announced among the hints."""
    names, _ = launched(ctx, lambda: run_attention(ctx, 700 + dim, [1, 6, 90], [700, 333, 1200], 2, 4, dim, 32, "f16", "f32", hints=(new, length), spare=1))
    assert names == form


@pytest.mark.parametrize("dim", [64, 128, 200, 256])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 40), (False, 33), (False, 0)])
def test_masks_of_many_rows(ctx, dim, causal, window):
    names, _ = launched(ctx, lambda: run_attention(ctx, 710 + dim, [90, 3, 300], [90, 200, 700], 1, 3, dim, 64, "bf16", "f32", causal, window, hints=(300, 0)))
    assert TILES in names and FEW not in names


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_many_rows_that_see_nothing_are_zeros(ctx, dim):
    """No positions, fewer than rows, pages that are not there, and sequences without rows."""
    def gone(c, table):
        table[2, :] = -1
        table[3, 0] = len(c)
        table[4, 1] = -5
        table[5, 7:9] = len(c) + 1
    names, (got, _) = launched(ctx, lambda: run_attention(ctx, 720, [2, 150, 3, 1, 200, 140, 0], [0, 2, 70, 20, 100, 500, 50], 2, 2, dim, 32, "bf16", "bf16",
                                                          hints=(200, 500), change=gone))
    assert names == {TILES}
    assert (got[:2] == 0).all() and (got[2:150] == 0).all() and (got[150:152] != 0).any() and (got[152:156] == 0).all() and (got[156:256] == 0).all()
    assert (got[257:] != 0).any((1, 2)).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 20])
def test_a_position_that_is_not_finite_among_many_rows(ctx, dim, window):
    lengths = [400, 64, 345]

    def mark(c, table):
        for s, pos in ((0, 399), (1, 40), (2, 344), (2, 70)):
            co.store(c[table[s, pos // 32]:][:1], np.full((1, 1, dim), np.nan if s else 1.0), np.full((1, 1, dim), 1.0 if s else np.inf), [pos % 32])
    names, (got, want) = launched(ctx, lambda: run_attention(ctx, 730, [5, 40, 300], lengths, 1, 2, dim, 32, "f16", "f32", window=window, hints=(300, 400), change=mark))
    assert names == {TILES}
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got).any() and not np.isnan(got).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", ["sink", "rising", "scales"])
def test_many_rows_with_one_score_far_above_the_others(ctx, dim, kind):
    """As for few rows: a weight of nearly 1 beside thousands that together still count, a maximum that rises from record to record, large and small scales."""
    r = rng(74, dim)
    page, n, added = 64, 3000, 300
    pages = -(-n // page)
    table = batch(r, [n], page, pages, pages)
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
    q = rounded(r.standard_normal((added, 1, dim)) * 0.3, "f16")
    q[..., 0] = 1.0
    want, weight, slack = co.attention(q, c, table, [0, added], [n], dim, 1.0)
    vmax = np.abs(co.load(c, np.arange(pages * page), dim)[1]).max((0, 1))
    for length, form in ((n, {TILES, JOIN}), (100, {TILES})):
        yd = torch.empty((added, dim), dtype=torch.float32, device="cuda")
        names, _ = launched(ctx, lambda: ctx.adadim_mx4_attention(torch.from_numpy(q.reshape(added, -1)).half().cuda(), torch.from_numpy(c).cuda(), ints(table),
                                                                  ints([0, added]), ints([n]), yd, dim, scale=1.0, max_new=added, max_length=length))
        assert names == form
        check(host(yd).astype(np.float64).reshape(want.shape), want, weight, slack, dim, n, vmax, "f32")


@pytest.mark.parametrize("n", [64, 65, 130, 400])
@pytest.mark.parametrize("long", [100, 3000])
@pytest.mark.parametrize("many", [False, True])
def test_many_sequences_of_unlike_lengths(ctx, n, long, many):
    """One to a few new tokens each (none at all for some), of which one sequence has several tiles; lengths from 0 on, one far beyond the others."""
    r = rng(75, n, long, many)
    lengths = r.integers(0, 60 if n > 64 else 120, n)
    lengths[r.integers(n)] = long
    added = np.where(r.random(n) < 0.15, 0, r.integers(1, 4, n))
    added[n // 2], added[n - 1] = 140 if many else 30, 20
    lengths = np.maximum(lengths, added - 2 * (r.random(n) < 0.1))
    names, _ = launched(ctx, lambda: run_attention(ctx, 750 + n, added.tolist(), lengths.tolist(), 1, 2, 64, 32, "f16", "f32", window=0 if n % 2 else 500,
                                                   hints=(int(added.max()), long), spare=2))
    assert (TILES if many else FEW) in names and (FEW if many else TILES) not in names


@pytest.mark.parametrize("hints", [False, True])
def test_a_mixed_batch_by_one_call_and_by_two(ctx, hints):
    """A chunk beside decoding sequences: each call writes the rows of its own sequences, in one form or in two."""
    r = rng(76)
    dim, page, heads, group = 128, 32, 2, 4
    added, lengths = [150, 1, 1, 2, 0, 1], [400, 300, 35, 90, 64, 700]
    width = max(lengths) // page + 1
    pages = sum(-(-n // page) for n in lengths)
    table = batch(r, lengths, page, pages, width)
    k, v = (r.standard_normal((pages * page, heads, dim)) for _ in range(2))
    cache = torch.empty(B.mx4_cache_shape(pages, page, heads, dim), dtype=torch.uint8, device="cuda")
    ctx.adadim_mx4_cache_store(*(torch.from_numpy(t.reshape(len(t), -1)).float().cuda() for t in (k, v)), ints(np.arange(pages * page)), cache)
    offsets = np.concatenate([[0], np.cumsum(added)])
    q = rounded(r.standard_normal((sum(added), heads * group, dim)) * 0.7, "f16")
    qd, t, o, n = torch.from_numpy(q.reshape(len(q), -1)).half().cuda(), ints(table), ints(offsets), ints(lengths)
    want, weight, slack = co.attention(q, cache.cpu().numpy(), table, offsets, lengths, dim, float(np.float32(dim ** -0.5)))

    def call(y, a, b):
        more = dict(max_new=max(added[a:b]), max_length=max(lengths[a:b])) if hints else {}
        ctx.adadim_mx4_attention(qd, cache, t[a:b], o[a:b + 1], n[a:b], y, dim, **more)
    whole, parts = (torch.full(qd.shape, 5.0, dtype=torch.float32, device="cuda") for _ in range(2))
    call(whole, 0, 6)
    names, _ = launched(ctx, lambda: call(parts, 0, 1))
    assert TILES in names and (parts[150:] == 5.0).all() and (parts[:150] != 5.0).any(1).all()
    first = parts[:150].clone()
    names, _ = launched(ctx, lambda: call(parts, 1, 6))
    assert names == {FEW} or not hints
    assert torch.equal(parts[:150], first)
    for y in (whole, parts):
        check(host(y).astype(np.float64).reshape(want.shape), want, weight, slack, dim, max(lengths), 12.0, "f32")
