"""The paged cache as a serving program uses it: pages, storing and attention together, on other streams, recorded as a graph."""
import importlib.util
import os
import sys

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2309_15531_amd import binding as B, mx4
from test_gpu_cache import check, host, ints
from test_gpu_mx4_streams import randn, slow

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADS, GROUP, DIM, PAGE = 2, 4, 96, 32


class Batch:
    """Three sequences with a cache, stepped with given numbers of new tokens."""

    def __init__(self, ctx, pool=40):
        self.pages = mx4.CachePages(ctx, pool, PAGE, 3, 12)
        self.cache = mx4.Mx4Cache(self.pages, HEADS, DIM)

    def step(self, qkv, added, tokens, **hints):
        rows = self.pages.add(added, tokens)
        q, k, v = qkv.split([HEADS * GROUP * DIM, HEADS * DIM, HEADS * DIM], 1)
        self.cache.store(k, v, rows.slots)
        return rows, self.cache.attend(q, rows.offsets, **hints)


def inputs(seed, tokens):
    return randn(seed, tokens, (HEADS * GROUP + 2 * HEADS) * DIM).half()


STEPS = [[100, 1, 33], [1, 1, 1], [5, 0, 2], [1, 70, 1], [0, 1, 0]]


def test_steps_are_the_oracles():
    """Prompts, decoding, drafted tokens that are taken back and a sequence that starts anew: results, pages and what the cache holds."""
    ctx = B.Context()
    b = Batch(ctx)
    table, free, count, lengths = np.full((3, 12), -1, np.int32), list(range(40)), 40, [0, 0, 0]
    mirror = np.zeros(b.cache.records.shape, np.uint8)
    for turn, added in enumerate(STEPS):
        tokens = sum(added) + turn % 2                        # (a padded batch now and then)
        x = inputs(turn, tokens)
        rows, y = b.step(x, ints(added), tokens, max_new=max(added))
        want = co.reserve(lengths, added, PAGE, table, free, count, tokens)
        assert rows.slots.tolist() == want["slots"] and rows.offsets.tolist() == want["offsets"] and rows.lacking.item() == 0
        table, count, lengths = want["table"], want["left"], want["lengths"]
        assert b.pages.lengths.tolist() == lengths and b.pages.count.item() == count
        q, k, v = (t.double().cpu().numpy().reshape(tokens, -1, DIM) for t in x.split([HEADS * GROUP * DIM, HEADS * DIM, HEADS * DIM], 1))
        co.store(mirror, k, v, want["slots"])
        ref, weight, slack = co.attention(q, mirror, table, want["offsets"], lengths, DIM, float(np.float32(DIM ** -0.5)))
        n = sum(added)
        check(host(y).astype(np.float64).reshape(ref.shape)[:n], ref[:n], weight[:n], slack[:n], DIM, max(lengths), 8.0, "f16")
        for got, ref in zip(b.cache.load(rows.slots), co.load(mirror, want["slots"], DIM)):
            assert np.array_equal(got.double().cpu().numpy().reshape(ref.shape), ref)
        kept = [lengths[0] - 2, lengths[1], 0] if turn == 2 else lengths
        b.pages.trim(ints(kept))
        want = co.trim(lengths, kept, PAGE, table, free, count)
        free, lengths, count = want["free"], want["lengths"], want["left"]
        assert b.pages.free.tolist()[:count] == free[:count] and b.pages.count.item() == count
    ctx.close()


def test_a_pool_without_pages_refuses_and_goes_on():
    ctx = B.Context()
    b = Batch(ctx, pool=4)
    rows, _ = b.step(inputs(0, 60), ints([30, 20, 10]), 60)
    assert rows.lacking.item() == 0 and b.pages.count.item() == 1
    before = b.cache.records.clone()
    rows, y = b.step(inputs(1, 90), ints([30, 30, 30]), 90)
    assert rows.lacking.item() == 2 and b.pages.lengths.tolist() == [30, 20, 10] and torch.equal(b.cache.records, before) and rows.offsets.tolist() == [0] * 4
    b.pages.trim(ints([0, 20, 10]))
    rows, _ = b.step(inputs(2, 30), ints([0, 30, 0]), 30)
    assert rows.lacking.item() == 0 and b.pages.lengths.tolist() == [0, 50, 10] and b.pages.count.item() == 1
    ctx.close()


def test_steps_take_part_in_the_current_stream():
    """Inputs that the current stream has yet to write and results it reads at once: the same bits as with everything on one stream."""
    plain = B.Context()
    b, want = Batch(plain), []
    for turn, added in enumerate(STEPS):
        rows, y = b.step(inputs(turn, sum(added)), ints(added), sum(added), max_new=max(added))
        want += [*(t.clone() for t in rows), y.clone(), b.pages.lengths.clone()]
    torch.cuda.synchronize()
    own, here = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(own):
        ctx = B.Context()
    with torch.cuda.stream(here):
        b, got = Batch(ctx), []
        for turn, added in enumerate(STEPS):
            x, a = torch.zeros((sum(added), (HEADS * GROUP + 2 * HEADS) * DIM), dtype=torch.float16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
            value, number = inputs(turn, sum(added)), ints(added)
            slow(4)
            x.copy_(value)
            a.copy_(number)
            rows, y = b.step(x, a, sum(added), max_new=max(added))
            x.fill_(float("nan"))
            a.fill_(-1)
            got += [*(t.clone() for t in rows), y.clone(), b.pages.lengths.clone()]
        here.synchronize()
    assert len(got) == len(want) and all(torch.equal(g, w) for g, w in zip(got, want))
    own.synchronize()
    ctx.close()
    plain.close()


@pytest.mark.parametrize("tokens,long", [(3, 12), (3, 200), (150, 12)])
def test_a_recorded_step_grows_the_sequences_at_every_replay(tokens, long):
    """One graph of reserve, store and attention, replayed with new inputs and numbers of tokens, between eager steps of another batch on the same context;
    each replay against an eager step on a copy of everything."""
    own = torch.cuda.Stream()
    with torch.cuda.stream(own):
        ctx = B.Context()
        b, other, eager = (Batch(ctx) for _ in range(3))
        x, added = inputs(0, tokens), ints([0, 0, 0])
        hints = dict(max_new=max(1, tokens // 3), max_length=long)
        b.step(x, added, tokens, **hints)                     # (nothing is added: scratch grows, lengths stay)
        ctx.adadim_capture_begin()
        try:
            rows, y = b.step(x, added, tokens, **hints)
        finally:
            graph = ctx.adadim_capture_end()
        torch.cuda.empty_cache()
        per = tokens // 3
        for turn in range(1, 6):
            a = [per, max(1, per - turn), per] if turn % 2 else [per, 0, max(1, per // 2)]
            x.copy_(inputs(turn, tokens))
            added.copy_(ints(a))
            y.fill_(3.0)
            ctx.adadim_graph_launch(graph)
            want_rows, want = eager.step(x, added, tokens, **hints)
            n = sum(a)
            assert torch.equal(y[:n], want[:n]) and torch.isfinite(y[:n]).all() and (y[n:] == 3.0).all(), turn
            assert all(torch.equal(g, w) for g, w in zip(rows, want_rows)) and rows.lacking.item() == 0
            assert torch.equal(b.pages.lengths, eager.pages.lengths) and torch.equal(b.pages.table, eager.pages.table)
            other.step(inputs(turn + 70, 350), ints([200, 100, 50]), 350, max_new=200)          # scratch that outgrows the recorded one
            other.pages.trim(ints([0, 0, 0]))
            own.synchronize()
        ctx.adadim_graph_destroy(graph)
    own.synchronize()
    ctx.close()


@pytest.mark.parametrize("added,group", [(1, 8), (4, 8), (400, 2)])
def test_a_recorded_attention_in_shares(added, group):
    """Long sequences, whose positions are shared between workgroups by way of scratch: replays between eager calls that need more of it, and less."""
    own = torch.cuda.Stream()
    dim, page, heads, n = 128, 64, 2, 9000
    with torch.cuda.stream(own):
        ctx = B.Context()
        pages = mx4.CachePages(ctx, 300, page, 1, 300)
        cache = mx4.Mx4Cache(pages, heads, dim)
        rows = pages.add(ints([n]), n)
        cache.store(randn(1, n, heads * dim).half(), randn(2, n, heads * dim).half(), rows.slots)
        q, offsets = randn(3, added, heads * group * dim).half(), ints([0, added])
        big = randn(4, 800, heads * 4 * dim).half()
        call = dict(max_new=added, max_length=n)
        cache.attend(q, offsets, **call)
        ctx.adadim_capture_begin()
        try:
            y = cache.attend(q, offsets, **call)
        finally:
            graph = ctx.adadim_capture_end()
        for turn in range(4):
            q.copy_(randn(10 + turn, added, heads * group * dim))
            y.fill_(float("nan"))
            ctx.adadim_graph_launch(graph)
            assert torch.equal(y, cache.attend(q, offsets, **call)) and torch.isfinite(y).all(), turn
            if turn:
                cache.attend(big[:200 * turn], ints([0, 200 * turn]), max_new=200 * turn)
            cache.attend(q[:1], ints([0, 1]), max_new=1)
            own.synchronize()
        ctx.adadim_graph_destroy(graph)
    own.synchronize()
    ctx.close()


def test_two_contexts_at_once():
    """Calls that share positions by way of scratch, on two streams at the same time: each context has its own."""
    dim, page, heads, group, n = 128, 64, 4, 4, 6000
    streams, made, got = [torch.cuda.Stream() for _ in range(2)], [], [[], []]
    for i, stream in enumerate(streams):
        with torch.cuda.stream(stream):
            ctx = B.Context()
            pages = mx4.CachePages(ctx, 300, page, 2, 100)
            cache = mx4.Mx4Cache(pages, heads, dim)
            rows = pages.add(ints([n, n // 3]), n + n // 3)
            cache.store(*(randn(20 + 2 * i + j, n + n // 3, heads * dim).half() for j in range(2)), rows.slots)
            q = [randn(30 + i, k, heads * group * dim).half() for k in (2, 300)]
            offsets = [ints([0, 1, 2]), ints([0, 200, 300])]
            made.append((ctx, cache, q, offsets, [cache.attend(x, o, max_new=m, max_length=n).clone() for x, o, m in zip(q, offsets, (1, 200))]))
    torch.cuda.synchronize()
    for turn in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                ctx, cache, q, offsets, _ = made[i]
                got[i].append(cache.attend(q[turn % 2], offsets[turn % 2], max_new=(1, 200)[turn % 2], max_length=n))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, made[i][4][turn % 2]) and torch.isfinite(y).all() for turn, y in enumerate(got[i]))
        made[i][0].close()


def test_the_example_runs(capsys, monkeypatch):
    monkeypatch.setattr(sys, "argv", ["mx4_attention.py", "--heads", "4", "--kv-heads", "2", "--dim", "64", "--prompt", "150", "--sequences", "3", "--steps", "2"])
    spec = importlib.util.spec_from_file_location("mx4_attention", os.path.join(ROOT, "examples", "mx4_attention.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    example.main()
    out = capsys.readouterr().out
    assert "all sequences ended: 12 of 12 pages free" in out and out.count("step") == 3
