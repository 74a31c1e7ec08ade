"""Performance cases of attention over a paged cache of microscaled 4-bit keys and values: what a serving program calls between a
layer's projections.

The cache is a pool of pages; a page holds `page` positions (a multiple of 32) of every key-value head.  Each 32 positions of a head
are one record: the codes of the keys, the codes of the values, the scales of the keys, the scales of the values, in blocks of 32
values along a head as everywhere in mx4 (E2M1 codes, a byte exponent + 127 per block).  Heads are filled up to D = 64, 128 or 256:

  keys    codes [32 positions][D / 2 bytes], the even element in the low half of a byte; scales [32][D / 32]
  values  codes [4][16][8][D / 32 bytes]: part (g, m, i) holds elements m D / 16 .. of position 4 g + i (i < 4) or 12 + 4 g + i;
          scales [4][D / 32][8]: (g, block, i)

Scales lie in 2^-23 .. 2^13, where fp16 holds every value; a position whose key or value is not finite has the key scales 255 (NaN) and
codes and value scales of zeros.

  reserve  pages for the tokens that a batch adds: block tables from a stack of free pages, slots and positions of the new rows
  trim     the other way: the pages of finished sequences and of drafted tokens that were turned down, back to the stack
  store    rows of keys and values to their slots, and back to values
  attend   softmax(scale Q K^T) V over the pages of each sequence, for one new token or many, causal, with or without a window

`listed()` are fixed sizes of the shapes this package names; `draw(rng)` takes further ones from the same ranges.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 32
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_CONTEXT = None


def _context():
    """The one library context a program keeps for its stream."""
    global _CONTEXT
    if _CONTEXT is None:
        from paper_2309_15531_amd import binding
        _CONTEXT = binding.Context()
    return _CONTEXT


# --------------------------------------------------------------------------------------------- cases
def _reserve(name, sequences, longest, most, page, spread):
    return {"name": name, "kind": "reserve", "sequences": sequences, "longest": longest, "most": most, "page": page, "spread": spread}


def _trim(name, sequences, longest, most, ended, page, spread):
    return {"name": name, "kind": "trim", "sequences": sequences, "longest": longest, "most": most, "ended": ended, "page": page,
            "spread": spread}


def _store(name, tokens, heads, dim, page, x, y):
    return {"name": name, "kind": "store", "tokens": tokens, "heads": heads, "dim": dim, "page": page, "x": x, "y": y}


def _attend(name, sequences, longest, most, heads, group, dim, page, x, causal=True, window=0, spread=1):
    """sequences of up to `longest` positions, the last up to `most` of them new; `group` query heads to each of `heads`."""
    return {"name": name, "kind": "attend", "sequences": sequences, "longest": longest, "most": most, "heads": heads, "group": group,
            "dim": dim, "page": page, "x": x, "causal": causal, "window": window, "spread": spread}


def listed():
    return [
        # one decoding step of a large batch: a token each, a page for those that cross into a new one
        _reserve("reserve_decode", 256, 8192, 1, 64, 1),
        # a batch of prompts that enters an empty cache
        _reserve("reserve_prompts", 64, 1, 2048, 64, 2),
        # drafted tokens that a verification turned down, and a few sequences that ended
        _trim("trim_drafts", 64, 8192, 6, 4, 64, 3),
        # a batch that goes out whole
        _trim("trim_batch", 256, 16384, 1, 256, 32, 4),
        # the keys and values of sixteen decoding sequences
        _store("store_decode", 16, 8, 128, 64, "bf16", "bf16"),
        # those of a batch of prompts, 32 heads as a 7B-shaped block has them
        _store("store_prompt", 8192, 32, 128, 64, "f16", "f16"),
        # one sequence, one token: latency
        _attend("attend_token", 1, 1000, 1, 8, 4, 128, 64, "f16", spread=5),
        # a decoding step of a 70B-shaped block: 64 heads over 8, ragged lengths
        _attend("attend_decode", 64, 8192, 1, 8, 8, 128, 64, "bf16", spread=6),
        # two sequences of very long context, heads of their own (7B-shaped): the cache is the work
        _attend("attend_long", 2, 100003, 1, 32, 1, 128, 128, "f16", spread=7),
        # drafted tokens to verify, heads of 80 in a group of five, a sliding window
        _attend("attend_drafts", 17, 5001, 6, 8, 5, 80, 32, "bf16", window=4096, spread=8),
        # a prompt into an empty cache, 7B-shaped
        _attend("attend_prompt", 1, 4096, 4096, 32, 1, 128, 64, "f16", spread=0),
        # chunks of two long prompts over what of them is there already, 70B-shaped
        _attend("attend_chunk", 2, 16384, 2048, 8, 8, 128, 64, "bf16", spread=9),
    ]


MOST_PAIRS = 6.0e10                                             # (query, key, element) triples of a drawn case
MOST_CACHE = 8.0e8                                              # values of keys and values it holds


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["reserve", "trim", "store", "attend", "attend", "attend", "attend", "attend"])
    page, spread = rng.choice([32, 64, 64, 128, 256]), rng.randrange(1, 1 << 20)
    if kind == "reserve":
        c = _reserve("", _log(rng, 1, 1024), _log(rng, 1, 16384), rng.choice([1, 1, _log(rng, 2, 2048)]), page, spread)
        while c["sequences"] * c["most"] > 1 << 17:
            c["sequences"] = (c["sequences"] + 1) // 2
    elif kind == "trim":
        n = _log(rng, 1, 1024)
        c = _trim("", n, _log(rng, 8, 16384), rng.choice([1, 4, 8]), rng.choice([0, n // 8, n]), page, spread)
    elif kind == "store":
        x = rng.choice(["f16", "f16", "bf16", "bf16", "f32"])
        c = _store("", _log(rng, 1, 8192), rng.choice([1, 2, 4, 8, 8, 32]), rng.choice([64, 80, 96, 100, 128, 128, 256]), page, x,
                   rng.choice([x, "f32"]))
        while c["tokens"] * c["heads"] * c["dim"] > 8192 * 32 * 128 / (2 if "f32" in (c["x"], c["y"]) else 1):
            c["tokens"] //= 2
    else:
        most = rng.choice([1, 1, 1, _log(rng, 2, 16), _log(rng, 16, 4096)])
        longest = max(most, _log(rng, 1, 32768))
        heads, group = rng.choice([(1, 8), (2, 4), (4, 7), (8, 1), (8, 4), (8, 5), (8, 8), (32, 1), (40, 1), (4, 16)])
        c = _attend("", _log(rng, 1, 128), longest, most, heads, group, rng.choice([64, 80, 96, 128, 128, 128, 256]), page,
                    rng.choice(["f16", "bf16"]), causal=rng.random() < 0.85, window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]),
                    spread=spread)
        while c["sequences"] > 1 and (c["sequences"] * float(most) * longest * heads * group * c["dim"] > MOST_PAIRS
                                      or 2.0 * c["sequences"] * longest * heads * c["dim"] > MOST_CACHE):
            c["sequences"] //= 2
        while c["most"] * float(longest) * heads * group * c["dim"] > MOST_PAIRS:
            c["most"] = (c["most"] + 1) // 2
        while 2.0 * c["longest"] * heads * c["dim"] > MOST_CACHE:
            c["longest"] = max(c["most"], c["longest"] // 2)
    c.pop("name", None)
    return c


def _lengths(case):
    """(held, added) of each sequence, in tokens; spread 0: the largest everywhere."""
    c, n = case, case["sequences"]
    if c["spread"] == 0:
        return [c["longest"] - c["most"]] * n, [c["most"]] * n
    r = random.Random(c["spread"])
    if c["kind"] == "attend":
        total = [c["longest"]] + [r.randint(max(1, c["longest"] // 8), c["longest"]) for _ in range(n - 1)]
        added = [min(t, c["most"] if c["most"] <= 8 else r.randint((c["most"] + 1) // 2, c["most"])) for t in total]
        added[0] = min(total[0], c["most"])
        return [t - a for t, a in zip(total, added)], added
    held = [r.randint(0, c["longest"]) if c["longest"] > 1 else 0 for _ in range(n)]
    return held, [c["most"] if c["most"] <= 8 else r.randint(1, c["most"]) for _ in range(n)]


def _pages(tokens, page):
    return (tokens + page - 1) // page


# --------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) & 0x7FFFFFFF)


def _randn(shape, g):
    return torch.randn(shape, dtype=torch.float32, device="cuda", generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _full(dim):
    """What a head is filled up to."""
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def _keys(tokens, heads, dim, g):
    """Keys: unit channels, and a few of each head several times as large, the same for all tokens."""
    x = _randn((tokens, heads, dim), g)
    return x.mul_(torch.where(torch.rand((heads, dim), device="cuda", generator=g) < 0.03, 6.0, 1.0))


def _codes(x):
    """(codes u8 0..15 [.., D], scale bytes [.., D / 32]) of fp32 rows whose length is a multiple of 32."""
    b = x.unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(-1)
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 3, 0).clamp(-23, 13)
    m = torch.ldexp(b.abs(), -e[..., None])
    q = torch.zeros_like(m, dtype=torch.uint8)
    for edge, even in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        q += (m >= edge) if even else (m > edge)
    q |= torch.signbit(b).to(torch.uint8) << 3
    return q.flatten(-2), (e + 127).to(torch.uint8)


def _paired(q):
    return q[..., 0::2] | (q[..., 1::2] << 4)


def _value_order(device):
    """The position that stands at (g, i) of a record's values."""
    g, i = torch.arange(4, device=device)[:, None], torch.arange(8, device=device)
    return 4 * g + torch.where(i < 4, i, 12 + i)


def _records(k, v):
    """[.., 32, D] keys and values to records [.., 34 D]."""
    full = k.shape[-1]
    (kq, ks), (vq, vs) = _codes(k), _codes(v)
    order = _value_order(k.device).reshape(-1)
    vq = _paired(vq)[..., order, :].unflatten(-1, (16, full // 32)).unflatten(-3, (4, 8)).transpose(-3, -2)
    vs = vs[..., order, :].unflatten(-2, (4, 8)).transpose(-2, -1)
    return torch.cat([_paired(kq).flatten(-2), vq.flatten(-4), ks.flatten(-2), vs.flatten(-3)], -1)


def _filled(pages, heads, page, dim, g):
    """A pool of pages with keys and values in all of them."""
    full, out = _full(dim), []
    step = max(1, (1 << 25) // (heads * page * full))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        k = _keys(n * page, heads, dim, g).view(n, page, heads, dim).transpose(1, 2)
        v = _randn((n, heads, page, dim), g)
        k, v = (torch.nn.functional.pad(t, (0, full - dim)).unflatten(2, (-1, BLOCK)) for t in (k, v))
        out.append(_records(k, v))
    return torch.cat(out)


def prepare(case, seed):
    c, g = case, _gen(seed * 7 + 3)
    st = {"case": c}
    if c["kind"] in ("reserve", "trim"):
        held, added = _lengths(c)
        page, n = c["page"], c["sequences"]
        width = max(_pages(h + a, page) for h, a in zip(held, added))
        used = [_pages(h, page) for h in held]
        pool = sum(_pages(h + a, page) for h, a in zip(held, added)) + 64
        ids = torch.randperm(pool, device="cuda", generator=g).to(torch.int32)
        st["page"] = page
        st["held"] = _ints(held)
        st["lengths"] = torch.empty(n, dtype=torch.int32, device="cuda")
        st["left"] = torch.empty(1, dtype=torch.int32, device="cuda")
        st["table"] = torch.zeros((n, width), dtype=torch.int32, device="cuda")
        at = torch.arange(width, device="cuda")
        mask = at < _ints(used)[:, None]
        st["table"][mask] = ids[:sum(used)]
        if c["kind"] == "reserve":
            st["added"], st["free"], tokens = _ints(added), ids[sum(used):].contiguous(), sum(added)
            st["count"] = _ints([pool - sum(used)])
            st["offsets"] = torch.empty(n + 1, dtype=torch.int32, device="cuda")
            st["slots"], st["positions"] = (torch.empty(tokens, dtype=torch.int32, device="cuda") for _ in range(2))
            st["lacking"] = torch.empty(1, dtype=torch.int32, device="cuda")
        else:
            r = random.Random(c["spread"] + seed)
            gone = set(r.sample(range(n), c["ended"]))
            kept = [0 if s in gone else max(0, held[s] - r.randint(0, c["most"])) for s in range(n)]
            st["kept"] = _ints(kept)
            st["free"] = torch.zeros(pool, dtype=torch.int32, device="cuda")
            st["free"][:pool - sum(used)] = ids[sum(used):]
            st["count"] = _ints([pool - sum(used)])
    elif c["kind"] == "store":
        t, h, d, page = c["tokens"], c["heads"], c["dim"], c["page"]
        pages = _pages(t, page) + 8
        order = torch.randperm(pages, device="cuda", generator=g)
        at = torch.arange(t, device="cuda") + page // 3          # runs of a sequence's positions, over pages in any order
        st["slots"] = (order[at // page] * page + at % page).to(torch.int32)
        st["K"] = _keys(t, h, d, g).view(t, h * d).to(TYPES[c["x"]])
        st["V"] = _randn((t, h * d), g).to(TYPES[c["x"]])
        st["cache"] = torch.zeros((pages, h, page // BLOCK, 34 * _full(d)), dtype=torch.uint8, device="cuda")
        st["YK"], st["YV"] = (torch.empty((t, h * d), dtype=TYPES[c["y"]], device="cuda") for _ in range(2))
    else:
        held, added = _lengths(c)
        page, n, h, d = c["page"], c["sequences"], c["heads"], c["dim"]
        st["lens"], st["new"] = [x + y for x, y in zip(held, added)], added
        used = [_pages(t, page) for t in st["lens"]]
        pages = sum(used) + 4
        ids = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        st["table"] = torch.full((n, max(used)), -1, dtype=torch.int32, device="cuda")
        st["table"][torch.arange(max(used), device="cuda") < _ints(used)[:, None]] = ids[:sum(used)]
        st["cache"] = _filled(pages, h, page, d, g)
        st["offsets"] = _ints([sum(added[:s]) for s in range(n + 1)])
        st["lengths"] = _ints(st["lens"])
        t, hq = sum(added), h * c["group"]
        st["Q"] = (_randn((t, hq * d), g) * 1.2).to(TYPES[c["x"]])
        st["Y"] = torch.empty((t, hq * d), dtype=TYPES[c["x"]], device="cuda")
    return st


# --------------------------------------------------------------------------------------------- the plain forms
def _grid(device):
    return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float32, device=device)


def _halves(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _sequence(st, s):
    """fp32 keys and values [heads, positions, dim] of a sequence, out of its pages."""
    c = st["case"]
    full, dim, length = _full(c["dim"]), c["dim"], st["lens"][s]
    r = st["cache"][st["table"][s, :_pages(length, c["page"])].long()].transpose(0, 1).flatten(1, 2)      # [heads, blocks, 34 D]
    kq, vq, ks, vs = r.split([16 * full, 16 * full, full, full], -1)
    grid = _grid(r.device)
    steps = torch.exp2(torch.arange(256, device=r.device).float() - 127.0)
    k = grid[_halves(kq).int()].unflatten(-1, (32, full // 32, 32)) * steps[ks.int()].unflatten(-1, (32, full // 32, 1))
    back = torch.argsort(_value_order(r.device).reshape(-1))
    v = grid[_halves(vq.unflatten(-1, (4, 16, 8, full // 32))).int()].transpose(-3, -2).flatten(-2).flatten(-3, -2)[..., back, :]
    w = steps[vs.int()].unflatten(-1, (4, full // 32, 8)).transpose(-2, -1).flatten(-3, -2)[..., back, :]
    v = v.unflatten(-1, (-1, 32)) * w[..., None]
    return k.flatten(-2).flatten(1, 2)[:, :length, :dim], v.flatten(-2).flatten(1, 2)[:, :length, :dim]


def _plain_attend(st):
    c = st["case"]
    h, gr, d = c["heads"], c["group"], c["dim"]
    rows = max(1, (1 << 28) // max(st["lens"]) // gr)           # (of the scores of a few heads at a time)
    q, y, at = st["Q"].float(), [], 0
    for s, new in enumerate(st["new"]):
        k, v = _sequence(st, s)
        length = st["lens"][s]
        qs = q[at:at + new].view(new, h, gr, d).transpose(0, 1)                                     # [heads, new, group, dim]
        o = torch.empty_like(qs)
        hs = max(1, min(h, rows // new))
        step = min(new, rows)
        for r in range(0, new, step):
            m = min(step, new - r)
            pos = torch.arange(length - new + r, length - new + r + m, device=q.device)[:, None]
            key = torch.arange(length, device=q.device)
            seen = torch.ones((m, length), dtype=torch.bool, device=q.device)
            if c["causal"]:
                seen &= key <= pos
            if c["window"]:
                seen &= key > pos - c["window"]
            for a in range(0, h, hs):
                score = torch.matmul(qs[a:a + hs, r:r + m].flatten(1, 2), k[a:a + hs].transpose(1, 2).contiguous()) * d ** -0.5
                score = torch.where(seen[:, None], score.unflatten(1, (m, gr)), -math.inf)
                p = torch.exp(score - score.amax(-1, keepdim=True))
                p = p / p.sum(-1, keepdim=True)
                o[a:a + hs, r:r + m] = torch.matmul(p.flatten(1, 2), v[a:a + hs].contiguous()).unflatten(1, (m, gr))
        y.append(o.transpose(0, 1).reshape(new, h * gr * d))
        at += new
    return torch.cat(y).to(TYPES[c["x"]])


def _plain_store(st):
    """The values that the rows' codes and scales stand for: nearest, ties to even, the scale from the block's largest."""
    c, out = st["case"], {}
    for name in ("K", "V"):
        x = st[name].float().view(c["tokens"], c["heads"], c["dim"])
        x = torch.nn.functional.pad(x, (0, _full(c["dim"]) - c["dim"])).unflatten(-1, (-1, BLOCK))
        amax = x.abs().amax(-1, keepdim=True)
        s = torch.exp2(torch.where(amax > 0, torch.frexp(amax).exponent - 3, 0).clamp(-23, 13).float())
        m = x.abs() / s
        step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
        m = torch.clamp(torch.round(m / step) * step, max=6.0)
        out[name] = (torch.copysign(m, x) * s).flatten(-2)[..., :c["dim"]].flatten(1).to(TYPES[c["y"]])
    return out


def _plain_reserve(st):
    page, table, n = st["page"], st["table"].clone(), st["held"].numel()
    held, added, tokens = st["held"].long(), st["added"].long(), st["slots"].numel()
    zero = held.new_zeros(1)
    offsets = torch.cat([zero, added.cumsum(0)])
    lengths = held + added
    had, has = (held + page - 1) // page, (lengths + page - 1) // page
    first = torch.cat([zero, (has - had).cumsum(0)])
    at = torch.arange(table.shape[1], device=table.device)
    place = first[:-1, None] + at - had[:, None]
    new = (at >= had[:, None]) & (at < has[:, None])
    table = torch.where(new, st["free"][(st["count"].long() - 1 - place).clamp(0, st["free"].numel() - 1)], table)
    row = torch.arange(tokens, device=table.device)
    seq = torch.searchsorted(offsets[1:].contiguous(), row, right=True).clamp(max=n - 1)
    pos = held[seq] + row - offsets[seq]
    slots = table[seq, pos // page].long() * page + pos % page
    return {"table": table, "lengths": lengths.int(), "offsets": offsets.int(), "slots": slots.int(), "positions": pos.int(),
            "left": (st["count"].long() - first[-1]).int(), "lacking": torch.zeros_like(st["count"])}


def _plain_trim(st):
    page, table, free = st["page"], st["table"], st["free"].clone()
    held, kept = st["held"].long(), torch.minimum(st["held"], st["kept"]).long()
    had, has = (held + page - 1) // page, (kept + page - 1) // page
    at = torch.arange(table.shape[1], device=table.device)
    gone = table[(at >= has[:, None]) & (at < had[:, None])]
    place = st["count"].long() + torch.arange(gone.numel(), device=table.device)
    free[place] = gone
    return {"free": free, "lengths": kept.int(), "left": (st["count"].long() + gone.numel()).int()}


PLAIN = {"reserve": _plain_reserve, "trim": _plain_trim, "store": _plain_store, "attend": _plain_attend}


# --------------------------------------------------------------------------------------------- one pass
def run(st):
    c = st["case"]
    if not own:
        return PLAIN[c["kind"]](st)
    ctx = _context()
    if c["kind"] == "reserve":
        ctx.adadim_cache_reserve(st["held"], st["added"], st["page"], st["table"], st["free"], st["count"], st["lengths"],
                                 st["offsets"], st["slots"], st["positions"], st["left"], st["lacking"])
        return {n: st[n] for n in ("table", "lengths", "offsets", "slots", "positions", "left", "lacking")}
    if c["kind"] == "trim":
        ctx.adadim_cache_trim(st["held"], st["kept"], st["page"], st["table"], st["free"], st["count"], st["lengths"], st["left"])
        return {n: st[n] for n in ("free", "lengths", "left")}
    if c["kind"] == "store":
        ctx.adadim_mx4_cache_store(st["K"], st["V"], st["slots"], st["cache"])
        ctx.adadim_mx4_cache_load(st["slots"], st["cache"], st["YK"], st["YV"])
        return {"K": st["YK"], "V": st["YV"]}
    ctx.adadim_mx4_attention(st["Q"], st["cache"], st["table"], st["offsets"], st["lengths"], st["Y"], c["dim"], causal=c["causal"],
                             window=c["window"], max_new=max(st["new"]), max_length=max(st["lens"]))
    return st["Y"]


# --------------------------------------------------------------------------------------------- what a pass needs
SIZE = {"f16": 2.0, "bf16": 2.0, "f32": 4.0}


def _seen(length, new, causal, window):
    """(keys that some row sees, pairs of a row and a key that it sees)."""
    first, pairs = length, 0
    for p in range(length - new, length):
        hi = p if causal else length - 1
        lo = max(0, p - window + 1) if window else 0
        first, pairs = min(first, lo), pairs + hi - lo + 1
    return length - first, pairs


def work(case):
    c = case
    if c["kind"] == "attend":
        held, added = _lengths(c)
        read = pairs = 0
        for x, a in zip(held, added):
            k, p = _seen(x + a, a, c["causal"], c["window"])
            read, pairs = read + k, pairs + p
        hq = c["heads"] * c["group"]
        blocks = (c["dim"] + BLOCK - 1) // BLOCK
        return {"bytes": 2.0 * 17 * blocks * c["heads"] * read + 2.0 * SIZE[c["x"]] * sum(added) * hq * c["dim"],
                "flops": 4.0 * c["dim"] * hq * pairs}
    if c["kind"] == "store":
        n = 2.0 * c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": n * (SIZE[c["x"]] + SIZE[c["y"]] + 2 * 17 / 32) + 8.0 * c["tokens"], "flops": 8.0 * n}
    held, added = _lengths(c)
    n, page = c["sequences"], c["page"]
    if c["kind"] == "reserve":
        new = sum(_pages(h + a, page) - _pages(h, page) for h, a in zip(held, added))
        return {"bytes": 16.0 * n + 8.0 * new + 8.0 * sum(added), "flops": 4.0 * (n + sum(added))}
    gone = sum(_pages(h, page) for h in held) * c["ended"] / n
    return {"bytes": 12.0 * n + 8.0 * gone, "flops": 4.0 * (n + gone)}


# --------------------------------------------------------------------------------------------- 64 bits
def _nearest64(x):
    """Each value's nearest among the sixteen of its block, of two equally near ones the one whose mantissa bit is 0."""
    grid = torch.tensor([0, 1, 2, 4, .5, 1.5, 3, 6], dtype=torch.float64, device=x.device)      # even mantissas first
    b = torch.nn.functional.pad(x, (0, -x.shape[-1] % BLOCK)).unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(-1, keepdim=True)
    s = torch.exp2((torch.floor(torch.log2(torch.where(amax > 0, amax, 4.0))) - 2.0).clamp(-23, 13))
    m = b.abs() / s
    best, dist = torch.zeros_like(m), m.clone()
    for v in grid[1:]:
        d = (m - v).abs()
        near = d < dist
        best, dist = torch.where(near, v, best), torch.where(near, d, dist)
    return (torch.sign(b) * best * s).flatten(-2)[..., :x.shape[-1]]


def _value64(code, scale):
    """From the fields of a code: (-1)^s 2^(max(x, 1) - 1) (m / 2 + (x > 0)), times 2^(scale - 127)."""
    code = code.int()
    x, m, sign = ((code >> 1) & 3).double(), (code & 1).double(), 1.0 - 2.0 * (code >> 3).double()
    return sign * torch.exp2(x.clamp(min=1.0) - 1.0) * (0.5 * m + (x > 0)) * torch.exp2(scale.double() - 127.0)


def _head64(st, s, head):
    """fp64 keys and values [positions, dim] of one head of a sequence: every element's byte looked up by its address."""
    c = st["case"]
    full, length = _full(c["dim"]), st["lens"][s]
    dev = st["cache"].device
    t, e = torch.arange(length, device=dev)[:, None], torch.arange(c["dim"], device=dev)
    flat = st["cache"].view(-1)
    record = (st["table"][s].long()[t // c["page"]] * c["heads"] + head) * (c["page"] // 32) + t % c["page"] // 32
    base, t = record * (34 * full), t % 32
    kb = flat[base + t * (full // 2) + e // 2]
    ks = flat[base + 32 * full + t * (full // 32) + e // 32]
    g, i, unit = t % 16 // 4, t % 4 + t // 16 * 4, full // 16
    vb = flat[base + 16 * full + ((g * 16 + e // unit) * 8 + i) * (unit // 2) + e % unit // 2]
    vs = flat[base + 33 * full + (g * (full // 32) + e // 32) * 8 + i]
    odd = e % 2 == 1
    return (_value64(torch.where(odd, b >> 4, b & 15), sc) for b, sc in ((kb, ks), (vb, vs)))


def exact(case, seed):
    c = case
    if c["kind"] in ("reserve", "trim"):
        return None                                             # whole numbers: equal to the plain form's
    st = prepare(case, seed)
    if c["kind"] == "store":
        shape = (c["tokens"], c["heads"], c["dim"])
        return {n: torch.cat([_nearest64(x.double()) for x in st[n].view(shape).split(1024)]).flatten(1) for n in ("K", "V")}
    d, gr, at = c["dim"], c["group"], 0
    y = torch.empty(st["Q"].shape, dtype=torch.float64, device="cuda")
    for length, new, s in zip(st["lens"], st["new"], range(c["sequences"])):
        for head in range(c["heads"]):
            k, v = _head64(st, s, head)
            for j in range(head * gr, (head + 1) * gr):
                for r in range(0, new, 2048):
                    rows = torch.arange(r, min(new, r + 2048), device="cuda")
                    score = (st["Q"][at + rows, j * d:(j + 1) * d].double() @ k.t()) / math.sqrt(d)
                    ahead = (length - new + rows)[:, None] - torch.arange(length, device="cuda")        # how far a key lies behind its query
                    hidden = torch.zeros_like(ahead, dtype=torch.bool)
                    if c["causal"]:
                        hidden |= ahead < 0
                    if c["window"]:
                        hidden |= ahead >= c["window"]
                    y[at + rows, j * d:(j + 1) * d] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v
        at += new
    return y
