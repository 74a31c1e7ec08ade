"""Performance cases of the microscaled 4-bit operators: what a serving program calls behind the weight quantization.

A microscaled ("mx4") row is cut into blocks of 32 consecutive values; a block stores one power-of-two scale in a byte
(exponent + 127; 255 is NaN) and 32 codes of 4 bits: sign, two bits of exponent, one of mantissa, the values
0, .5, 1, 1.5, 2, 3, 4, 6.  Two codes to a byte, the even element in the low half.  A row is held in pieces of 128 values, 64
bytes of codes and a word of 4 scale bytes, the last piece filled up with zeros of scale 1; the words of a piece lie together for
all rows: codes u8 [rows, 64 * pieces], scales u8 [pieces, rows, 4].

  quantize  rows of 16- or 32-bit values to codes and scales, and back to values
  matmul    Y = X W^T with W in mx4, X in 16 bits (weight-only) or in mx4 itself
  experts   the same with one weight per expert, the rows of X sorted by expert in ragged groups
  route     router scores to the k experts of each token, their shares, and the rows sorted by expert
  combine   the experts' outputs of a token, weighted and added up

`listed()` are fixed sizes of the shapes this package names; `draw(rng)` takes further ones from the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK, PIECE = 32, 128
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
def _quantize(name, rows, cols, x, y):
    return {"name": name, "kind": "quantize", "rows": rows, "cols": cols, "x": x, "y": y}


def _matmul(name, tokens, out, inn, x, y):
    return {"name": name, "kind": "matmul", "tokens": tokens, "out": out, "in": inn, "x": x, "y": y}


def _experts(name, tokens, k, experts, out, inn, x, y):
    return {"name": name, "kind": "experts", "tokens": tokens, "k": k, "experts": experts, "out": out, "in": inn, "x": x, "y": y}


def _route(name, tokens, k, experts, x, renormalize):
    return {"name": name, "kind": "route", "tokens": tokens, "k": k, "experts": experts, "x": x, "renormalize": renormalize}


def _combine(name, tokens, k, cols, x, y):
    return {"name": name, "kind": "combine", "tokens": tokens, "k": k, "cols": cols, "x": x, "y": y}


def listed():
    return [
        # the activations of sixteen sequences that decode together, ahead of a 4-bit by 4-bit product
        _quantize("quantize_tokens", 16, 4096, "bf16", "bf16"),
        # a weight of a 70B-shaped block, once per model load
        _quantize("quantize_weight", 28672, 8192, "f16", "f16"),
        # one token through the gate projection of a 7B-shaped block: a read of the weight
        _matmul("linear_token", 1, 11008, 4096, "f16", "f16"),
        # a few dozen tokens through a layer whose sizes are no multiple of anything
        _matmul("linear_ragged", 37, 2761, 1721, "bf16", "f32"),
        # a prompt through the down projection of that block, activations as they are
        _matmul("linear_prompt", 2048, 4096, 11008, "f16", "f16"),
        # a batch of prompts through the gate projection of a 70B-shaped block, activations in mx4 too
        _matmul("mx4_prompt", 8192, 28672, 8192, "mx4", "bf16"),
        # sixteen decoding sequences, two of eight experts each: a read of nearly all experts
        _experts("experts_decode", 16, 2, 8, 11008, 4096, "f16", "f16"),
        # a batch of prompts, two of sixteen experts per token, groups of uneven length
        _experts("experts_prompt", 4096, 2, 16, 4096, 5120, "mx4", "bf16"),
        # the router of that decode step, and of a large batch over many experts
        _route("route_decode", 16, 2, 8, "f32", True),
        _route("route_prompt", 16384, 8, 128, "bf16", True),
        # the experts' outputs back to their tokens, for both
        _combine("combine_decode", 16, 2, 4096, "f16", "f16"),
        _combine("combine_prompt", 8192, 8, 4096, "bf16", "bf16"),
    ]


MOST_FLOPS = 2.0 * 8192 * 28672 * 8192
MOST_EXPERTS = 2.0 * 4096 * 2 * 4096 * 5120 * 2


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // step, max(1, int(round(v / step)))) * step


def draw(rng):
    kind = rng.choice(["quantize", "matmul", "matmul", "matmul", "experts", "experts", "route", "combine"])
    step = rng.choice([1, 8, 32, 32, 128])                      # of the contracted axis
    if kind == "quantize":
        x = rng.choice(["f16", "f16", "bf16", "f32"])
        c = _quantize("", _log(rng, 1, 28672), _log(rng, 64, 8192, step), x, rng.choice(["bf16", "f32", x]))
    elif kind == "matmul":
        tokens, out, inn = _log(rng, 1, 8192), _log(rng, 64, 28672, rng.choice([1, 8, 64])), _log(rng, 64, 11008, step)
        x = rng.choice(["f16", "f16", "bf16", "mx4", "mx4"])
        y = rng.choice(["f16", "bf16", "bf16", "f32"]) if x == "mx4" else rng.choice([x, x, "f32"])
        c = _matmul("", tokens, out, inn, x, y)
        while 2.0 * c["tokens"] * out * inn > MOST_FLOPS / 4:
            c["tokens"] //= 2
    elif kind == "experts":
        experts = rng.choice([4, 8, 8, 16, 32, 64])
        k = rng.choice([1, 2, 2, 4])
        tokens, out, inn = _log(rng, 1, 4096), _log(rng, 256, 11008, rng.choice([1, 8, 64])), _log(rng, 256, 5120, step)
        while experts * out * inn > 8 * 11008 * 4096:
            out = max(256, out // 2)
            inn = max(256, inn // 2 // step * step)
        x = rng.choice(["f16", "bf16", "mx4"])
        c = _experts("", tokens, k, experts, out, inn, x, rng.choice(["f16", "bf16"]) if x == "mx4" else x)
        while 2.0 * c["tokens"] * k * out * inn > MOST_EXPERTS:
            c["tokens"] //= 2
    elif kind == "route":
        experts = rng.choice([4, 8, 16, 60, 64, 128, 256])
        k = min(experts, rng.choice([1, 2, 2, 4, 6, 8]))
        c = _route("", _log(rng, 1, 16384), k, experts, rng.choice(["f32", "f16", "bf16"]), rng.random() < 0.7)
        while c["tokens"] * experts > 16384 * 128:
            c["tokens"] //= 2
    else:
        k = rng.choice([1, 2, 2, 4, 8])
        x = rng.choice(["f16", "bf16", "bf16", "f32"])
        c = _combine("", _log(rng, 1, 16384), k, _log(rng, 64, 8192, rng.choice([1, 8, 64])), x, rng.choice([x, x, "f32"]))
        while c["tokens"] * k * c["cols"] > 8192 * 8 * 4096 / (2 if x == "f32" else 1):
            c["tokens"] //= 2
    c.pop("name", None)
    return {n: v + 32 if v == 3072 else v for n, v in c.items()}    # (a width that no shape of this package has)


# --------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) & 0x7FFFFFFF)


def _randn(shape, g):
    return torch.randn(shape, dtype=torch.float32, device="cuda", generator=g)


def _acts(rows, cols, g):
    """Activations: ordinary channels of unit size and a few heavy ones."""
    x = _randn((rows, cols), g)
    heavy = torch.randint(0, cols, (max(1, min(8, cols // 64)),), device="cuda", generator=g)
    x[:, heavy] *= 30.0
    return x


def _weights(rows, cols, g):
    """N(0, 0.02^2) with a hundredth of the columns five times as large."""
    w = _randn((rows, cols), g).mul_(0.02)
    w.mul_(torch.where(torch.rand(cols, device="cuda", generator=g) < 0.01, 5.0, 1.0))
    return w


def _padded(x):
    pad = -x.shape[-1] % PIECE
    return torch.nn.functional.pad(x, (0, pad)) if pad else x


def _scale(amax, steps):
    """(exponent + 127, the power of two itself) that brings a block's largest value into [4, 8); 1 for a block of zeros."""
    e = (torch.where(amax > 0, torch.frexp(amax).exponent - 3, 0).clamp(-127, 127) + 127).int()
    return e, steps.index_select(0, e.reshape(-1)).view(amax.shape)


def _quantized(x, steps):
    """(codes u8, scales u8) of fp32 rows: the operands that a program holds in mx4."""
    xb = _padded(x).unflatten(-1, (-1, BLOCK))
    e, s = _scale(xb.abs().amax(-1), steps)
    m = xb.abs() / s[..., None]
    q = torch.zeros_like(m, dtype=torch.uint8)
    for edge, even in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        q += (m >= edge) if even else (m > edge)
    q |= torch.signbit(xb).to(torch.uint8) << 3
    q = q.flatten(-2)
    return (q[..., 0::2] | (q[..., 1::2] << 4)).contiguous(), e.to(torch.uint8).unflatten(-1, (-1, 4)).transpose(0, 1).contiguous()


def _quantized_experts(experts, out, inn, g, steps):
    pairs = [_quantized(_weights(out, inn, g), steps) for _ in range(experts)]
    return torch.stack([p[0] for p in pairs]), torch.stack([p[1] for p in pairs])


def _routed(tokens, k, experts, g):
    """(offsets, rows) of a router that prefers some experts: the rows of each expert in the order of the tokens."""
    score = _randn((tokens, experts), g) + 0.7 * _randn((experts,), g)
    chosen = score.topk(k, -1).indices.reshape(-1)
    order = torch.argsort(chosen, stable=True)
    counts = torch.bincount(chosen, minlength=experts)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return offsets.to(torch.int32), (order // k).to(torch.int32)


def _tables():
    """The values of the 256 bytes: pairs of codes, scales."""
    v = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float32)
    b = torch.arange(256)
    s = torch.ldexp(torch.ones(256, dtype=torch.float64), b - 127).float()
    s[255] = float("nan")
    return torch.stack([v[b & 15], v[b >> 4]], 1).cuda(), s.cuda()


def _pieces(cols):
    return (cols + PIECE - 1) // PIECE


def _empty(*shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    c, g = case, _gen(seed * 7 + 1)
    st = {"case": c}
    st["pairs"], st["steps"] = _tables()
    if c["kind"] == "quantize":
        rows, cols = c["rows"], c["cols"]
        make = _weights if c["x"] == "f16" else _acts
        st["X"] = make(rows, cols, g).to(TYPES[c["x"]])
        st["codes"] = _empty(rows, 64 * _pieces(cols), dtype=torch.uint8)
        st["scales"] = _empty(_pieces(cols), rows, 4, dtype=torch.uint8)
        st["Y"] = _empty(rows, cols, dtype=TYPES[c["y"]])
    elif c["kind"] in ("matmul", "experts"):
        x = _acts(c["tokens"], c["in"], g)
        st["X"], st["x_scales"] = _quantized(x, st["steps"]) if c["x"] == "mx4" else (x.to(TYPES[c["x"]]), None)
        if c["kind"] == "matmul":
            st["codes"], st["scales"] = _quantized(_weights(c["out"], c["in"], g), st["steps"])
            st["Y"] = _empty(c["tokens"], c["out"], dtype=TYPES[c["y"]])
        else:
            st["codes"], st["scales"] = _quantized_experts(c["experts"], c["out"], c["in"], g, st["steps"])
            st["offsets"], st["rows"] = _routed(c["tokens"], c["k"], c["experts"], g)
            st["Y"] = _empty(c["tokens"] * c["k"], c["out"], dtype=TYPES[c["y"]])
    elif c["kind"] == "route":
        t, k, e = c["tokens"], c["k"], c["experts"]
        st["logits"] = (_randn((t, e), g) + 0.7 * _randn((e,), g)).to(TYPES[c["x"]])
        st["chosen"], st["weights"] = _empty(t, k, dtype=torch.int32), _empty(t, k, dtype=torch.float32)
        st["offsets"], st["rows"], st["slots"] = (_empty(e + 1, dtype=torch.int32), _empty(t * k, dtype=torch.int32),
                                                  _empty(t, k, dtype=torch.int32))
    else:
        t, k = c["tokens"], c["k"]
        st["Z"] = _randn((t * k, c["cols"]), g).to(TYPES[c["x"]])
        st["weights"] = torch.softmax(_randn((t, k), g), -1)
        st["slots"] = torch.randperm(t * k, device="cuda", generator=g).to(torch.int32).view(t, k)
        st["Y"] = _empty(t, c["cols"], dtype=TYPES[c["y"]])
    return st


# --------------------------------------------------------------------------------------------- the plain forms
def _values(codes, scales, cols, st):
    """fp32 values [.., cols] of mx4 rows."""
    s = scales.transpose(-3, -2).flatten(-2)                    # [.., rows, blocks]
    v = st["pairs"].index_select(0, codes.reshape(-1).int()).view(*s.shape, BLOCK)
    return (v * st["steps"].index_select(0, s.reshape(-1).int()).view(*s.shape, 1)).flatten(-2)[..., :cols]


def _plain_quantize(st):
    """Scale: the power of two that brings the block's largest value into [4, 8); codes: nearest, ties to even."""
    c = st["case"]
    x = _padded(st["X"].float()).unflatten(-1, (-1, BLOCK))
    s = _scale(x.abs().amax(-1, keepdim=True), st["steps"])[1]
    m = x.abs() / s
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    m = torch.clamp(torch.round(m / step) * step, max=6.0)
    return (torch.copysign(m, x) * s).flatten(-2)[..., :c["cols"]].to(TYPES[c["y"]])


def _plain_input(st):
    c = st["case"]
    return _values(st["X"], st["x_scales"], c["in"], st) if c["x"] == "mx4" else st["X"].float()


def _plain_matmul(st):
    c = st["case"]
    w = _values(st["codes"], st["scales"], c["in"], st)
    return (_plain_input(st) @ w.t()).to(TYPES[c["y"]])


def _plain_experts(st):
    """The groups, filled up to the longest one, in one batch of products."""
    c = st["case"]
    w = _values(st["codes"], st["scales"], c["in"], st)
    x = _plain_input(st)[st["rows"]]
    n = st["offsets"][1:] - st["offsets"][:-1]
    at = torch.arange(int(n.max()), device=x.device)
    have = at < n[:, None]
    place = torch.where(have, st["offsets"][:-1, None] + at, 0)
    y = torch.bmm(x[place], w.transpose(1, 2))
    return y[have].to(TYPES[c["y"]])


def _plain_route(st):
    c = st["case"]
    t, k, e = c["tokens"], c["k"], c["experts"]
    l = st["logits"].float()
    top, chosen = torch.sort(l, dim=-1, descending=True, stable=True)
    top, chosen = top[:, :k], chosen[:, :k]
    p = torch.exp(top - top[:, :1])
    weights = p / (p if c["renormalize"] else torch.exp(l - top[:, :1])).sum(-1, keepdim=True)
    order = torch.argsort(chosen.reshape(-1), stable=True)
    slots = torch.empty_like(order)
    slots[order] = torch.arange(t * k, device=l.device)
    counts = (chosen.reshape(-1, 1) == torch.arange(e, device=l.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return {"chosen": chosen.int(), "weights": weights, "offsets": offsets.int(), "rows": (order // k).int(),
            "slots": slots.view(t, k).int()}


def _plain_combine(st):
    c = st["case"]
    return (st["Z"].float()[st["slots"]] * st["weights"][..., None]).sum(1).to(TYPES[c["y"]])


PLAIN = {"quantize": _plain_quantize, "matmul": _plain_matmul, "experts": _plain_experts, "route": _plain_route,
         "combine": _plain_combine}


# --------------------------------------------------------------------------------------------- one pass
def run(st):
    c = st["case"]
    if not own:
        return PLAIN[c["kind"]](st)
    ctx = _context()
    if c["kind"] == "quantize":
        ctx.adadim_mx4_quantize(st["X"], st["codes"], st["scales"])
        ctx.adadim_mx4_dequantize(st["codes"], st["scales"], st["Y"])
        return st["Y"]
    if c["kind"] == "matmul":
        ctx.adadim_mx4_matmul(st["X"], st["codes"], st["scales"], st["Y"], in_f=c["in"], x_scales=st["x_scales"])
        return st["Y"]
    if c["kind"] == "experts":
        ctx.adadim_mx4_matmul_experts(st["X"], st["codes"], st["scales"], st["offsets"], st["Y"], in_f=c["in"],
                                      x_scales=st["x_scales"], rows=st["rows"])
        return st["Y"]
    if c["kind"] == "route":
        ctx.adadim_expert_route(st["logits"], st["chosen"], st["weights"], st["offsets"], st["rows"], st["slots"],
                                renormalize=c["renormalize"])
        return {n: st[n] for n in ("chosen", "weights", "offsets", "rows", "slots")}
    ctx.adadim_expert_combine(st["Z"], st["slots"], st["weights"], st["Y"])
    return st["Y"]


# --------------------------------------------------------------------------------------------- what a pass needs
SIZE = {"f16": 2.0, "bf16": 2.0, "f32": 4.0}


def _mx4_bytes(rows, cols):
    return 17.0 * rows * ((cols + BLOCK - 1) // BLOCK)


def work(case):
    c = case
    if c["kind"] == "quantize":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (SIZE[c["x"]] + SIZE[c["y"]]) + _mx4_bytes(c["rows"], c["cols"]), "flops": 8.0 * n}
    if c["kind"] in ("matmul", "experts"):
        t, k = c["tokens"], c.get("k", 1)
        x = _mx4_bytes(t, c["in"]) if c["x"] == "mx4" else SIZE[c["x"]] * t * c["in"]
        # of the experts' weights those that a token asks for (as many as even choices leave out, at most)
        e = c.get("experts")
        read = 1.0 if e is None else max(float(k), e * (1.0 - (1.0 - k / e) ** t))
        return {"bytes": read * _mx4_bytes(c["out"], c["in"]) + x + SIZE[c["y"]] * t * k * c["out"],
                "flops": 2.0 * t * k * c["out"] * c["in"]}
    if c["kind"] == "route":
        t, k, e = c["tokens"], c["k"], c["experts"]
        return {"bytes": SIZE[c["x"]] * t * e + 16.0 * t * k + 4 * (e + 1), "flops": 4.0 * t * e}
    t, k, n = c["tokens"], c["k"], c["cols"]
    return {"bytes": SIZE[c["x"]] * t * k * n + SIZE[c["y"]] * t * n + 8.0 * t * k, "flops": 2.0 * t * k * n}


# --------------------------------------------------------------------------------------------- 64 bits
def _values64(codes, scales, cols):
    """fp64 values of mx4 rows, from the fields of a code: (-1)^s * 2^(max(x, 1) - 1) * (m / 2 + (x > 0))."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    x, m = ((q >> 1) & 3).double(), (q & 1).double()
    v = torch.exp2(x.clamp(min=1.0) - 1.0) * (0.5 * m + (x > 0)) * (1.0 - 2.0 * (q >> 3).double())
    return (v.unflatten(-1, (-1, BLOCK)) * torch.exp2(scales.transpose(0, 1).flatten(1).double() - 127.0)[..., None]).flatten(-2)[..., :cols]


def _nearest64(x):
    """The values that codes and scales of x stand for: each the nearest of the eight, of two equally near ones the one
    whose mantissa bit is 0."""
    grid = torch.tensor([0, 1, 2, 4, .5, 1.5, 3, 6], dtype=torch.float64, device=x.device)      # even mantissas first
    b = _padded(x).unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(-1, keepdim=True)
    s = torch.exp2((torch.floor(torch.log2(torch.where(amax > 0, amax, 4.0))) - 2.0).clamp(-127, 127))
    m = b.abs() / s
    best, dist = torch.zeros_like(m), m.clone()
    for v in grid[1:]:
        d = (m - v).abs()
        near = d < dist
        best, dist = torch.where(near, v, best), torch.where(near, d, dist)
    return (torch.sign(b) * best * s).flatten(-2)[..., :x.shape[-1]]


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["kind"] == "quantize":
        return torch.cat([_nearest64(x.double()) for x in st["X"].split(4096)])
    if c["kind"] == "route":
        l = st["logits"].double()
        left, t, k = l.clone(), c["tokens"], c["k"]
        chosen = torch.empty((t, k), dtype=torch.int64, device=l.device)
        for j in range(k):                                      # the largest one left, the first of equal ones
            best = left == left.amax(-1, keepdim=True)
            chosen[:, j] = torch.where(best, torch.arange(c["experts"], device=l.device), c["experts"]).amin(-1)
            left.scatter_(1, chosen[:, j:j + 1], -math.inf)
        p = torch.softmax(l, -1).gather(1, chosen)
        return {"chosen": None, "weights": p / p.sum(-1, keepdim=True) if c["renormalize"] else p, "offsets": None,
                "rows": None, "slots": None}
    if c["kind"] == "combine":
        parts = zip(st["slots"].split(1024), st["weights"].split(1024))
        return torch.cat([torch.matmul(w.double()[:, None], st["Z"][s.long()].double()).squeeze(1) for s, w in parts])
    x = _values64(st["X"], st["x_scales"], c["in"]) if c["x"] == "mx4" else st["X"].double()
    if c["kind"] == "matmul":
        parts = zip(st["codes"].split(4096), st["scales"].split(4096, 1))
        return torch.cat([x @ _values64(q, s, c["in"]).t() for q, s in parts], 1)
    at, y = st["offsets"].tolist(), []
    for e in range(c["experts"]):
        rows = st["rows"][at[e]:at[e + 1]].long()
        y.append(x[rows] @ _values64(st["codes"][e], st["scales"][e], c["in"]).t())
    return torch.cat(y)
