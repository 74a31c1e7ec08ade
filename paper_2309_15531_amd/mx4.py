"""Layers of microscaled 4-bit weights: a linear layer, and a layer of experts behind a router; and a paged cache of keys and values in the
same format with the attention over it.

Allocation and call order only; all arithmetic happens in libadadim.so, but for the activation between an expert's two products, which
is the caller's.

A call is part of the stream that is torch's current one, as torch's own operations are, whichever stream the context has.  While the context
records a graph its stream has to be the current one; what the calls allocate then, results and the activation's tensors among it, is the
graph's alone until the graph is destroyed.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B


# torch.cuda.current_stream() makes an object of the stream first: 2.6 us, where this takes 0.1 and a call of the library 3.
_current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _raw_stream(X):
    """The hipStream_t that torch's work on X's device goes to now; None for a host tensor (which the call refuses)."""
    return _current(X.get_device()) if X.is_cuda else None


def _ordered(ctx, X, body, *args):
    """body(*args): library calls and torch's own work, both on the context's stream.

    Where torch's current stream is another one, the context's waits for it first and it waits for the context's behind the body: what came
    before is done for the body, and what follows finds the body done.  So memory may go back to either stream's pool when the call
    returns; what the caller gets is allocated before, from the current stream's.  While a graph is recorded the body's memory is the
    recording's (a replay writes to the same addresses, whenever it comes)."""
    same = _raw_stream(X) in (ctx.stream, None)
    if ctx.recording is not None:
        if not same:
            raise ValueError("a graph is being recorded: the context's stream has to be torch's current stream")
        with torch.cuda.use_mem_pool(_recordings_pool(ctx)):
            return body(*args)
    if same:
        return body(*args)
    here = torch.cuda.current_stream(X.device)
    there = torch.cuda.ExternalStream(ctx.stream, X.device) if ctx.stream else torch.cuda.default_stream(X.device)
    there.wait_stream(here)
    try:
        with torch.cuda.stream(there):
            return body(*args)
    finally:
        here.wait_stream(there)


def _recordings_pool(ctx):
    """The memory that the graph being recorded has to itself."""
    if not ctx.recording:
        ctx.recording.append(torch.cuda.MemPool())
    return ctx.recording[0]


def _output(ctx, shape, dtype, device):
    """What the caller gets from a call."""
    if ctx.recording is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.use_mem_pool(_recordings_pool(ctx)):
        return torch.empty(shape, dtype=dtype, device=device)


class Mx4Weight:
    """An [out, in] weight in mx4 on the device, or one for each of `experts` side by side."""

    def __init__(self, ctx: B.Context, out_f: int, in_f: int, experts: int = 0, device="cuda"):
        self.ctx, self.out_f, self.in_f, self.experts = ctx, out_f, in_f, experts
        lead = (experts,) if experts else ()
        codes, scales = B.mx4_shapes(out_f, in_f)
        self.codes = torch.empty(lead + codes, dtype=torch.uint8, device=device)
        self.scales = torch.empty(lead + scales, dtype=torch.uint8, device=device)

    def _part(self, expert):
        if (expert is None) != (self.experts == 0):
            raise ValueError("name an expert where there are several weights, and none where there is one")
        if expert is None:
            return self.codes, self.scales
        if not 0 <= expert < self.experts:
            raise ValueError(f"expert {expert} of {self.experts}")
        return self.codes[expert], self.scales[expert]

    def store(self, W, expert: int | None = None, hp=None):
        """Quantizes W (fp16, bf16 or fp32 [out, in]).  hp: a prepared Hessian (search.PreparedHessian) of the layer's inputs; the result is
        then the reconstruction error ||X W^T - X Q(W)^T||_F^2 as a device scalar, to be held against the per-OC and per-IC ones."""
        if tuple(W.shape) != (self.out_f, self.in_f):
            raise ValueError(f"W: expected {(self.out_f, self.in_f)}, got {tuple(W.shape)}")
        codes, scales = self._part(expert)
        if hp is None:
            return _ordered(self.ctx, W, self.ctx.adadim_mx4_quantize, W, codes, scales)
        loss = _output(self.ctx, (1,), torch.float32, W.device)
        _ordered(self.ctx, W, self._store_scored, W, codes, scales, hp, loss)
        return loss

    def _store_scored(self, W, codes, scales, hp, loss):
        dW = self.ctx.alloc_score(self.out_f, self.in_f, W.device)
        self.ctx.adadim_mx4_quantize(W, codes, scales, dW, B.DW_F16_SCALED, hp.colscale)
        self.ctx.adadim_layer_error_prepared(dW, B.DW_F16_SCALED, hp.Hs, hp.hmeta, loss, shape=(self.out_f, self.in_f))

    def values(self, expert: int | None = None, dtype=torch.float32):
        """The stored weight as [out, in] of `dtype`."""
        Y = _output(self.ctx, (self.out_f, self.in_f), dtype, self.codes.device)
        _ordered(self.ctx, Y, self.ctx.adadim_mx4_dequantize, *self._part(expert), Y)
        return Y


def quantize_rows(ctx: B.Context, X):
    """(codes, scales) of the rows of X, as a product's left operand."""
    codes, scales = (_output(ctx, n, torch.uint8, X.device) for n in B.mx4_shapes(*X.shape))
    _ordered(ctx, X, ctx.adadim_mx4_quantize, X, codes, scales)
    return codes, scales


def _quantized(ctx, X):
    """The same where the call is ordered already."""
    codes, scales = (torch.empty(n, dtype=torch.uint8, device=X.device) for n in B.mx4_shapes(*X.shape))
    ctx.adadim_mx4_quantize(X, codes, scales)
    return codes, scales


class Mx4Linear:
    """Y = X W^T for X fp16 or bf16 [tokens, in].

    mx4_inputs: from that many tokens on X is quantized as well (0: never), and the product runs at the 4-bit rate: 4096 tokens through
    [4096, 4096] take 47 us with the quantization, 117 us as bf16."""

    def __init__(self, weight: Mx4Weight, mx4_inputs: int = 0):
        if weight.experts:
            raise ValueError("a linear layer has one weight")
        self.weight, self.mx4_inputs = weight, mx4_inputs

    def __call__(self, X, Y=None):
        w = self.weight
        if Y is None:
            Y = _output(w.ctx, (X.shape[0], w.out_f), X.dtype, X.device)
        _ordered(w.ctx, X, self._run, X, Y)
        return Y

    def _run(self, X, Y):
        w = self.weight
        if self.mx4_inputs and X.shape[0] >= self.mx4_inputs:
            codes, scales = _quantized(w.ctx, X)
            w.ctx.adadim_mx4_matmul(codes, w.codes, w.scales, Y, in_f=w.in_f, x_scales=scales)
        else:
            w.ctx.adadim_mx4_matmul(X, w.codes, w.scales, Y, in_f=w.in_f)


class Mx4Experts:
    """Y[t] = sum over the k experts e chosen for token t of weight(t, e) down_e(activation(up_e(X[t]))).

    activation takes the rows [rows, up.out] to [rows, down.in] (fp16 or bf16); it may see rows that no expert has written where the
    router's mask leaves a token fewer than k experts: nothing reads them afterwards.  mx4_inputs as in Mx4Linear, by the rows
    of each product.  The host learns neither the choices nor how many rows an expert has: nothing here waits for the device, and
    with the activation a layer can be recorded as a graph (adadim_capture_begin; make the same call once before)."""

    def __init__(self, up: Mx4Weight, down: Mx4Weight, k: int, activation, renormalize: bool = True, mx4_inputs: int = 0):
        if up.experts != down.experts or not up.experts or up.in_f != down.out_f:
            raise ValueError("up and down have the same experts, and down leads back to up's inputs")
        if not 1 <= k <= up.experts:
            raise ValueError(f"{k} of {up.experts} experts")
        self.ctx, self.up, self.down, self.k = up.ctx, up, down, k
        self.activation, self.renormalize, self.mx4_inputs = activation, renormalize, mx4_inputs

    def _product(self, X, weight, offsets, n_rows, rows=None):
        Y = torch.empty((n_rows, weight.out_f), dtype=X.dtype, device=X.device)
        if self.mx4_inputs and n_rows >= self.mx4_inputs:
            codes, scales = _quantized(self.ctx, X)
            self.ctx.adadim_mx4_matmul_experts(codes, weight.codes, weight.scales, offsets, Y, in_f=weight.in_f, x_scales=scales, rows=rows)
        else:
            self.ctx.adadim_mx4_matmul_experts(X, weight.codes, weight.scales, offsets, Y, in_f=weight.in_f, rows=rows)
        return Y

    def __call__(self, X, logits, Y=None):
        """X [tokens, in] fp16 or bf16, logits [tokens, experts] (-infinity: an expert this token must not have)."""
        if Y is None:
            Y = _output(self.ctx, (X.shape[0], self.down.out_f), X.dtype, X.device)
        _ordered(self.ctx, X, self._run, X, logits, Y)
        return Y

    def _run(self, X, logits, Y):
        tokens, k, dev = X.shape[0], self.k, X.device
        chosen, slots = (torch.empty((tokens, k), dtype=torch.int32, device=dev) for _ in range(2))
        weights = torch.empty((tokens, k), dtype=torch.float32, device=dev)
        offsets = torch.empty(self.up.experts + 1, dtype=torch.int32, device=dev)
        rows = torch.empty(tokens * k, dtype=torch.int32, device=dev)
        self.ctx.adadim_expert_route(logits, chosen, weights, offsets, rows, slots, renormalize=self.renormalize)
        h = self._product(X, self.up, offsets, tokens * k, rows)
        z = self._product(self.activation(h), self.down, offsets, tokens * k)
        self.ctx.adadim_expert_combine(z, slots, weights, Y)


class NewRows(NamedTuple):
    """What CachePages.add gives, all int32 on the device."""
    offsets: torch.Tensor                 # [sequences + 1]: where each sequence's new rows begin
    slots: torch.Tensor                   # [tokens]: a row's place in the caches, -1 behind the last sequence's rows
    positions: torch.Tensor               # [tokens]: its position in its sequence, -1 there
    lacking: torch.Tensor                 # [1]: 0, or why nothing was added: pages short, or -1 (table or rows too small, a negative number)


class CachePages:
    """Which pages hold what, for the caches of all layers of a model: `pages` pages of `page` positions for up to `sequences` sequences of up to
    `width` pages.  All of it lives on the device, and no call waits for it; a step can be recorded as a graph."""

    def __init__(self, ctx: B.Context, pages: int, page: int, sequences: int, width: int, device="cuda"):
        self.ctx, self.pages, self.page = ctx, pages, page
        self.table = torch.full((sequences, width), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.free = torch.arange(pages, dtype=torch.int32, device=device)
        self.count = torch.full((1,), pages, dtype=torch.int32, device=device)

    def add(self, added, tokens: int) -> NewRows:
        """added[s] (int32, device) more tokens for each sequence, `tokens` at most in all.  All or nothing: where lacking is not 0 no sequence
        has grown and no row has a slot."""
        n, dev = self.lengths.numel(), added.device
        rows = NewRows(*(_output(self.ctx, (k,), torch.int32, dev) for k in (n + 1, tokens, tokens, 1)))
        _ordered(self.ctx, added, self.ctx.adadim_cache_reserve, self.lengths, added, self.page, self.table, self.free, self.count, self.lengths,
                 rows.offsets, rows.slots, rows.positions, self.count, rows.lacking)
        return rows

    def trim(self, kept):
        """Each sequence keeps its first kept[s] (int32, device) tokens; the pages behind them are free again."""
        _ordered(self.ctx, kept, self.ctx.adadim_cache_trim, self.lengths, kept, self.page, self.table, self.free, self.count, self.lengths, self.count)


class Mx4Cache:
    """A layer's keys and values, `heads` heads of `dim` elements, filled up to 64, 128 or 256 and 4.25 bits each: 4.25 KB a token for 32 heads of 128,
    where fp16 takes 16."""

    def __init__(self, pages: CachePages, heads: int, dim: int):
        self.ctx, self.pages, self.heads, self.dim = pages.ctx, pages, heads, dim
        self.records = torch.empty(B.mx4_cache_shape(pages.pages, pages.page, heads, dim), dtype=torch.uint8, device=pages.table.device)

    def store(self, K, V, slots):
        """Rows [tokens, heads * dim] (fp16, bf16 or fp32; views of one projection's output will do) to their slots."""
        _ordered(self.ctx, K, self.ctx.adadim_mx4_cache_store, K, V, slots, self.records)

    def load(self, slots, dtype=torch.float32):
        """(K, V) [tokens, heads * dim] as stored."""
        K, V = (_output(self.ctx, (slots.numel(), self.heads * self.dim), dtype, slots.device) for _ in range(2))
        _ordered(self.ctx, slots, self.ctx.adadim_mx4_cache_load, slots, self.records, K, V)
        return K, V

    def attend(self, Q, offsets, Y=None, scale: float | None = None, causal: bool = True, window: int = 0, max_new: int = 0, max_length: int = 0):
        """Attention of the rows of Q [tokens, query heads * dim] (fp16 or bf16), whose keys and values are stored already, to their sequences.
        max_new, max_length: the most new rows and positions of a sequence, where the host knows them (a decoding step: 1); they lay the
        launch out for all sequences, the result does not depend on them.  Rows in no sequence are left as they are (without Y: not initialized)."""
        if Y is None:
            Y = _output(self.ctx, tuple(Q.shape), Q.dtype, Q.device)
        p = self.pages
        _ordered(self.ctx, Q, lambda: self.ctx.adadim_mx4_attention(Q, self.records, p.table, offsets, p.lengths, Y, self.dim, scale=scale, causal=causal,
                                                                    window=window, max_new=max_new, max_length=max_length))
        return Y
