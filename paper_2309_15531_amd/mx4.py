"""Layers of microscaled 4-bit weights: a linear layer, and a layer of experts behind a router.

Allocation and call order only; all arithmetic happens in libadadim.so, but for the activation between an expert's two products, which
is the caller's.

A call is part of the stream that is torch's current one, as torch's own operations are, whichever stream the context has.  While the context
records a graph its stream has to be the current one; what the calls allocate then, the activation's tensors among it, stays until the graph is
destroyed, and the results of the recorded calls with it.
"""
from __future__ import annotations

import torch

from . import binding as B


class _Ordered:
    """The body's library calls and torch's own work in it, both on the context's stream.

    Where torch's current stream is another one, the context's waits for it first and it waits for the context's behind the body: what came
    before is done for the body, and what follows finds the body done.  So memory may go back to either stream's pool when the call
    returns; what the caller gets is allocated before, from the current stream's.  While a graph is recorded the body's memory is the
    recording's (a replay writes to the same addresses, whenever it comes)."""

    __slots__ = ("ctx", "here", "there", "switch")

    def __init__(self, ctx):
        self.ctx = ctx

    def __enter__(self):
        ctx = self.ctx
        here = torch.cuda.current_stream()
        self.there = self.switch = None
        if here.cuda_stream != ctx.stream:
            if ctx.recording is not None:
                raise ValueError("a graph is being recorded: the context's stream has to be torch's current stream")
            self.here, self.there = here, torch.cuda.ExternalStream(ctx.stream) if ctx.stream else torch.cuda.default_stream()
            self.there.wait_stream(here)
            self.switch = torch.cuda.stream(self.there)
        elif ctx.recording is not None:
            self.switch = torch.cuda.use_mem_pool(_recordings_pool(ctx))
        if self.switch is not None:
            self.switch.__enter__()

    def __exit__(self, *error):
        if self.switch is not None:
            self.switch.__exit__(*error)
        if self.there is not None:
            self.here.wait_stream(self.there)


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
            with _Ordered(self.ctx):
                self.ctx.adadim_mx4_quantize(W, codes, scales)
            return None
        loss = _output(self.ctx, (1,), torch.float32, W.device)
        with _Ordered(self.ctx):
            dW = self.ctx.alloc_score(self.out_f, self.in_f, W.device)
            self.ctx.adadim_mx4_quantize(W, codes, scales, dW, B.DW_F16_SCALED, hp.colscale)
            self.ctx.adadim_layer_error_prepared(dW, B.DW_F16_SCALED, hp.Hs, hp.hmeta, loss, shape=(self.out_f, self.in_f))
        return loss

    def values(self, expert: int | None = None, dtype=torch.float32):
        """The stored weight as [out, in] of `dtype`."""
        Y = _output(self.ctx, (self.out_f, self.in_f), dtype, self.codes.device)
        with _Ordered(self.ctx):
            self.ctx.adadim_mx4_dequantize(*self._part(expert), Y)
        return Y


def quantize_rows(ctx: B.Context, X):
    """(codes, scales) of the rows of X, as a product's left operand."""
    codes, scales = (_output(ctx, n, torch.uint8, X.device) for n in B.mx4_shapes(*X.shape))
    with _Ordered(ctx):
        ctx.adadim_mx4_quantize(X, codes, scales)
    return codes, scales


def _quantized(ctx, X):
    """The same where the call is ordered already."""
    codes, scales = (torch.empty(n, dtype=torch.uint8, device=X.device) for n in B.mx4_shapes(*X.shape))
    ctx.adadim_mx4_quantize(X, codes, scales)
    return codes, scales


class Mx4Linear:
    """Y = X W^T for X fp16 or bf16 [tokens, in].

    mx4_inputs: from that many tokens on X is quantized as well (0: never), and the product runs at the 4-bit rate: 4096 tokens through
    [4096, 4096] take 48 us with the quantization, 115 us as bf16."""

    def __init__(self, weight: Mx4Weight, mx4_inputs: int = 0):
        if weight.experts:
            raise ValueError("a linear layer has one weight")
        self.weight, self.mx4_inputs = weight, mx4_inputs

    def __call__(self, X, Y=None):
        w = self.weight
        if Y is None:
            Y = _output(w.ctx, (X.shape[0], w.out_f), X.dtype, X.device)
        with _Ordered(w.ctx):
            if self.mx4_inputs and X.shape[0] >= self.mx4_inputs:
                codes, scales = _quantized(w.ctx, X)
                w.ctx.adadim_mx4_matmul(codes, w.codes, w.scales, Y, in_f=w.in_f, x_scales=scales)
            else:
                w.ctx.adadim_mx4_matmul(X, w.codes, w.scales, Y, in_f=w.in_f)
        return Y


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
        tokens, k, dev = X.shape[0], self.k, X.device
        if Y is None:
            Y = _output(self.ctx, (tokens, self.down.out_f), X.dtype, dev)
        with _Ordered(self.ctx):
            chosen, slots = (torch.empty((tokens, k), dtype=torch.int32, device=dev) for _ in range(2))
            weights = torch.empty((tokens, k), dtype=torch.float32, device=dev)
            offsets = torch.empty(self.up.experts + 1, dtype=torch.int32, device=dev)
            rows = torch.empty(tokens * k, dtype=torch.int32, device=dev)
            self.ctx.adadim_expert_route(logits, chosen, weights, offsets, rows, slots, renormalize=self.renormalize)
            h = self._product(X, self.up, offsets, tokens * k, rows)
            z = self._product(self.activation(h), self.down, offsets, tokens * k)
            self.ctx.adadim_expert_combine(z, slots, weights, Y)
        return Y
