"""Every form of the microscaled products at sizes that lead to it, in a call of its own and recorded with the routing around it.

The exact result is taken on the device in 64 bits from the dequantized values (which are the oracle's bit for bit, in a test of
their own).  Tolerance as for every product: fp32 sums of n exact terms of magnitude sum S are within 2 n 2^-24 S."""
import numpy as np
import pytest
import torch

from mx4_forms import MX4_FORMS
from paper_2309_15531_amd import binding as B
from test_gpu_mx4 import check_experts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


def quantized(ctx, x):
    """Codes, scales and values (fp32) of a device matrix."""
    codes, scales = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in B.mx4_shapes(*x.shape))
    ctx.adadim_mx4_quantize(x, codes, scales)
    v = torch.empty(x.shape, dtype=torch.float32, device="cuda")
    ctx.adadim_mx4_dequantize(codes, scales, v)
    return codes, scales, v


def randn(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


def check(Y, x, w):
    want, mags = x.double() @ w.double().t().contiguous(), x.double().abs() @ w.double().abs().t().contiguous()
    off = (Y.double() - want).abs() / (2.0 * x.shape[1] * 2.0 ** -24 * mags + 2.0 ** -24 * want.abs() + 2.0 ** -150)
    assert bool((off <= 1.0).all()), float(off.max())


@pytest.mark.parametrize("x", ["f16", "bf16", "mx4"])
@pytest.mark.parametrize("wide", [False, True])
def test_every_form(ctx, x, wide):
    """Y in fp32 with room behind its rows; `wide` weights have scales beyond fp16's, so that fp16 X takes its second way."""
    for (mx, experts, rows, out, inn), form in MX4_FORMS.items():
        if mx != (x == "mx4") or (wide and x != "f16"):
            continue
        print((mx, experts, rows, out, inn), form, flush=True)
        n = max(1, experts)
        w = [quantized(ctx, randn(rows + e, out, inn) * (2.0 ** -30 if wide else 0.05))
             for e in range(n)]
        a = randn(out, rows, inn)
        if mx:
            X, xs, xv = quantized(ctx, a)
        else:
            X, xs = a.to(torch.float16 if x == "f16" else torch.bfloat16), None
            xv = X.float()
        full = torch.full((rows + 1, out + 4), 9.0, device="cuda")
        Y = full[:rows, :out]
        if not experts:
            ctx.adadim_mx4_matmul(X, w[0][0], w[0][1], Y, in_f=inn, x_scales=xs)
            check(Y, xv, w[0][2])
        else:
            # groups of unlike sizes, one of them empty; Y's rows in another order than X's
            cuts = np.sort(np.random.default_rng(rows).integers(0, rows + 1, experts - 1))
            cuts[-1] = cuts[-2] if experts > 2 else cuts[-1]
            offsets = np.concatenate([[0], cuts, [rows]]).astype(np.int32)
            order = np.random.default_rng(out).permutation(rows).astype(np.int32)
            codes, scales = torch.stack([p[0] for p in w]), torch.stack([p[1] for p in w])
            ctx.adadim_mx4_matmul_experts(X, codes, scales, torch.from_numpy(offsets).cuda(), Y, in_f=inn, x_scales=xs,
                                          rows=torch.from_numpy(order).cuda())
            for e in range(experts):
                lo, hi = offsets[e], offsets[e + 1]
                if hi > lo:
                    check(Y[lo:hi], xv[torch.from_numpy(order[lo:hi]).long().cuda()], w[e][2])
        assert bool((full[rows] == 9.0).all()) and bool((full[:, out:] == 9.0).all()), "writes outside Y"


@pytest.mark.parametrize("x", ["f16", "bf16", "mx4"])
def test_a_shared_contraction_gives_the_same_bits_every_time(ctx, x):
    """Shares are added up in their own order, whoever ends last; and one call leaves nothing behind for the next."""
    for (mx, experts, rows, out, inn), form in MX4_FORMS.items():
        if mx != (x == "mx4") or form[1] == 1:
            continue
        print((mx, experts, rows, out, inn), form, flush=True)
        codes, scales, _ = quantized(ctx, randn(1, out, inn))
        a = randn(2, rows, inn)
        X, xs = quantized(ctx, a)[:2] if mx else (a.to(torch.float16 if x == "f16" else torch.bfloat16), None)
        ys = torch.empty((6, rows, out), device="cuda")
        for Y in ys:
            ctx.adadim_mx4_matmul(X, codes, scales, Y, in_f=inn, x_scales=xs)
        assert bool((ys == ys[0]).all())


@pytest.mark.parametrize("tokens", [1, 64, 700])
def test_a_recorded_layer(ctx, tokens):
    """Quantize, route, products, combine, and a product with a shared contraction, recorded once and replayed between other work:
    every replay reads the inputs as they are then."""
    E, k, hidden, inner = 8, 2, 512, 4096
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = B.Context()
        up = [quantized(c, randn(e, inner, hidden) * 0.05)[:2] for e in range(E)]
        down = [quantized(c, randn(100 + e, hidden, inner) * 0.05)[:2] for e in range(E)]
        up, down = ([torch.stack(t) for t in zip(*m)] for m in (up, down))
        out_w = quantized(c, randn(7, 96, hidden))[:2]
        X = torch.empty((tokens, hidden), dtype=torch.bfloat16, device="cuda")
        logits = torch.empty((tokens, E), dtype=torch.float32, device="cuda")
        xq, xs = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in B.mx4_shapes(tokens, hidden))
        chosen, slots = (torch.empty((tokens, k), dtype=torch.int32, device="cuda") for _ in range(2))
        weights = torch.empty((tokens, k), device="cuda")
        offsets, rows = torch.empty(E + 1, dtype=torch.int32, device="cuda"), torch.empty(tokens * k, dtype=torch.int32, device="cuda")
        h = torch.empty((tokens * k, inner), dtype=torch.bfloat16, device="cuda")
        z = torch.empty((tokens * k, hidden), dtype=torch.bfloat16, device="cuda")
        y = torch.empty((tokens, hidden), dtype=torch.bfloat16, device="cuda")
        last = torch.empty((tokens, 96), device="cuda")

        def layer():
            c.adadim_mx4_quantize(X, xq, xs)
            c.adadim_expert_route(logits, chosen, weights, offsets, rows, slots)
            c.adadim_mx4_matmul_experts(xq, *up, offsets, h, in_f=hidden, x_scales=xs, rows=rows)
            c.adadim_mx4_matmul_experts(h, *down, offsets, z)
            c.adadim_expert_combine(z, slots, weights, y)
            c.adadim_mx4_matmul(y, *out_w, last)

        def fill(seed):
            X.copy_(randn(seed, tokens, hidden))
            logits.copy_(randn(seed + 50, tokens, E))

        fill(0)
        layer()                                               # workspaces have their size
        c.adadim_capture_begin()
        try:
            layer()
        finally:
            graph = c.adadim_capture_end()
        try:
            for seed in range(1, 6):
                fill(seed)
                layer()
                want = [t.clone() for t in (chosen, weights, offsets, rows, slots, h, z, y, last)]
                for t in (chosen, weights, offsets, rows, slots, h, z, y, last):
                    t.zero_()
                for _ in range(seed % 2 + 1):
                    c.adadim_graph_launch(graph)
                for t, w in zip((chosen, weights, offsets, rows, slots, h, z, y, last), want):
                    assert torch.equal(t, w), seed
                side.synchronize()
        finally:
            c.adadim_graph_destroy(graph)
    side.synchronize()
    c.close()


def test_rows_of_x_beyond_4_gb(ctx):
    """Rows named by the routing that lie further from the first than 32 bits of bytes reach: they are brought together first."""
    inn, out = 4096, 256
    tokens = (2 ** 32 + 2 ** 28) // (2 * inn)
    codes, scales, wv = quantized(ctx, randn(1, out, inn))
    X = torch.zeros((tokens, inn), dtype=torch.float16, device="cuda")
    named = torch.tensor([0, tokens - 1, 2 ** 31 // (2 * inn), tokens - 2, 5, 2 ** 32 // (2 * inn) + 3], device="cuda")
    X[named] = randn(3, len(named), inn).half()
    for reps in (1, 40):                                      # few rows, and tiles
        rows = named.repeat(reps).int()
        Y = torch.full((len(rows), out), 9.0, device="cuda")
        offsets = torch.tensor([0, len(rows)], dtype=torch.int32, device="cuda")
        ctx.adadim_mx4_matmul_experts(X, codes[None], scales[None], offsets, Y, rows=rows)
        check(Y, X[rows.long()].float(), wv)


@pytest.mark.parametrize("x,y", [("f16", "f16"), ("bf16", "f32"), ("mx4", "bf16")])
@pytest.mark.parametrize("places", [(0,), (129,), (3, 64), (63, 64, 65), (1, 1, 127, 128, 128, 129), (5,) * 20])
def test_fewer_rows_than_experts(ctx, places, x, y):
    """Groups with rows are found among many empty ones; rows in front of the first and behind the last stay."""
    sizes = [places.count(e) for e in range(130)]
    check_experts(ctx, sizes, 70, 260, x, y, lead=2, tail=1)
    check_experts(ctx, sizes, 70, 260, x, y, seed=1)
