"""Edges of the microscaled operators and of the routing that other tests do not reach."""
import numpy as np
import pytest
import torch

from mx4_group_forms import MX4_GROUP_FORMS
from paper_2309_15531_amd import binding as B
from test_gpu_mx4 import TYPES, check_route, mx4, rng, spread
from test_gpu_mx4_forms import check, quantized, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


@pytest.mark.parametrize("x", ["f16", "bf16", "mx4"])
@pytest.mark.parametrize("rows,out,inn", [(3, 40, 200), (90, 40, 200), (900, 270, 136), (700, 520, 1024)])
def test_experts_without_tokens(ctx, x, rows, out, inn):
    """rows[] can name no row of X then: the groups' rows are zeros, the others stay."""
    codes, scales = (torch.stack([t, t, t]) for t in mx4(ctx, spread(rng(rows, out), out, inn)))
    c, s = B.mx4_shapes(0, inn)
    X = torch.empty(c, dtype=torch.uint8, device="cuda") if x == "mx4" else torch.empty((0, inn), dtype=TYPES[x], device="cuda")
    xs = torch.empty(s, dtype=torch.uint8, device="cuda") if x == "mx4" else None
    offsets = torch.tensor([1, 2, 2, rows - 1], dtype=torch.int32, device="cuda")
    named = torch.from_numpy(rng(rows).integers(-1, 5, rows).astype(np.int32)).cuda()
    Y = torch.full((rows, out + 2), 9.0, device="cuda")
    ctx.adadim_mx4_matmul_experts(X, codes, scales, offsets, Y[:, :out], in_f=inn, x_scales=xs, rows=named)
    assert bool((Y[1:rows - 1, :out] == 0.0).all())
    assert bool((Y[0] == 9.0).all()) and bool((Y[rows - 1] == 9.0).all()) and bool((Y[:, out:] == 9.0).all())


def test_a_recording_outlives_larger_calls(ctx):
    """Recorded at decode sizes, then larger calls of every kind on the same context, then replayed: counters, partial sums, the router's masks
    and a copied X are still the recording's own."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = B.Context()

        def made(tokens, inn, out, experts):
            g = torch.Generator(device="cuda").manual_seed(tokens + out)
            codes, scales = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in B.mx4_shapes(out, inn))
            c.adadim_mx4_quantize(torch.randn((out, inn), generator=g, device="cuda"), codes, scales)
            X = torch.randn((tokens, inn), generator=g, device="cuda").bfloat16()
            logits = torch.randn((tokens, experts), generator=g, device="cuda")
            i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")
            routed = [i32(tokens, 2), torch.zeros((tokens, 2), device="cuda"), i32(experts + 1), i32(2 * tokens), i32(tokens, 2)]
            return X, codes, scales, logits, routed, torch.zeros((tokens, out), device="cuda")

        def go(X, codes, scales, logits, routed, Y):
            c.adadim_expert_route(logits, *routed)
            c.adadim_mx4_matmul(X, codes, scales, Y)

        # a shared contraction; rows whose X is copied; each outgrown in turn
        small = [made(12, 8192, 96, 16), made(700, 333, 512, 16)]
        large = [made(40, 8192, 1500, 16), made(5000, 333, 512, 16)]
        for s in small:
            go(*s)
        want = [[t.clone() for t in (*s[4], s[5])] for s in small]
        c.adadim_capture_begin()
        try:
            for s in small:
                go(*s)
        finally:
            graph = c.adadim_capture_end()
        for l in large:
            go(*l)
        for turn in range(3):
            for s in small:
                for t in (*s[4], s[5]):
                    t.zero_()
            c.adadim_graph_launch(graph)
            go(*large[turn % 2])
            for s, w in zip(small, want):
                assert all(torch.equal(t, v) for t, v in zip((*s[4], s[5]), w)), turn
        c.adadim_graph_destroy(graph)
    side.synchronize()
    c.close()


# ------------------------------------------------------------------------------------------ loops that go round more than once
@pytest.mark.parametrize("tokens,experts,k", [(16385, 8, 2), (40000, 6, 3), (2200, 1024, 2), (7000, 300, 4)])
def test_route_of_more_chunks_than_workgroups_or_rounds(ctx, tokens, experts, k):
    """Above 16384 tokens a workgroup places several chunks; with many experts the counts of the chunks are added up in several rounds.  Some
    tokens have no expert, so that rows end in -1."""
    l = rng(tokens, experts).standard_normal((tokens, experts))
    l[5::97] = -np.inf
    l[6::89, 1:] = -np.inf
    check_route(ctx, l, k, True, torch.float32)


@pytest.mark.parametrize("x", ["f16", "bf16", "mx4"])
def test_tiles_of_more_experts_than_a_wave_has_lanes(ctx, x):
    """Uneven groups, empty ones among them on both sides of every multiple of 64, rows in front of the first and behind the last."""
    for (mx, experts, rows, out, inn), form in MX4_GROUP_FORMS.items():
        if mx != (x == "mx4"):
            continue
        print((mx, experts, rows, out, inn), form, flush=True)
        w = [quantized(ctx, randn(rows + e, out, inn) * 0.05) for e in range(experts)]
        a = randn(out, 997, inn)
        if mx:
            X, xs, xv = quantized(ctx, a)
        else:
            X, xs = a.to(TYPES[x]), None
            xv = X.float()
        r = np.random.default_rng(rows + out)
        share = r.random(experts) ** 3
        share[[0, 62, 64, 65, 127, experts - 1]] = 0.0
        share[[63, 66, 128]] = 2.0
        lead, tail = 7, 11
        sizes = np.floor(share / share.sum() * (rows - lead - tail)).astype(int)
        offsets = (lead + np.concatenate([[0], np.cumsum(sizes)])).astype(np.int32)
        named = r.integers(0, 997, rows).astype(np.int32)
        full = torch.full((rows, out + 4), 9.0, device="cuda")
        codes, scales = torch.stack([p[0] for p in w]), torch.stack([p[1] for p in w])
        ctx.adadim_mx4_matmul_experts(X, codes, scales, torch.from_numpy(offsets).cuda(), full[:, :out], in_f=inn, x_scales=xs,
                                      rows=torch.from_numpy(named).cuda())
        at = torch.from_numpy(named).long().cuda()
        for e in range(experts):
            lo, hi = offsets[e], offsets[e + 1]
            if hi > lo:
                check(full[lo:hi, :out], xv[at[lo:hi]], w[e][2])
        assert bool((full[:lead] == 9.0).all()) and bool((full[offsets[-1]:] == 9.0).all()) and bool((full[:, out:] == 9.0).all())


# ------------------------------------------------------------------------------------------ products are exact
FORM_SIZES = [1, 20, 40, 130, 700, 3000]                       # rows: few, and tiles of every height


def every_weight():
    """Codes and scales [255, 128]: row b has the scale byte b, its values all codes in turn."""
    codes = torch.from_numpy(np.tile(np.arange(0x10, dtype=np.uint8).reshape(8, 2) @ np.array([1, 16], np.uint8), (253, 8)))
    scales = torch.from_numpy(np.arange(253, dtype=np.uint8)[None, :, None].repeat(4, 2))
    return codes.cuda(), scales.contiguous().cuda()


@pytest.mark.parametrize("x", ["f16", "bf16", "mx4"])
@pytest.mark.parametrize("rows", FORM_SIZES)
@pytest.mark.parametrize("power", [10, -10])
def test_a_product_of_one_term_is_exact(ctx, x, rows, power):
    """One value of X that is not zero, a power of two: Y is the weight times it to the last bit, from the smallest weight that there is to the largest
    that fp32 holds."""
    codes, scales = every_weight()
    w = torch.empty((253, 128), device="cuda")
    ctx.adadim_mx4_dequantize(codes, scales, w)
    keep = slice(0, 127) if power > 0 else slice(127, 253)     # products that fp32 holds as normal numbers
    codes, scales, w = codes[keep].contiguous(), scales[:, keep].contiguous(), w[keep]
    at = (torch.arange(rows, device="cuda") * 37) % 128
    a = torch.zeros((rows, 128), device="cuda")
    a[torch.arange(rows), at] = 2.0 ** power
    X, xs = quantized(ctx, a)[:2] if x == "mx4" else (a.to(TYPES[x]), None)
    Y = torch.empty((rows, len(w)), device="cuda")
    ctx.adadim_mx4_matmul(X, codes, scales, Y, in_f=128, x_scales=xs)
    want = w.double()[:, at].t() * 2.0 ** power
    assert bool((want.abs()[want != 0] >= 2.0 ** -126).all())
    off = Y.double() != want
    assert not bool(off.any()), (off.nonzero()[:5].tolist(), Y[off][:5].tolist(), want[off][:5].tolist())


@pytest.mark.parametrize("rows", FORM_SIZES)
def test_the_largest_fp16_times_weights_beyond_fp16(ctx, rows):
    """A number just below a power of two must not be taken for that power: 65504 x 2^112 is in fp32's range, 65536 x 2^112 is not."""
    codes = torch.full((40, 64), 0x22, dtype=torch.uint8, device="cuda")           # ones
    scales = torch.full((1, 40, 4), 112 + 127, dtype=torch.uint8, device="cuda")
    X = torch.zeros((rows, 128), dtype=torch.float16, device="cuda")
    X[:, 77] = 65504.0
    X[rows // 2:, 77] = -65504.0
    Y = torch.empty((rows, 40), device="cuda")
    ctx.adadim_mx4_matmul(X, codes, scales, Y)
    want = torch.full((rows, 40), 65504.0, dtype=torch.float64, device="cuda") * 2.0 ** 112
    want[rows // 2:] *= -1.0
    assert bool((Y.double() == want).all()), Y[:, 0]
