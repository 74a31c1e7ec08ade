"""Edges of the microscaled operators and of the routing that other tests do not reach."""
import numpy as np
import pytest
import torch

from paper_2309_15531_amd import binding as B
from test_gpu_mx4 import TYPES, mx4, rng, spread

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
