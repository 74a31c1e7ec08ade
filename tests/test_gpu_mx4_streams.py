"""The layers over the microscaled operators where torch's current stream is not the context's, with slow work in front of each."""
import pytest
import torch

from paper_2309_15531_amd import binding as B, mx4, search as S

pytestmark = pytest.mark.gpu
HIDDEN, INNER, EXPERTS = 256, 320, 4


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def silu(h):
    return torch.nn.functional.silu(h)


def slow(n=12):
    """Some milliseconds of work on the current stream."""
    m = torch.ones((4096, 4096), device="cuda")
    for _ in range(n):
        m = m @ m * 2.0 ** -12
    return m


def layers(ctx):
    one, up, down = mx4.Mx4Weight(ctx, 512, HIDDEN), mx4.Mx4Weight(ctx, INNER, HIDDEN, EXPERTS), mx4.Mx4Weight(ctx, HIDDEN, INNER, EXPERTS)
    return one, up, down


def store(one, up, down, weights):
    one.store(weights[0])
    for e in range(EXPERTS):
        up.store(weights[1][e], e)
        down.store(weights[2][e], e)


def results(ctx, one, up, down, x, logits):
    return [mx4.Mx4Linear(one)(x), mx4.Mx4Linear(one, mx4_inputs=1)(x), mx4.Mx4Experts(up, down, 2, silu)(x, logits),
            mx4.Mx4Experts(up, down, 2, silu, mx4_inputs=1)(x, logits), one.values(), *mx4.quantize_rows(ctx, x)]


@pytest.mark.parametrize("tokens", [3, 200])
def test_layers_take_part_in_the_current_stream(tokens):
    """Inputs that the current stream has yet to write, results that it reads at once, and memory of the call that goes back to the allocator
    and is filled with other values right behind it: the same bits as with everything on one stream."""
    weights = [randn(1, 512, HIDDEN) * 0.05, randn(2, EXPERTS, INNER, HIDDEN) * 0.05, randn(3, EXPERTS, HIDDEN, INNER) * 0.05]
    x, logits = randn(4, tokens, HIDDEN).bfloat16(), randn(5, tokens, EXPERTS)
    plain = B.Context()
    made = layers(plain)
    store(*made, weights)
    want = [t.clone() for t in results(plain, *made, x, logits)]
    hessian = S.PreparedHessian(plain, HIDDEN).update_prepared(x.half().repeat(4, 1))
    want_loss = made[0].store(weights[0], hp=hessian).clone()
    torch.cuda.synchronize()
    own, here = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(own):
        ctx = B.Context()
    with torch.cuda.stream(here):
        for turn in range(3):
            made = layers(ctx)
            late = [torch.zeros_like(w) for w in weights]
            late_x, late_logits = torch.zeros_like(x), torch.zeros_like(logits)
            with torch.cuda.stream(own):
                slow(4 * turn)
            slow()
            for t, v in zip((*late, late_x, late_logits), (*weights, x, logits)):
                t.copy_(v)
            store(*made, late)
            for t in late:
                t.fill_(float("nan"))
            got = results(ctx, *made, late_x, late_logits)
            junk = [torch.full((tokens * 2, n), float("nan"), dtype=torch.bfloat16, device="cuda") for n in (HIDDEN, INNER, HIDDEN, INNER, 512)]
            got = [t.clone() for t in got]
            late_x.fill_(float("nan"))
            late_logits.fill_(float("nan"))
            loss = made[0].store(weights[0], hp=hessian).clone()
            here.synchronize()
            for i, (g, w) in enumerate(zip(got, want)):
                assert torch.equal(g, w), (turn, i)
            assert torch.equal(loss, want_loss), turn
            del junk
    own.synchronize()
    ctx.close()
    plain.close()


@pytest.mark.parametrize("tokens", [1, 64, 300])
@pytest.mark.parametrize("least", [0, 1])
def test_recorded_layers_between_other_work(tokens, least):
    """Two layers recorded as one graph; everything that the recording handed out is let go of but the result, the allocator is emptied and
    memory filled with NaN.  Every replay gives what the eager calls give on the same inputs, and nobody else's memory is written."""
    own = torch.cuda.Stream()
    with torch.cuda.stream(own):
        ctx = B.Context()
        made = layers(ctx)
        store(*made, [randn(1, 512, HIDDEN) * 0.05, randn(2, EXPERTS, INNER, HIDDEN) * 0.05, randn(3, EXPERTS, HIDDEN, INNER) * 0.05])
        one, up, down = made
        linear, experts = mx4.Mx4Linear(one, mx4_inputs=least), mx4.Mx4Experts(up, down, 2, silu, mx4_inputs=least)
        x, logits = torch.empty((tokens, HIDDEN), dtype=torch.bfloat16, device="cuda"), torch.empty((tokens, EXPERTS), device="cuda")

        def fill(seed):
            x.copy_(randn(seed, tokens, HIDDEN))
            logits.copy_(randn(seed + 50, tokens, EXPERTS))

        def layer():
            return linear(experts(x, logits) + x)             # (the sum is torch's own: recorded, and its memory the caller's)

        fill(0)
        layer()
        sums = torch.empty_like(x)
        ctx.adadim_capture_begin()
        try:
            first = experts(x, logits)
            torch.add(first, x, out=sums)
            y = linear(sums)
            del first
        finally:
            graph = ctx.adadim_capture_end()
        torch.cuda.empty_cache()
        shapes = [(tokens, HIDDEN), (2 * tokens, INNER), (2 * tokens, HIDDEN), (tokens, 512), (2 * tokens,), (1 << 20,)]
        for seed in range(1, 6):
            fill(seed)
            junk = [torch.full(s, float("nan"), dtype=t, device="cuda") for s in shapes for t in (torch.bfloat16, torch.float32)]
            y.zero_()
            for _ in range(seed % 2 + 1):
                ctx.adadim_graph_launch(graph)
            got = y.clone()
            assert all(bool(j.isnan().all()) for j in junk), seed
            want = layer()
            assert torch.equal(got, want), seed
            own.synchronize()
            del junk
        ctx.adadim_graph_destroy(graph)
        assert torch.equal(y, want), "a result outlives the graph for whoever holds it"
    own.synchronize()
    with pytest.raises(ValueError, match="stream"):
        with torch.cuda.stream(own):
            ctx.adadim_capture_begin()
        try:
            linear(x)
        finally:
            with torch.cuda.stream(own):
                ctx.adadim_graph_destroy(ctx.adadim_capture_end())
    ctx.close()
