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
