"""The layers over the microscaled operators, and the example that uses them.

A layer is held against the same steps taken from the stored values in fp32 or 64 bits: what separates them is the rounding of the
intermediate rows to bf16 (2^-9 relative each, twice) and that of the output; 2 % of the largest output is several times their sum."""
import importlib.util
import os
import sys

import pytest
import torch

from paper_2309_15531_amd import binding as B, mx4, search as S

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def relu2(h):
    return torch.relu(h) ** 2


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_a_weight_and_its_error(ctx, dtype):
    """The loss of store() is that of the stored values on the calibration activations (fp16 dW, fp32 sums: 1e-3 as in the search)."""
    out, inn = 96, 256
    W, X = (randn(1, out, inn) * 0.05).to(dtype), randn(2, 512, inn).half()
    hp = S.PreparedHessian(ctx, inn).update_prepared(X)
    w = mx4.Mx4Weight(ctx, out, inn)
    loss = w.store(W, hp=hp)
    want = ((W.double() - w.values().double()) @ X.double().t().contiguous()).square().sum()
    assert abs(loss.item() - want.item()) <= 1e-3 * want.item()
    assert w.store(W) is None


@pytest.mark.parametrize("tokens", [0, 1, 5, 300])
@pytest.mark.parametrize("least", [0, 1, 100])
def test_linear(ctx, tokens, least):
    out, inn = 200, 320
    w = mx4.Mx4Weight(ctx, out, inn)
    w.store(randn(1, out, inn) * 0.05)
    x = randn(2, tokens, inn).bfloat16()
    layer = mx4.Mx4Linear(w, mx4_inputs=least)
    v = x.float()
    if least and tokens >= least:
        v = torch.empty((tokens, inn), device="cuda")
        ctx.adadim_mx4_dequantize(*mx4.quantize_rows(ctx, x), v)
    want = v.double() @ w.values().double().t().contiguous()
    got = layer(x)
    assert got.dtype == torch.bfloat16 and got.shape == (tokens, out)
    if tokens:
        assert float((got.double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max())
        y = torch.empty((tokens, out), device="cuda")
        assert layer(x, y) is y and torch.equal(y.bfloat16(), got)


@pytest.mark.parametrize("tokens", [0, 1, 7, 250])
@pytest.mark.parametrize("least", [0, 1])
@pytest.mark.parametrize("renormalize", [True, False])
def test_experts(ctx, tokens, least, renormalize):
    """Tokens whose mask leaves fewer than k experts, or none, and an expert that nobody may choose."""
    E, k, hidden, inner = 6, 3, 192, 160
    up, down = mx4.Mx4Weight(ctx, inner, hidden, E), mx4.Mx4Weight(ctx, hidden, inner, E)
    for e in range(E):
        up.store(randn(e, inner, hidden) * 0.1, e)
        down.store(randn(50 + e, hidden, inner) * 0.1, e)
    x, logits = randn(9, tokens, hidden).bfloat16(), randn(10, tokens, E)
    logits[:, 4] = float("-inf")
    logits[1::5, :4] = float("-inf")                          # one expert left
    logits[2::5] = float("-inf")                              # none
    y = mx4.Mx4Experts(up, down, k, relu2, renormalize=renormalize, mx4_inputs=least)(x, logits)

    def rounded(v):
        if not least:
            return v.float()
        r = torch.empty(v.shape, device="cuda")
        ctx.adadim_mx4_dequantize(*mx4.quantize_rows(ctx, v), r)
        return r
    want = torch.zeros((tokens, hidden), device="cuda")
    if tokens:
        scores = torch.softmax(torch.where(torch.isfinite(logits), logits, torch.full_like(logits, -1e30)).double(), dim=1)
        scores[torch.isinf(logits)] = 0.0
        share, index = scores.topk(k, dim=1)
        if renormalize:
            share = share / share.sum(dim=1, keepdim=True).clamp(min=1e-30)
        v = rounded(x)
        for e in range(E):
            h = rounded(relu2((v @ up.values(e).t()).bfloat16()))
            want += ((share * (index == e)).sum(dim=1)[:, None].float()) * (h @ down.values(e).t())
        assert bool((y[2::5] == 0).all())
        assert float((y.float() - want).abs().max()) <= 0.02 * float(want.abs().max())
    assert y.shape == want.shape


def test_refusals(ctx):
    one, some, other = mx4.Mx4Weight(ctx, 64, 32), mx4.Mx4Weight(ctx, 64, 32, 4), mx4.Mx4Weight(ctx, 32, 64, 4)
    for call in (lambda: mx4.Mx4Linear(some), lambda: one.store(randn(0, 32, 64)), lambda: one.store(randn(0, 64, 32), expert=0),
                 lambda: some.store(randn(0, 64, 32)), lambda: some.store(randn(0, 64, 32), expert=4),
                 lambda: mx4.Mx4Experts(one, one, 1, relu2), lambda: mx4.Mx4Experts(some, some, 1, relu2),
                 lambda: mx4.Mx4Experts(some, other, 0, relu2), lambda: mx4.Mx4Experts(some, other, 5, relu2)):
        with pytest.raises(ValueError):
            call()


def test_the_example_runs(monkeypatch, capsys):
    spec = importlib.util.spec_from_file_location("mx4_layer", os.path.join(ROOT, "examples", "mx4_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    monkeypatch.setattr(sys, "argv", ["mx4_layer.py", "--hidden", "256", "--inner", "320", "--experts", "4", "--tokens", "1,70"])
    example.main()
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 5 and "in mx4" in lines[0]
    # a value in mx4 is some 0.115 of itself off: gate and up by 0.16 each with both operands in mx4, their product by 0.23, the output by 0.28
    assert all(float(l.split(", ")[-1].split()[0]) < 40.0 for l in lines[1:])
