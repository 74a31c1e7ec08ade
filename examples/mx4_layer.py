"""A transformer block's expert layer and a linear layer in microscaled 4-bit weights, from fp16 weights to outputs:

    python examples/mx4_layer.py [--hidden 1024] [--inner 2816] [--experts 8] [--k 2] [--tokens 1,64,2048]

Weights are quantized once and scored on calibration activations beside the per-OC and per-IC ones of the search; then tokens are routed
and pass through their experts, by mx4 weights with bf16 activations and with both in mx4, against the fp16 weights in fp32."""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2309_15531_amd import binding as B, mx4, search as S  # noqa: E402


def gated(h):
    """silu of one half times the other."""
    gate, up = h.chunk(2, dim=1)
    return torch.nn.functional.silu(gate) * up


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--hidden", type=int, default=1024)
    p.add_argument("--inner", type=int, default=2816)
    p.add_argument("--experts", type=int, default=8)
    p.add_argument("--k", type=int, default=2)
    p.add_argument("--tokens", default="1,64,2048")
    args = p.parse_args()
    g = torch.Generator(device="cuda").manual_seed(0)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    ctx = B.Context()

    # ---- weights in, with their error beside the search's at 4 bits
    X = randn(4096, args.hidden).half()
    hp = S.PreparedHessian(ctx, args.hidden).update_prepared(X)
    up_w = [(randn(2 * args.inner, args.hidden) * 0.03).half() for _ in range(args.experts)]
    down_w = [(randn(args.hidden, args.inner) * 0.03).half() for _ in range(args.experts)]
    up = mx4.Mx4Weight(ctx, 2 * args.inner, args.hidden, args.experts)
    down = mx4.Mx4Weight(ctx, args.hidden, args.inner, args.experts)
    losses = [up.store(w, e, hp) for e, w in enumerate(up_w)]
    for e, w in enumerate(down_w):
        down.store(w, e)
    if args.hidden % 128 == 0 and args.inner % 64 == 0:
        ls = S.LayerSearch(ctx, 2 * args.inner, args.hidden, bits=4, group=128, keep_winner=False)
        ls.score_all(up_w[0], hp)
        oc, ic = ls.losses.tolist()
        print(f"expert 0, up: error {losses[0].item():.4g} in mx4 (4.25 bits a weight), {oc:.4g} per-OC and {ic:.4g} per-IC in INT4 g128")

    # ---- tokens through their experts
    router = randn(args.experts, args.hidden) * 0.05
    for tokens in (int(t) for t in args.tokens.split(",")):
        x = randn(tokens, args.hidden).bfloat16()
        logits = x.float() @ router.t()
        chosen = logits.topk(args.k, dim=1)
        share = torch.softmax(chosen.values, dim=1)
        want = torch.zeros((tokens, args.hidden), device="cuda")
        for e in range(args.experts):
            t, j = (chosen.indices == e).nonzero(as_tuple=True)
            want[t] += share[t, j, None] * (gated(x[t].float() @ up_w[e].float().t()) @ down_w[e].float().t())
        for what, least in (("bf16 activations", 0), ("mx4 activations", 1)):
            layer = mx4.Mx4Experts(up, down, args.k, gated, mx4_inputs=least)
            y = layer(x, logits)
            torch.cuda.synchronize()
            start = time.perf_counter()
            for _ in range(10):
                layer(x, logits)
            torch.cuda.synchronize()
            us = (time.perf_counter() - start) * 1e5
            off = ((y.float() - want).norm() / want.norm()).item()
            print(f"{tokens:6d} tokens, {what}: {us:8.1f} us a layer, {100 * off:.1f} % from the fp16 weights' result")
    ctx.close()


if __name__ == "__main__":
    main()
