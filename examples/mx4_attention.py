"""An attention layer as it serves: projections in microscaled 4-bit weights, keys and values in a paged cache in the same format.

    python examples/mx4_attention.py [--heads 32] [--kv-heads 8] [--dim 128] [--prompt 512] [--sequences 8] [--steps 4]

A batch of prompts goes in, then each sequence decodes a few tokens, some of which are taken back; every step's result is held against attention
in fp32 over the keys and values before they were stored."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2309_15531_amd import binding as B, mx4  # noqa: E402


class Attention:
    """X -> o(attention(q(X), k(X), v(X))) of new tokens, given the sequences' earlier ones in the cache."""

    def __init__(self, ctx, pages, hidden, heads, kv_heads, dim, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.qkv = mx4.Mx4Weight(ctx, (heads + 2 * kv_heads) * dim, hidden)
        self.o = mx4.Mx4Weight(ctx, hidden, heads * dim)
        self.qkv.store(torch.randn((self.qkv.out_f, hidden), generator=g, device=device) * hidden ** -0.5)
        self.o.store(torch.randn((hidden, heads * dim), generator=g, device=device) * hidden ** -0.5)
        self.cache = mx4.Mx4Cache(pages, kv_heads, dim)
        self.qkv_layer, self.o_layer = mx4.Mx4Linear(self.qkv), mx4.Mx4Linear(self.o)

    def split(self, x):
        """Queries, keys and values as views of one product."""
        y, a, b = self.qkv_layer(x), self.heads * self.dim, self.kv_heads * self.dim
        return y[:, :a], y[:, a:a + b], y[:, a + b:]

    def __call__(self, x, rows, max_new):
        q, k, v = self.split(x)
        self.cache.store(k, v, rows.slots)
        return self.o_layer(self.cache.attend(q, rows.offsets, max_new=max_new))


def plain(q, k, v, group):
    """Causal attention in fp32 of the last rows of a sequence: q [new, heads, dim], k and v [positions, kv_heads, dim]."""
    k, v = (t.float().repeat_interleave(group, 1).transpose(0, 1) for t in (k, v))
    s = torch.matmul(q.float().transpose(0, 1), k.transpose(1, 2).contiguous()) * q.shape[-1] ** -0.5
    new, n = s.shape[1:]
    s.masked_fill_(torch.arange(n, device=s.device) > torch.arange(n - new, n, device=s.device)[:, None], float("-inf"))
    return torch.matmul(torch.softmax(s, -1), v).transpose(0, 1)


def main():
    p = argparse.ArgumentParser()
    for name, value in (("heads", 32), ("kv-heads", 8), ("dim", 128), ("prompt", 512), ("sequences", 8), ("steps", 4)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    ctx = B.Context()
    hidden, n, page = a.heads * a.dim, a.sequences, 64
    width = (a.prompt + a.steps * 3) // page + 2
    pages = mx4.CachePages(ctx, n * width, page, n, width)
    layer = Attention(ctx, pages, hidden, a.heads, a.kv_heads, a.dim)
    g = torch.Generator(device="cuda").manual_seed(1)
    kept = [(torch.empty((0, a.kv_heads, a.dim), device="cuda"),) * 2 for _ in range(n)]        # keys and values as they were
    lengths = [0] * n
    for step in range(a.steps + 1):
        added = [max(1, a.prompt - 37 * s) if step == 0 else 1 + (s + step) % 3 for s in range(n)]
        tokens = sum(added)
        x = torch.randn((tokens, hidden), generator=g, device="cuda").bfloat16()
        rows = pages.add(torch.tensor(added, dtype=torch.int32, device="cuda"), tokens)
        y = layer(x, rows, max(added))
        q, k, v = layer.split(x)
        at, want = 0, []
        for s in range(n):
            new = slice(at, at + added[s])
            k_s, v_s = (torch.cat([old, t[new].view(-1, a.kv_heads, a.dim).float()]) for old, t in zip(kept[s], (k, v)))
            kept[s] = (k_s, v_s)
            want.append(plain(q[new].reshape(-1, a.heads, a.dim), k_s, v_s, a.heads // a.kv_heads).reshape(added[s], -1))
            at += added[s]
        want = layer.o_layer(torch.cat(want).bfloat16()).float()
        off = ((y.float() - want).norm() / want.norm()).item()
        lengths = [l + d for l, d in zip(lengths, added)]
        print(f"step {step}: {tokens} new tokens, {sum(lengths)} in the cache, {int(pages.count)} pages left, {100 * off:.1f} % from unquantized keys and values")
        if step:                                              # of a sequence's tokens of this step one stays
            lengths = [l - d + 1 for l, d in zip(lengths, added)]
            pages.trim(torch.tensor(lengths, dtype=torch.int32, device="cuda"))
            kept = [(k_s[:l], v_s[:l]) for (k_s, v_s), l in zip(kept, lengths)]
    pages.trim(torch.zeros(n, dtype=torch.int32, device="cuda"))
    print(f"all sequences ended: {int(pages.count)} of {pages.pages} pages free")
    ctx.close()


if __name__ == "__main__":
    main()
