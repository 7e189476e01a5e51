"""A transformer block of the Diffusion stage with its projections in 8 bits: self-attention and the feed-forward layer,

    h += x;  x = out_proj(attention(qkv_proj(norm(h))))
    h += x;  x = down(gelu(up(norm(h))))

where h is the residual stream and x what the last sublayer left to be added to it (the addition is part of the next norm).
Weights are quantised once (a scale for each output channel); activations as they come (a scale for each token), by the norm
ahead of a projection, from attention's output, and behind the GELU.  block_16 is the same block on 16-bit weights, with
torch for what is not a projection or attention; run as a program this file times both and says how far apart they are:

    python examples/int8_block.py [--heads 12] [--grid 9x30x52]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_20655_amd import binding as dit  # noqa: E402

SPLIT, D, EPS = (44, 42, 42), 128, 1e-6  # rotary channels per axis (t, h, w), head_dim


def make_weights(heads, seed=0, device="cuda"):
    """Random 16-bit weights of one block, [out features, in features], and the norms' channel weights."""
    gen = torch.Generator(device=device).manual_seed(seed)
    C = heads * D

    def linear(n, k):
        return (torch.randn((n, k), generator=gen, device=device) * k ** -0.5).bfloat16()

    def bias(n):
        return (0.1 * torch.randn(n, generator=gen, device=device)).bfloat16()

    def gamma():
        return 1.0 + 0.25 * torch.randn(C, generator=gen, device=device)

    return dict(heads=heads, norm1=gamma(), norm2=gamma(), qkv=(linear(3 * C, C), bias(3 * C)), out=(linear(C, C), bias(C)),
                up=(linear(4 * C, C), bias(4 * C)), down=(linear(C, 4 * C), bias(C)))


def quantise_weights(w):
    """The same weights in 8 bits: (8-bit rows, scales, bias) for each projection."""
    q = dict(w)
    for name in ("qkv", "out", "up", "down"):
        q[name] = dit.dit_quant_rows_forward(w[name][0]) + (w[name][1],)
    return q


def attention(qkv, heads, grid, workspace):
    L = qkv.shape[0]
    q, k, v = qkv.view(1, L, 3 * heads, D).split(heads, dim=2)
    return dit.dit_attn_forward(q, k, v, grid, SPLIT, workspace=workspace).view(L, heads * D)


def block_8(h, x, w, grid, workspace=None):
    """One block in 8 bits: (h, x) before it to (h, x) behind it; h [L, C] bf16 or float32, x [L, C] bf16."""
    q, s, h = dit.dit_rms_norm_quant_forward(x, w["norm1"], EPS, residual=h)
    a = attention(dit.dit_linear_quant_forward(q, s, *w["qkv"]), w["heads"], grid, workspace)
    q, s = dit.dit_quant_rows_forward(a)
    x = dit.dit_linear_quant_forward(q, s, *w["out"])
    q, s, h = dit.dit_rms_norm_quant_forward(x, w["norm2"], EPS, residual=h)
    u = dit.dit_linear_quant_forward(q, s, *w["up"])
    q, s = dit.dit_quant_rows_forward(u, act="gelu")
    return h, dit.dit_linear_quant_forward(q, s, *w["down"])


def block_16(h, x, w, grid, workspace=None):
    """The same block on 16-bit weights and activations."""
    def norm(t, gamma):
        t = t.float()
        return (t * torch.rsqrt((t * t).mean(1, keepdim=True) + EPS) * gamma).bfloat16()

    h = h + x
    a = attention(dit.dit_linear_forward(norm(h, w["norm1"]), *w["qkv"]), w["heads"], grid, workspace)
    h = h + dit.dit_linear_forward(a, *w["out"])
    u = dit.dit_linear_forward(norm(h, w["norm2"]), *w["up"])
    return h, dit.dit_linear_forward(torch.nn.functional.gelu(u, approximate="tanh"), *w["down"])


def make_rows(heads, grid, seed=1, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)
    shape = (grid[0] * grid[1] * grid[2], heads * D)
    return tuple(torch.randn(shape, generator=gen, device=device).bfloat16() for _ in range(2))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--grid", default="9x30x52")
    args = ap.parse_args()
    grid = tuple(int(n) for n in args.grid.split("x"))
    w = make_weights(args.heads)
    h, x = make_rows(args.heads, grid)
    results = []
    for name, block, weights in (("16 bits", block_16, w), ("8 bits", block_8, quantise_weights(w))):
        out = block(h, x, weights, grid)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        for _ in range(5):
            out = block(h, x, weights, grid)
        end.record()
        torch.cuda.synchronize()
        results.append((out[0] + out[1]).float())
        print("%-8s %9.3f ms a block, %d tokens, %d heads" % (name, start.elapsed_time(end) / 5, h.shape[0], args.heads))
    off = results[1] - results[0]
    print("difference of the residual stream behind the block: %.4f of its RMS" % (off.square().mean() / results[0].square().mean()) ** 0.5)


if __name__ == "__main__":
    main()
