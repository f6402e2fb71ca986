"""Frames arrive one at a time: each is attended against everything that came before it.

    python examples/stream_frames.py [--frames 40] [--grid 28x37] [--dtype e4m3] [--window 20000]

Prints the time of a frame's layer as the sequence grows, and how far the 8-bit cache is from the whole sequence in one go.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_04939_b200 import LiteVGGT, StreamingGlobalAttention  # noqa: E402


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--frames", type=int, default=40)
    ap.add_argument("--grid", default="28x37")
    ap.add_argument("--dtype", default="e4m3", choices=("bf16", "e4m3"))
    ap.add_argument("--window", type=int, default=None, help="tokens that are kept at least (default: all)")
    a = ap.parse_args()
    grid_h, grid_w = map(int, a.grid.split("x"))
    rows = grid_h * grid_w + 5
    ctx = LiteVGGT(a.frames, grid_h, grid_w, 0.0)  # merges nothing: its global layer is the check at the end
    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g, device="cuda")).bfloat16()

    x = normal(a.frames * rows, ctx.dim)
    weights = normal(3 * ctx.dim, ctx.dim, scale=0.02), normal(3 * ctx.dim, scale=0.02), normal(ctx.dim, ctx.dim, scale=0.02), normal(ctx.dim, scale=0.02)
    capacity = a.frames * rows if a.window is None else a.window + 2 * rows
    layer = StreamingGlobalAttention(ctx, capacity, a.dtype, window=a.window)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    layer.step(x[:rows], *weights)
    layer.reset()
    for f in range(a.frames):
        begin.record()
        out = layer.step(x[f * rows:(f + 1) * rows], *weights)
        end.record()
        torch.cuda.synchronize()
        if f % max(1, a.frames // 10) == 0 or f == a.frames - 1:
            print(f"frame {f:4d}: {layer.length:7d} tokens held, {begin.elapsed_time(end):7.3f} ms")
    layer.cache.poll()
    if a.window is None:
        whole = ctx.global_attn(x, *weights)[-rows:].float()
        ctx.poll()
        print(f"last frame against all frames at once: rms difference {((out.float() - whole).norm() / whole.norm()).item():.2e}")


if __name__ == "__main__":
    main()
