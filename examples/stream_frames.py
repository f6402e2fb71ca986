"""Frames arrive one at a time: each is attended against everything that came before it.

    python examples/stream_frames.py [--frames 40] [--grid 28x37] [--dtype e4m3] [--window 20000 | --keep 10000] [--rotary]

Prints the time of a frame's layer as the sequence grows, and how far a cache in codes is from the whole sequence in one go.  With --keep
the cache holds twice as many tokens and a frame, and when it is full every head keeps those that drew most of the attention; --rotary turns
queries and keys by time, height and width.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_04939_b200 import LiteVGGT, RotaryAxes, StreamingGlobalAttention  # noqa: E402


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--frames", type=int, default=40)
    ap.add_argument("--grid", default="28x37")
    ap.add_argument("--dtype", default="e4m3", choices=("bf16", "e4m3", "e2m1"))
    ap.add_argument("--window", type=int, default=None, help="tokens that are kept at least (default: all)")
    ap.add_argument("--keep", type=int, default=None, help="tokens that every head keeps when the cache is full")
    ap.add_argument("--rotary", action="store_true", help="positions in time, height and width")
    a = ap.parse_args()
    grid_h, grid_w = map(int, a.grid.split("x"))
    rows = grid_h * grid_w + 5
    ctx = LiteVGGT(a.frames, grid_h, grid_w, 0.0)  # merges nothing: its global layer is the check at the end
    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g, device="cuda")).bfloat16()

    x = normal(a.frames * rows, ctx.dim)
    weights = normal(3 * ctx.dim, ctx.dim, scale=0.02), normal(3 * ctx.dim, scale=0.02), normal(ctx.dim, ctx.dim, scale=0.02), normal(ctx.dim, scale=0.02)
    capacity = 2 * a.keep + rows if a.keep else a.frames * rows if a.window is None else a.window + 2 * rows
    kept = dict(keep=a.keep, first=min(5, a.keep), recent=min(rows, a.keep // 2)) if a.keep else {}
    rotary = RotaryAxes(ctx.dim // ctx.cfg.heads, (16, 24, 24), (10000.0, 100.0, 100.0)) if a.rotary else None
    layer = StreamingGlobalAttention(ctx, capacity, a.dtype, window=a.window, rotary=rotary, **kept)
    patch = torch.arange(-5, rows - 5, device="cuda").clamp(min=0)  # special tokens are nowhere in the frame
    there = (torch.arange(rows, device="cuda") >= 5).int()

    def where(f):
        """Time, height and width of a frame's tokens."""
        return torch.stack([torch.full_like(there, f), (patch // grid_w + 1).int() * there, (patch % grid_w + 1).int() * there]) if rotary else None

    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    layer.step(x[:rows], *weights, positions=where(0))
    layer.reset()
    for f in range(a.frames):
        begin.record()
        out = layer.step(x[f * rows:(f + 1) * rows], *weights, positions=where(f))
        end.record()
        torch.cuda.synchronize()
        if f % max(1, a.frames // 10) == 0 or f == a.frames - 1:
            print(f"frame {f:4d}: {layer.length:7d} tokens held, {begin.elapsed_time(end):7.3f} ms")
    layer.cache.poll()
    if a.window is None and a.keep is None and rotary is None:
        whole = ctx.global_attn(x, *weights)[-rows:].float()
        ctx.poll()
        print(f"last frame against all frames at once: rms difference {((out.float() - whole).norm() / whole.norm()).item():.2e}")


if __name__ == "__main__":
    main()
