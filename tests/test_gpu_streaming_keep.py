"""Streams without an end on the GPU: a cache that keeps what drew most of the attention, in every type, with positions.

A step's output is compared with that of the same operators called one by one; the bits are the same.
"""
import os
import subprocess
import sys

import pytest
import torch

import paper_2512_04939_b200 as pkg
from test_gpu_streaming import GRID, ROWS, close, make

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def where(f):
    i = torch.arange(ROWS, device="cuda")
    patch = (i - 5).clamp(min=0)
    return torch.stack([torch.full_like(i, f), (patch // GRID[1] + 1) * (i >= 5), (patch % GRID[1] + 1) * (i >= 5)]).int()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "e2m1"])
def test_a_stream_keeps_what_drew_most(dtype):
    x, w = make(8)
    ctx = pkg.LiteVGGT(1, *GRID, 0.0)
    rotary = pkg.RotaryAxes(64, (16, 24, 24), (10000.0, 100.0, 100.0))
    layer = pkg.StreamingGlobalAttention(ctx, 4 * ROWS, dtype, page_size=32, keep=2 * ROWS, first=5, recent=ROWS, decay=0.9, rotary=rotary)
    cache = pkg.KVCache.empty(40, 64, 16, 64, dtype, weights=True)
    pages, spare, held, cuts = list(range(20)), list(range(20, 40)), 0, 0
    for f in range(8):
        out = layer.step(x[f * ROWS:(f + 1) * ROWS], *w, positions=where(f))
        q, k, v = (t.unflatten(1, (16, 64)) for t in ctx.linear(x[f * ROWS:(f + 1) * ROWS], w[0], w[1]).split(1024, 1))
        q, k = rotary.rotate(where(f), q, k)
        if held + ROWS > 4 * ROWS:
            kept = cache.evict(cache.batch([0], [held], [pages]), cache.batch([2 * ROWS], [2 * ROWS], [spare]), 5, ROWS)
            assert torch.equal(kept, layer.kept)
            pages, spare, held, cuts = spare, pages, 2 * ROWS, cuts + 1
        held += ROWS
        batch = cache.batch([ROWS], [held], [pages])
        cache.append(batch, k, v)
        y, lse = cache.attend(batch, q, lse=True)
        cache.weigh(batch, q, lse, decay=0.9)
        assert torch.equal(out, ctx.linear(y.flatten(1), w[2], w[3])) and layer.length == held
    assert cuts == 2
    layer.cache.poll()


def test_one_frame_with_positions_is_the_layer_with_them():
    """Height and width alone, as the global layer's own rotation has them (no frame's time, no merging)."""
    x, w = make(1)
    ctx = pkg.LiteVGGT(1, *GRID, 0.0)
    plan = ctx.merge_plan(x, torch.zeros(1, *GRID, device="cuda"))
    whole = ctx.global_attn_ext(plan, x, *w, rope=True, rope_base=100.0)
    rotary = pkg.RotaryAxes(64, (32, 32), (100.0, 100.0))
    layer = pkg.StreamingGlobalAttention(ctx, ROWS, rotary=rotary)
    assert close(layer.step(x, *w, positions=where(0)[1:]), whole)


@pytest.mark.parametrize("args", [["--dtype", "e2m1", "--keep", "300", "--rotary"], ["--dtype", "e2m1"], ["--rotary", "--window", "400"]])
def test_the_example_runs(args):
    subprocess.run([sys.executable, os.path.join(ROOT, "examples", "stream_frames.py"), "--frames", "9", "--grid", "9x11", *args], check=True, timeout=300)


def test_refusals():
    ctx = pkg.LiteVGGT(1, *GRID, 0.0)
    with pytest.raises(ValueError):
        pkg.StreamingGlobalAttention(ctx, 100, rotary=pkg.RotaryAxes(128, (64, 64), (100.0, 100.0)))
    x, w = make(1)
    layer = pkg.StreamingGlobalAttention(ctx, 4 * ROWS, rotary=pkg.RotaryAxes(64, (32, 32), (100.0, 100.0)))
    for positions in (None, where(0), where(0)[1:, :9], where(0)[1:].long()):
        with pytest.raises(ValueError):
            layer.step(x, *w, positions=positions)
    assert layer.length == 0 and layer.pages == []
