"""The layer for frames that keep arriving against the layer over all frames at once.

Both round Q, K, V and the attention's output to bfloat16 at the same places, the one-go layer K after it has been multiplied by the
softmax scale, so a row's output differs by the rounding of what each stores: LAYER_NOISE (helpers) covers that for one
layer against an oracle that rounds nothing, so twice it covers two such layers against each other, beside the outputs' own
rounding (2^-8 of an entry each).
"""
import pytest
import torch

import paper_2512_04939_b200 as pkg
from helpers import LAYER_NOISE

pytestmark = pytest.mark.gpu

GRID, ROWS = (9, 11), 9 * 11 + 5


def make(frames):
    g = torch.Generator().manual_seed(21)
    x = torch.randn(frames * ROWS, 1024, generator=g).bfloat16().cuda()
    w = [(0.02 * torch.randn(*s, generator=g)).bfloat16().cuda() for s in ((3072, 1024), (3072,), (1024, 1024), (1024,))]
    return x, w


def close(got, want):
    got, want = got.double(), want.double()
    rms = want.square().mean().sqrt()
    return bool(((got - want).abs() <= 2 * LAYER_NOISE * rms + 2.0 ** -7 * want.abs()).all())


@pytest.mark.parametrize("chunks", [[1] * 6, [2, 1, 3], [6]])
def test_frames_one_after_another_are_the_whole_sequence(chunks):
    """A chunk's last frame sees all frames up to it; so does that frame in the layer over those frames at once."""
    x, w = make(6)
    layer = pkg.StreamingGlobalAttention(pkg.LiteVGGT(1, *GRID, 0.0), 6 * ROWS, page_size=16)
    at = 0
    for n in chunks:
        out = layer.step(x[at * ROWS:(at + n) * ROWS], *w, frame_rows=ROWS)
        for f in range(n):
            upto = at + f + 1
            whole = pkg.LiteVGGT(upto, *GRID, 0.0).global_attn(x[:upto * ROWS], *w)
            assert close(out[f * ROWS:(f + 1) * ROWS], whole[-ROWS:])
        at += n
    layer.cache.poll()


def test_a_window_keeps_the_last_tokens_and_uses_their_pages_again():
    x, w = make(8)
    layer = pkg.StreamingGlobalAttention(pkg.LiteVGGT(1, *GRID, 0.0), 4 * ROWS, page_size=32, window=2 * ROWS)
    for f in range(8):
        out = layer.step(x[f * ROWS:(f + 1) * ROWS], *w)
        assert min(f + 1, 2) * ROWS <= layer.length < 2 * ROWS + 32
        alone = pkg.StreamingGlobalAttention(layer.ctx, 4 * ROWS, page_size=128)
        again = alone.step(x[(f + 1) * ROWS - layer.length:(f + 1) * ROWS], *w)
        assert close(out, again[-ROWS:])


def test_eight_bits_follow_sixteen_and_a_reset_forgets():
    """Rounding K and V to E4M3 changes every score and value by up to 2^-4 of itself, independently: the outputs stay within a
    tenth of their size of one another."""
    x, w = make(3)
    ctx = pkg.LiteVGGT(1, *GRID, 0.0)
    outs = []
    for dtype in ("bf16", "e4m3"):
        layer = pkg.StreamingGlobalAttention(ctx, 3 * ROWS, dtype)
        for _ in range(2):
            for f in range(3):
                out = layer.step(x[f * ROWS:(f + 1) * ROWS], *w)
            assert layer.length == 3 * ROWS
            layer.reset()
        outs.append(out.double())
    assert (outs[1] - outs[0]).norm() <= 0.1 * outs[0].norm()


def test_refusals():
    ctx = pkg.LiteVGGT(1, *GRID, 0.0)
    x, w = make(2)
    with pytest.raises(ValueError):
        pkg.StreamingGlobalAttention(ctx, 0)
    with pytest.raises(ValueError):
        pkg.StreamingGlobalAttention(ctx, 100, window=101)
    layer = pkg.StreamingGlobalAttention(ctx, ROWS)
    layer.step(x[:ROWS], *w)
    with pytest.raises(ValueError, match="pages"):
        layer.step(x[ROWS:], *w)
