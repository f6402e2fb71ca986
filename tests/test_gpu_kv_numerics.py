"""Scores, probabilities and values far from the ordinary, every operator of the paged K/V cache against its definition in float64.
Tolerances are those of test_gpu_kv_cache."""
import math

import pytest
import torch

import kv_reference as ref
from test_gpu_kv_cache import DTYPES, Scene, f64

pytestmark = pytest.mark.gpu


def run(scene, rows, q, causal_block=0, scale=None):
    scene.store()
    batch = scene.cache.batch(rows, scene.lengths, scene.pages, q_heads=q.shape[1], causal_block=causal_block)
    out = scene.cache.attend(batch, q.cuda(), scale=scale)
    scene.cache.poll()
    scene.check(rows, q, out, causal_block, scale)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("power", [20, 23, 25, 26, 27, 28, 29])
def test_one_score_far_above_the_first_keys(power, head_dim):
    """One key a head, behind the first tile of keys, whose score is about 2^power for all rows and the others' zero: it takes all of their
    weight.  Scores beyond 2^22 have no fraction left that a polynomial could take its power of, and some of them, from
    2^26 on, made one whose exponent ran over: next to no weight, and a row's sum that looked fine."""
    heads, rows = 16, 17
    for seed in range(12):
        scene = Scene([384], heads, head_dim, "bf16", 32, seed=100 + seed)
        scene.k_new.zero_()
        q = torch.zeros(rows, heads, head_dim)
        for h in range(heads):
            a, b = (1 + torch.rand(2, generator=scene.g)).tolist()
            scene.k_new[128 + 32 * (h % 8) + h % 4, h, 3] = a * 2.0 ** (power - power // 2 + 2)
            q[:, h, 3] = b * 2.0 ** (power // 2)
        run(scene, [rows], q.bfloat16())


@pytest.mark.parametrize("rows", [5, 40])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("power", [8, 22, 26, 30, 36, 47, 60, 100])
def test_scores_of_any_size_above_and_below_the_first_keys(power, head_dim, rows):
    """One key a head, behind the first tile of keys, whose scores lie about 2^power above the others' zeros for one half of the
    rows and below them for the other: it takes all of a row's weight, or none however large its value is.  A largest score of 2^30
    and more is rounded by its scaling to something that is not the largest any more."""
    heads = 16
    scene = Scene([640], heads, head_dim, "bf16", 32, seed=30)
    scene.k_new.zero_()
    g = scene.g
    for h in range(heads):
        at = 128 + 32 * h + h % 4
        scene.k_new[at, h, 3] = float(2.0 ** (power - power // 2 + 2) * (1 + torch.rand(1, generator=g)))
        scene.v_new[at, h] *= 2.0 ** 40
    q = torch.zeros(rows, heads, head_dim)
    q[:, :, 3] = 2.0 ** (power // 2) * (1 + torch.rand(rows, heads, generator=g))
    q[1::2] *= -1
    run(scene, [rows], q.bfloat16())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [1, 14, 200])
def test_probabilities_that_all_round_the_same_way(rows, head_dim, dtype):
    """In front of every 127 keys that are alike one of four times their weight, so that wherever the keys are cut their probabilities
    lie just above a tie of bfloat16, and one value: what the rounding takes from the product it takes from the sum as well, or
    the whole row is off by it."""
    scene = Scene([4096], 2, head_dim, dtype, 128, seed=31)
    scene.k_new.zero_()
    scene.k_new[::128, :, 0] = 16.0
    scene.v_new.fill_(1.125)
    q = torch.zeros(rows, 2, head_dim)
    q[:, :, 0] = 8.0
    apart = 2.0 - math.log2(1 + 2.0 ** -8 + 2.0 ** -12)  # p = 2^-2 (1 + 2^-8 + 2^-12)
    run(scene, [rows], q.bfloat16(), scale=apart / (16.0 * 8.0 * 1.4426950408889634))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [1, 3, 14, 40])
def test_values_at_the_end_of_the_range(rows, head_dim, dtype):
    """A key of 2^5 times the others' weight, anywhere among them, with a value of 2^125: the sums of probabilities of at most 1 hold."""
    heads = 32
    scene = Scene([8192], heads, head_dim, dtype, 128, seed=32)
    scene.k_new.zero_()
    for h in range(heads):
        at = 200 + 250 * h
        scene.k_new[at, h, 0] = 8.0
        scene.v_new[at, h] = 2.0 ** 125 * torch.sign(scene.v_new[at, h].float()).bfloat16()
    q = torch.zeros(rows, heads, head_dim)
    q[:, :, 0] = 8.0
    run(scene, [rows], q.bfloat16(), scale=5.0 / (64.0 * 1.4426950408889634))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [1, 14, 40, 300])
@pytest.mark.parametrize("low", [60, 121, 124])
def test_scores_of_minus_infinity_in_front(low, rows, head_dim):
    """The first 150 keys have scores of minus infinity, all others scores of -low in base-2 units: only those count, and alike."""
    scene = Scene([900], 2, head_dim, "bf16", 64, seed=33)
    scene.k_new.zero_()
    scene.k_new[:, :, 0] = -8.0
    scene.k_new[:150, :, 1] = float("-inf")
    scene.v_new *= 2.0 ** -12
    q = torch.zeros(rows, 2, head_dim)
    q[:, :, 0] = 8.0
    q[:, :, 1] = 1.0
    run(scene, [rows], q.bfloat16(), scale=low / (64.0 * 1.4426950408889634))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [1, 14])
@pytest.mark.parametrize("length", [1, 700])
def test_values_at_the_lower_end_of_the_range(length, rows, head_dim, dtype):
    """Values of 2^-112 and, as bfloat16, of 2^-123: the tolerance of the other tests, and half a step of the output."""
    scene = Scene([length], 2, head_dim, dtype, 16, seed=34)
    scene.v_new *= 2.0 ** (-112 if dtype == "e4m3" else -123)
    scene.store()
    batch = scene.cache.batch([rows], [length], scene.pages)
    q = scene.queries([rows], 2)
    out = f64(scene.cache.attend(batch, q.cuda()))
    want, spread = ref.attend(f64(q), *scene.held(0), 0, head_dim ** -0.5)
    assert (abs(out - want) <= 2.0 ** -9 * abs(want) + 2.0 ** -8 * spread + 2.0 ** -134).all()
