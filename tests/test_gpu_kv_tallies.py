"""Tallies on the GPU where test_gpu_kv_evict.py does not go: see there for the tolerance of what a row gives out."""
import pytest
import torch

import paper_2512_04939_b200 as pkg
from test_gpu_kv_cache import f64
from test_gpu_kv_evict import Tallied, check_lse, evict, scene_of, weigh

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,length", [(3, 700), (1000, 1000)])
def test_tallies_that_come_after_the_batch(rows, length):
    """A batch that was planned for a cache without tallies keeps its rows whole; what they give out is the same, summed in another order:
    the smaller of the two orders' chains has 32 numbers and tiles, 2^-19, as the longer one."""
    g = torch.Generator(device="cuda").manual_seed(60)
    k, v = (torch.randn(length, 1, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    q, got = torch.randn(rows, 4, 64, generator=g, device="cuda").bfloat16(), []
    for late in (False, True):
        weights = torch.zeros(8, 1, 128, device="cuda")
        cache = pkg.KVCache(*(torch.zeros(8, 1, 128, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)), weights=None if late else weights)
        batch = cache.batch([rows], [length], [range(8)], q_heads=4, causal_block=1)
        cache.append(cache.batch([length], [length], [range(8)]), k, v)
        out, lse = cache.attend(batch, q, lse=True)
        stream = torch.cuda.current_stream().cuda_stream
        if late:
            assert cache.lib.litevggt_kv_track(cache.handle, weights.data_ptr()) == 0
            assert cache.lib.litevggt_kv_weigh(cache.handle, batch.handle, q.data_ptr(), 256, 64, 0.125, lse.data_ptr(), 1.0, stream) == 0
        else:
            cache.weigh(batch, q, lse)
        cache.poll()
        got.append(weights.flatten()[:length].double())
    assert ((got[0] - got[1]).abs() <= 2.0 ** -18 * got[0]).all() and got[0].sum() > 3.9 * rows


@pytest.mark.parametrize("head_dim,dtype", [(64, "bf16"), (128, "bf16"), (64, "e4m3"), (128, "e2m1")])
def test_many_tiles_of_rows_in_turn(head_dim, dtype):
    """256,000 rows a K/V head, 2000 tiles that one thread adds up.  Keys of zeros: every p is exp(-lse), in every head another one, so each
    addition is rounded the same way.  Allowed are 2^-18 (1 + |lse|) of the sum.  The k-th addition of a chain is off by half a step, from 2^-24
    of the k numbers' sum down to half of that, so n equal numbers by 3/4 n/2 2^-24 of theirs at most: chains of 32 rows, 32 tiles and 63 such sums
    by 3/4 (16 + 16 + 32) 2^-24 = 3/4 2^-18; the exponential and its argument by 2^-22 + 2^-23 (1 + |lse|)."""
    heads, rows, length = 16, 32_000, 4_752
    cache = pkg.KVCache.empty(38, 128, heads, head_dim, dtype, weights=True)
    nothing = torch.zeros(1, 1, head_dim, dtype=torch.bfloat16, device="cuda").expand(length, heads, head_dim)
    cache.append(cache.batch([length], [length], [range(38)]), nothing, nothing)
    batch = cache.batch([rows], [length], [range(38)], q_heads=8 * heads)
    q = torch.randn(1, 1, head_dim, device="cuda").bfloat16().expand(rows, 8 * heads, head_dim)
    lse = 0.03 + torch.arange(heads, device="cuda") / 16
    cache.weigh(batch, q, lse.repeat_interleave(8).expand(rows, -1).contiguous(), decay=0.0)
    cache.poll()
    got = cache.weights.transpose(1, 2).reshape(-1, heads)[:length].double()
    want = 8 * rows * torch.exp(-lse.double())
    over = (got - want).abs() / (2.0 ** -18 * (1 + lse.double()) * want)
    assert (got == got[0]).all() and over.max() <= 1.0, f"{over.max().item()} of the tolerance"


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_sequences_of_few_rows_beside_one_of_many_leave_most_parts_empty(head_dim, dtype):
    rows = [4000, 17, 20, 40, 30, 9]
    scene = Tallied([300, 300, 280, 900, 500, 260], 4, head_dim, dtype, 32, seed=61)
    batch, q, _, lse, start = weigh(scene, rows, 16, decay=0.5)
    once = scene.weights.clone()
    for _ in range(3):
        scene.weights.copy_(start)
        scene.cache.weigh(batch, q.cuda(), lse, decay=0.5)
        assert torch.equal(once, scene.weights)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("rows", [1, 40])
def test_log_sums_of_scores_whose_terms_cancel(dtype, rows):
    """Products of 2^11 times the score: the bound that include/litevggt.h states, with the scores' own term."""
    scene = Tallied([500], 1, 64, dtype, 64, seed=62)
    scene.k_new[..., 32:] = scene.k_new[..., :32]
    scene.store()
    q = 48.0 * torch.randn(rows, 1, 64, generator=scene.g).bfloat16()
    q[..., 32:] = -q[..., :32] + (q[..., :32] * 2.0 ** -7 * torch.randint(-1, 2, (rows, 1, 32), generator=scene.g)).bfloat16()
    lse = scene.cache.attend(scene.cache.batch([rows], [500], scene.pages), q.cuda(), lse=True)[1]
    check_lse(scene, [rows], q, f64(lse), 0, 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows,q_heads", [([1, 1, 1, 1, 1, 0, 1], 12), ([1, 3, 2, 1, 1, 0, 8], 24)])
def test_warps_that_take_several_units_of_few_rows(head_dim, dtype, rows, q_heads):
    """More units of 32 keys than there are warps on the chip, three to five for each: runs that go over from keys to keys, from head to head and
    from sequence to sequence, some of which have no units; at most eight rows of a head, and more."""
    scene = Tallied([9000, 33, 0, 5000, 1, 250, 64], 12, head_dim, dtype, 64, seed=63)
    batch, q, _, lse, start = weigh(scene, rows, q_heads, causal_block=1, decay=0.5)
    once = scene.weights.clone()
    scene.weights.copy_(start)
    scene.cache.weigh(batch, q.cuda(), lse, decay=0.5)
    assert torch.equal(once, scene.weights)


@pytest.mark.parametrize("lengths,kv_heads", [([513], 4), ([700], 2), ([2000], 3), ([4096], 4), ([600, 5000, 513, 20000, 40] * 8, 8)])
def test_many_equal_tallies_in_one_block(lengths, kv_heads):
    """Tallies that nobody has taken, and others of which more are alike than are compared with one another."""
    scene = scene_of(lengths, kv_heads, 64, "bf16", 64, sum(-(-n // 64) for n in lengths), 64)
    keep = [n // 2 for n in lengths]
    for values in ([0.0], [0.0, 1.0], [3.0, 3.0, 3.0, 0.5, 7.0], [1.0, 1.0 + 2.0 ** -23, 1.0 + 2.0 ** -13, -1.0, float("nan")]):
        choice = torch.randint(0, len(values), scene.weights.shape, device="cuda")
        scene.weights.copy_(torch.tensor(values, device="cuda")[choice])
        evict(scene, keep, 3, 4)
    evict(scene, [n - 1 for n in lengths])
    evict(scene, [1 for _ in lengths])
