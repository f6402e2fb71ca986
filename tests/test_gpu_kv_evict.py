"""Tallies of the attention that cached tokens draw, and eviction by them, on the GPU against their definitions in float64.

Tolerance of a tally w_j = decay w_j + sum_i p_ij, p_ij = exp(x_ij), x_ij = scale q_i . k_j - lse_i: a score's products are added in 32 bits, in
up to 8 steps of 16, off by 2^-23 each of what they add up to at most, B_ij = scale sum_c |q_c k_c|; scaling it, the constants and the
exponential's argument take 2^-23 (B_ij + |lse_i|) more, the exponential 2^-22 and a sum of up to 32 rows in turn (and as many tiles) 2^-19.
Together less than 2^-18 (1 + B_ij + |lse_i|) of each p_ij, and 2^-22 of decay w_j; and 2^-125 for every row, what an exponential may come
out as where it is less.

Tolerance of lse: 2^-8 + 2^-20 (B + |lse|), B the row's largest B_ij: its terms may be rounded to bfloat16.  Which tokens are kept, and what is
moved, is exact.
"""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2512_04939_b200 as pkg
from test_gpu_kv_cache import CHUNKS, Scene, f64
from test_gpu_kv_four_bits import quantised

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "e4m3", "e2m1"]


class Tallied(Scene):
    """A scene whose cache has tallies, all of them 7 where nobody has begun any."""

    def __init__(self, lengths, kv_heads, head_dim, dtype, page_size, seed=0):
        super().__init__(lengths, kv_heads, head_dim, dtype, page_size, seed)
        c = self.cache
        if dtype == "e2m1":
            c.k_exp.fill_(0xFF)
            c.v_exp.fill_(0xFF)
        self.dtype = dtype
        self.weights = torch.full(c.k.shape[:3], 7.0, device="cuda")
        self.cache = pkg.KVCache(c.k, c.v, c.k_exp, c.v_exp, weights=self.weights)

    def held(self, i):
        if self.dtype != "e2m1":
            return super().held(i)
        lo = sum(self.lengths[:i])
        return [quantised(f64(t[lo:lo + self.lengths[i]]))[0] for t in (self.k_new, self.v_new)]

    def tallies(self, i):
        """Of sequence i, float64 [length, kv_heads]."""
        ids = torch.tensor(self.pages[i], dtype=torch.int64)
        return f64(self.weights[ids.cuda()].transpose(1, 2).reshape(-1, self.kv_heads)[:self.lengths[i]])


def drawn(q, k, lse, causal_block, scale):
    """sum_i p_ij and its tolerance, [length, kv_heads], one row at a time."""
    rows, q_heads, _ = q.shape
    length, kv_heads = k.shape[:2]
    total, allowed = np.zeros((length, kv_heads)), np.zeros((length, kv_heads))
    with np.errstate(all="ignore"):
        for h in range(q_heads):
            kh = k[:, h * kv_heads // q_heads]
            for i in range(rows):
                n = ref.seen(length, rows, causal_block, i)
                x = scale * (kh[:n] @ q[i, h]) if np.isfinite(kh[:n]).all() else scale * (kh[:n] * q[i, h]).sum(1)
                p = np.exp(x - lse[i, h])
                size = scale * (np.abs(kh[:n]) @ np.abs(q[i, h]))
                total[:n, h * kv_heads // q_heads] += p
                allowed[:n, h * kv_heads // q_heads] += 2.0 ** -18 * (1 + size + abs(lse[i, h])) * p
    return total, allowed


def check_lse(scene, rows, q, lse, causal_block, scale):
    at = 0
    for i, r in enumerate(rows):
        k = scene.held(i)[0]
        for h in range(q.shape[1]):
            kh = k[:, h * scene.kv_heads // q.shape[1]]
            for row in range(r):
                n, got = ref.seen(len(k), r, causal_block, row), lse[at + row, h]
                if n == 0:
                    assert got == -np.inf
                    continue
                x = scale * (kh[:n] @ f64(q[at + row, h]))
                want = x.max() + np.log(np.exp(x - x.max()).sum())
                size = scale * (np.abs(kh[:n]) @ np.abs(f64(q[at + row, h]))).max()
                assert abs(got - want) <= 2.0 ** -8 + 2.0 ** -20 * (size + abs(want))
        at += r


def weigh(scene, rows, q_heads, causal_block=0, scale=None, decay=1.0, q=None, before=None):
    scene.store()
    if before is not None:
        scene.weights.copy_(before)
    batch = scene.cache.batch(rows, scene.lengths, scene.pages, q_heads=q_heads, causal_block=causal_block)
    q = scene.queries(rows, q_heads) if q is None else q
    out, lse = scene.cache.attend(batch, q.cuda(), scale=scale, lse=True)
    assert torch.equal(out, scene.cache.attend(batch, q.cuda(), scale=scale)) or not out.isfinite().all()
    start = scene.weights.clone()
    was = [scene.tallies(i) for i in range(len(rows))]
    scene.cache.weigh(batch, q.cuda(), lse, scale=scale, decay=decay)
    scene.cache.poll()
    check(scene, rows, q, f64(lse), causal_block, scale, decay, was, start)
    return batch, q, out, lse, start


def check(scene, rows, q, lse, causal_block, scale, decay, was, start):
    scale, at = scene.head_dim ** -0.5 if scale is None else scale, 0
    for i, r in enumerate(rows):
        got = scene.tallies(i)
        if r == 0:
            assert np.array_equal(got, was[i], equal_nan=True)
            continue
        total, allowed = drawn(f64(q[at:at + r]), scene.held(i)[0], lse[at:at + r], causal_block, scale)
        at += r
        want = total if decay == 0 else total + decay * was[i]
        allowed += 2.0 ** -22 * (np.abs(want) if decay == 0 else np.abs(want) + decay * np.abs(was[i])) + 1e-37 + r * q.shape[1] * 2.0 ** -125
        assert np.array_equal(np.isnan(want), np.isnan(got)) and np.array_equal(want[np.isinf(want)], got[np.isinf(want)]), f"sequence {i}"
        with np.errstate(invalid="ignore"):
            over = np.where(np.isfinite(want), np.abs(got - want) / allowed, 0.0)
        assert over.max(initial=0.0) <= 1.0, f"sequence {i}: {over.max()} of the tolerance at {np.unravel_index(over.argmax(), over.shape)}"
    # what belongs to no token is as it was
    inside = torch.zeros_like(scene.weights, dtype=torch.bool)
    for n, pages in zip(scene.lengths, scene.pages):
        for j, page in enumerate(pages):
            inside[page, :, :max(0, min(scene.cache.page_size, n - j * scene.cache.page_size))] = True
    assert torch.equal(scene.weights[~inside].view(torch.int32), start[~inside].view(torch.int32))


# ------------------------------------------------------------------ log-sum-exp
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows,lengths,q_heads,kv_heads,causal_block", [
    ([1, 1], [1, 700], 2, 2, 0), ([3, 5], [300, 5], 12, 4, 1), ([16], [2500], 1, 1, 0), ([40, 300], [30, 300], 2, 1, 1), ([200], [3000], 1, 1, 7), ([2, 20], [0, 0], 2, 2, 0)])
def test_log_sums(dtype, head_dim, rows, lengths, q_heads, kv_heads, causal_block):
    scene = Tallied(lengths, kv_heads, head_dim, dtype, 32, seed=20)
    scene.store()
    batch = scene.cache.batch(rows, lengths, scene.pages, q_heads=q_heads, causal_block=causal_block)
    q = scene.queries(rows, q_heads, 2.0)
    out, lse = scene.cache.attend(batch, q.cuda(), lse=True)
    assert torch.equal(out, scene.cache.attend(batch, q.cuda()))
    check_lse(scene, rows, q, f64(lse), causal_block, head_dim ** -0.5)
    given = torch.full_like(lse, 3.0)
    again = scene.cache.attend(batch, q.cuda(), lse=given)
    assert again[1] is given and torch.equal(given, lse)


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_log_sums_of_pieces_that_are_done_again(rows):
    """Scores that leave the first keys' maximum far behind, whole rows and rows in parts."""
    scene = Tallied([3000, 200], 1, 64, "bf16", 64, seed=21)
    line = torch.randn(64, generator=scene.g)
    line /= line.norm()
    scene.k_new = (line * torch.linspace(-40, 40, 3200)[:, None]).unsqueeze(1).bfloat16()
    scene.store()
    batch = scene.cache.batch([rows, rows], [3000, 200], scene.pages)
    q = (line * 9.0 + 0.1 * torch.randn(2 * rows, 1, 64, generator=scene.g)).bfloat16()
    for x in (q, -q):
        check_lse(scene, [rows, rows], x, f64(scene.cache.attend(batch, x.cuda(), lse=True)[1]), 0, 0.125)


# ------------------------------------------------------------------ tallies
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("lengths,page_size", [([1], 16), ([2, 15, 16, 17], 16), ([31, 32, 33, 640], 128), ([1000, 0, 48], 32)])
def test_single_tokens(dtype, head_dim, lengths, page_size):
    weigh(Tallied(lengths, 2, head_dim, dtype, page_size, seed=22), [1] * len(lengths), 2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim,q_heads,kv_heads,rows", [(64, 16, 2, 1), (128, 8, 1, 1), (64, 12, 4, 5), (128, 16, 1, 1), (128, 6, 2, 4), (64, 7, 7, 16), (64, 9, 1, 1)])
def test_shared_heads_and_drafts(dtype, head_dim, q_heads, kv_heads, rows):
    weigh(Tallied([rows + 250, rows, 829], kv_heads, head_dim, dtype, 64, seed=23), [rows] * 3, q_heads, causal_block=1, decay=0.75)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows,lengths,q_heads,kv_heads,page_size,causal_block", CHUNKS + [([150], [600], 1, 1, 16, 1), ([20, 17], [40, 1030], 8, 1, 128, 1)])
def test_chunks(dtype, head_dim, rows, lengths, q_heads, kv_heads, page_size, causal_block):
    scene = Tallied(lengths, kv_heads, head_dim, dtype, page_size, seed=24)
    batch, q, _, lse, start = weigh(scene, rows, q_heads, causal_block, decay=0.5)
    once = scene.weights.clone()
    scene.weights.copy_(start)
    scene.cache.weigh(batch, q.cuda(), lse, decay=0.5)
    assert torch.equal(once, scene.weights)  # nothing depends on who comes first


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim,rows,length,q_heads", [(64, 1500, 1500, 4), (128, 900, 300, 2), (64, 300, 9000, 1)])
def test_rows_in_parts_and_many_items(dtype, head_dim, rows, length, q_heads):
    """Few keys of many rows are shared out by rows and added up again; twice, since the counters have to be zero again."""
    scene = Tallied([length], 1, head_dim, dtype, 128, seed=25)
    batch, q, _, lse, start = weigh(scene, [rows], q_heads, causal_block=1)
    once = scene.weights.clone()
    scene.weights.copy_(start)
    scene.cache.weigh(batch, q.cuda(), lse)
    assert torch.equal(once, scene.weights)


def test_more_items_than_ctas():
    """CTAs that take several items each, of several sequences and heads, some of which no row sees."""
    weigh(Tallied([5000, 300, 4000, 17, 900], 4, 64, "bf16", 64, seed=26), [40, 300, 200, 17, 0], 8, causal_block=1)


@pytest.mark.parametrize("head_dim,dtype", [(64, "bf16"), (64, "e2m1"), (128, "bf16"), (128, "e4m3")])
def test_two_items_of_many_rows_for_a_cta(head_dim, dtype):
    """More tiles of rows, one after the other and from item to item, than there is memory for at once; frames see their past only."""
    scene = Tallied([8000], 5, head_dim, dtype, 64, seed=40)
    batch, q, _, lse, start = weigh(scene, [600], 5, causal_block=150, decay=0.5)
    once = scene.weights.clone()
    for _ in range(3):
        scene.weights.copy_(start)
        scene.cache.weigh(batch, q.cuda(), lse, decay=0.5)
        assert torch.equal(once, scene.weights)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [3, 30, 200])
def test_rows_that_see_nothing_and_sequences_without_rows(dtype, rows):
    """They draw nothing, and tallies without rows are not even weakened."""
    for causal_block in (0, 1):
        weigh(Tallied([0, max(1, rows // 2), 64, 40], 2, 64, dtype, 16, seed=27), [rows, rows, rows, 0], 2, causal_block, decay=0.25)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [8, 14, 150])
def test_what_a_row_does_not_see_has_no_influence(dtype, head_dim, rows):
    """A key and a row that are not finite spoil the tallies of what sees them or what they see, and no others."""
    scene = Tallied([rows + 60, rows + 40], 1, head_dim, dtype, 16, seed=28)
    scene.k_new[rows + 60 - 3, 0, 1] = float("nan")
    q = scene.queries([rows, rows], 1)
    q[rows + rows // 2, 0, 5] = float("nan")  # of the second sequence: it sees 40 + rows / 2 + 1 tokens
    weigh(scene, [rows, rows], 1, causal_block=1, q=q)
    second = scene.tallies(1)[:, 0]
    assert np.array_equal(np.isnan(second), np.arange(rows + 40) <= 40 + rows // 2)
    # the first sequence's rows that see the key have no sum: everything that they see is spoilt, and nothing behind
    assert np.isnan(scene.tallies(0)[:rows + 60, 0]).any() and not np.isnan(second[-1])


@pytest.mark.parametrize("rows", [2, 40])
def test_tallies_begin_anew_whatever_they_held(rows):
    scene = Tallied([300], 2, 64, "bf16", 16, seed=29)
    before = torch.full_like(scene.weights, float("nan"))
    weigh(scene, [rows], 2, decay=0.0, before=before)
    before = torch.full_like(scene.weights, -3.0)
    before[:, :, ::3] = float("inf")
    scene.weights.copy_(before)
    weigh(scene, [rows], 2, decay=1.0, before=before)


def test_appended_tokens_begin_with_nothing():
    scene = Tallied([100, 33], 4, 64, "e2m1", 16, seed=30)
    scene.store()
    assert all(not scene.tallies(i).any() for i in range(2)) and scene.weights.eq(7.0).sum() == scene.weights.numel() - 133 * 4
    scene.weights.fill_(5.0)
    tail = scene.cache.batch([7, 0], [100, 33], scene.pages)
    scene.cache.append(tail, scene.k_new[:7].cuda(), scene.v_new[:7].cuda())
    assert np.array_equal(scene.tallies(0)[:, 0], np.where(np.arange(100) < 93, 5.0, 0.0)) and (scene.tallies(1) == 5.0).all()


def test_strided_queries_and_scale():
    for rows in (2, 150):
        scene = Tallied([rows + 11], 2, 64, "bf16", 32, seed=31)
        q = scene.queries([rows], 4)
        wide = torch.zeros(rows, 9, 72, dtype=torch.bfloat16)
        wide[:, 1::2, 8:] = q
        scene.store()
        batch = scene.cache.batch([rows], [rows + 11], scene.pages, q_heads=4)
        strided = wide.cuda()[:, 1::2, 8:]
        _, lse = scene.cache.attend(batch, strided, scale=0.3, lse=True)
        was, start = [scene.tallies(0)], scene.weights.clone()
        scene.cache.weigh(batch, strided, lse, scale=0.3)
        check(scene, [rows], q, f64(lse), 0, 0.3, 1.0, was, start)


# ------------------------------------------------------------------ eviction
def kept_by(tallies, m, first, last):
    """Token numbers [m, kv_heads] from the definition."""
    n, heads = tallies.shape
    if m == n:
        return np.tile(np.arange(n)[:, None], (1, heads))
    out = []
    for h in range(heads):
        free = np.where(np.isnan(tallies[:, h]), -np.inf, tallies[:, h])[first:n - last]
        nan = np.isnan(tallies[first:n - last, h])
        order = sorted(range(len(free)), key=lambda i: (-free[i], bool(nan[i]), i)) if nan.any() else np.argsort(-free, kind="stable")
        out.append(np.concatenate([np.arange(first), np.sort(np.asarray(order[:m - first - last], np.int64)) + first, np.arange(n - last, n)]))
    return np.stack(out, 1)


def evict(scene, keep, first=0, last=0):
    """Eviction from the scene as it is, into pages behind a gap, checked in full."""
    c = scene.cache
    spare = [i for i in range(c.pages) if i not in {p for pages in scene.pages for p in pages}]
    into_pages, at = [], 0
    for m in keep:
        n = -(-m // c.page_size)
        into_pages.append(spare[at:at + n])
        at += n
    assert at <= len(spare)
    into = c.batch(keep, keep, into_pages)
    batch = c.batch([0] * len(keep), scene.lengths, scene.pages)
    pools = [t for t in (c.k, c.v, c.k_exp, c.v_exp, c.weights) if t is not None]
    before = [t.clone() for t in pools]
    kept = c.evict(batch, into, first, last)
    c.poll()
    got, at = kept.cpu().numpy(), 0
    want = [t.clone() for t in before]
    for i, m in enumerate(keep):
        mine = kept_by(scene.tallies(i), m, first, last)
        assert np.array_equal(got[at:at + m], mine), f"sequence {i}"
        at += m
        if m == 0:
            continue
        token, slot, heads = torch.from_numpy(mine).cuda(), torch.arange(m, device="cuda")[:, None], torch.arange(c.kv_heads, device="cuda")
        source = (torch.tensor(scene.pages[i], device="cuda")[token // c.page_size], heads, token % c.page_size)
        target = (torch.tensor(into_pages[i], device="cuda")[slot // c.page_size], heads, slot % c.page_size)
        for a, b in zip(before, want):
            a, b = (x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x for x in (a, b))
            b[target] = a[source]
    for a, b in zip(pools, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))  # in the new pages what was chosen, everywhere else what was there
    return batch, into, kept


def scene_of(lengths, kv_heads, head_dim, dtype, page_size, spare, seed):
    """Contents and tallies of any bits: moving is exact."""
    g = torch.Generator().manual_seed(seed)
    counts = [-(-n // page_size) for n in lengths]
    scene = Tallied.__new__(Tallied)
    pages = sum(counts) + spare
    order = torch.randperm(pages, generator=g).tolist()
    scene.pages = [order[sum(counts[:i]):sum(counts[:i + 1])] for i in range(len(counts))]
    scene.lengths, scene.kv_heads, scene.head_dim, scene.g = list(lengths), kv_heads, head_dim, g
    scene.cache = pkg.KVCache.empty(pages, page_size, kv_heads, head_dim, dtype, weights=True)
    gpu = torch.Generator(device="cuda").manual_seed(seed)
    for t in (scene.cache.k, scene.cache.v, scene.cache.k_exp, scene.cache.v_exp):
        if t is not None:
            t.view(torch.uint8).random_(generator=gpu)
    scene.weights = scene.cache.weights
    scene.weights.normal_(generator=gpu).mul_(2).exp_()
    return scene


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim,page_size,kv_heads", [(64, 16, 16), (64, 128, 1), (128, 32, 3), (128, 64, 8)])
def test_ragged_sequences(dtype, head_dim, page_size, kv_heads):
    scene = scene_of([1, 17, 1500, 64, 0, 45, 700, 2], kv_heads, head_dim, dtype, page_size, 400, 40)
    evict(scene, [1, 9, 700, 64, 0, 0, 699, 1])
    evict(scene, [1, 17, 41, 30, 0, 45, 41, 2], 5, 25)
    evict(scene, [1, 17, 1500, 64, 0, 45, 700, 2], 3, 2)


@pytest.mark.parametrize("n,m,first,last,kv_heads", [
    (520500, 131072, 1041, 4164, 1), (100003, 1, 0, 0, 3), (99999, 99998, 7, 0, 2), (65536, 32768, 0, 32768, 1), (40000, 5000, 5000, 0, 2), (9000, 4500, 5, 100, 16)])
def test_long_sequences(n, m, first, last, kv_heads):
    scene = scene_of([n], kv_heads, 64, "e2m1", 128, -(-m // 128), 41)
    scene.weights *= torch.rand_like(scene.weights) > 0.1
    evict(scene, [m], first, last)


@pytest.mark.parametrize("n", [40, 5000, 70000])
def test_equal_and_unusual_tallies(n):
    """Equal ones everywhere, zeros of both signs, infinities, NaN, negative and subnormal ones: the earlier of equals stays."""
    scene = scene_of([n], 4, 64, "bf16", 64, -(-n // 64), 42)
    scene.weights.fill_(0.0)
    evict(scene, [n // 2])
    scene.weights.copy_(torch.randint(0, 3, scene.weights.shape, device="cuda") - 1.0)
    scene.weights[scene.weights == 0] *= -1.0
    scene.weights[::2] += 0.0
    evict(scene, [n // 2], 1, 1)
    odd = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, 1e-45, -1e-45, 3e38, -3e38, 1.0, 1.0000001], device="cuda")
    scene.weights.copy_(odd[torch.randint(0, len(odd), scene.weights.shape, device="cuda")])
    for m in (n // 11, n // 2, n - 1):
        evict(scene, [m], 0, 2)
    scene.weights.fill_(math.nan)
    evict(scene, [n // 3], 2, 2)


def test_pool_beyond_32_bits():
    pages = (1 << 32) // (128 * 64 * 2) + 60
    scene = scene_of([128], 2, 64, "bf16", 128, 0, 43)
    scene.cache = pkg.KVCache.empty(pages, 128, 2, 64, weights=True)
    scene.pages, scene.lengths, scene.weights = [[pages - 1, 3, pages - 7]], [300], scene.cache.weights
    g = torch.Generator().manual_seed(3)
    k, v, q = (torch.randn(n, 2, 64, generator=g).bfloat16().cuda() for n in (300, 300, 20))
    c = scene.cache
    c.append(c.batch([300], [300], scene.pages), k, v)
    for rows in (1, 20):
        batch = c.batch([rows], [300], scene.pages)
        _, lse = c.attend(batch, q[:rows], lse=True)
        c.weigh(batch, q[:rows], lse)
    assert abs(scene.tallies(0).sum() - 2 * 21) < 2 * 21 * 2.0 ** -7  # every row gives out one (within its sum's rounding)
    into = c.batch([150], [150], [[pages - 3, pages - 20]])
    kept = c.evict(c.batch([0], [300], scene.pages), into).long()
    assert np.array_equal(kept.cpu().numpy(), kept_by(scene.tallies(0), 150, 0, 0))
    got = c.gather(into)
    for x, y in zip(got, (k, v)):
        assert torch.equal(x, y.gather(0, kept.unsqueeze(-1).expand(-1, -1, 64)))


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_run_as_it_is_used_captured_and_on_another_stream(dtype):
    """Chunks turned by their positions, stored, attended and weighed; then the cache is halved, and the next chunk sees what stayed."""
    heads, d, rows = 4, 64, 50
    rotary = pkg.RotaryAxes(d, (16, 24, 24), (10000.0, 100.0, 100.0))
    cache = pkg.KVCache.empty(40, 16, heads, d, dtype, weights=True)
    g = torch.Generator().manual_seed(5)
    fused = torch.randn(4 * rows, 3 * heads * d, generator=g).bfloat16().cuda()
    positions = torch.stack([torch.arange(4 * rows) // 50, torch.arange(4 * rows) % 7, torch.arange(4 * rows) % 5]).int().cuda()

    def chunk(i, batch):
        q, k, v = (t.unflatten(1, (heads, d)) for t in fused[i * rows:(i + 1) * rows].split(heads * d, 1))
        q, k = rotary.rotate(positions[:, i * rows:(i + 1) * rows], q, k)
        cache.append(batch, k, v)
        out, lse = cache.attend(batch, q, lse=True)
        cache.weigh(batch, q, lse, decay=0.9)
        return out

    def run():
        for i in range(3):
            chunk(i, whole[i])
        kept = cache.evict(whole[2], into, first=5, last=20)
        return chunk(3, after), kept, cache.gather(after_all)

    pages = list(range(10))
    whole = [cache.batch([rows], [(i + 1) * rows], [pages], causal_block=10) for i in range(3)]
    into, after = cache.batch([75], [75], [list(range(20, 25))]), cache.batch([rows], [125], [list(range(20, 28))], causal_block=10)
    after_all = cache.batch([125], [125], [list(range(20, 28))])
    out, kept, (k, v) = run()
    tallies = cache.weights.clone()
    # the last chunk over the kept tokens, one head at a time
    q, k_new = rotary.rotate(positions[:, 150:], *(fused[150:, a * 256:a * 256 + 256].unflatten(1, (heads, d)) for a in (0, 1)))
    want, size = ref.attend(f64(q), f64(k), f64(v), 10, 0.125)
    assert np.all(np.abs(f64(out) - want) <= 2.0 ** -7 * (np.abs(want) + size))
    assert kept[:5].eq(torch.arange(5, device="cuda")[:, None]).all() and kept[-20:].eq(torch.arange(130, 150, device="cuda")[:, None]).all()
    assert (kept[1:] > kept[:-1]).all()
    if dtype == "bf16":
        assert torch.equal(k[75:], k_new)
    # the same from a graph, and on another stream
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        again = run()
    for _ in range(2):
        cache.weights.fill_(float("nan")), cache.k.view(torch.uint8).zero_()
        graph.replay()
        assert torch.equal(again[0], out) and torch.equal(again[1], kept) and torch.equal(again[2][0], k)
        assert torch.equal(cache.weights[20:27], tallies[20:27])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = run()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other[0], out) and torch.equal(other[1], kept)
    cache.poll()


def test_refusals():
    cache = pkg.KVCache.empty(8, 16, 2, 64, weights=True)
    plain = pkg.KVCache.empty(8, 16, 2, 64)
    batch, into = cache.batch([3], [40], [[2, 0, 1]], q_heads=4), cache.batch([20], [20], [[5, 6]])
    q, lse = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 4, device="cuda")
    for bad in (lse[:2], lse.half(), lse.cpu(), torch.zeros(3, 8, device="cuda")[:, ::2]):
        with pytest.raises(ValueError):
            cache.weigh(batch, q, bad)
        with pytest.raises(ValueError):
            cache.attend(batch, q, lse=bad)
    for kw in (dict(decay=1.5), dict(decay=-1.0), dict(decay=math.nan), dict(scale=0.0)):
        with pytest.raises(pkg.LiteVGGTError):
            cache.weigh(batch, q, lse, **kw)
    other = plain.batch([3], [40], [[2, 0, 1]], q_heads=4)
    with pytest.raises(ValueError):
        plain.weigh(other, q, lse)
    with pytest.raises(ValueError):
        plain.evict(other, other)
    with pytest.raises(pkg.LiteVGGTError):
        cache.weigh(other, q, lse)
    twice = cache.batch([3, 1], [20, 5], [[2, 0], [2]], q_heads=4)
    with pytest.raises(pkg.LiteVGGTError):
        cache.weigh(twice, torch.zeros(4, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 4, device="cuda"))
    for args in ((batch, into, 5, 16), (batch, into, -1), (batch, cache.batch([20], [20], [[5, 1]])), (batch, cache.batch([0], [20], [[5, 6]])),
                 (batch, cache.batch([41], [41], [[5, 6, 7]])), (batch, cache.batch([20, 1], [20, 1], [[5, 6], [7]]))):
        with pytest.raises(pkg.LiteVGGTError):
            cache.evict(*args)
    with pytest.raises(ValueError):
        cache.evict(batch, into, 2 ** 31)
    for weights in (torch.zeros(8, 2, 16, device="cuda").half(), torch.zeros(8, 2, 15, device="cuda"), torch.zeros(8, 2, 16), torch.zeros(8, 2, 32, device="cuda")[:, :, ::2]):
        with pytest.raises(ValueError):
            pkg.KVCache(plain.k, plain.v, weights=weights)
    # sums may not lie where the queries or the output are
    buf = torch.zeros(64, 4, 64, dtype=torch.bfloat16, device="cuda")
    for at in (0, 3 * 4 * 64 * 2 - 4):
        inside = buf.view(torch.float32).flatten()[at // 4:at // 4 + 12].view(3, 4)
        with pytest.raises(pkg.LiteVGGTError):
            cache.attend(batch, buf[:3], out=buf[8:11], lse=inside)
        with pytest.raises(pkg.LiteVGGTError):
            cache.attend(batch, buf[8:11], out=buf[:3], lse=inside)
