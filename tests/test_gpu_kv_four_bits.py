"""The paged K/V cache in 4 bits on the GPU, every operator against its definition in float64.

What is stored and read back is exact.  The attention is that over the values that the codes stand for, which bfloat16 holds
exactly.  Its tolerance, entry by entry: where every probability is rounded by r_j, |r_j| <= 2^-8, in the sum as in the product, the row is off
by sum_j p_j r_j (v_j - o) / (1 + sum_j p_j r_j), at most 2^-8 D with D = sum_j p_j |v_j - o|, but for the divisor, at most 1 / (1 - 2^-8);
rounding it takes 2^-8 |o| more (and of what it is off by, 2^-16 D).  2^-12 A, A = sum_j p_j |v_j|, is for powers of two from a cubic
(7.5e-5 < 2^-13) and for scores in 32 bits, of up to 2^7, off by 2^-16.  Altogether 1.01 2^-8 (D + |o|) + 2^-12 A.
"""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2512_04939_b200 as pkg
from test_gpu_kv_cache import CHUNKS, Scene, attend, f64

pytestmark = pytest.mark.gpu

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantised(x):
    """What rows (last axis) stand for once they are held as codes, and e + 127 of every 32 elements."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(-1, 32)
    top = np.abs(blocks).max(1)
    finite = np.isfinite(top)
    e = np.full(len(blocks), -126.0)
    while (more := finite & (top > 6.0 * 2.0 ** e)).any():
        e[more] += 1
    far = np.abs(LEVELS - np.abs(np.where(finite[:, None], blocks, 0.0) * 2.0 ** -e[:, None])[..., None])
    nearest = far == far.min(-1, keepdims=True)
    # of two that are equally near the even code
    code = np.where(nearest.sum(-1) > 1, (nearest * [1, 0, 1, 0, 1, 0, 1, 0]).argmax(-1), nearest.argmax(-1))
    size = np.minimum(LEVELS[code] * 2.0 ** e[:, None], 3.0 * 2.0 ** 126)  # where bfloat16 ends
    values = np.where(finite[:, None], np.copysign(size, blocks), np.nan)
    exps = np.where(finite, e + 127, 255).astype(np.int64)
    return values.reshape(x.shape), exps.reshape(*x.shape[:-1], x.shape[-1] // 32)


class Four(Scene):
    def __init__(self, lengths, kv_heads, head_dim, page_size, seed=0):
        super().__init__(lengths, kv_heads, head_dim, "e2m1", page_size, seed)
        self.cache.k_exp.fill_(0xFF)
        self.cache.v_exp.fill_(0xFF)

    def held(self, i):
        lo = sum(self.lengths[:i])
        return [quantised(f64(t[lo:lo + self.lengths[i]]))[0] for t in (self.k_new, self.v_new)]

    def check(self, rows, q, out, causal_block=0, scale=None):
        scale, at = self.head_dim ** -0.5 if scale is None else scale, 0
        for i, r in enumerate(rows):
            k, v = self.held(i)
            want, size = ref.attend(f64(q[at:at + r]), k, v, causal_block, scale)
            got = f64(out[at:at + r])
            assert np.array_equal(np.isnan(want), np.isnan(got)), f"sequence {i}"
            fine = np.isfinite(want)
            assert np.array_equal(want[~fine & ~np.isnan(want)], got[~fine & ~np.isnan(want)]), f"sequence {i}"
            apart = np.zeros_like(want)
            for h in range(q.shape[1]):
                kh, vh = (x[:, h * self.kv_heads // q.shape[1]] for x in (k, v))
                for row in range(r):
                    n = ref.seen(len(k), r, causal_block, row)
                    if n == 0:
                        continue
                    with np.errstate(all="ignore"):
                        p = scale * (kh[:n] @ f64(q[at + row, h]))
                        p = np.exp(p - p.max())
                        apart[row, h] = (p[:, None] / p.sum() * np.abs(vh[:n] - want[row, h])).sum(0)
            at += r
            with np.errstate(invalid="ignore"):
                allowed = 1.01 * 2.0 ** -8 * (apart + np.abs(want)) + 2.0 ** -12 * size + 1e-30
                over = np.where(fine, np.abs(got - want) / allowed, 0.0)
            assert over.max(initial=0.0) <= 1.0, f"sequence {i}: {over.max()} of the tolerance at {np.unravel_index(over.argmax(), over.shape)}"


def exact_rows(n, head_dim, g):
    """Rows that codes hold exactly: every block's largest magnitude is 6 times a power of two of its own, 2^-2 to 2^1."""
    levels = torch.tensor(LEVELS, device="cuda")
    x = levels[torch.randint(0, 8, (n, head_dim // 32, 32), generator=g, device="cuda")]
    x[..., 0] = 6.0
    x *= torch.randint(0, 2, x.shape, generator=g, device="cuda") * 2 - 1
    return (x * torch.exp2(torch.randint(-2, 2, (n, head_dim // 32, 1), generator=g, device="cuda").double())).view(n, 1, head_dim)


@pytest.mark.parametrize("head_dim,lengths", [(64, [640_000, 1, 650_003]), (128, [310_000, 33, 330_001])])
@pytest.mark.parametrize("rows,page_size", [(1, 128), (3, 16), (8, 64)])
def test_pieces_of_many_keys(head_dim, lengths, rows, page_size):
    """So many keys that every CTA has thousands in a row."""
    g = torch.Generator(device="cuda").manual_seed(41)
    cache = pkg.KVCache.empty(sum(-(-n // page_size) for n in lengths), page_size, 1, head_dim, "e2m1")
    ids, pages = torch.randperm(cache.pages).tolist(), []
    for n in lengths:
        pages.append(ids[:-(-n // page_size)])
        ids = ids[len(pages[-1]):]
    k, v = exact_rows(sum(lengths), head_dim, g), exact_rows(sum(lengths), head_dim, g)
    cache.append(cache.batch(lengths, lengths, pages), k.bfloat16(), v.bfloat16())
    q = (2.0 * torch.randn(3 * rows, 1, head_dim, generator=g, device="cuda")).bfloat16()
    out, lse = cache.attend(cache.batch([rows] * 3, lengths, pages, causal_block=1), q, lse=True)
    at = 0
    for i, n in enumerate(lengths):
        for row in range(rows):
            sees = ref.seen(n, rows, 1, row)
            got = out[i * rows + row, 0].double()
            if sees == 0:
                assert not got.any()
                continue
            kh, vh = k[at:at + sees, 0], v[at:at + sees, 0]
            x = head_dim ** -0.5 * (kh @ q[i * rows + row, 0].double())
            p = torch.softmax(x, 0)[:, None]
            want = (p * vh).sum(0)
            allowed = 1.01 * 2.0 ** -8 * ((p * (vh - want).abs()).sum(0) + want.abs()) + 2.0 ** -12 * (p * vh.abs()).sum(0)
            assert ((got - want).abs() <= allowed).all(), f"sequence {i}, row {row}: {((got - want).abs() / allowed).max()} of the tolerance"
            assert abs(lse[i * rows + row, 0].item() - x.logsumexp(0).item()) <= 2.0 ** -8 + 2.0 ** -22 * 100
        at += n


# ------------------------------------------------------------------ store, read back
@pytest.mark.parametrize("head_dim,page_size,kv_heads", [(64, 16, 16), (64, 128, 1), (128, 32, 3), (128, 64, 8)])
def test_stored_rows_read_back(head_dim, page_size, kv_heads):
    scene = Four([1, 17, 150, 64, 0, 45], kv_heads, head_dim, page_size)
    whole = scene.store()
    k, v = scene.cache.gather(whole)
    want = [np.concatenate([scene.held(i)[n] for i in range(6)]) for n in range(2)]
    assert np.array_equal(f64(k), want[0]) and np.array_equal(f64(v), want[1])
    rows = sum(scene.lengths) * kv_heads
    for exps in (scene.cache.k_exp, scene.cache.v_exp):
        assert exps.view(-1, head_dim // 32).eq(0xFF).all(1).sum().item() == scene.cache.pages * kv_heads * page_size - rows
    # in which half of which byte a code lies
    first = scene.cache.k[scene.pages[1][0], kv_heads - 1, 3].cpu().numpy()
    exps = scene.cache.k_exp[scene.pages[1][0], kv_heads - 1, 3].cpu().numpy().astype(np.float64)
    codes = np.stack([first & 15, first >> 4], -1).reshape(-1)
    values = np.where(codes & 8, -1, 1) * LEVELS[codes & 7] * np.repeat(2.0 ** (exps - 127), 32)
    assert np.array_equal(values, scene.held(1)[0][3, kv_heads - 1])


def test_many_rows_at_once():
    """More rows than are on the chip at once, in chunks, as slices of one projection; the tail is read back."""
    g = torch.Generator().manual_seed(3)
    heads, n = 16, 30000
    cache = pkg.KVCache.empty(n // 128 + 1, 128, heads, 64, "e2m1")
    ids = torch.randperm(cache.pages, generator=g).tolist()
    fused = torch.randn(n, 3 * heads * 64 + 8, generator=g).bfloat16().cuda()
    k, v = (fused[:, a:a + heads * 64].unflatten(1, (heads, 64)) for a in (heads * 64, 2 * heads * 64))
    for lo, hi in ((0, 29000), (29000, n)):
        cache.append(cache.batch([hi - lo], [hi], [ids]), k[lo:hi], v[lo:hi])
    for rows in (n, 17):
        for got, x in zip(cache.gather(cache.batch([rows], [n], [ids])), (k, v)):
            y = x[n - rows:].float().unflatten(2, (2, 32))
            top = y.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(top.double() / 6)).float()
            step = torch.exp2(torch.floor(torch.log2((y / torch.exp2(e)).abs().clamp(min=1))) - 1)
            assert torch.equal(got.float(), (torch.round(y / torch.exp2(e) / step) * step * torch.exp2(e)).flatten(2))


def test_codes_at_the_ends_of_their_range():
    """Every level and every tie between two of them, under powers of two from the least to the largest, zeros, blocks that are not finite."""
    ties = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 0.2490234375])
    block = torch.cat([ties, -ties])
    rows = torch.zeros(32, 64)
    for i, e in enumerate([-126, -125, -60, -1, 0, 1, 2, 3, 100, 124]):
        rows[i, :32] = block * 2.0 ** e
    rows[10, 0], rows[10, 33] = 6.03125, 2.0 ** -133       # just over; the least magnitude
    rows[11, 5], rows[11, 40] = 2.0 ** -128, -1.5 * 2.0 ** -127
    rows[12, 7], rows[13, 35] = float("nan"), float("inf")
    rows[14, 31], rows[14, 32] = float("-inf"), 1.0
    rows[15, 2] = -0.0
    rows[16] = 3.5 * 2.0 ** 126 * torch.linspace(-1, 1, 64)
    rows[17, :32], rows[17, 32:] = 12.0 * block / 6, 12.0625 * block / 6  # where a second multiplication begins
    rows[18:] = torch.randn(14, 64, generator=torch.Generator().manual_seed(1)) * torch.exp2(torch.arange(-120, 121, 18)[:14, None].float())
    x = rows.bfloat16().unsqueeze(1)
    cache = pkg.KVCache.empty(2, 16, 1, 64, "e2m1")
    batch = cache.batch([32], [32], [[1, 0]])
    cache.append(batch, x.cuda(), x.cuda())
    want, exps = quantised(f64(x))
    assert np.array_equal(cache.k_exp[[1, 0]].cpu().numpy().reshape(32, 1, 2), exps)
    for got in cache.gather(batch):
        assert np.array_equal(f64(got), want, equal_nan=True)


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("lengths", [[1], [2, 15, 16, 17], [127, 128, 129, 640], [1000, 0, 31]])
def test_single_tokens(head_dim, lengths):
    attend(Four(lengths, 2, head_dim, 16), [1] * len(lengths), 2)


@pytest.mark.parametrize("page_size", [16, 128])
@pytest.mark.parametrize("head_dim,q_heads,kv_heads,rows", [(64, 16, 2, 1), (128, 8, 1, 1), (64, 12, 4, 5), (128, 16, 1, 1), (128, 6, 2, 4), (64, 7, 7, 16)])
def test_shared_heads_and_drafts(head_dim, q_heads, kv_heads, rows, page_size):
    attend(Four([rows + 250, rows, 829], kv_heads, head_dim, page_size, seed=2), [rows] * 3, q_heads, causal_block=1)


@pytest.mark.parametrize("head_dim", [64, 128])
def test_long_cache_is_cut_and_joined(head_dim):
    scene = Four([9001], 1, head_dim, 128, seed=3)
    batch, q, out = attend(scene, [1], 4, q_scale=2.0)
    assert torch.equal(out, scene.cache.attend(batch, q.cuda()))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows,lengths,q_heads,kv_heads,page_size,causal_block", CHUNKS)
def test_chunks(head_dim, rows, lengths, q_heads, kv_heads, page_size, causal_block):
    scene = Four(lengths, kv_heads, head_dim, page_size, seed=4)
    batch, q, out = attend(scene, rows, q_heads, causal_block)
    assert torch.equal(out, scene.cache.attend(batch, q.cuda()))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_scores_that_grow_along_the_keys(rows, head_dim):
    """Keys in order of growing scores: references follow, and pieces are done again."""
    scene = Four([900, 300], 1, head_dim, 64, seed=6)
    line = torch.randn(head_dim, generator=scene.g)
    line /= line.norm()
    scene.k_new = (line * torch.linspace(-40, 40, 1200)[:, None]).unsqueeze(1).bfloat16()
    scene.store()
    batch = scene.cache.batch([rows, 5], [900, 300], scene.pages, causal_block=1)
    q = (line * 8.0 + 0.1 * torch.randn(rows + 5, 1, head_dim, generator=scene.g)).bfloat16()
    for x in (q, -q):
        out = scene.cache.attend(batch, x.cuda())
        scene.check([rows, 5], x, out, 1)
        assert torch.equal(out, scene.cache.attend(batch, x.cuda()))
    scene.cache.poll()


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [3, 30, 200])
def test_rows_that_see_nothing(head_dim, rows):
    scene = Four([0, max(1, rows // 2), 64], 2, head_dim, 16, seed=7)
    scene.store()
    for causal_block in (0, 1):
        batch = scene.cache.batch([rows, rows, rows], scene.lengths, scene.pages, causal_block=causal_block)
        q = scene.queries([rows] * 3, 2)
        out = scene.cache.attend(batch, q.cuda())
        scene.check([rows] * 3, q, out, causal_block)
        assert not f64(out[:rows]).any()


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [8, 14, 150])
def test_what_a_row_does_not_see_has_no_influence(head_dim, rows):
    """Blocks that are not finite, and elements at the end of the range, in tokens that some rows of a chunk see and others do not."""
    scene = Four([rows + 60, rows + 2], 1, head_dim, 16, seed=8)
    n = rows + 60
    scene.v_new[n - 3, 0, 5] = float("nan")
    scene.v_new[n - 5, 0, 40] = float("inf")
    scene.k_new[n - 2, 0, 1] = float("nan")
    scene.v_new[n + 4, 0, head_dim - 1] = 3.2e38  # 3.76 * 2^126
    scene.v_new[n + 6, 0, 0] = -3.2e38
    attend(scene, [rows, rows], 1, causal_block=1)


@pytest.mark.parametrize("rows", [3, 14, 40])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_values_of_very_different_size(head_dim, rows):
    """Within rows and between them, over powers of two from one multiplication to two; large ones that a row does not see."""
    scene = Four([200, 500, 300], 1, head_dim, 16, seed=17)
    scene.v_new[200 - rows // 2:200] *= 2.0 ** 60
    scene.v_new[200:700] *= torch.exp2(torch.randint(-20, 20, (500, 1, head_dim // 32), generator=scene.g).float()).repeat_interleave(32, 2).bfloat16()
    scene.k_new[700:, :, :32] *= 16.0
    scene.store()
    batch = scene.cache.batch([rows] * 3, scene.lengths, scene.pages, causal_block=1)
    q = scene.queries([rows] * 3, 1, 0.5)
    out = scene.cache.attend(batch, q.cuda())
    scene.cache.poll()
    scene.check([rows] * 3, q, out, 1)


@pytest.mark.parametrize("head_dim", [64, 128])
def test_many_short_pieces_that_are_done_again(head_dim):
    rows = [18 + i % 23 for i in range(200)]
    scene = Four([r + 3 for r in rows], 2, head_dim, 16, seed=16)
    at = 0
    for i, r in enumerate(rows):
        if i % 5:
            scene.v_new[at + 3 + (7 * i) % r, i % 2, i % head_dim] = float("nan") if i % 3 else float("inf")
        at += r + 3
    attend(scene, rows, 2, causal_block=1)


def test_mixed_batch_in_a_graph_and_on_another_stream():
    rows, lengths = [1, 90, 0, 5, 300], [700, 90, 50, 1200, 333]
    scene = Four(lengths, 2, 64, 32, seed=11)
    scene.store()
    batch = scene.cache.batch(rows, lengths, scene.pages, q_heads=4, causal_block=1)
    q = scene.queries(rows, 4)
    qd, side, graph = q.cuda(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = scene.cache.attend(batch, qd)
    torch.cuda.current_stream().wait_stream(side)
    out = torch.empty_like(first)
    with torch.cuda.graph(graph):
        scene.cache.attend(batch, qd, out=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first)
    scene.check(rows, q, out, 1)


def test_pool_beyond_32_bits():
    pages = (1 << 32) // (128 * 32) + 40
    cache = pkg.KVCache.empty(pages, 128, 1, 64, "e2m1")
    assert cache.k.numel() > 1 << 32
    g = torch.Generator().manual_seed(13)
    k, v, q = (torch.randn(n, 1, 64, generator=g).bfloat16() for n in (300, 300, 150))
    ids = [pages - 1, 3, pages - 7]
    whole = cache.batch([300], [300], [ids])
    cache.append(whole, k.cuda(), v.cuda())
    k, v = (quantised(f64(x))[0] for x in (k, v))
    got = cache.gather(whole)
    assert np.array_equal(f64(got[0]), k) and np.array_equal(f64(got[1]), v)
    for rows in (1, 150):
        want, spread = ref.attend(f64(q[:rows]), k, v, 0, 0.125)
        out = f64(cache.attend(cache.batch([rows], [300], [ids]), q[:rows].cuda()))
        assert np.all(np.abs(out - want) <= 2.0 ** -9 * np.abs(want) + 2.0 ** -8 * spread)


def test_refusals():
    u8 = dict(dtype=torch.uint8, device="cuda")
    k, e = torch.zeros(4, 2, 16, 32, **u8), torch.zeros(4, 2, 16, 2, **u8)
    assert pkg.KVCache(k, k, e, e).head_dim == 64
    for pools in ((k, k), (k, k, e), (k, k, e, e[..., :1]), (k, k.bfloat16(), e, e), (k, k, e[..., 0], e[..., 0]), (k, k, e, e.cpu()),
                  (k, k, e, e.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            pkg.KVCache(*pools)
    with pytest.raises(pkg.LiteVGGTError):
        pkg.KVCache(k[..., :16].contiguous(), k[..., :16].contiguous(), e[..., :1].contiguous(), e[..., :1].contiguous())  # 32 channels
    for args in ((64, "e3m0"), (65, "e2m1"), (80, "e2m1")):
        with pytest.raises(ValueError):
            pkg.KVCache.empty(4, 16, 2, *args)
