"""The paged K/V cache on the GPU, every operator against its definition in float64 (kv_reference).

Tolerance of the attention, entry by entry, with A = sum_j p_j |v_j| >= |o|: 2^-9 |o| + 2^-8 A.  The output's rounding to
bfloat16 takes up to 2^-8 |o| <= 2^-9 |o| + 2^-9 A of it.  The other 2^-9 A is for the probabilities' rounding as operands
of the second product, up to 2^-8 each but of either sign, and none for a row's largest, whose probability is 1 (their sum
is that of the rounded ones, so one or two keys leave p1 p2 |v1 - v2| 2^-8 <= 2^-9 A of it, and many average out), and for
scores accumulated in 32 bits.  Storing and reading back are exact.
"""
import ctypes as C

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2512_04939_b200 as pkg

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Scene:
    """Sequences in pages of a pool that is NaN wherever nothing was stored, and their contents in float64."""

    def __init__(self, lengths, kv_heads, head_dim, dtype, page_size, seed=0, lean=1.0):
        g = torch.Generator().manual_seed(seed)
        counts = [-(-n // page_size) for n in lengths]
        n_pages = sum(counts) + 3
        order = torch.randperm(n_pages, generator=g).tolist()
        self.pages, at = [], 0
        for n in counts:
            self.pages.append(order[at:at + n])
            at += n
        self.lengths, self.kv_heads, self.head_dim = list(lengths), kv_heads, head_dim
        self.cache = pkg.KVCache.empty(n_pages, page_size, kv_heads, head_dim, dtype)
        self.cache.k.view(torch.uint8).fill_(0xFF)
        self.cache.v.view(torch.uint8).fill_(0xFF)
        if dtype == "e4m3":
            self.cache.k_exp.fill_(0xFF)
            self.cache.v_exp.fill_(0xFF)
        total = sum(lengths)
        shift = lean * torch.randn(1, kv_heads, head_dim, generator=g)
        self.k_new = (torch.randn(total, kv_heads, head_dim, generator=g) + shift).bfloat16()
        self.v_new = torch.randn(total, kv_heads, head_dim, generator=g).bfloat16()
        self.narrow = dtype == "e4m3"
        self.g = g

    def store(self):
        """Everything that the sequences hold, in one append."""
        whole = self.cache.batch(self.lengths, self.lengths, self.pages)
        self.cache.append(whole, self.k_new.cuda(), self.v_new.cuda())
        return whole

    def held(self, i):
        """K and V of sequence i in float64 [length, kv_heads, head_dim]."""
        lo = sum(self.lengths[:i])
        both = [f64(t[lo:lo + self.lengths[i]]) for t in (self.k_new, self.v_new)]
        return [ref.quantised(x)[0] if self.narrow else x for x in both]

    def queries(self, rows, q_heads, scale=1.0):
        return (scale * torch.randn(sum(rows), q_heads, self.head_dim, generator=self.g)).bfloat16()

    def check(self, rows, q, out, causal_block=0, scale=None):
        scale = self.head_dim ** -0.5 if scale is None else scale
        at = 0
        for i, r in enumerate(rows):
            want, spread = ref.attend(f64(q[at:at + r]), *self.held(i), causal_block, scale)
            got = f64(out[at:at + r])
            at += r
            assert np.array_equal(np.isnan(want), np.isnan(got)), f"sequence {i}"
            fine = np.isfinite(want)
            assert np.array_equal(want[~fine & ~np.isnan(want)], got[~fine & ~np.isnan(want)]), f"sequence {i}"
            allowed = 2.0 ** -9 * np.abs(want) + (2.0 ** -9 + 2.0 ** -9) * spread + 1e-30
            with np.errstate(invalid="ignore"):
                over = np.where(fine, np.abs(got - want) / allowed, 0.0)
            assert over.max(initial=0.0) <= 1.0, f"sequence {i}: {over.max()} of the tolerance at {np.unravel_index(over.argmax(), over.shape)}"


def attend(scene, rows, q_heads, causal_block=0, scale=None, q_scale=1.0):
    scene.store()
    batch = scene.cache.batch(rows, scene.lengths, scene.pages, q_heads=q_heads, causal_block=causal_block)
    q = scene.queries(rows, q_heads, q_scale)
    out = scene.cache.attend(batch, q.cuda(), scale=scale)
    scene.cache.poll()
    scene.check(rows, q, out, causal_block, scale)
    return batch, q, out


DTYPES = ["bf16", "e4m3"]


# ------------------------------------------------------------------ store, read back
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim,page_size,kv_heads", [(64, 16, 16), (64, 128, 1), (128, 32, 3), (128, 64, 8)])
def test_stored_rows_read_back(dtype, head_dim, page_size, kv_heads):
    scene = Scene([1, 17, 300, 128, 0, 45], kv_heads, head_dim, dtype, page_size)
    whole = scene.store()
    k, v = scene.cache.gather(whole)
    want = [np.concatenate([scene.held(i)[n] for i in range(6)]) for n in range(2)]
    assert np.array_equal(f64(k), want[0]) and np.array_equal(f64(v), want[1])
    # no other row of the pool was touched
    rows = sum(scene.lengths) * kv_heads
    untouched = scene.cache.k.view(torch.uint8).view(-1, head_dim * (1 if scene.narrow else 2)).eq(0xFF).all(1).sum().item()
    assert untouched == scene.cache.pages * kv_heads * page_size - rows


@pytest.mark.parametrize("dtype", DTYPES)
def test_chunk_by_chunk_from_a_fused_projection(dtype):
    """Rows arrive in chunks, K and V as strided slices of one projection; the tail is read back, not the whole."""
    scene = Scene([100, 33], 4, 64, dtype, 16)
    fused = torch.zeros(133, 3 * 4 * 64 + 16, dtype=torch.bfloat16).cuda()
    k = fused[:, 256:512].unflatten(1, (4, 64))
    v = fused[:, 512:768].unflatten(1, (4, 64))
    done = [0, 0]
    for rows in ([1, 0], [60, 3], [38, 29], [1, 1]):
        take = [range(0 + d, d + r) for d, r in zip(done, rows)]
        ids = list(take[0]) + [100 + i for i in take[1]]
        done = [d + r for d, r in zip(done, rows)]
        batch = scene.cache.batch(rows, done, scene.pages)
        k[:len(ids)].copy_(scene.k_new[ids])
        v[:len(ids)].copy_(scene.v_new[ids])
        scene.cache.append(batch, k[:len(ids)], v[:len(ids)])
    tail = scene.cache.batch([7, 33], [100, 33], scene.pages)
    got = scene.cache.gather(tail)
    for n in range(2):
        assert np.array_equal(f64(got[n]), np.concatenate([scene.held(0)[n][93:], scene.held(1)[n]]))


def test_codes_at_the_ends_of_their_range():
    """Largest, smallest and uneven magnitudes, ties between codes, zeros, rows that are not finite."""
    rows = torch.zeros(16, 64)
    rows[0] = torch.linspace(-448, 448, 64)
    rows[1, 0], rows[1, 1] = 449.0, 2.0 ** -12
    rows[2, :3] = torch.tensor([17.0, 19.0, 448.0])                 # ties between neighbouring codes
    rows[3, :4] = torch.tensor([2.0 ** -9, 1.5 * 2.0 ** -9, 2.0 ** -10, 256.0])  # subnormal codes and ties among them
    rows[4] = 1e38 * torch.linspace(-1, 1, 64)
    rows[5] = 2.0 ** -130
    rows[6, 5] = 2.0 ** -133
    rows[7, 9] = -1.5 * 2.0 ** -116
    rows[8, 1] = float("nan")
    rows[9, 63] = float("inf")
    rows[10, 2] = -0.0
    rows[11] = 57344.0 * torch.linspace(-1, 1, 64)
    rows[12] = 57600.0 * torch.linspace(-1, 1, 64)
    rows[13] = 2.0 ** 120 * torch.linspace(-1, 1, 64)
    rows[14, 7], rows[14, 8] = -3e38, 1e30
    rows[15] = torch.randn(64, generator=torch.Generator().manual_seed(1)) * 1e-20
    x = rows.bfloat16().unsqueeze(1)
    cache = pkg.KVCache.empty(1, 16, 1, 64, "e4m3")
    batch = cache.batch([16], [16], [[0]])
    cache.append(batch, x.cuda(), x.cuda())
    want, exps = ref.quantised(f64(x))
    assert np.array_equal(cache.k_exp.cpu().numpy().reshape(16), exps.reshape(16) + 127)
    for got in cache.gather(batch):
        assert np.array_equal(f64(got), want, equal_nan=True)


# ------------------------------------------------------------------ few rows
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("lengths", [[1], [2, 15, 16, 17], [127, 128, 129, 640], [1000, 0, 31]])
def test_single_tokens(dtype, head_dim, lengths):
    attend(Scene(lengths, 2, head_dim, dtype, 16), [1] * len(lengths), 2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim,q_heads,kv_heads,rows", [(64, 16, 2, 1), (128, 8, 1, 1), (64, 12, 4, 5), (128, 16, 1, 1), (128, 6, 2, 4), (64, 7, 7, 16)])
def test_shared_heads_and_drafts(dtype, head_dim, q_heads, kv_heads, rows):
    attend(Scene([rows + 250, rows, 1029], kv_heads, head_dim, dtype, 64, seed=2), [rows] * 3, q_heads, causal_block=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_long_cache_is_cut_and_joined(dtype, head_dim):
    """One token over many pages: every CTA takes a part of the keys.  Twice, since the counters have to be zero again."""
    scene = Scene([9001], 2, head_dim, dtype, 128, seed=3)
    batch, q, out = attend(scene, [1], 4, q_scale=2.0)
    assert torch.equal(out, scene.cache.attend(batch, q.cuda()))


# ------------------------------------------------------------------ chunks
CHUNKS = [
    # rows, lengths, q_heads, kv_heads, page_size, causal_block
    ([17], [17], 1, 1, 16, 0),
    ([33, 300], [400, 300], 2, 2, 16, 1),
    ([128, 129, 1], [128, 1000, 777], 2, 1, 32, 1),
    ([256], [513], 2, 2, 64, 0),
    ([257, 100], [257, 1300], 3, 1, 128, 1),
    ([522], [1044], 1, 1, 64, 261),
    ([600, 5], [700, 2000], 4, 2, 32, 7),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows,lengths,q_heads,kv_heads,page_size,causal_block", CHUNKS)
def test_chunks(dtype, head_dim, rows, lengths, q_heads, kv_heads, page_size, causal_block):
    scene = Scene(lengths, kv_heads, head_dim, dtype, page_size, seed=4)
    batch, q, out = attend(scene, rows, q_heads, causal_block)
    assert torch.equal(out, scene.cache.attend(batch, q.cuda()))  # nothing depends on who comes first


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_chunk_over_a_long_cache(dtype, head_dim):
    """Rows whose keys are cut into parts that several CTAs take."""
    attend(Scene([140, 6007], 1, head_dim, dtype, 128, seed=5), [140, 200], 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_scores_that_grow_along_the_keys(dtype, rows):
    """Keys in order of growing scores, up to 60 in base-2 units: the reference has to follow."""
    scene = Scene([900], 1, 64, dtype, 64, seed=6)
    line = torch.randn(64, generator=scene.g)
    line /= line.norm()
    scene.k_new = (line * torch.linspace(-40, 40, 900)[:, None] + 0.1 * torch.randn(900, 64, generator=scene.g)).unsqueeze(1).bfloat16()
    scene.store()
    batch = scene.cache.batch([rows], [900], scene.pages)
    q = (line * 8.0 + 0.1 * torch.randn(rows, 1, 64, generator=scene.g)).bfloat16()
    scene.check([rows], q, scene.cache.attend(batch, q.cuda()))
    scene.check([rows], -q, scene.cache.attend(batch, -q.cuda()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_pieces_that_are_done_again(dtype, head_dim):
    """Many pieces a CTA, whole ones and parts, and in some heads scores that leave the first keys' maximum far behind (by more
    than 2^60): those pieces are done again, the others are not, and nothing of it is left for the next call."""
    heads, lengths, rows = 6, [3000, 401, 64], [300, 200, 40]
    scene = Scene(lengths, heads, head_dim, dtype, 64, seed=14)
    line = torch.randn(head_dim, generator=scene.g)
    line /= line.norm()
    at = 0
    for n in lengths:
        for h in (1, 4):
            scene.k_new[at:at + n, h] += (line * torch.linspace(-45, 45, n)[:, None]).bfloat16()
        at += n
    scene.store()
    batch = scene.cache.batch(rows, lengths, scene.pages, causal_block=1)
    q = (line * 8.0 * (head_dim / 64) ** 0.5 + 0.3 * torch.randn(sum(rows), heads, head_dim, generator=scene.g)).bfloat16()
    out = scene.cache.attend(batch, q.cuda())
    scene.check(rows, q, out, 1)
    assert torch.equal(out, scene.cache.attend(batch, q.cuda()))
    calm = scene.queries(rows, heads, 0.1)
    scene.check(rows, calm, scene.cache.attend(batch, calm.cuda()), 1)
    scene.cache.poll()


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_keys_than_a_piece_takes(dtype):
    attend(Scene([70001], 1, 64, dtype, 128, seed=15), [70], 1)


# ------------------------------------------------------------------ edges
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("rows", [3, 30, 200])
def test_rows_that_see_nothing(dtype, head_dim, rows):
    """Queries of a sequence without tokens, and causal rows ahead of a sequence's first token, come out as zero."""
    scene = Scene([0, max(1, rows // 2), 64], 2, head_dim, dtype, 16, seed=7)
    scene.store()
    for causal_block in (0, 1):
        batch = scene.cache.batch([rows, rows, rows], scene.lengths, scene.pages, causal_block=causal_block)
        q = scene.queries([rows] * 3, 2)
        out = scene.cache.attend(batch, q.cuda())
        scene.check([rows] * 3, q, out, causal_block)
        assert not f64(out[:rows]).any()
        if causal_block:
            assert not f64(out[rows:rows + rows - scene.lengths[1]]).any()


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [8, 14, 150])
def test_what_a_row_does_not_see_has_no_influence(dtype, head_dim, rows):
    """NaN and infinity in K and V of tokens that some rows of a chunk see and others do not."""
    scene = Scene([rows + 60], 1, head_dim, dtype, 16, seed=8)
    n = rows + 60
    scene.v_new[n - 3, 0, 5] = float("nan")
    scene.v_new[n - 5, 0, 9] = float("inf")
    scene.v_new[n - 4, 0, head_dim - 1] = float("-inf")
    scene.k_new[n - 2, 0, 1] = float("nan")
    attend(scene, [rows], 1, causal_block=1)


@pytest.mark.parametrize("rows", [3, 14, 40])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_values_of_very_different_size(dtype, head_dim, rows):
    """Large values that a row does not see, or that hardly weigh for it, take nothing from the small ones that do."""
    scene = Scene([200, 500, 300], 1, head_dim, dtype, 16, seed=17)
    scene.v_new[200 - rows // 2:200] *= 2.0 ** 60  # unseen by the sequence's rows before them
    scene.v_new[200:700] *= torch.exp2(torch.randint(-20, 20, (500, 1, 1), generator=scene.g).float()).bfloat16()
    scene.k_new[700:] += 8.0
    scene.k_new[::150][5:6] = -24.0  # the third sequence's queries lean this way: about 2^-300 of their weight
    scene.v_new[::150][5:6] *= 2.0 ** 60
    scene.store()
    batch = scene.cache.batch([rows] * 3, scene.lengths, scene.pages, causal_block=1)
    q = scene.queries([rows] * 3, 1)
    q[2 * rows:] = (0.25 * q[2 * rows:] + 0.75 * 8.0 / head_dim ** 0.5 * 1.0).bfloat16()
    out = scene.cache.attend(batch, q.cuda())
    scene.cache.poll()
    scene.check([rows] * 3, q, out, 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_many_short_pieces_that_are_done_again(dtype, head_dim):
    """A CTA's pieces are one key tile each and nearly all of them hold values that are not finite where not all rows see them, in
    other places each, so whatever looks after V may be ahead of the rows by several pieces."""
    rows = [18 + i % 23 for i in range(400)]
    scene = Scene([r + 3 for r in rows], 2, head_dim, dtype, 16, seed=16)
    at = 0
    for i, r in enumerate(rows):
        if i % 5:
            scene.v_new[at + 3 + (7 * i) % r, i % 2, i % head_dim] = float("nan") if i % 3 else float("inf")
        at += r + 3
    attend(scene, rows, 2, causal_block=1)


@pytest.mark.parametrize("rows", [1, 200])
def test_not_finite_where_it_is_seen(rows):
    scene = Scene([300], 1, 64, "bf16", 16, seed=9)
    scene.v_new[7, 0, 3] = float("inf")
    scene.v_new[8, 0, 4] = float("nan")
    attend(scene, [rows], 1)
    scene.k_new[100, 0, 0] = float("nan")
    attend(scene, [rows], 1)


@pytest.mark.parametrize("rows", [2, 150])
def test_strided_queries_scale_and_given_output(rows):
    scene = Scene([rows + 11], 2, 64, "bf16", 32, seed=10)
    scene.store()
    batch = scene.cache.batch([rows], [rows + 11], scene.pages, q_heads=4)
    q = scene.queries([rows], 4)
    wide = torch.zeros(rows, 9, 72, dtype=torch.bfloat16).cuda()
    strided = wide[:, 1::2, 8:]
    strided.copy_(q)
    out = torch.full((rows, 4, 64), 7.0, dtype=torch.bfloat16).cuda()
    assert scene.cache.attend(batch, strided, scale=0.3, out=out) is out
    scene.check([rows], q, out, scale=0.3)


def test_mixed_batch_on_another_stream():
    """Single tokens and chunks in one batch; the batch is made on one stream and used on another."""
    rows, lengths = [1, 90, 0, 5, 300], [700, 90, 50, 1200, 333]
    scene = Scene(lengths, 2, 64, "e4m3", 32, seed=11)
    scene.store()
    batch = scene.cache.batch(rows, lengths, scene.pages, q_heads=4, causal_block=1)
    q = scene.queries(rows, 4)
    qd, side = q.cuda(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = scene.cache.attend(batch, qd)
        del batch
    torch.cuda.current_stream().wait_stream(side)
    scene.check(rows, q, out, 1)


def test_calls_in_a_graph():
    scene = Scene([400], 2, 64, "bf16", 32, seed=12)
    scene.store()
    batch = scene.cache.batch([40], [400], scene.pages, causal_block=1)
    q, k, v = scene.queries([40], 2).cuda(), scene.k_new[360:].cuda(), scene.v_new[360:].cuda()
    out = torch.empty_like(q)

    def step():
        scene.cache.append(batch, k, v)
        scene.cache.attend(batch, q, out=out)

    step()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_pool_beyond_32_bits():
    """Rows that lie more than 2^32 bytes and elements into the pool."""
    pages = (1 << 32) // (128 * 64) + 40
    cache = pkg.KVCache.empty(pages, 128, 1, 64, "bf16")
    assert cache.k.numel() > 1 << 32
    g = torch.Generator().manual_seed(13)
    k, v, q = (torch.randn(n, 1, 64, generator=g).bfloat16() for n in (300, 300, 150))
    ids = [pages - 1, 3, pages - 7]
    whole = cache.batch([300], [300], [ids])
    cache.append(whole, k.cuda(), v.cuda())
    got = cache.gather(whole)
    assert torch.equal(got[0].cpu(), k) and torch.equal(got[1].cpu(), v)
    for rows in (1, 150):
        want, spread = ref.attend(f64(q[:rows]), f64(k), f64(v), 0, 0.125)
        out = f64(cache.attend(cache.batch([rows], [300], [ids]), q[:rows].cuda()))
        assert np.all(np.abs(out - want) <= 2.0 ** -9 * np.abs(want) + 2.0 ** -8 * spread)


# ------------------------------------------------------------------ refusals
def test_refusals():
    cache = pkg.KVCache.empty(4, 16, 2, 64)
    batch = cache.batch([3], [20], [[2, 0]], q_heads=4)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    ok = torch.zeros(3, 4, 64, **bf)
    for bad in (torch.zeros(2, 4, 64, **bf), torch.zeros(3, 2, 64, **bf), torch.zeros(3, 4, 64, device="cuda"), ok.cpu(),
                torch.zeros(3, 64, 4, **bf).transpose(1, 2), torch.zeros(3, 4, 65, **bf)[..., :64], torch.zeros(3, 4, 65, **bf)[..., 1:]):
        with pytest.raises(ValueError):
            cache.attend(batch, bad)
    with pytest.raises(ValueError):
        cache.attend(batch, ok, out=torch.zeros(3, 4, 128, **bf)[..., :64])
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(pkg.LiteVGGTError):
            cache.attend(batch, ok, scale=scale)
    for rows, lengths, pages in (([3], [20], [[2]]), ([3], [20], [[2, 4]]), ([3], [20], [[2, -1]]), ([-1], [20], [[2, 0]]), ([3], [-1], [[]]),
                                 ([], [], []), ([3, 1], [20], [[2, 0]]), ([2 ** 31], [20], [[2, 0]])):
        with pytest.raises(ValueError):
            cache.batch(rows, lengths, pages)
    for extra in (dict(q_heads=3), dict(q_heads=0), dict(causal_block=-1)):
        with pytest.raises(pkg.LiteVGGTError):
            cache.batch([3], [20], [[2, 0]], **extra)
    with pytest.raises(pkg.LiteVGGTError):
        cache.batch([2 ** 30], [20], [[2, 0]], q_heads=4)  # rows times heads
    with pytest.raises(pkg.LiteVGGTError):
        cache.batch([1], [2 ** 30 + 1], [np.zeros(2 ** 26 + 1, np.int32)])  # tokens
    other = pkg.KVCache.empty(4, 16, 2, 64)
    with pytest.raises(pkg.LiteVGGTError, match="stale or foreign"):
        other.attend(batch, ok)
    beyond = cache.batch([21], [20], [[2, 0]])
    with pytest.raises(pkg.LiteVGGTError, match="shape"):
        cache.append(beyond, torch.zeros(21, 2, 64, **bf), torch.zeros(21, 2, 64, **bf))
    with pytest.raises(pkg.LiteVGGTError, match="shape"):
        cache.gather(beyond)
    for shape in ((4, 2, 8, 64), (4, 2, 256, 64), (4, 2, 16, 96)):
        with pytest.raises(pkg.LiteVGGTError, match="config"):
            pkg.KVCache(torch.zeros(shape, **bf), torch.zeros(shape, **bf))
    pool = torch.zeros(4, 2, 16, 64, **bf)
    codes = pool.to(torch.float8_e4m3fn)
    exps = torch.zeros(4, 2, 16, dtype=torch.uint8, device="cuda")
    for args in ((pool, pool[:2]), (pool.float(), pool.float()), (codes, codes), (codes, codes, exps, exps[:2]), (pool, pool, exps, exps),
                 (pool.cpu(), pool.cpu()), (pool.transpose(0, 1), pool.transpose(0, 1)), (pool, codes)):
        with pytest.raises(ValueError):
            pkg.KVCache(*args)
    with pytest.raises(ValueError):
        pkg.KVCache.empty(4, 16, 2, 64, "int8")
    # the C entries refuse what the wrapper cannot pass
    lib = pkg.load_library()
    assert lib.litevggt_kv_attend(cache.handle, batch.handle, ok.data_ptr(), 3, 64, 1.0, ok.data_ptr(), None) == 4  # alignment
    assert lib.litevggt_kv_attend(cache.handle, batch.handle, ok.data_ptr(), -8, 64, 1.0, ok.data_ptr(), None) == 3
    assert lib.litevggt_kv_attend(cache.handle, batch.handle, ok.data_ptr() + 8, 256, 64, 1.0, ok.data_ptr(), None) == 4
    assert lib.litevggt_kv_attend(cache.handle, batch.handle, None, 256, 64, 1.0, ok.data_ptr(), None) == 1
    assert lib.litevggt_kv_attend(None, batch.handle, ok.data_ptr(), 256, 64, 1.0, ok.data_ptr(), None) == 1
    handle, n_bytes, one = C.c_void_p(), C.c_size_t(), (C.c_int32 * 1)(1)
    assert lib.litevggt_kv_batch_create(cache.handle, 1, one, one, one, 2, 0, C.byref(handle), C.byref(n_bytes)) == 0
    assert lib.litevggt_kv_attend(cache.handle, handle, ok.data_ptr(), 256, 64, 1.0, ok.data_ptr(), None) == 8  # not placed
    assert lib.litevggt_kv_batch_place(handle, ok.data_ptr(), n_bytes.value - 1, None) == 3
    assert lib.litevggt_kv_batch_place(handle, ok.data_ptr() + 16, n_bytes.value, None) == 4
    assert lib.litevggt_kv_batch_destroy(handle) == 0
