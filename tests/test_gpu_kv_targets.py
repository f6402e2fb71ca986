"""Batches without queries on the GPU: they store, read back and evict like any other, bit for bit, and hold their pages' numbers only."""
import pytest
import torch

import paper_2512_04939_b200 as pkg
from test_gpu_kv_evict import scene_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "e2m1"])
def test_they_store_read_back_and_evict(dtype):
    lengths, keep = [300, 0, 1200, 17], [150, 0, 700, 17]
    scene = scene_of(lengths, 3, 64, dtype, 32, 60, 50)
    c, g = scene.cache, torch.Generator(device="cuda").manual_seed(51)
    k, v = (torch.randn(sum(lengths), 3, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    tallies = scene.weights.clone()
    taken = {p for pages in scene.pages for p in pages}
    spare, into_pages = [i for i in range(c.pages) if i not in taken], []
    for m in keep:
        into_pages.append(spare[:-(-m // 32)])
        spare = spare[len(into_pages[-1]):]
    results = []
    for heads in (None, pkg.NO_QUERIES):
        whole, into = c.batch(lengths, lengths, scene.pages, heads), c.batch(keep, keep, into_pages, heads)
        c.append(whole, k, v)
        scene.weights.copy_(tallies)
        kept = c.evict(whole, into, first=2, last=11)
        results.append([kept, *c.gather(whole), *c.gather(into), scene.weights.clone()])
        for t in (c.k, c.v):
            t.view(torch.uint8).zero_()
    c.poll()
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert into.memory.numel() < 4 * sum(map(len, into_pages)) + 4096
    q = torch.zeros(sum(keep), 3, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        c.attend(into, q)
    with pytest.raises(pkg.LiteVGGTError):
        c.attend(into, q[:, :0])
    with pytest.raises(ValueError):
        c.weigh(into, q, torch.zeros(sum(keep), 3, device="cuda"))


def test_a_stream_that_keeps_many_tokens_makes_room_without_a_plan_for_their_attention():
    """100,000 tokens of 16 heads kept: the target of an eviction took 0.9 GB when it was planned as an attention over itself."""
    ctx = pkg.LiteVGGT(1, 9, 11, 0.0)
    layer = pkg.StreamingGlobalAttention(ctx, 100_400, "e2m1", page_size=128, keep=100_000, recent=64)
    g = torch.Generator(device="cuda").manual_seed(52)
    d = ctx.dim
    w = [(0.02 * torch.randn(*s, generator=g, device="cuda")).bfloat16() for s in ((3 * d, d), (3 * d,), (d, d), (d,))]
    x = torch.randn(300, d, generator=g, device="cuda").bfloat16()
    # as after many steps: all but the last rows are there, and have drawn something
    c = layer.cache
    for t in (c.k, c.v):
        t.random_(generator=g)
    c.k_exp.fill_(126), c.v_exp.fill_(126)
    c.weights.uniform_(generator=g)
    layer.pages, layer.free, layer.length = layer.free[:782], layer.free[782:], 100_096
    layer.step(x, *w)
    assert layer.kept is None
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    layer.step(x, *w)
    layer.cache.poll()
    assert layer.kept.shape == (100_000, 16) and layer.length == 100_300
    assert torch.cuda.max_memory_allocated() - held < 100 << 20
