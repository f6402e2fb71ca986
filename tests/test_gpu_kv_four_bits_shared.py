"""Long 4-bit caches whose K/V heads are shared by several query heads: pieces of thousands of keys, at most eight rows of a head.  The tolerance is
that of test_gpu_kv_four_bits.py."""
import pytest
import torch

import kv_reference as ref
import paper_2512_04939_b200 as pkg
from test_gpu_kv_four_bits import exact_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("head_dim,lengths", [(64, [700_000, 650_003]), (128, [310_000, 350_001])])
@pytest.mark.parametrize("rows,q_heads,page_size", [(1, 8, 128), (2, 4, 16), (4, 2, 64), (1, 3, 32)])
def test_pieces_of_many_keys_with_shared_heads(head_dim, lengths, rows, q_heads, page_size):
    g = torch.Generator(device="cuda").manual_seed(65)
    cache = pkg.KVCache.empty(sum(-(-n // page_size) for n in lengths), page_size, 1, head_dim, "e2m1")
    ids, pages = torch.randperm(cache.pages).tolist(), []
    for n in lengths:
        pages.append(ids[:-(-n // page_size)])
        ids = ids[len(pages[-1]):]
    k, v = exact_rows(sum(lengths), head_dim, g), exact_rows(sum(lengths), head_dim, g)
    cache.append(cache.batch(lengths, lengths, pages), k.bfloat16(), v.bfloat16())
    q = (2.0 * torch.randn(2 * rows, q_heads, head_dim, generator=g, device="cuda")).bfloat16()
    batch = cache.batch([rows] * 2, lengths, pages, q_heads=q_heads, causal_block=1)
    out, lse = cache.attend(batch, q, lse=True)
    again = cache.attend(batch, q, lse=True)
    cache.poll()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    at = 0
    for i, n in enumerate(lengths):
        for row in range(rows):
            sees = ref.seen(n, rows, 1, row)
            kh, vh, mine = k[at:at + sees, 0], v[at:at + sees, 0], q[i * rows + row].double()
            x = head_dim ** -0.5 * (kh @ mine.T)  # [keys, q_heads]
            p = torch.softmax(x, 0)
            want = p.T @ vh
            size = head_dim ** -0.5 * (kh.abs() @ mine.abs().T).amax(0)
            for h in range(q_heads):
                got, ph = out[i * rows + row, h].double(), p[:, h:h + 1]
                allowed = 1.01 * 2.0 ** -8 * ((ph * (vh - want[h]).abs()).sum(0) + want[h].abs()) + 2.0 ** -12 * (ph * vh.abs()).sum(0)
                assert ((got - want[h]).abs() <= allowed).all(), f"sequence {i}, row {row}, head {h}"
                off = abs(lse[i * rows + row, h].item() - x[:, h].logsumexp(0).item())
                assert off <= 2.0 ** -8 + 2.0 ** -20 * (size[h].item() + abs(x[:, h].logsumexp(0).item()))
        at += n
