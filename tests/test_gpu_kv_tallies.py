"""Tallies on the GPU where test_gpu_kv_evict.py does not go: see there for the tolerance of what a row gives out."""
import pytest
import torch

import paper_2512_04939_b200 as pkg

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
