"""What the paged K/V cache's calls take and refuse on the GPU, beside test_gpu_kv_cache."""
import pytest
import torch

import paper_2512_04939_b200 as pkg

pytestmark = pytest.mark.gpu


def zeros(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")


def test_batches_are_made_outside_a_capture():
    """A batch's arrays are copied from its own host memory, which a graph would read again at every replay."""
    cache = pkg.KVCache.empty(4, 16, 2, 64)
    x, graph = zeros(8), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(pkg.LiteVGGTError):
            cache.batch([3], [20], [[2, 0]])
    graph.replay()
    assert x.eq(1).all()
    assert cache.batch([3], [20], [[2, 0]]).rows == 3


@pytest.mark.parametrize("rows", [3, 40])
def test_queries_are_not_written_over(rows):
    """A piece that is done again reads its queries once more."""
    cache = pkg.KVCache.empty(4, 16, 2, 64)
    cache.k.zero_(), cache.v.zero_()
    batch = cache.batch([rows], [50], [[2, 0, 1, 3]])
    buf = zeros(2 * rows, 2, 64)
    for q, out in ((buf[:rows], buf[:rows]), (buf[1:rows + 1], buf[:rows]), (buf[::2], buf[:rows])):
        with pytest.raises(pkg.LiteVGGTError):
            cache.attend(batch, q, out=out)
    cache.attend(batch, buf[:rows], out=buf[rows:])
    cache.poll()
