"""The numbers that KVCache.batch hands to the library: it must refuse what it cannot pass on as it is.  No GPU."""
import ctypes as C
import types

import numpy as np
import pytest

from paper_2512_04939_b200.kv_cache import KVCache


class Reached(Exception):
    pass


def cache():
    """A cache without pools, whose library notes what comes in."""
    c = KVCache.__new__(KVCache)
    c.pages, c.page_size, c.kv_heads, c.head_dim, c.handle = 8, 16, 2, 64, None

    def create(handle, n, rows, lengths, pages, q_heads, causal_block, *_):
        take = lambda at, count: list((C.c_int32 * count).from_address(at))
        lengths = take(lengths, n)
        raise Reached(take(rows, n), lengths, take(pages, sum(-(-x // 16) for x in lengths)), q_heads, causal_block)

    c.lib = types.SimpleNamespace(litevggt_kv_batch_create=create)
    return c


@pytest.mark.parametrize("rows,lengths,pages", [
    ([3, 1], [20, 0], [[2, 0], []]), (np.array([3, 1], np.uint8), (20, 0), [range(2, 5), np.empty(0, np.int32)]), ([3.0, 1.0], [20.0, 0], [(2, 7.0, 1), []])])
def test_whole_numbers_arrive(rows, lengths, pages):
    with pytest.raises(Reached) as e:
        cache().batch(rows, lengths, pages, q_heads=4, causal_block=5)
    assert e.value.args == ([3, 1], [20, 0], [2, int(pages[0][1])], 4, 5)


@pytest.mark.parametrize("rows,lengths,pages,extra", [
    ([2.5], [20], [[2, 0]], {}), ([3], [20.5], [[2, 0]], {}), ([3], [20], [[2, 0.5]], {}), ([3], [20], [[float("nan"), 0]], {}),
    ([[3, 1]], [[20, 4]], [[2, 0]], {}), ([3], [20], [[[2, 0], [1, 1]]], {}),
    ([3], [20], [[2, 0]], dict(causal_block=2 ** 32 + 1)), ([3], [20], [[2, 0]], dict(causal_block=2 ** 31)),
    ([3], [20], [[2, 0]], dict(q_heads=2 ** 32 + 2)), ([3], [20], [[2, 0]], dict(causal_block=-2 ** 32))])
def test_other_numbers_are_refused(rows, lengths, pages, extra):
    """A fraction cut off is another row count or another page; of a number beyond 32 bits ctypes passes the lower 32."""
    with pytest.raises(ValueError):
        cache().batch(rows, lengths, pages, **extra)
