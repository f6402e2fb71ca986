"""Batches that store, read back and evict, and are never attended with: they hold their pages' numbers and nothing of an attention's plan.
On stand-ins for the CUDA runtime and the kernel launchers.  No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import test_kv_evict_host as base
import test_streaming_keep as keep
from paper_2512_04939_b200 import streaming
from test_kv_evict_host import OK, SHAPE, evict, host, weigh  # noqa: F401
from test_streaming_pages import WEIGHTS, Context, tokens

NO_QUERIES = -1


def create(host, cache, rows, lengths, pages, q_heads, causal_block=0):
    handle, size = C.c_void_p(), C.c_size_t()
    arrays = [np.ascontiguousarray(x, np.int32) for x in (rows, lengths, pages)]
    code = host.litevggt_kv_batch_create(cache, len(rows), *(C.c_void_p(a.ctypes.data) for a in arrays), q_heads, causal_block, C.byref(handle),
                                         C.byref(size))
    return code, handle, size.value


@pytest.mark.parametrize("length", [131072, 400000])
def test_memory_of_a_target_grows_with_its_pages(host, length):
    """An attention of so many rows over themselves would need gigabytes for the parts of its rows."""
    pages = -(-length // 128)
    cache = base.base.cache_of(host, pages=pages, page_size=128, kv_heads=16)
    assert host.litevggt_kv_track(cache, base.base.memory(64)) == OK
    code, handle, size = create(host, cache, [length], [length], np.arange(pages), NO_QUERIES)
    assert code == OK and size <= 4 * pages + 4096
    host.litevggt_kv_batch_destroy(handle)


def test_what_a_batch_without_queries_does(host):
    cache, p, i64 = base.tracked(host), base.base.memory(64), C.c_int64
    source = base.batch(host, cache, [3], [40], [1, 0, 5])
    code, into, size = create(host, cache, [20], [20], [6, 7], NO_QUERIES)
    assert code == OK and host.litevggt_kv_batch_place(into, base.base.memory(size), C.c_size_t(size), None) == OK
    assert host.litevggt_kv_append(cache, into, p, i64(128), i64(64), p, i64(128), i64(64), None) == OK
    assert host.litevggt_kv_gather(cache, into, p, p, None) == OK
    assert evict(host, cache, source, into, 5, 15) == OK
    before = host.fake_launches(), host.fake_weighs()
    q = base.base.memory(1 << 16)
    assert host.litevggt_kv_attend(cache, into, q, i64(128), i64(64), C.c_float(0.125), base.base.memory(1 << 16), None) == SHAPE
    assert weigh(host, cache, into) == SHAPE
    assert (host.fake_launches(), host.fake_weighs()) == before
    assert evict(host, cache, into, create(host, cache, [0], [0], [], NO_QUERIES)[1], 0, 0) != OK  # (not in place)


def test_numbers_of_heads_that_are_refused(host):
    cache = base.tracked(host)
    for q_heads in (0, -2, 3):
        assert create(host, cache, [3], [20], [1, 0], q_heads)[0] == SHAPE
    for rows in (-1, 2 ** 30):  # rows times heads fit 31 bits, as everywhere
        assert create(host, cache, [rows], [20], [1, 0], NO_QUERIES)[0] == SHAPE
    assert create(host, cache, [3], [20], [1, 16], NO_QUERIES)[0] == SHAPE


def test_a_stream_makes_room_with_such_a_batch(monkeypatch):
    asked = []

    class Cache(keep.Cache):
        def batch(self, rows, lengths, pages, q_heads=None, causal_block=0):
            asked.append((rows[0], lengths[0], q_heads))
            return super().batch(rows, lengths, pages, causal_block)

    monkeypatch.setattr(streaming, "KVCache", Cache)
    layer = streaming.StreamingGlobalAttention(Context(), 200, page_size=16, keep=100, decay=0.5)
    for at in range(0, 210, 30):
        layer.step(tokens(at, 30), *WEIGHTS)
    assert [a for a in asked if a[:2] == (100, 100)] == [(100, 100, NO_QUERIES)] and layer.length == 130
    assert all(q_heads is None for rows, _, q_heads in asked if rows == 30)


def test_the_binding_knows_them():
    from paper_2512_04939_b200 import NO_QUERIES as public
    from test_kv_numbers import Reached, cache

    assert public == NO_QUERIES
    with pytest.raises(Reached) as e:
        cache().batch([3], [20], [[2, 0]], q_heads=public)
    assert e.value.args[3] == NO_QUERIES
