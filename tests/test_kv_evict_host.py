"""Tallies and eviction (kv_evict_api.cu) linked against stand-ins for the CUDA runtime and the kernel launchers: refusals, and how the work
of taking tallies is cut.  No GPU."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import test_kv_host as base

HERE, CSRC = base.HERE, base.CSRC
OK, NULL, SHAPE, ALIGN, CUDA, STALE = 0, 1, 3, 4, 6, 8


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host") / "libkvevict.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-w", "-Wl,-Bsymbolic", "-I/usr/local/cuda/include", "-x", "c++",
                    os.path.join(CSRC, "kv_api.cu"), os.path.join(CSRC, "kv_evict_api.cu"), os.path.join(HERE, "kv_host_fakes.cpp"),
                    os.path.join(HERE, "kv_evict_fakes.cpp"), "-o", so], check=True)
    return C.CDLL(so)


def batch(host, cache, rows, lengths, pages, q_heads=2, causal_block=0, place=True):
    handle, size = C.c_void_p(), C.c_size_t()
    arrays = [np.ascontiguousarray(x, np.int32) for x in (rows, lengths, pages)]
    assert host.litevggt_kv_batch_create(cache, len(rows), *(C.c_void_p(a.ctypes.data) for a in arrays), q_heads, causal_block, C.byref(handle),
                                         C.byref(size)) == OK
    if place:
        assert host.litevggt_kv_batch_place(handle, base.memory(size.value), size, None) == OK
    return handle


def weigh(host, cache, b, q="p", lse="p", scale=0.125, decay=1.0, row=128, head=64):
    p = base.memory(64)
    q, lse = (p if x == "p" else x for x in (q, lse))
    return host.litevggt_kv_weigh(cache, b, q, C.c_int64(row), C.c_int64(head), C.c_float(scale), lse, C.c_float(decay), None)


def evict(host, cache, a, b, first=0, last=0, kept="p"):
    return host.litevggt_kv_evict(cache, a, b, first, last, base.memory(64) if kept == "p" else kept, None)


def tracked(host, **kw):
    cache = base.cache_of(host, pages=16, **kw)
    assert host.litevggt_kv_track(cache, base.memory(64)) == OK
    return cache


def test_tallies_are_wanted_and_taken(host):
    cache = base.cache_of(host)
    b = batch(host, cache, [3], [20], [1, 0])
    assert weigh(host, cache, b) == NULL and evict(host, cache, b, b) == NULL
    odd = C.c_void_p(base.memory(64).value + 8)
    assert host.litevggt_kv_track(cache, odd) == ALIGN and host.litevggt_kv_track(None, odd) == NULL
    assert host.litevggt_kv_track(cache, base.memory(64)) == OK
    before = host.fake_weighs()
    assert weigh(host, cache, b) == OK and host.fake_weighs() == before + 1
    assert host.litevggt_kv_track(cache, None) == OK and weigh(host, cache, b) == NULL


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(lse=None), NULL), (dict(scale=0.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=1e30), SHAPE),
    (dict(decay=-0.1), SHAPE), (dict(decay=1.001), SHAPE), (dict(decay=float("nan")), SHAPE), (dict(row=-8), SHAPE), (dict(head=4), ALIGN),
    (dict(row=1 << 33), SHAPE), (dict(q=C.c_void_p(1 << 20 | 8)), ALIGN), (dict(lse=C.c_void_p(1 << 20 | 2)), ALIGN)])
def test_weighings_that_are_refused(host, kw, code):
    cache = tracked(host)
    b, before = batch(host, cache, [3], [20], [1, 0]), host.fake_weighs()
    assert weigh(host, cache, b, **kw) == code and host.fake_weighs() == before


def test_batches_that_are_refused(host):
    cache, other = tracked(host), tracked(host)
    b = batch(host, cache, [3, 1], [20, 5], [1, 0, 2])
    unplaced = batch(host, cache, [3], [20], [1, 0], place=False)
    shared = batch(host, cache, [3, 1], [20, 5], [1, 0, 1])
    assert weigh(host, other, b) == STALE and weigh(host, cache, unplaced) == STALE and weigh(host, cache, None) == NULL
    assert weigh(host, cache, shared) == SHAPE and weigh(host, cache, shared) == SHAPE and weigh(host, cache, b) == OK
    assert weigh(host, cache, batch(host, cache, [0, 0], [20, 5], [1, 0, 2]), q=None, lse=None) == OK  # no rows


def test_evictions_that_are_refused(host):
    cache, other = tracked(host), tracked(host)
    a = batch(host, cache, [1, 0], [40, 20], [1, 0, 5, 2, 3])
    into = batch(host, cache, [20, 20], [20, 20], [6, 7, 8, 9])
    before = host.fake_evicts()
    assert evict(host, cache, a, into, 5, 15) == OK and host.fake_evicts() == before + 1  # (the second sequence keeps all of its own)
    for args in ((a, into, 5, 16), (a, into, -1, 0), (a, into, 0, -1), (a, into, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert evict(host, cache, *args) == SHAPE
    for rows, lengths, pages in (([20], [20], [6, 7]),                       # another number of sequences
                                 ([20, 21], [20, 21], [6, 7, 8, 9]),         # more than there is
                                 ([0, 0], [20, 20], [6, 7, 8, 9]), ([20, 19], [20, 20], [6, 7, 8, 9]),  # not whole sequences
                                 ([20, 20], [20, 20], [6, 7, 8, 7]),         # a page twice
                                 ([20, 20], [20, 20], [6, 7, 8, 1])):        # a page that is read
        assert evict(host, cache, a, batch(host, cache, rows, lengths, pages)) == SHAPE
    assert evict(host, cache, a, into, kept=None) == NULL
    assert evict(host, cache, a, into, kept=C.c_void_p(1 << 20 | 2)) == ALIGN
    assert evict(host, other, a, into) == STALE and evict(host, cache, a, batch(host, other, [20, 20], [20, 20], [6, 7, 8, 9])) == STALE
    assert host.fake_evicts() == before + 1
    nothing = batch(host, cache, [0, 0], [0, 0], [])
    assert evict(host, cache, a, nothing, kept=None) == OK and host.fake_evicts() == before + 1


def plan(host, b):
    out = (C.c_longlong * 10)()
    host.fake_weigh_plan(b, out)
    return dict(zip(("parts", "block", "items", "few", "few_at", "tiles_at", "joins", "sums", "bytes", "image"), out))


@pytest.mark.parametrize("rows,lengths,q_heads", [
    ([1], [262], 2), ([9], [500], 2), ([1, 40, 0, 8, 300], [70, 90, 50, 120, 333], 4), ([17], [17], 2), ([2000], [2048], 2), ([300], [300], 20),
    ([0, 0], [5, 6], 2), ([400], [100], 2)])
def test_every_key_is_in_one_unit_and_its_memory_in_the_batch(host, rows, lengths, q_heads):
    ps, group = 128, q_heads // 2
    cache = tracked(host, page_size=ps)
    counts = [-(-n // ps) for n in lengths]
    b = batch(host, cache, rows, lengths, np.arange(sum(counts)) % 16, q_heads)
    p = plan(host, b)
    few = sum(-(-n // 32) for r, n in zip(rows, lengths) if 0 < r * group <= 16)
    many = [(r, n) for r, n in zip(rows, lengths) if r * group > 16]
    assert p["few"] == few and p["items"] == 2 * sum(-(-n // p["block"]) for _, n in many) and p["block"] in (128, 256)
    assert 1 <= p["parts"] <= max([1] + [-(-r * group // 128) for r, _ in many])
    assert p["image"] <= p["bytes"] and p["few_at"] + 8 * (len(rows) + 1) <= p["image"] and p["tiles_at"] + 8 * (len(rows) + 1) <= p["image"]
    if p["parts"] > 1:
        assert p["joins"] + 4 * p["items"] <= p["image"]
        assert p["sums"] + 4 * p["items"] * p["parts"] * p["block"] <= p["bytes"]


def test_few_keys_of_many_rows_are_shared_out_by_rows(host):
    cache = tracked(host, page_size=128, kv_heads=1)
    p = plan(host, batch(host, cache, [1000], [1000], list(range(8)), q_heads=8))
    assert p["items"] * p["parts"] >= 100
    cache = base.cache_of(host, pages=300, page_size=128, kv_heads=16)
    assert plan(host, batch(host, cache, [1041], [38000], list(range(297)), q_heads=16))["parts"] == 1
