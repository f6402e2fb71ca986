"""The paged K/V cache's entry points (kv_api.cu) linked against stand-ins for the CUDA runtime, two devices of it, and for the kernel
launchers (kv_host_fakes.cpp).  No GPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2512_04939_b200.binding import KVConfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2512_04939_b200", "csrc")


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host") / "libkvhost.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-w", "-Wl,-Bsymbolic", "-I/usr/local/cuda/include", "-x", "c++",
                    os.path.join(CSRC, "kv_api.cu"), os.path.join(HERE, "kv_host_fakes.cpp"), "-o", so], check=True)
    return C.CDLL(so)


@pytest.fixture(autouse=True)
def fresh(host):
    host.fake_current_device(0)
    host.fake_capture(0)
    host.fake_forget()


_KEPT = []


def memory(size):
    _KEPT.append(C.create_string_buffer(size + 256))
    return C.c_void_p((C.addressof(_KEPT[-1]) + 255) & ~255)


def cache_of(host, device=0, pages=8, page_size=16, kv_heads=2, head_dim=64):
    cfg, handle, p = KVConfig(pages, page_size, kv_heads, head_dim, 0), C.c_void_p(), memory(64)
    assert host.litevggt_kv_create(C.byref(cfg), device, p, p, None, None, p, C.byref(handle)) == 0
    return handle


def batch_of(host, cache, rows=3, length=20, pages=(1, 0), q_heads=2, place=True):
    handle, size = C.c_void_p(), C.c_size_t()
    assert host.litevggt_kv_batch_create(cache, 1, (C.c_int32 * 1)(rows), (C.c_int32 * 1)(length), (C.c_int32 * len(pages))(*pages), q_heads, 0,
                                         C.byref(handle), C.byref(size)) == 0
    if place:
        assert host.litevggt_kv_batch_place(handle, memory(size.value), size, None) == 0
    return handle, size


def calls(host, cache, batch):
    """Every call that takes a batch: append, gather, attend."""
    p, i64 = memory(64), C.c_int64
    return [host.litevggt_kv_append(cache, batch, p, i64(128), i64(64), p, i64(128), i64(64), None),
            host.litevggt_kv_gather(cache, batch, p, p, None),
            host.litevggt_kv_attend(cache, batch, p, i64(128), i64(64), C.c_float(0.125), memory(1 << 14), None)]


@pytest.mark.parametrize("device,current", [(1, 0), (0, 1), (1, 1)])
def test_every_stream_call_is_made_on_the_caches_device(host, device, current):
    """Streams are named by handles that mean another stream on another device (the default ones do): a batch's arrays have to be
    on their way in the stream that its kernels follow in, whatever device is current, and that stays current."""
    cache = cache_of(host, device)
    host.fake_current_device(current)
    batch, _ = batch_of(host, cache)
    assert (host.fake_stream_calls(device), host.fake_stream_calls(1 - device)) == (1, 0)
    assert calls(host, cache, batch) == [0, 0, 0]
    host.fake_forget()
    assert host.litevggt_kv_poll(cache, None) == 0
    assert host.fake_stream_calls(device) == 3 and host.fake_stream_calls(1 - device) == 0
    assert host.fake_get_device() == current


def test_a_batch_does_not_outlive_its_cache(host):
    """The next cache may lie where the last one did; a batch whose page numbers were checked against that one is refused."""
    for _ in range(20):
        old = cache_of(host, pages=8)
        batch, _ = batch_of(host, old, pages=(7, 6))
        assert calls(host, old, batch) == [0, 0, 0]
        assert host.litevggt_kv_destroy(old) == 0
        new = cache_of(host, pages=2)
        host.fake_forget()
        assert calls(host, new, batch) == [8, 8, 8] and host.fake_launches() == 0
        assert host.litevggt_kv_batch_destroy(batch) == 0 and host.litevggt_kv_destroy(new) == 0


def test_a_batch_is_not_placed_while_its_stream_is_captured(host):
    """The copy would be of the batch's own host memory, again at every replay, when the batch may be gone."""
    cache = cache_of(host)
    batch, size = batch_of(host, cache, place=False)
    host.fake_capture(1)
    assert host.litevggt_kv_batch_place(batch, memory(size.value), size, None) == 6
    assert host.fake_stream_calls(0) == 0 and calls(host, cache, batch) == [8, 8, 8]
    host.fake_capture(0)
    assert host.litevggt_kv_batch_place(batch, memory(size.value), size, None) == 0
    host.fake_capture(1)
    assert calls(host, cache, batch) == [0, 0, 0]  # calls with a batch that is in place may be captured


@pytest.mark.parametrize("at,row_stride,refused", [
    (0, 128, True), (8, 128, True), (-8, 128, True), (376, 128, True), (-376, 128, True),  # of 3 rows of 2 heads of 64
    (384, 128, False), (-384, 128, False),
    (-384, 4096, False), (120, 4096, True), (128, 4096, False), (3712, 4096, False), (3720, 4096, True), (4216, 4096, True), (4224, 4096, False),
    (8192 + 120, 4096, True), (8192 + 128, 4096, False), (120, 0, True), (128, 0, False)])
def test_outputs_lie_beside_the_queries(host, at, row_stride, refused):
    """`at`: where the output begins, in elements behind the queries.  A piece that is done again reads its queries again, so they must not
    have been written over; an output between rows of queries is none of that."""
    cache = cache_of(host)
    batch, _ = batch_of(host, cache)
    q = memory(1 << 16).value + (1 << 14)
    st = host.litevggt_kv_attend(cache, batch, C.c_void_p(q), C.c_int64(row_stride), C.c_int64(64), C.c_float(0.125), C.c_void_p(q + 2 * at), None)
    assert st == (3 if refused else 0)
