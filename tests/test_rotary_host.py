"""The rotary entry points (rotary_api.cu) linked against stand-ins for the CUDA runtime and the kernel launch: what they refuse, how planes
are laid out and how a launch is cut.  No GPU."""
import ctypes as C
import math
import os
import subprocess

import pytest

from paper_2512_04939_b200.binding import RotaryConfig, RotaryTensor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2512_04939_b200", "csrc")
OK, NULL, BAD_CONFIG, SHAPE, ALIGN, CUDA = 0, 1, 2, 3, 4, 6
BASE = 1 << 30  # an address that nothing follows


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host") / "librotaryhost.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-w", "-Wl,-Bsymbolic", "-I/usr/local/cuda/include", "-x", "c++",
                    os.path.join(CSRC, "rotary_api.cu"), os.path.join(HERE, "rotary_host_fakes.cpp"), "-o", so], check=True)
    return C.CDLL(so)


def config(head_dim=64, sections=(16, 24, 24), bases=None, layout=0):
    bases = (100.0,) * len(sections) if bases is None else bases
    pad = 4 - len(sections)
    return RotaryConfig(head_dim, len(sections), (C.c_int32 * 4)(*sections, *[0] * pad), (C.c_double * 4)(*bases, *[0.0] * pad), layout)


_KEPT = []


def memory(size=2048):
    _KEPT.append(C.create_string_buffer(size + 16))
    return C.c_void_p((C.addressof(_KEPT[-1]) + 15) & ~15)


def create(host, cfg, handle, device=0, at="own", size=2048):
    return host.litevggt_rotary_create(None if cfg is None else C.byref(cfg), device, memory() if at == "own" else at, C.c_size_t(size), None,
                                       None if handle is None else C.byref(handle))


def made(host, device=0, **kw):
    handle = C.c_void_p()
    assert create(host, config(**kw), handle, device) == OK
    return handle


def tensor(src=BASE, dst=2 * BASE, row=1024, head=64, heads=16, out_row=None, out_head=None):
    return RotaryTensor(src, row, head, dst, row if out_row is None else out_row, head if out_head is None else out_head, heads)


def apply(host, handle, *tensors, rows=7, dtype=0, positions=4 * BASE, axis_stride=7, row_stride=1, n=None):
    i64 = C.c_int64
    many = (RotaryTensor * max(len(tensors), 1))(*tensors)
    return host.litevggt_rotary_apply(handle, C.c_void_p(positions), i64(axis_stride), i64(row_stride), i64(rows), dtype, 0, many,
                                      len(tensors) if n is None else n, None)


def last(host):
    out = (C.c_int * 11)()
    host.fake_last(out)
    return dict(zip(("width", "neighbours", "units", "turned", "slots", "block_rows", "blocks", "planes", "threads", "across",
                     "all_slots"), out))


@pytest.mark.parametrize("bad", [
    dict(head_dim=0), dict(head_dim=258, sections=(2,)), dict(sections=(16, 24, 26)), dict(sections=(16, 25, 23)), dict(sections=(0, 0)),
    dict(sections=(-2, 66)), dict(bases=(1.0, 100.0, 100.0)), dict(bases=(float("nan"), 100.0, 100.0)), dict(bases=(100.0, math.inf, 2.0)),
    dict(layout=3), dict(layout=-1)])
def test_configurations_that_are_refused(host, bad):
    handle, cfg = C.c_void_p(5), config(**bad)
    assert create(host, cfg, handle) == BAD_CONFIG
    assert handle.value is None


def test_axes_devices_and_handles_that_are_refused(host):
    handle, cfg = C.c_void_p(), config()
    for n in (0, 5, -1):
        cfg.n_axes = n
        assert create(host, cfg, handle) == BAD_CONFIG
    cfg.n_axes = 3
    assert create(host, cfg, handle, 2) == CUDA
    assert create(host, None, handle) == NULL and create(host, cfg, None) == NULL and create(host, cfg, handle, at=None) == NULL
    assert create(host, cfg, handle, size=1000) == SHAPE and create(host, cfg, handle, at=C.c_void_p(memory().value + 8)) == ALIGN
    host.fake_capture(1)
    assert create(host, cfg, handle) == CUDA and handle.value is None
    host.fake_capture(0)
    assert create(host, cfg, handle, 1) == OK and host.fake_copied_on() == 1 and host.fake_get_device() == 0
    assert host.litevggt_rotary_destroy(handle) == OK and host.litevggt_rotary_destroy(None) == OK
    assert apply(host, None, tensor()) == NULL


@pytest.mark.parametrize("layout", [0, 1, 2])
@pytest.mark.parametrize("head_dim,sections,bases", [(64, (16, 24, 24), (10000.0, 100.0, 50.0)), (128, (2, 66, 0, 30), (3.0, 100.0, 7.0, 1e6)), (6, (6,), (10.0,))])
def test_planes_and_their_turns(host, layout, head_dim, sections, bases):
    handle = made(host, head_dim=head_dim, sections=sections, bases=bases, layout=layout)
    assert apply(host, handle, tensor(row=head_dim * 16, head=head_dim)) == OK
    total, p, at = sum(sections) // 2, 0, 0
    assert last(host)["planes"] == total
    first, second, axis, turn = C.c_int(), C.c_int(), C.c_int(), C.c_ulonglong()
    for a, n in enumerate(sections):
        for i in range(n // 2):
            host.fake_plane(p, C.byref(first), C.byref(second), C.byref(axis), C.byref(turn))
            want = [(at + i, at + n // 2 + i), (at + 2 * i, at + 2 * i + 1), (p, total + p)][layout]
            assert (first.value, second.value, axis.value) == (*want, a)
            share = p / total if layout == 2 else i / (n // 2)
            frequency = bases[a] ** -share
            # float64's power, and half of the turn's own unit, 2^-64
            assert abs(turn.value / 2.0 ** 64 * 2 * math.pi - frequency) <= 4e-15 * frequency + 2 * math.pi * 2.0 ** -65
            p += 1
        at += n


@pytest.mark.parametrize("kw,t,dtype,width", [
    (dict(sections=(16, 16, 32)), {}, 0, 8), (dict(sections=(16, 24, 24)), {}, 0, 4), (dict(sections=(16, 24, 24), layout=2), {}, 0, 8),
    (dict(sections=(16, 24, 24), layout=1), {}, 0, 8), (dict(sections=(16, 24, 24), layout=2), {}, 2, 4), (dict(sections=(2, 30, 32)), {}, 1, 1),
    (dict(sections=(4, 28, 32)), {}, 1, 2), (dict(sections=(2, 2), layout=1), {}, 0, 4), (dict(sections=(6,), layout=1), {}, 0, 2),
    (dict(layout=1), dict(src=BASE + 2), 0, 1), (dict(layout=1), dict(dst=2 * BASE + 4), 0, 2), (dict(layout=1), dict(row=1028), 0, 4),
    (dict(layout=1), dict(row=1025), 2, 1), (dict(layout=1), dict(head=66, row=2048), 0, 2)])
def test_widths_follow_sections_and_alignment(host, kw, t, dtype, width):
    handle = made(host, **kw)
    assert apply(host, handle, tensor(**t), dtype=dtype) == OK
    got = last(host)
    assert got["width"] == width and got["neighbours"] == (kw.get("layout") == 1 and width > 1)
    assert got["units"] * got["slots"] * got["block_rows"] <= 256
    channels = got["turned"] * width * (1 if got["neighbours"] else 2) + (got["units"] - got["turned"]) * width
    assert channels == 64
    assert got["blocks"] * got["block_rows"] >= 7


def test_every_head_dim_is_cut_into_whole_units(host):
    for head_dim in range(2, 257):
        for width in {2, head_dim // 2 * 2, head_dim // 4 * 2} - {0}:
            for layout in (0, 1, 2):
                handle = made(host, head_dim=head_dim, sections=(width,), layout=layout)
                assert apply(host, handle, tensor(row=head_dim * 16, head=head_dim), rows=100000) == OK
                got = last(host)
                covered = got["turned"] * got["width"] * (1 if got["neighbours"] else 2) + (got["units"] - got["turned"]) * got["width"]
                assert covered == head_dim and 1 <= got["units"] * got["slots"] * got["block_rows"] <= got["threads"] <= 256
                assert got["slots"] * got["across"] == got["all_slots"] <= 16
                host.litevggt_rotary_destroy(handle)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(dtype=3), SHAPE), (dict(n=0), SHAPE), (dict(n=3), SHAPE),
    (dict(axis_stride=-1), SHAPE), (dict(row_stride=1 << 40), SHAPE), (dict(positions=0), NULL), (dict(positions=4 * BASE + 2), ALIGN)])
def test_calls_that_are_refused(host, kw, code):
    handle, before = made(host), host.fake_launches()
    assert apply(host, handle, tensor(), **kw) == code
    assert host.fake_launches() == before


@pytest.mark.parametrize("t,code", [
    (dict(src=0), NULL), (dict(dst=0), NULL), (dict(heads=0), SHAPE), (dict(heads=16385), SHAPE), (dict(row=-1), SHAPE), (dict(head=-64), SHAPE),
    (dict(row=1 << 40), SHAPE), (dict(src=BASE + 1), ALIGN), (dict(out_head=0), SHAPE), (dict(out_row=0), SHAPE), (dict(out_row=960), SHAPE),
    (dict(out_head=63), SHAPE), (dict(dst=BASE + 2048), SHAPE), (dict(dst=BASE, out_row=2048), SHAPE), (dict(dst=BASE + 128), SHAPE)])
def test_tensors_that_are_refused(host, t, code):
    handle, before = made(host), host.fake_launches()
    assert apply(host, handle, tensor(**t)) == code
    assert host.fake_launches() == before
    assert apply(host, handle, tensor(src=3 * BASE, dst=3 * BASE), tensor(**t)) == code


def test_what_may_lie_where(host):
    handle = made(host)
    fused = dict(row=4096, out_row=4096)
    assert apply(host, handle, tensor(dst=BASE)) == OK                                          # in place
    assert apply(host, handle, tensor(dst=BASE, **fused), tensor(src=BASE + 2048, dst=BASE + 2048, **fused)) == OK  # slices of one projection
    assert apply(host, handle, tensor(dst=BASE + 4096, **fused)) == OK                          # into another slice of it
    assert apply(host, handle, tensor(row=0, head=0, out_row=1024, out_head=64)) == OK          # an input that is the same for all
    assert apply(host, handle, tensor(row=64, head=7 * 64)) == OK                               # heads outside rows
    assert apply(host, handle, tensor(row=4, head=4, heads=1, out_row=64, out_head=0)) == OK    # rows of an input that overlap
    # one tensor's output in another's input, or both outputs in one place
    assert apply(host, handle, tensor(), tensor(src=3 * BASE, dst=BASE)) == SHAPE
    assert apply(host, handle, tensor(), tensor(src=3 * BASE, dst=2 * BASE + 64)) == SHAPE
    # an output over the positions
    assert apply(host, handle, tensor(), positions=2 * BASE + 128) == SHAPE and apply(host, handle, tensor(dst=4 * BASE)) == SHAPE
    assert apply(host, handle, tensor(dst=BASE), positions=BASE) == SHAPE
    # no rows: nothing is looked at
    assert apply(host, handle, tensor(src=0, dst=0), rows=0, positions=0) == OK


def test_calls_run_on_their_own_device(host):
    handle = made(host, device=1)
    assert apply(host, handle, tensor()) == OK
    assert host.fake_launched_on() == 1 and host.fake_get_device() == 0
