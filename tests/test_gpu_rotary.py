"""Rotary positions of several axes on the GPU, against their definition in float64.

Tolerance of an entry y = x_a c - x_b s: half a step of its type (finfo.eps / 2 of |y|; half its least step where it is subnormal), and
6e-7 (|x_a| + |x_b|) for what is computed in 32 bits: the angle is off by at most pi 2^-25 (24 bits of a half turn) + 2 pi 2^-32, cosine and sine
by 2^-23 more (two units in the last place), a product and a fused sum by 2^-24 each: together less than 4e-7.
"""
import math

import pytest
import torch

import paper_2512_04939_b200 as pkg

pytestmark = pytest.mark.gpu

LAYOUTS = ["halves", "pairs", "across"]
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def reference(x, positions, sections, bases, layout, back=False):
    """In float64, plane by plane; and |x_a| + |x_b| of every entry."""
    y, size = x.double().clone(), x.double().abs()
    at = done = 0
    for a, n in enumerate(sections):
        for i in range(n // 2):
            if layout == "across":
                one, two, share = done + i, sum(sections) // 2 + done + i, (done + i) / (sum(sections) // 2)
            else:
                one, two = (at + i, at + n // 2 + i) if layout == "halves" else (at + 2 * i, at + 2 * i + 1)
                share = i / (n // 2)
            t = positions[a].double()[:, None] * bases[a] ** -share * (-1 if back else 1)
            p, q = x[..., one].double(), x[..., two].double()
            y[..., one], y[..., two] = p * t.cos() - q * t.sin(), p * t.sin() + q * t.cos()
            size[..., one] = size[..., two] = p.abs() + q.abs()
        at += n
        done += n // 2
    return y, size


def check(got, x, positions, sections, bases, layout, back=False):
    want, size = reference(x, positions, sections, bases, layout, back)
    info = torch.finfo(x.dtype)
    allowed = info.eps / 2 * torch.clamp(want.abs(), min=info.tiny) + 6e-7 * size
    over = ((got.double() - want).abs() / allowed).max().item() if got.numel() else 0.0
    assert over <= 1.0, over
    turned = sum(sections)
    assert torch.equal(got[..., turned:], x[..., turned:])


def inputs(rows, heads, head_dim, dtype, axes, seed=0, far=1000):
    g = torch.Generator().manual_seed(seed)
    x = [torch.randn(rows, h, head_dim, generator=g).to(dtype).cuda() for h in heads]
    positions = torch.randint(-far, far, (axes, rows), generator=g, dtype=torch.int32).cuda()
    return x, positions


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rows,heads,head_dim,sections", [
    (1, (16, 16), 64, (16, 24, 24)), (333, (16, 16), 64, (16, 16, 32)), (5000, (32, 8), 128, (32, 48, 48)), (77, (8, 1), 128, (2, 60, 66)),
    (40, (12, 4), 80, (16, 24, 24)), (9, (3, 1), 6, (2, 2)), (64, (1, 1), 256, (64, 64, 64, 64)), (31, (5, 2), 50, (14, 0, 30)),
    (2, (300, 7), 64, (64,))])
def test_rotated_and_rotated_back(dtype, layout, rows, heads, head_dim, sections):
    bases = (10000.0, 100.0, 37.5, 2.0)[:len(sections)]
    rotary = pkg.RotaryAxes(head_dim, sections, bases, layout)
    (q, k), positions = inputs(rows, heads, head_dim, dtype, len(sections))
    for back, turn in ((False, rotary.rotate), (True, rotary.rotate_back)):
        for got, x in zip(turn(positions, q, k), (q, k)):
            check(got, x, positions, sections, bases, layout, back)
    assert torch.equal(rotary.rotate(positions, q), rotary.rotate(positions, q, k)[0])


@pytest.mark.parametrize("layout", LAYOUTS)
def test_slices_of_a_projection_in_place_and_odd_addresses(layout):
    sections, bases = (16, 24, 16), (10000.0, 100.0, 100.0)
    rotary = pkg.RotaryAxes(64, sections, bases, layout)
    (fused,), positions = inputs(200, (1,), 16 * 64 * 3 + 8, torch.bfloat16, 3)
    for shift in (0, 1, 2, 4):  # elements: widths of 16, 2, 4 and 8 bytes
        whole = fused[:, 0].clone()
        q, k = (whole[:, shift + lo:shift + lo + 1024].unflatten(1, (16, 64)) for lo in (0, 1024))
        before = q.clone(), k.clone()
        got = rotary.rotate(positions, q, k, out=(q, k))
        assert got[0].data_ptr() == q.data_ptr()
        for x, y in zip(before, (q, k)):
            check(y, x, positions, sections, bases, layout)
        assert torch.equal(whole[:, shift + 2048:], fused[:, 0, shift + 2048:]) and torch.equal(whole[:, :shift], fused[:, 0, :shift])
    # heads outside rows, positions by rows, queries shared by all heads
    x = before[0].transpose(0, 1).contiguous().transpose(0, 1)
    check(rotary.rotate(positions.T.contiguous().T, x), x, positions, sections, bases, layout)
    x = before[0][:, :1].expand(-1, 16, -1)
    check(rotary.rotate(positions, x), x, positions, sections, bases, layout)


def test_far_positions_keep_their_angle():
    """At position 2^31 - 1 a 32-bit product would be off by many turns; what is left of float64's own is 2^31 2^-53."""
    sections, bases = (32, 32), (10000.0, 3.0)
    rotary = pkg.RotaryAxes(64, sections, bases)
    (x,), _ = inputs(6, (4,), 64, torch.float32, 2)
    positions = torch.tensor([[2 ** 31 - 1, -2 ** 31, 0, 1, 10 ** 9, 1 << 20]] * 2, dtype=torch.int32).cuda()
    check(rotary.rotate(positions, x), x, positions, sections, bases, "halves")
    assert torch.equal(rotary.rotate(positions, x)[2], x[2])


def test_values_that_are_not_finite_stay_in_their_plane():
    rotary = pkg.RotaryAxes(64, (32, 16), (100.0, 100.0))
    (x,), positions = inputs(8, (4,), 64, torch.bfloat16, 2)
    x[3, 1, 5], x[2, 0, 60], x[4, 2, 63] = math.inf, math.nan, -math.inf
    got = rotary.rotate(positions, x)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[3, 1, [5, 21]] = bad[2, 0, 60] = bad[4, 2, 63] = True
    assert torch.equal(~torch.isfinite(got), bad)
    assert got[2, 0, 60].isnan() and got[4, 2, 63] == -math.inf


@pytest.mark.parametrize("layout", LAYOUTS)
def test_the_gradient_against_differences(layout):
    """f = sum g . rotate(x) is linear in x, so its differences are exact but for roundings: 2 * 1e-6 of the terms."""
    sections, bases = (10, 12, 8), (10000.0, 100.0, 100.0)
    rotary = pkg.RotaryAxes(32, sections, bases, layout)
    (x, g), positions = inputs(3, (2, 2), 32, torch.float32, 3)
    grad = rotary.rotate_back(positions, g)
    f0 = (g.double() * rotary.rotate(positions, x).double()).sum()
    for i in range(0, 3 * 2 * 32, 7):
        step = torch.zeros(3 * 2 * 32, device="cuda")
        step[i] = 1.0
        f1 = (g.double() * rotary.rotate(positions, x + step.view_as(x)).double()).sum()
        assert abs((f1 - f0 - grad.flatten()[i].double()).item()) <= 2e-6 * (g.abs().max() * (x.abs().max() + 1)).item() * 4
    # and the rotation keeps lengths, so turning back gives the input
    assert (rotary.rotate_back(positions, rotary.rotate(positions, x)) - x).abs().max() <= 2e-6 * 2 * x.abs().max()


def test_captured_replayed_and_on_another_stream():
    sections, bases = (16, 24, 24), (10000.0, 100.0, 100.0)
    rotary = pkg.RotaryAxes(64, sections, bases)
    (q, k), positions = inputs(100, (16, 16), 64, torch.bfloat16, 3)
    out = torch.empty_like(q), torch.empty_like(k)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = rotary.rotate(positions, q, k)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        rotary.rotate(positions, q, k, out=out)
    for _ in range(2):
        q.neg_(), positions.neg_()
        graph.replay()
        for got, x in zip(out, (q, k)):
            check(got, x, positions, sections, bases, "halves")
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_made_outside_a_capture():
    """The table is copied from the call's own memory, which a graph would read again at every replay."""
    x, graph = torch.zeros(8, device="cuda"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(pkg.LiteVGGTError):
            pkg.RotaryAxes(64, (64,), (100.0,))
    graph.replay()
    assert x.eq(1).all()


def test_no_rows_and_refusals():
    rotary = pkg.RotaryAxes(64, (16, 24, 24), (10000.0, 100.0, 100.0))
    (q, k), positions = inputs(10, (16, 4), 64, torch.bfloat16, 3)
    assert rotary.rotate(positions[:, :0], q[:0], k[:0])[1].shape == (0, 4, 64)
    for args in ((positions[:2], q), (positions.long(), q), (positions.cpu(), q), (positions[:, :9], q), (positions, q[:, :, :32]), (positions, q.double()),
                 (positions, q, k.float()), (positions, q, k[:9]), (positions, q.cpu()), (positions, q[0]), (positions, q.transpose(1, 2)), (positions, q[:, :0])):
        with pytest.raises(ValueError):
            rotary.rotate(*args)
    for out in ((q,), (q, k, k), (q, k[:, :2]), (q.float(), k)):
        with pytest.raises(ValueError):
            rotary.rotate(positions, q, k, out=out)
    buf = torch.zeros(11, 16, 64, dtype=torch.bfloat16, device="cuda")
    for src, dst in ((buf[:10], buf[1:]), (buf[1:], buf[:10])):
        with pytest.raises(pkg.LiteVGGTError):
            rotary.rotate(positions, src, out=dst)
    for bad in (dict(sections=(16, 24, 23)), dict(sections=(64, 2, 2)), dict(bases=(1.0, 2.0, 2.0)), dict(layout="thirds"), dict(bases=(2.0,)), dict(sections=(1.5, 2, 2)),
                dict(device=99)):
        kw = dict(sections=(16, 24, 24), bases=(10000.0, 100.0, 100.0))
        with pytest.raises((ValueError, pkg.LiteVGGTError)):
            pkg.RotaryAxes(64, **{**kw, **bad})
