"""Where the rotary calls' outputs may lie beside inputs and one another: tensors whose heads lie outside their rows, interleaved head by head.
On the stand-ins of test_rotary_host.py.  No GPU."""
import random

import pytest
import torch

from test_rotary_host import BASE, OK, SHAPE, apply, host, made, tensor  # noqa: F401


@pytest.mark.parametrize("kv_heads", [16, 4, 1])
def test_slices_of_heads_that_lie_outside_rows(host, kv_heads):
    """Queries and keys of [heads, 3, rows, head_dim], seven rows of 64 in two bytes each, turned where they are."""
    handle, piece = made(host), 7 * 64
    q = dict(row=64, head=3 * piece, out_row=64, out_head=3 * piece)
    k = dict(q, heads=kv_heads)
    assert apply(host, handle, tensor(dst=BASE, **q), tensor(src=BASE + 2 * piece, dst=BASE + 2 * piece, **k)) == OK
    assert apply(host, handle, tensor(dst=BASE + 4 * piece, **q)) == OK  # into the values' place
    # a row or a byte too near
    assert apply(host, handle, tensor(dst=BASE, **q), tensor(src=BASE + 2 * piece - 128, dst=BASE + 2 * piece - 128, **k)) == SHAPE
    assert apply(host, handle, tensor(dst=BASE + 4 * piece + 128, **q)) == SHAPE
    assert apply(host, handle, tensor(dst=BASE, **q), tensor(src=BASE + 6 * piece - 16, dst=BASE + 6 * piece - 16, **k)) == SHAPE


def test_what_is_let_through_never_meets(host):
    """Any strides: an accepted call's output shares no element with another tensor of it."""
    rng, handle, let = random.Random(80), made(host, head_dim=2, sections=(2,)), 0
    for _ in range(20000):
        rows, heads = rng.randint(1, 4), (rng.randint(1, 3), rng.randint(1, 3))
        step = [(rng.randint(0, 12), rng.randint(0, 24)) for _ in range(4)]
        if rng.random() < 0.7:
            step = [step[0]] * 4
        at = [rng.randint(0, 60) for _ in range(4)]
        if rng.random() < 0.5:
            at[1], at[3], step[1], step[3] = at[0], at[2], step[0], step[2]
        many = [tensor(BASE + 2 * at[2 * i], BASE + 2 * at[2 * i + 1], *step[2 * i], heads[i], *step[2 * i + 1]) for i in range(2)]
        for t, (row, head), (out_row, out_head), n in zip(many, step[::2], step[1::2], heads):
            t.in_row, t.in_head, t.out_row, t.out_head, t.heads = row, head, out_row, out_head, n
        if apply(host, handle, *many, rows=rows) != OK:
            continue
        let += 1
        places = [[at[i] + r * step[i][0] + h * step[i][1] + c for r in range(rows) for h in range(heads[i // 2]) for c in range(2)] for i in range(4)]
        for o in (1, 3):
            assert len(set(places[o])) == len(places[o])
            for other in {0, 1, 2, 3} - {o}:
                assert not set(places[o]) & set(places[other]) or places[o] == places[other] and other == o - 1
    assert let > 2000


@pytest.mark.gpu
def test_heads_outside_rows_in_place():
    import paper_2512_04939_b200 as pkg

    rotary = pkg.RotaryAxes(64, (16, 24, 24), (10000.0, 100.0, 100.0))
    g = torch.Generator(device="cuda").manual_seed(81)
    whole = torch.randn(8, 3, 100, 64, generator=g, device="cuda").bfloat16()
    positions = torch.randint(0, 1000, (3, 100), generator=g, device="cuda", dtype=torch.int32)
    q, k = (whole[:, i].transpose(0, 1) for i in (0, 1))
    want, values = rotary.rotate(positions, q, k), whole[:, 2].clone()
    rotary.rotate(positions, q, k, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(whole[:, 2], values)
