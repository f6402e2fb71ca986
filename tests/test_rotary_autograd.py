"""Rotations and autograd: what would lose a gradient without a word is refused, and an autograd.Function around the two calls gives it."""
import types

import pytest
import torch

from paper_2512_04939_b200 import RotaryAxes


class Reached(Exception):
    pass


def on_the_host():
    """An object whose tensors are on the CPU and whose library call says that it was reached."""
    r = RotaryAxes.__new__(RotaryAxes)
    r._index, r._axes, r.head_dim, r.device, r.handle = -1, 1, 4, torch.device("cpu"), None
    return r


@pytest.mark.parametrize("call", ["rotate", "rotate_back"])
def test_tensors_that_require_a_gradient_are_refused(call):
    r, positions = on_the_host(), torch.zeros(1, 3, dtype=torch.int32)
    plain, leaf = torch.ones(3, 2, 4), torch.ones(3, 2, 4, requires_grad=True)
    for args, out in (((leaf,), None), ((plain, leaf), None), ((leaf * 2.0, plain), None), ((plain,), leaf), ((plain, plain), (torch.ones(3, 2, 4), leaf)),
                      ((leaf,), leaf)):
        with pytest.raises(ValueError, match="autograd"):
            getattr(r, call)(positions, *args, out=out)
    assert leaf.grad is None and (leaf == 1.0).all()


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_they_are_taken_where_gradients_are_off(mode, monkeypatch):
    r, leaf = on_the_host(), torch.ones(3, 2, 4, requires_grad=True)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0, raising=False)

    def reached(*_):
        raise Reached

    r._home, r._apply = 0, reached
    with mode(), pytest.raises(Reached):
        r.rotate(torch.zeros(1, 3, dtype=torch.int32), leaf)


@pytest.mark.gpu
def test_a_function_around_them_gives_the_gradient():
    rotary = RotaryAxes(64, (16, 24, 24), (10000.0, 100.0, 100.0))
    g = torch.Generator(device="cuda").manual_seed(70)
    positions = torch.randint(0, 1000, (3, 33), generator=g, device="cuda", dtype=torch.int32)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k):
            return rotary.rotate(positions, q, k)

        @staticmethod
        def backward(ctx, dq, dk):
            return rotary.rotate_back(positions, dq, dk)

    q, k = (torch.randn(33, h, 64, generator=g, device="cuda", requires_grad=True) for h in (4, 2))
    with pytest.raises(ValueError, match="autograd"):
        rotary.rotate(positions, q, k)
    with pytest.raises(ValueError, match="autograd"):
        rotary.rotate(positions, q, out=q)
    wq, wk = (torch.randn(33, h, 64, generator=g, device="cuda") for h in (4, 2))
    yq, yk = Turn.apply(q, k)
    ((yq * wq).sum() + (yk * wk).sum()).backward()
    dq, dk = rotary.rotate_back(positions, wq, wk)
    assert torch.equal(q.grad, dq) and torch.equal(k.grad, dk)
    # <rotate(x), w> = <x, rotate_back(w)>: cosines and sines are the same bits both ways, so only the product's rounding and the sum's differ, 2 2^-24
    # of |x_a| + |x_b| in each of a plane's two, 2^-22 of a row's norm, once each way
    left, right = (yq.double() * wq.double()).sum(2), (q.detach().double() * dq.double()).sum(2)
    assert ((left - right).abs() <= 2.0 ** -20 * q.detach().double().norm(dim=2) * wq.double().norm(dim=2)).all()
