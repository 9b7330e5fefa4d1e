"""CPU tests of the Python autograd node of rotary(), its kernel replaced by a multiple of the frequencies."""
import pytest
import torch

from paper_2511_02043_amd import functional as F


@pytest.fixture(autouse=True)
def plain(monkeypatch):
    def turn(q, k, how, inverse):
        positions, inv_freq = how[:2]
        f = (positions[:, None, :, 0].float() * inv_freq[0])[..., None] * (-1 if inverse else 1)
        return tuple(None if x is None else x * f for x in (q, k))
    monkeypatch.setattr(F, "_rotary_plain", turn)


def call():
    q = torch.ones(1, 2, 4, 16, requires_grad=True)
    pos, inv = torch.arange(1, 5, dtype=torch.int32).reshape(1, 4, 1), torch.ones(8)
    return q, pos, inv, F._Rotary.apply(q, None, pos, inv, (8,), False, False)[0]


def test_gradient_of_the_positions_of_the_call():
    q, pos, inv, y = call()
    y.sum().backward()
    assert torch.equal(q.grad[0, 0, :, 0], -pos[0, :, 0].float())


@pytest.mark.parametrize("which", ["positions", "inv_freq"])
def test_what_the_backward_pass_reads_may_not_change(which):
    q, pos, inv, y = call()
    (pos if which == "positions" else inv).add_(6)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_positions_made_in_inference_mode():
    q = torch.ones(1, 2, 4, 16, requires_grad=True)
    with torch.inference_mode():
        pos, inv = torch.full((1, 4, 1), 3, dtype=torch.int32), torch.ones(8)
    F._Rotary.apply(q, None, pos, inv, (8,), False, False)[0].sum().backward()
    assert torch.equal(q.grad, torch.full_like(q, -3.0))


def test_func_grad_looks_into_the_node():
    pos, inv = torch.arange(1, 5, dtype=torch.int32).reshape(1, 4, 1), torch.ones(8)
    f = pos.reshape(1, 1, 4, 1).float()
    cube = lambda q: (F._Rotary.apply(q, None, pos, inv, (8,), False, False)[0] ** 3).sum()
    both = lambda q, k: sum((x ** 3).sum() for x in F._Rotary.apply(q, k, pos, inv, (8,), False, False))
    torch.manual_seed(0)
    q, k = torch.randn(1, 2, 4, 16), torch.randn(1, 1, 4, 16)
    # y = f q, and the stand-in's turn back is -f
    assert torch.allclose(torch.func.grad(cube)(q), -3 * f ** 3 * q ** 2)
    for got, x in zip(torch.func.grad(both, argnums=(0, 1))(q, k), (q, k)):
        assert torch.allclose(got, -3 * f ** 3 * x ** 2)
    twice = torch.func.grad(lambda x: torch.func.grad(cube)(x).sum())(q)
    # back through the turn back (a turn, f), the square's 6 y, and the first turn (-f)
    assert torch.allclose(twice, -6 * f ** 3 * q)


@pytest.mark.parametrize("transform", [lambda f, q: torch.func.vmap(f)(q[None]), lambda f, q: torch.func.jvp(f, (q,), (q,))])
def test_transforms_without_a_rule_are_refused(transform):
    pos, inv = torch.ones(1, 4, 1, dtype=torch.int32), torch.ones(8)
    with pytest.raises(RuntimeError):
        transform(lambda q: F._Rotary.apply(q, None, pos, inv, (8,), False, False)[0], torch.ones(1, 2, 4, 16))
