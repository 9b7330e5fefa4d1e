"""rotary() under torch.func on the GPU."""
import pytest
import torch

from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def inputs():
    torch.manual_seed(0)
    q, k = (torch.randn(2, h, 9, 32, device="cuda") for h in (4, 2))
    return q, k, torch.randint(0, 99, (1, 9, 2), device="cuda", dtype=torch.int32), torch.rand(16, device="cuda")


def test_func_grad_is_the_ordinary_gradient():
    q, k, pos, inv = inputs()
    loss = lambda q, k: sum((x ** 3).sum() for x in F.rotary(q, k, pos, inv, sections=(5, 11)))
    got = torch.func.grad(loss, argnums=(0, 1))(q, k)
    q.requires_grad_(True), k.requires_grad_(True)
    want = torch.autograd.grad(loss(q, k), (q, k))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_func_grad_of_a_sum_and_of_a_gradient():
    """A gradient that arrives as one number, expanded; and the second derivative: |R x|^4 / 4 has the gradient |x|^2 x."""
    q, k, pos, inv = inputs()
    total = torch.func.grad(lambda x: F.rotary(x, None, pos, inv, sections=(5, 11))[0].sum())(q)
    x = q.clone().requires_grad_(True)
    F.rotary(x, None, pos, inv, sections=(5, 11))[0].sum().backward()
    assert torch.equal(total, x.grad)
    fourth = lambda x: (F.rotary(x, None, pos, inv, sections=(5, 11))[0].square().sum() ** 2) / 4
    u = torch.randn_like(q)
    second = torch.func.grad(lambda x: (torch.func.grad(fourth)(x) * u).sum())(q).double()
    qd, ud = q.double(), u.double()
    want = 2 * (qd * ud).sum() * qd + qd.square().sum() * ud
    assert torch.allclose(second, want, rtol=1e-4, atol=1e-4 * float(want.abs().max()))


@pytest.mark.parametrize("transform", [lambda f, q: torch.func.vmap(f)(q[None]), lambda f, q: torch.func.jvp(f, (q,), (q,))])
def test_transforms_without_a_rule_raise(transform):
    q, _, pos, inv = inputs()
    with pytest.raises(RuntimeError):
        transform(lambda x: F.rotary(x, None, pos, inv, sections=(5, 11))[0], q)
