"""norm_rotary() under torch's transforms on the GPU: torch.compile gives what the call gives, and the transforms that it has no rule for raise."""
import pytest
import torch

from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def inputs():
    torch.manual_seed(0)
    q, k = (torch.randn(2, h, 9, 32, device="cuda") for h in (4, 2))
    return q, k, torch.randint(0, 99, (1, 9, 2), device="cuda", dtype=torch.int32), torch.rand(16, device="cuda"), torch.rand(32, device="cuda")


@pytest.mark.parametrize("transform", [lambda f, q: torch.func.vmap(f)(q[None]), lambda f, q: torch.func.jvp(f, (q,), (q,))], ids=["vmap", "jvp"])
def test_transforms_without_a_rule_raise(transform):
    q, _, pos, inv, w = inputs()
    with pytest.raises(RuntimeError):
        transform(lambda x: F.norm_rotary(x, None, pos, inv, w, sections=(5, 11))[0], q)


def test_forward_mode_raises():
    q, _, pos, inv, w = inputs()
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(q, torch.ones_like(q))
        with pytest.raises(RuntimeError):
            F.norm_rotary(dual, None, pos, inv, w, sections=(5, 11))


def test_compiled_calls():
    q, k, pos, inv, w = inputs()

    def step(q, k, w):
        return sum((x ** 3).sum() for x in F.norm_rotary(q, k, pos, inv, w, w, sections=(5, 11)))

    leaves = [x.requires_grad_(True) for x in (q, k, w)]
    want = step(*leaves)
    grads = torch.autograd.grad(want, leaves)
    got = torch.compile(step, backend="eager")(*leaves)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(got, leaves), grads))
