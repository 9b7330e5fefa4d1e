"""What rotary()'s backward pass reads again, on the GPU: positions and frequencies as they were in the forward pass, or an error."""
import pytest
import torch

from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def native(q, k, pos, inv):
    return F.rotary(q, k, pos, inv)


def python(q, k, pos, inv):
    return F._Rotary.apply(q, k, pos, inv, (16,), False, False)


def inputs(rows=2):
    torch.manual_seed(0)
    q, k = (torch.randn(2, h, 9, 32, device="cuda", requires_grad=True) for h in (4, 2))
    return q, k, torch.randint(0, 99, (rows, 9, 1), device="cuda", dtype=torch.int32), torch.rand(16, device="cuda")


@pytest.mark.parametrize("node", [native, python])
@pytest.mark.parametrize("which", ["positions", "inv_freq"])
def test_in_place_changes_raise(node, which):
    q, k, pos, inv = inputs()
    qo, ko = node(q, k, pos, inv)
    (pos if which == "positions" else inv).add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (qo.sum() + ko.sum()).backward()


def test_one_row_of_positions_for_all_sequences():
    """The call expands it: the version is that of the caller's tensor all the same."""
    q, k, pos, inv = inputs(1)
    qo, _ = F.rotary(q, k, pos, inv)
    pos.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        qo.sum().backward()


@pytest.mark.parametrize("node", [native, python])
def test_changes_behind_the_backward_pass_are_fine(node):
    q, k, pos, inv = inputs()
    want = [torch.autograd.grad(F.rotary(q, k, pos + n, inv)[0].square().sum() + F.rotary(q, k, pos + n, inv)[1].sum(), (q, k)) for n in range(2)]
    for n in range(2):
        qo, ko = node(q, k, pos, inv)
        got = torch.autograd.grad(qo.square().sum() + ko.sum(), (q, k))
        assert all(torch.equal(x, y) for x, y in zip(got, want[n]))
        pos.add_(1)


@pytest.mark.parametrize("node", [native, python])
def test_tensors_made_in_inference_mode(node):
    q, k, pos, inv = inputs()
    want = torch.autograd.grad(F.rotary(q, k, pos, inv)[0].sum(), q)[0]
    with torch.inference_mode():
        pos, inv = pos.clone(), inv.clone()
    assert torch.equal(torch.autograd.grad(node(q, k, pos, inv)[0].sum(), q)[0], want)


def test_frequencies_that_want_a_gradient():
    q, k, pos, inv = inputs()
    inv.requires_grad_(True)
    with pytest.raises(ValueError, match="inv_freq"):
        F.rotary(q, k, pos, inv)
    with torch.no_grad():
        want = F.rotary(q, k, pos, inv)
    got = F.rotary(q, k, pos, inv.detach())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
