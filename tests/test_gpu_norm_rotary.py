"""Heads normalised and turned on the GPU against the fp64 oracle: forward pass and gradients.

Tolerances.  A row's sum of D <= 1032 squares in fp32, at most 40 of them one after the other in a lane and a tree of six: off by 46 * 2^-24 of itself, its
root by half of that, two roundings for root and quotient: the norm within 25 * 2^-24 = 1.5e-6, two products and the turn's three roundings 5 * 2^-24:
below 2e-6 of a pair's length.  In bf16 the machine's sine and cosine take 2^-14 of that length and the result's rounding 2^-8 of it.  A gradient is two
such terms, whose mean over D is formed like the norm, with r^3: 5e-6 (bf16: 2^-13) of their sizes.  A weight's gradient is a sum of N terms in fp32, at
most 200 of them one after the other (heads and tokens of a lane, 64th rows of partial sums) beside trees: 200 * 2^-24 = 1.2e-5 of the sum of their sizes,
in bf16 2^-14 more.
"""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def f64(x):
    return x.detach().double().cpu().numpy()


def setup(B, H, Hkv, S, D, sections, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    make = lambda h: (torch.randn(B, S, h, D, generator=g) * torch.exp(torch.randn(B, S, h, 1, generator=g))).to(DT[dtype]).cuda().transpose(1, 2)
    n = sum(sections)
    inv = (10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)).float().cuda()
    pos = torch.randint(-500, 9000, (B, S, len(sections)), generator=g).int().cuda()
    qw, kw = (torch.exp(0.5 * torch.randn(D, generator=g)).cuda() for _ in range(2))
    return make(H), make(Hkv), pos, inv, qw, kw


def check_forward(got, x, w, pos, inv, sections, interleaved, dtype):
    x, pos, inv = f64(x), pos.cpu().numpy(), f64(inv)
    w = None if w is None else f64(w)
    ref = mo.norm_rotary(x, w, pos, inv, sections, eps=EPS, interleaved=interleaved)
    z = mo.norm_rotary(x, w, 0 * pos, inv, sections, eps=EPS, interleaved=interleaved)
    length = mo.pair_lengths(z, sections, interleaved)
    bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -14 + 2e-6) * length if dtype == "bf16" else 2e-6 * length
    bad = ~(np.abs(f64(got) - ref) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:4], f64(got)[bad][:4], ref[bad][:4])


def check_gradient(dx, dw, x, w, dy, pos, inv, sections, interleaved, dtype):
    ref, ref_w, size, size_w = mo.norm_rotary_gradient(f64(x), None if w is None else f64(w), f64(dy), pos.cpu().numpy(), f64(inv), sections, eps=EPS,
                                                       interleaved=interleaved)
    if dx is not None:
        bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -13 * size if dtype == "bf16" else 5e-6 * size
        bad = ~(np.abs(f64(dx) - ref) <= bound)
        assert not bad.any(), (np.argwhere(bad)[:4], f64(dx)[bad][:4], ref[bad][:4])
    if dw is not None:
        bad = ~(np.abs(f64(dw) - ref_w) <= (1.2e-5 + (2.0 ** -14 if dtype == "bf16" else 0)) * size_w)
        assert not bad.any(), (np.argwhere(bad)[:4], f64(dw)[bad][:4], ref_w[bad][:4])


CASES = [
    (2, 4, 2, 37, 128, (16, 24, 24), False), (1, 3, 1, 1, 64, (8, 12, 12), True), (3, 2, 2, 5, 80, (40,), False), (1, 8, 8, 64, 32, (8, 8), True),
    (2, 2, 1, 9, 64, (10,), False), (1, 2, 1, 9, 40, (3, 4), True), (1, 1, 1, 3, 256, (32, 32, 32, 32), False), (2, 16, 2, 130, 128, (32,), False),
    (1, 2, 2, 7, 640, (150, 150), False), (1, 40, 8, 700, 64, (0, 32), True), (1, 1, 1, 2, 1024, (5,), False), (1, 2, 1, 3, 1024, (512,), True),
    (1, 2, 1, 5, 16, (8,), False), (1, 1, 2, 3, 8, (1,), False), (2, 5, 3, 3, 128, (13,), True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,S,D,sections,interleaved", CASES)
def test_forward_and_gradients(B, H, Hkv, S, D, sections, interleaved, dtype):
    q, k, pos, inv, qw, kw = setup(B, H, Hkv, S, D, sections, dtype)
    leaves = [x.requires_grad_(True) for x in (q, k, qw, kw)]
    qo, ko = F.norm_rotary(q, k, pos, inv, qw, kw, eps=EPS, sections=sections, interleaved=interleaved)
    assert qo.shape == q.shape and ko.shape == k.shape and qo.dtype == q.dtype
    dq, dk = torch.randn_like(qo), torch.randn_like(ko)
    gq, gk, gqw, gkw = torch.autograd.grad((qo, ko), leaves, (dq, dk))
    for got, x, w, dy, dx, dw in ((qo, q, qw, dq, gq, gqw), (ko, k, kw, dk, gk, gkw)):
        check_forward(got, x, w, pos, inv, sections, interleaved, dtype)
        check_gradient(dx, dw, x, w, dy, pos, inv, sections, interleaved, dtype)


def test_many_tokens_share_out_the_weights_gradient():
    q, k, pos, inv, qw, kw = setup(3, 3, 1, 5001, 64, (32,), "bf16")
    leaves = [x.requires_grad_(True) for x in (q, k, qw, kw)]
    out = F.norm_rotary(q, k, pos, inv, qw, kw, eps=EPS)
    dy = [torch.randn_like(x) for x in out]
    g = torch.autograd.grad(out, leaves, dy)
    again = torch.autograd.grad(F.norm_rotary(q, k, pos, inv, qw, kw, eps=EPS), leaves, dy)
    assert all(torch.equal(a, b) for a, b in zip(g, again))
    check_gradient(g[0], g[2], q, qw, dy[0], pos, inv, (32,), False, "bf16")
    check_gradient(g[1], g[3], k, kw, dy[1], pos, inv, (32,), False, "bf16")


def test_gradients_against_differences():
    """<dy, f(x + h u) - f(x - h u)> / 2 h in fp32: roundings of 4e-6 * |dy| |y| / h beside h^2 of a third derivative; the sums here have 800 terms of size 1."""
    q, k, pos, inv, qw, kw = setup(1, 2, 1, 6, 64, (16, 8), "f32")
    leaves = [x.requires_grad_(True) for x in (q, k, qw, kw)]
    dy = [torch.randn_like(x) for x in (q, k)]
    call = lambda *a: sum((y.double() * d.double()).sum() for y, d in zip(F.norm_rotary(a[0], a[1], pos, inv, a[2], a[3], eps=EPS, sections=(16, 8)), dy))
    g = torch.autograd.grad(F.norm_rotary(q, k, pos, inv, qw, kw, eps=EPS, sections=(16, 8)), leaves, dy)
    with torch.no_grad():
        for n in range(4):
            u, h = torch.randn_like(leaves[n]) * leaves[n].abs().mean(), 2.0 ** -8
            plus, minus = ([x + s * h * u if i == n else x for i, x in enumerate(leaves)] for s in (1, -1))
            quotient, want = (call(*plus) - call(*minus)) / (2 * h), (g[n].double() * u.double()).sum()
            assert abs(float(quotient - want)) <= 0.02 + 2e-3 * abs(float(want)), (n, float(quotient), float(want))


@pytest.mark.parametrize("which", ["q", "k", "q_weight", "k_weight", "q alone", "no weights", "broadcast", "one output"])
def test_gradients_that_are_wanted_or_arrive(which):
    q, k, pos, inv, qw, kw = setup(2, 4, 2, 11, 64, (32,), "f32")
    named = dict(q=q, k=k, q_weight=qw, k_weight=kw)
    if which in named:
        named[which].requires_grad_(True)
    else:
        for x in named.values():
            x.requires_grad_(True)
    if which == "q alone":
        k = kw = None
    if which == "no weights":
        qw = kw = None
    qo, ko = F.norm_rotary(q, k, pos, inv, qw, kw, eps=EPS)
    if which == "q alone":
        assert ko is None
    check_forward(qo, q, qw, pos, inv, (32,), False, "f32")
    if which == "broadcast":                       # a gradient of one number, expanded
        (qo.sum() + 2 * ko.sum()).backward()
        dy = torch.ones_like(qo), 2 * torch.ones_like(ko)
    elif which == "one output":
        dy = torch.randn_like(qo), None
        qo.backward(dy[0])
        assert k.grad is None and kw.grad is None
    else:
        dy = torch.randn_like(qo), None if ko is None else torch.randn_like(ko)
        torch.autograd.backward([y for y in (qo, ko) if y is not None and y.requires_grad], [d for d, y in zip(dy, (qo, ko)) if y is not None and y.requires_grad])
    for x, w, d in ((q, qw, dy[0]), (k, kw, dy[1])):
        if x is not None and d is not None:
            check_gradient(x.grad, None if w is None else w.grad, x, w, d, pos, inv, (32,), False, "f32")
    for name, x in named.items():
        if not x.requires_grad:
            assert x.grad is None, name


def test_shared_weight_takes_both_gradients():
    q, k, pos, inv, w, _ = setup(1, 4, 2, 13, 64, (32,), "f32")
    w.requires_grad_(True)
    qo, ko = F.norm_rotary(q, k, pos, inv, w, w, eps=EPS)
    dq, dk = torch.randn_like(qo), torch.randn_like(ko)
    torch.autograd.backward((qo, ko), (dq, dk))
    parts = [mo.norm_rotary_gradient(f64(x), f64(w), f64(d), pos.cpu().numpy(), f64(inv), (32,), eps=EPS) for x, d in ((q, dq), (k, dk))]
    assert (np.abs(f64(w.grad) - parts[0][1] - parts[1][1]) <= 1.3e-5 * (parts[0][3] + parts[1][3])).all()


def test_second_derivative_raises():
    q, k, pos, inv, qw, kw = setup(1, 2, 1, 4, 64, (32,), "f32")
    q.requires_grad_(True)
    y, _ = F.norm_rotary(q, k, pos, inv, qw, kw)
    (g,) = torch.autograd.grad((y ** 3).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        torch.autograd.grad(g.square().sum(), q)
    y, _ = F._NormRotary.apply(q, k, qw, kw, pos, inv, (32,), False, 1e-6)
    (h,) = torch.autograd.grad((y ** 3).sum(), q, create_graph=True)
    assert torch.equal(g, h)
    with pytest.raises(RuntimeError, match="no second derivative"):
        torch.autograd.grad(h.square().sum(), q)


def test_func_grad_is_the_ordinary_gradient():
    q, k, pos, inv, qw, kw = setup(2, 4, 2, 9, 64, (5, 11), "f32")
    loss = lambda q, k, qw, kw: sum((x ** 3).sum() for x in F.norm_rotary(q, k, pos, inv, qw, kw, sections=(5, 11)))
    got = torch.func.grad(loss, argnums=(0, 1, 2, 3))(q, k, qw, kw)
    leaves = [x.requires_grad_(True) for x in (q, k, qw, kw)]
    for a, b in zip(got, torch.autograd.grad(loss(*leaves), leaves)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("node", ["native", "python"])
@pytest.mark.parametrize("which", range(6))
def test_in_place_changes_raise(node, which):
    q, k, pos, inv, qw, kw = setup(2, 2, 1, 5, 64, (32,), "f32")
    k.requires_grad_(True)                         # q is saved as well; the leaves that want a gradient are not changed
    x = (q, k * 1.0, qw, kw, pos, inv)
    if node == "native":
        qo, ko = F.norm_rotary(x[0], x[1], x[4], x[5], x[2], x[3])
    else:
        qo, ko = F._NormRotary.apply(*x, (32,), False, 1e-6)
    with torch.no_grad():
        x[which].add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        ko.sum().backward()


def test_tensors_made_in_inference_mode():
    q, k, pos, inv, qw, kw = setup(2, 2, 1, 5, 64, (32,), "f32")
    q.requires_grad_(True)
    want = torch.autograd.grad(F.norm_rotary(q, k, pos, inv, qw, kw)[0].sum(), q)[0]
    with torch.inference_mode():
        k, pos, inv, qw, kw = (x.clone() for x in (k, pos, inv, qw, kw))
    assert torch.equal(torch.autograd.grad(F.norm_rotary(q, k, pos, inv, qw, kw)[0].sum(), q)[0], want)


def test_strides_views_and_one_row_of_positions():
    """Heads out of a fused projection, positions [axes, B, S] and one row of positions for all sequences; gradients the same way."""
    B, S, H, D, sections = 2, 19, 4, 64, (10, 11, 11)
    proj = torch.randn(B, S, 3 * H, D, device="cuda").bfloat16()
    q, k = proj[:, :, :H].transpose(1, 2), proj[:, :, H:2 * H].transpose(1, 2)
    inv, w = torch.rand(32, device="cuda"), torch.rand(D, device="cuda")
    pos = torch.randint(0, 90, (3, B, S), device="cuda", dtype=torch.int32)
    qo, ko = F.norm_rotary(q, k, pos.permute(1, 2, 0), inv, w, None, eps=EPS, sections=sections)
    check_forward(qo, q, w, pos.permute(1, 2, 0), inv, sections, False, "bf16")
    check_forward(ko, k, None, pos.permute(1, 2, 0), inv, sections, False, "bf16")
    q2 = q.detach().requires_grad_(True)
    wide = torch.randn(B, S, 2 * H, D, device="cuda").bfloat16()[:, :, H:].transpose(1, 2)
    (g,) = torch.autograd.grad(F.norm_rotary(q2, None, pos[:, 1:].permute(1, 2, 0), inv, w, eps=EPS, sections=sections)[0], q2, wide)
    check_gradient(g, None, q, w, wide, pos[:, [1, 1]].permute(1, 2, 0), inv, sections, False, "bf16")


def test_rows_of_zeros_and_of_far_sizes():
    """A row of zeros stays zeros (eps > 0) and has the gradient w dz / sqrt(eps); rows of 2^-40 and 2^40 keep their digits."""
    q, _, pos, inv, qw, _ = setup(1, 3, 1, 5, 64, (32,), "f32")
    q[:, 0] = 0
    q[:, 1] *= 2.0 ** -40
    q[:, 2] *= 2.0 ** 40
    q.requires_grad_(True)
    qo, _ = F.norm_rotary(q, None, pos, inv, qw, eps=EPS)
    dy = torch.randn_like(qo)
    (g,) = torch.autograd.grad(qo, q, dy)
    check_forward(qo, q, qw, pos, inv, (32,), False, "f32")
    check_gradient(g, None, q, qw, dy, pos, inv, (32,), False, "f32")
    assert not qo[:, 0].any()


def test_a_row_that_is_not_finite_stays_alone():
    q, k, pos, inv, qw, kw = setup(1, 4, 2, 40, 128, (64,), "bf16")
    want = F.norm_rotary(q, k, pos, inv, qw, kw)
    q2 = q.clone()
    q2[0, 1, 7, 5], q2[0, 2, 8, 3] = float("nan"), float("inf")
    got = F.norm_rotary(q2, k, pos, inv, qw, kw)
    same = torch.ones(4, 40, dtype=torch.bool, device="cuda")
    same[1, 7] = same[2, 8] = False
    assert torch.equal(got[0][0][same], want[0][0][same]) and torch.equal(got[1], want[1]) and bool(got[0][0, 1, 7].isnan().all())


def test_in_place_through_the_abi():
    from paper_2511_02043_amd import binding as fb
    q, k, pos, inv, qw, kw = setup(2, 4, 2, 33, 64, (32,), "bf16")
    q = q.contiguous()
    want, _ = F.norm_rotary(q, k, pos, inv, qw, kw)
    t = fb.tensor_desc(q[:, None])
    fb.check(fb.fl_norm_rotary(t, None, fb.rotary_desc(pos, inv, (32,)), fb.head_norm(eps=1e-6, q_weight=qw), t, None, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(q, want)


def test_empty_tensors():
    for B, S, H, Hkv in ((0, 4, 2, 1), (2, 0, 2, 1), (2, 4, 0, 1), (2, 4, 0, 0)):
        q, k = (torch.zeros(B, h, S, 64, device="cuda", requires_grad=True) for h in (H, Hkv))
        qw, kw = (torch.ones(64, device="cuda", requires_grad=True) for _ in range(2))
        pos, inv = torch.zeros(B, S, 1, device="cuda", dtype=torch.int32), torch.ones(32, device="cuda")
        qo, ko = F.norm_rotary(q, k, pos, inv, qw, kw)
        assert qo.shape == q.shape and ko.shape == k.shape
        (qo.sum() + ko.sum()).backward()
        assert not qw.grad.any() and not kw.grad.any() and q.grad.shape == q.shape


def test_another_stream():
    q, k, pos, inv, qw, kw = setup(2, 8, 2, 500, 128, (64,), "bf16")
    leaves = [x.requires_grad_(True) for x in (q, k, qw, kw)]
    dy = torch.randn_like(q), torch.randn_like(k)
    want = torch.autograd.grad(F.norm_rotary(q, k, pos, inv, qw, kw), leaves, dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = torch.autograd.grad(F.norm_rotary(q, k, pos, inv, qw, kw), leaves, dy)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_training_step_replays_from_a_graph():
    """Forward and backward pass captured together, several replays on new inputs with eager calls between them."""
    q, k, pos, inv, qw, kw = setup(2, 4, 2, 300, 128, (16, 24, 24), "bf16")
    dy = torch.randn_like(q), torch.randn_like(k)

    def step(q, k, qw, kw):
        leaves = [x.detach().requires_grad_(True) for x in (q, k, qw, kw)]
        out = F.norm_rotary(leaves[0], leaves[1], pos, inv, leaves[2], leaves[3], sections=(16, 24, 24))
        return list(out) + list(torch.autograd.grad(out, leaves, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step(q, k, qw, kw)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(q, k, qw, kw)
    for n in range(4):
        with torch.no_grad():
            q.copy_(torch.randn_like(q))
            k.copy_(torch.randn_like(k))
            qw.copy_(torch.rand_like(qw) + 0.5)
        want = step(q, k, qw, kw)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b.detach()) for a, b in zip(want, held)), n
