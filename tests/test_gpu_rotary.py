"""Rotary positions on the GPU against the fp64 oracle: forward and backward pass, and the write of new tokens into a paged cache.

Tolerances.  A pair turns with a relative error of its length: bf16 the rounding of the result, at most 2^-8 of it (eight significant bits), and 2^-14 of the length for sine,
cosine and the products; fp32 an angle within 2 pi 2^-25, sine and cosine within 2 units in the last place and three roundings: below 1e-6.
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def setup(B, H, Hkv, S, D, sections, dtype, seed=0, layout="bshd", far=0):
    g = torch.Generator().manual_seed(seed)
    def make(h):
        x = torch.randn(B, S, h, D, generator=g).to(DT[dtype]).cuda()
        return x.transpose(1, 2) if layout == "bshd" else x.transpose(1, 2).contiguous()
    n = sum(sections)
    inv = (10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)).float().cuda()
    pos = (torch.randint(0, 500, (B, S, len(sections)), generator=g) + far).int().cuda()
    return make(H), make(Hkv), pos, inv


def f64(x):
    return x.detach().double().cpu().numpy()


def close(got, ref, x, sections, interleaved, dtype):
    """Element by element, relative to the length of the element's pair."""
    n = sum(sections)
    length = np.zeros(x.shape)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        length[..., a] = length[..., b] = np.hypot(x[..., a], x[..., b])
    bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -14 * length if dtype == "bf16" else 1e-6 * length
    bad = np.abs(got - ref) > bound
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - ref)[bad][:4], bound[bad][:4])
    assert np.array_equal(got[..., 2 * n:], x[..., 2 * n:])


CASES = [
    (2, 4, 2, 37, 128, (16, 24, 24), False), (1, 3, 1, 1, 64, (8, 12, 12), True), (3, 2, 2, 5, 80, (40,), False), (1, 8, 8, 64, 32, (8, 8), True),
    (2, 2, 1, 9, 64, (10,), False), (1, 2, 1, 9, 40, (3, 4), True), (1, 1, 1, 3, 256, (32, 32, 32, 32), False), (2, 16, 2, 130, 128, (32,), False),
    (1, 2, 2, 7, 640, (150, 150), False), (1, 40, 8, 700, 64, (0, 32), True), (1, 1, 1, 2, 1032, (5,), False),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,S,D,sections,interleaved", CASES)
def test_forward_and_gradient(B, H, Hkv, S, D, sections, interleaved, dtype):
    q, k, pos, inv = setup(B, H, Hkv, S, D, sections, dtype)
    q.requires_grad_(True)
    k.requires_grad_(True)
    qo, ko = F.rotary(q, k, pos, inv, sections=sections, interleaved=interleaved)
    assert qo.shape == q.shape and ko.shape == k.shape and qo.dtype == q.dtype
    dq, dk = torch.randn_like(qo), torch.randn_like(ko)
    gq, gk = torch.autograd.grad((qo, ko), (q, k), (dq, dk))
    for got, x, inverse in ((qo, q, False), (ko, k, False), (gq, dq, True), (gk, dk, True)):
        ref = co.rotary(f64(x), pos.cpu().numpy(), inv.cpu().numpy(), sections, interleaved=interleaved, inverse=inverse)
        close(f64(got), ref, f64(x), sections, interleaved, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions_keep_their_phase(dtype):
    for far in (1 << 20, 1 << 28, -(1 << 28)):
        q, k, pos, inv = setup(1, 2, 1, 50, 64, (16, 16), dtype, far=far)
        qo, _ = F.rotary(q, k, pos, inv, sections=(16, 16))
        close(f64(qo), co.rotary(f64(q), pos.cpu().numpy(), inv.cpu().numpy(), (16, 16)), f64(q), (16, 16), False, dtype)


def test_gradient_against_differences():
    """<dy, f(x + h u) - f(x - h u)> / 2 h for fp32: the map is linear, so the quotient is exact but for roundings of 1e-6 / h."""
    q, k, pos, inv = setup(1, 2, 1, 6, 32, (4, 4), "f32")
    q.requires_grad_(True)
    qo, _ = F.rotary(q, k, pos, inv, sections=(4, 4))
    dy, u = torch.randn_like(qo), torch.randn_like(q)
    (g,) = torch.autograd.grad(qo, q, dy)
    with torch.no_grad():
        f = lambda x: F.rotary(x, None, pos, inv, sections=(4, 4))[0].double()
        quotient = ((f(q + u) - f(q - u)) * dy.double()).sum() / 2
    assert abs(float(quotient - (g.double() * u.double()).sum())) <= 1e-4


@pytest.mark.parametrize("which", ["q", "k", "q alone", "both", "broadcast"])
def test_gradients_that_are_wanted_or_arrive(which):
    q, k, pos, inv = setup(2, 4, 2, 11, 64, (32,), "f32")
    q.requires_grad_(which != "k")
    k.requires_grad_(which in ("k", "both", "broadcast"))
    qo, ko = F.rotary(q, None if which == "q alone" else k, pos, inv)
    if which == "q alone":
        assert ko is None
    if which == "broadcast":                       # a gradient of one number, expanded
        (qo.sum() + 2 * ko.sum()).backward()
        ones = np.ones(q.shape)
        assert np.allclose(f64(q.grad), co.rotary(ones, pos.cpu().numpy(), inv.cpu().numpy(), (32,), inverse=True), atol=1e-6)
        assert np.allclose(f64(k.grad), 2 * co.rotary(np.ones(k.shape), pos.cpu().numpy(), inv.cpu().numpy(), (32,), inverse=True), atol=2e-6)
        return
    x, y = (k, ko) if which == "k" else (q, qo)
    y.square().sum().backward()                    # a turn keeps lengths: the gradient of |y|^2 is 2 x
    assert torch.allclose(x.grad, 2 * x.detach(), atol=1e-5)
    other = q if which == "k" else k
    assert other.grad is None


def test_second_derivative():
    q, k, pos, inv = setup(1, 2, 2, 5, 32, (16,), "f32")
    q.requires_grad_(True)
    y, _ = F.rotary(q, k, pos, inv)
    (g,) = torch.autograd.grad((y ** 3).sum(), q, create_graph=True)
    (h,) = torch.autograd.grad((g * g).sum() / 2, q)
    # g = R' 3 y^2, h = R' diag(6 y) R g
    yd = co.rotary(f64(q), pos.cpu().numpy(), inv.cpu().numpy(), (16,))
    R = lambda x, inverse: co.rotary(x, pos.cpu().numpy(), inv.cpu().numpy(), (16,), inverse=inverse)
    want = R(6 * yd * R(R(3 * yd ** 2, True), False), True)
    assert np.allclose(f64(h), want, rtol=1e-4, atol=1e-4 * np.abs(want).max())


def test_func_transform_takes_the_python_node():
    q, k, pos, inv = setup(1, 2, 1, 4, 32, (16,), "f32")
    from paper_2511_02043_amd.functional import _Rotary
    x = q.clone().requires_grad_(True)
    out = _Rotary.apply(x, k, pos, inv, (16,), False, False)
    (g,) = torch.autograd.grad(out[0], x, torch.ones_like(out[0]), retain_graph=True)
    x2 = q.clone().requires_grad_(True)
    (g2,) = torch.autograd.grad(F.rotary(x2, k, pos, inv)[0], x2, torch.ones_like(out[0]))
    assert torch.equal(g, g2)


def test_strides_and_positions_views():
    """Heads out of a fused projection, positions [axes, B, S] and one row of positions for all sequences."""
    B, S, H, D = 2, 19, 4, 64
    proj = torch.randn(B, S, 3 * H, D, device="cuda").bfloat16()
    q, k = proj[:, :, :H].transpose(1, 2), proj[:, :, H:2 * H].transpose(1, 2)
    inv = torch.rand(32, device="cuda")
    pos = torch.randint(0, 90, (3, B, S), device="cuda", dtype=torch.int32)
    qo, ko = F.rotary(q, k, pos.permute(1, 2, 0), inv, sections=(10, 11, 11))
    for got, x in ((qo, q), (ko, k)):
        ref = co.rotary(f64(x), pos.permute(1, 2, 0).cpu().numpy(), inv.cpu().numpy(), (10, 11, 11))
        close(f64(got), ref, f64(x), (10, 11, 11), False, "bf16")
    one, _ = F.rotary(q, k, pos[:, 1:].permute(1, 2, 0), inv, sections=(10, 11, 11))
    both, _ = F.rotary(q, k, pos[:, [1, 1]].permute(1, 2, 0), inv, sections=(10, 11, 11))
    assert torch.equal(one, both)


def test_in_place_through_the_abi():
    from paper_2511_02043_amd import binding as fb
    q, k, pos, inv = setup(2, 4, 2, 33, 64, (32,), "bf16", layout="bhsd")
    want, _ = F.rotary(q, k, pos, inv)
    t = fb.tensor_desc(q[:, None])
    fb.check(fb.fl_rotary_embed(t, None, fb.rotary_desc(pos, inv, (32,)), t, None, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(q, want)


def test_empty_tensors():
    for B, S, H in ((0, 4, 2), (2, 0, 2), (2, 4, 0)):
        q, k = torch.zeros(B, H, S, 64, device="cuda"), torch.zeros(B, 1, S, 64, device="cuda")
        pos, inv = torch.zeros(B, S, 1, device="cuda", dtype=torch.int32), torch.ones(32, device="cuda")
        qo, ko = F.rotary(q, k, pos, inv)
        assert qo.shape == q.shape and ko.shape == k.shape


# ---- the serving form ----

def pool(B, Hkv, D, page, per, seed=0):
    g = torch.Generator().manual_seed(seed)
    kc, vc = (torch.randn(B * per + 3, page, Hkv, D, generator=g).bfloat16().cuda() for _ in range(2))
    table = torch.randperm(B * per + 3, generator=g)[:B * per].reshape(B, per).int().cuda()
    return kc, vc, table


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,lens,page,D,sections", [(1, [1, 17, 64], 16, 128, (16, 24, 24)), (5, [5, 3, 0, 40], 8, 64, (32,)), (70, [70, 129, 12], 64, 64, (10, 6)),
                                                    (3, [9, 30], 32, 80, (20, 20)), (1, [2], 16, 40, (3,))])
def test_append(T, lens, page, D, sections, interleaved):
    B, H, Hkv = len(lens), 4, 2
    q, k, pos, inv = setup(B, H, Hkv, T, D, sections, "bf16")
    v = torch.randn_like(k)
    per = -(-max(lens) // page)
    kc, vc, table = pool(B, Hkv, D, page, per)
    want_k, want_v = kc.clone(), vc.clone()
    turned_q, turned_k = F.rotary(q, k, pos, inv, sections=sections, interleaved=interleaved)
    for b, n in enumerate(lens):
        for t in range(T):
            slot = n - T + t
            if slot >= 0:
                want_k[table[b, slot // page], slot % page] = turned_k[b, :, t]
                want_v[table[b, slot // page], slot % page] = v[b, :, t]
    args = (pos, inv, kc, vc, torch.tensor(lens, dtype=torch.int32, device="cuda"), table)
    if T == 1:                                     # without the axis of tokens
        got = F.rotary_append(q[:, :, 0], k[:, :, 0], v[:, :, 0], *args, sections=sections, interleaved=interleaved)
        assert torch.equal(got, turned_q[:, :, 0])
    else:
        assert torch.equal(F.rotary_append(q, k, v, *args, sections=sections, interleaved=interleaved), turned_q)
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


def test_append_without_a_table_and_with_other_strides():
    B, Hkv, D, S = 2, 2, 64, 24
    q, k, pos, inv = setup(B, 4, Hkv, 3, D, (32,), "bf16")
    v = torch.randn_like(k)
    kc = torch.zeros(B, Hkv, S, D, device="cuda").bfloat16().transpose(1, 2)       # [B, S, Hkv, D] over [B, Hkv, S, D]
    vc = torch.zeros(B, S, Hkv, D, device="cuda").bfloat16()
    lens = torch.tensor([24, 11], dtype=torch.int32, device="cuda")
    F.rotary_append(q, k, v, pos, inv, kc, vc, lens)
    _, turned = F.rotary(q, k, pos, inv)
    for b, n in enumerate((24, 11)):
        assert torch.equal(kc[b, n - 3:n].transpose(0, 1), turned[b]) and torch.equal(vc[b, n - 3:n].transpose(0, 1), v[b])
        assert not kc[b, :n - 3].any() and not kc[b, n:].any()


def test_append_passes_over_entries_that_name_no_page():
    q, k, pos, inv = setup(3, 2, 1, 1, 64, (32,), "bf16")
    kc, vc, table = pool(3, 1, 64, 16, 1)
    table[0, 0], table[1, 0] = -1, kc.shape[0]
    before_k, before_v = kc.clone(), vc.clone()
    F.rotary_append(q, k, k, pos, inv, kc, vc, torch.full((3,), 4, dtype=torch.int32, device="cuda"), table)
    changed = (kc != before_k).flatten(1).any(1).nonzero().flatten().tolist()
    assert changed == [int(table[2, 0])] and (vc != before_v).flatten(1).any(1).sum() == 1


def test_another_stream():
    q, k, pos, inv = setup(2, 4, 2, 300, 128, (64,), "bf16")
    want, _ = F.rotary(q, k, pos, inv)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got, _ = F.rotary(q, k, pos, inv)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
