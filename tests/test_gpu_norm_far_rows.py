"""The gradient of normalised heads at rows far from one, where r^3 = (mean x^2 + eps)^(-3/2) is no fp32 number though r, the row over its size and the result are.

Tolerances: a row's norm in fp32 is within 1.5e-6 (64 squares: 64 / 2 roundings and those of root and quotient), u = x r and the mean of u g within 2e-6 of their
sizes, and dx = r (g - u mean(u g)) is two such terms: 5e-6 of the sum of their sizes, as at ordinary rows; in bf16 the machine's sine and cosine and
the result's own rounding, 2^-13 of that sum and 2^-8 of the result.  A weight's gradient: at most 40 terms, 1.2e-5 (bf16 2^-14 more) of the sum of their sizes.
"""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
D = 64


def f64(x):
    return x.detach().double().cpu().numpy()


def check(power, eps, dtype, sections, interleaved, zero_row=False):
    g = torch.Generator().manual_seed(0)
    make = lambda: torch.randn(1, 2, 9, D, generator=g)
    x = make() * 2.0 ** power
    if zero_row:
        x[0, 1, 3] = 0
    x, dy = x.to(DT[dtype]).cuda().requires_grad_(True), make().to(DT[dtype]).cuda()
    w = torch.exp(0.5 * torch.randn(D, generator=g)).cuda().requires_grad_(True)
    pos = torch.randint(-500, 9000, (1, 9, 1), generator=g).int().cuda()
    inv = (10000.0 ** (-torch.arange(sum(sections), dtype=torch.float64) / sum(sections))).float().cuda()
    y, _ = F.norm_rotary(x, None, pos, inv, w, eps=eps, sections=sections, interleaved=interleaved)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    ref, ref_w, size, size_w = mo.norm_rotary_gradient(f64(x), f64(w), f64(dy), pos.cpu().numpy(), f64(inv), sections, eps=eps, interleaved=interleaved)
    bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -13 * size if dtype == "bf16" else 5e-6 * size
    bad = ~(np.abs(f64(dx) - ref) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:4], f64(dx)[bad][:4], ref[bad][:4])
    bad = ~(np.abs(f64(dw) - ref_w) <= (1.2e-5 + (2.0 ** -14 if dtype == "bf16" else 0)) * size_w)
    assert not bad.any(), (np.argwhere(bad)[:4], f64(dw)[bad][:4], ref_w[bad][:4])


SHAPES = [((32,), False), ((5,), True)]                  # pieces of 16 bytes; single elements


@pytest.mark.parametrize("sections,interleaved", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [46, 50, 58])
def test_large_rows(power, dtype, sections, interleaved):
    check(power, 1e-5, dtype, sections, interleaved)


@pytest.mark.parametrize("sections,interleaved", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [-44, -50, -58])
def test_small_rows_without_eps(power, dtype, sections, interleaved):
    check(power, 0.0, dtype, sections, interleaved)


@pytest.mark.parametrize("sections,interleaved", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [1e-26, 1e-30])
def test_a_row_of_zeros_with_little_eps(eps, dtype, sections, interleaved):
    check(0, eps, dtype, sections, interleaved, zero_row=True)
