"""Soft-caps so far below the scale that 2 scale / cap is no fp32 number, with raw scores of zero: the calls that attend to dense keys, to bf16 pages and to 4-bit pages.

Every score is 0 or at the cap, at most 1e-10 here, so that a row's result is the mean of the values that it sees.  Error: P rounded to bf16 (at most 2^-8 of it, and n of 1 / n
each add up to 2^-8 of the mean magnitude) and the result's rounding, 2^-8; the log-sum-exp is log n within 1e-5."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu
H, HKV, N, PAGE = 4, 2, 100, 16


def setup(D):
    r = np.random.default_rng(0)
    codes, e = r.integers(0, 16, (2, 7, HKV, PAGE, D)).astype(np.uint8), r.integers(124, 128, (2, 7, HKV, PAGE, D // 32)).astype(np.uint8)
    codes[0, :, :, 5] = 0                          # every sixteenth key is zero, and so is its score
    cache4 = [torch.from_numpy(mo.pages_of(codes[i], e[i])).cuda() for i in range(2)]
    rows = [torch.from_numpy(mo.values(codes[i], e[i])).bfloat16().cuda() for i in range(2)]        # [pages, Hkv, page, D]: bf16 numbers
    table = torch.from_numpy(r.permutation(7).astype(np.int32))[None].cuda()
    k, v = (x[table[0].long()].transpose(0, 1).flatten(1, 2)[None, :, :N].contiguous() for x in rows)
    return k, v, [x.transpose(1, 2).contiguous() for x in rows], cache4, table, torch.tensor([N], dtype=torch.int32, device="cuda")


def check(out, lse, v, rows):
    """The last `rows` tokens' results, out [1, H, rows, D]."""
    v = v[0].double().repeat_interleave(H // HKV, 0)
    n = torch.arange(1, N + 1, device="cuda").double()[:, None]
    mean, size = (v.cumsum(1) / n)[:, N - rows:], (v.abs().cumsum(1) / n)[:, N - rows:]
    assert bool(((out[0].double() - mean).abs() <= 2.0 ** -8 * (1.01 * size + mean.abs())).all())
    if lse is not None:
        assert bool(((lse[0].double() - n[N - rows:, 0].log()).abs() <= 1e-5).all())


@pytest.mark.parametrize("scale,cap", [(1e3, 1e-40), (1e20, 1e-37), (1e30, 1e-10), (3e38, 1e-20)])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_zero_stay_zero(D, scale, cap):
    k, v, (k16, v16), (k4, v4), table, lens = setup(D)
    how, rows = dict(scale=scale, softcap=cap), 40
    q = torch.randn(1, H, N, D, device="cuda").bfloat16()
    check(F.attention(q, k, v, causal=True, **how), None, v, N)
    last, chunk = q[:, :, -1].contiguous(), q[:, :, -rows:].contiguous()
    paged = dict(how, return_lse=True)
    for call, caches in ((F.decode_attention, (k16, v16)), (F.decode_attention_mx4, (k4, v4))):
        out, lse = call(last, *caches, lens, table, **paged)
        check(out[:, :, None], lse[:, :, None], v, 1)
    for call, caches in ((F.paged_prefill_attention, (k16, v16)), (F.paged_prefill_attention_mx4, (k4, v4))):
        for x in (chunk, q):
            out, lse = call(x, *caches, lens, table, **paged)
            check(out, lse, v, x.shape[2])
    weights = torch.zeros(1, HKV, 112, device="cuda")
    F.decode_attention_weights(last, k16, v16, weights, lens, table, **how)
    assert bool(((weights[0, :, :N] - 2 / N).abs() <= 1e-5).all())
    out, lse = F.paged_prefill_attention(last[:, :, None], k16, v16, lens, table, **paged)
    F.prefill_key_weights(last[:, :, None], k16, lse, weights.zero_(), lens, table, **how)
    assert bool(((weights[0, :, :N] - 2 / N).abs() <= 1e-5).all())
