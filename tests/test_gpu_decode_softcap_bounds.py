"""The decode step under soft-caps at the ends of fp32: twice the cap in the log2 domain, and scores over the cap, stay finite."""
import numpy as np
import pytest
import torch

from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [1e-40, 1e-37, 1e30, 3e38])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_caps_that_leave_every_score_zero(cap, weights, D):
    """As in the forward kernels such caps level the scores: out is the mean of the values (a bf16 rounding of the probabilities and one of the
    result), each weight one over the length."""
    H, Hkv, n = 4, 2, 100
    torch.manual_seed(0)
    q, kc, vc = torch.randn(1, H, D, device="cuda").bfloat16(), *(torch.randn(7, 16, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    kc[3, 5] = 0                                           # a score of zero
    table, sl = torch.randperm(7, device="cuda").reshape(1, 7).int(), torch.tensor([n], dtype=torch.int32, device="cuda")
    if weights:
        w = torch.zeros(1, Hkv, 112, device="cuda")
        out, lse = F.decode_attention_weights(q, kc, vc, w, sl, table, softcap=cap, return_lse=True)
        assert torch.all((w[0, :, :n] - 2 / n).abs() <= 1e-5) and not w[0, :, n:].any()
    else:
        out, lse = F.decode_attention(q, kc, vc, sl, table, softcap=cap, return_lse=True)
    mean = vc[table[0].long()].flatten(0, 1)[:n].double().mean(0).repeat_interleave(2, 0)
    assert torch.all((out[0].double() - mean).abs() <= 2.0 ** -7 * float(vc.abs().max()) / 10 + 2.0 ** -8 * mean.abs())
    assert torch.all((lse - np.log(n)).abs() <= 1e-5)
