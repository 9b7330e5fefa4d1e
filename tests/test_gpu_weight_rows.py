"""Weights in unusual orders whose rows lie apart: each call leaves in them what it leaves in contiguous ones, and nothing in between."""
import pytest
import torch

from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("strides", [(160, 480), (320, 480), (163, 500), (480, 160)])
def test_orders_of_rows(strides):
    B, H, Hkv, D, page, C = 3, 4, 2, 64, 16, 160
    torch.manual_seed(0)
    kc, vc = (torch.randn(30, page, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    table = torch.randperm(30, device="cuda").reshape(B, 10).int()
    sl = torch.tensor([150, 7, 99], dtype=torch.int32, device="cuda")
    q = torch.randn(B, H, 20, D, device="cuda").bfloat16()
    buffer = torch.rand(2000, device="cuda")
    view = buffer.as_strided((B, Hkv, C), strides + (1,))
    plain, rest = view.clone().contiguous(), buffer.clone()
    lse = F.paged_prefill_attention(q, kc, vc, sl, table, return_lse=True)[1]
    for w in (plain, view):
        F.prefill_key_weights(q, kc, lse, w, sl, table)
        F.decode_attention_weights(q[:, :, 0].contiguous(), kc, vc, w, sl, table)
    assert torch.equal(view, plain)
    rest.as_strided((B, Hkv, C), strides + (1,)).copy_(plain)
    assert torch.equal(buffer, rest)
