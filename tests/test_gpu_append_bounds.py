"""rotary_append() where a sequence is longer than the bound that the host gave: the new tokens keep their slots, those past the bound are passed over."""
import pytest
import torch

from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("table", [True, False])
@pytest.mark.parametrize("bound", [16, 18, 19, 20, 32])
def test_slots_come_from_the_true_length(bound, table):
    Hkv, D, T, n, page = 2, 64, 3, 20, 16 if table else 32
    torch.manual_seed(0)
    q, k, v = (torch.randn(1, h, T, D, device="cuda").bfloat16() for h in (4, Hkv, Hkv))
    kc, vc = (torch.randn(5, page, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    pos, inv = torch.arange(n - T, n, dtype=torch.int32, device="cuda").reshape(1, T, 1), torch.rand(32, device="cuda")
    pages = torch.tensor([[3, 1]], dtype=torch.int32, device="cuda") if table else None
    turned_q, turned_k = F.rotary(q, k, pos, inv)
    want_k, want_v = kc.clone(), vc.clone()
    for t in range(T):
        slot = n - T + t
        if slot < bound:
            to = (int(pages[0, slot // page]), slot % page) if table else (0, slot)
            want_k[to], want_v[to] = turned_k[0, :, t], v[0, :, t]
    got = F.rotary_append(q, k, v, pos, inv, kc, vc, torch.tensor([n], dtype=torch.int32, device="cuda"), pages, max_seq_len=bound)
    assert torch.equal(got, turned_q) and torch.equal(kc, want_k) and torch.equal(vc, want_v)
