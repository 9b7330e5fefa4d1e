"""Eviction where its arguments lie in one another's gaps: no memory is shared, so the call is taken."""
import pytest
import torch

from paper_2511_02043_amd import binding as fb
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def test_views_that_take_turns_in_one_buffer():
    """Old and new weights of a (sequence, kv head) beside each other, and tables, lengths and slots in one array of int32."""
    B, Hkv, D, page, n, budget = 3, 2, 64, 16, 90, 40
    torch.manual_seed(0)
    kc, vc = (torch.randn(40, page, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    both = torch.rand(B, Hkv, 96 + 40, device="cuda")
    w = both[:, :, :96]
    tables = torch.randperm(40, device="cuda")[:B * 9].reshape(B, 9).int()
    lens = torch.tensor([n, 50, 7], dtype=torch.int32, device="cuda")
    want = F.evict_cache(w, kc.clone(), vc.clone(), lens, tables[:, :6], tables[:, 6:], budget, sinks=2, recent=20, max_seq_len=n)

    new_lens, kept = torch.empty(2 * B, dtype=torch.int32, device="cuda")[B:], torch.empty(B, Hkv, budget, dtype=torch.int32, device="cuda")
    e = fb.evict_desc(budget=budget, sinks=2, recent=20, dst_table=tables[:, 6:], new_lens=new_lens, kept=kept)
    kv = fb.paged_kv(seq_lens=lens, page_size=page, max_seq_len=n, block_table=tables[:, :6])
    cache = lambda c: fb.tensor_desc(c.transpose(1, 2)[:, None])
    fb.check(fb.fl_cache_evict(fb.weights_desc(w), cache(kc), cache(vc), kv, e, fb.weights_desc(both[:, :, 96:]), torch.cuda.current_stream().cuda_stream))
    assert torch.equal(new_lens, want[0]) and torch.equal(both[:, :, 96:], want[1]) and torch.equal(kept, want[2])
