"""evict_cache() where the table of a sequence names no page: its tokens have no keys and values, zeros take their places."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def test_sources_that_name_no_page():
    B, Hkv, D, page, n, budget = 2, 2, 64, 16, 90, 40
    torch.manual_seed(0)
    kc, vc = (torch.randn(20, page, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    table = torch.arange(12, dtype=torch.int32, device="cuda").reshape(B, 6)
    table[0, 1], table[1, 4] = -1, 20
    dst = torch.arange(12, 18, dtype=torch.int32, device="cuda").reshape(B, 3)
    w = torch.rand(B, Hkv, 96, device="cuda")
    want_k, want_v = kc.clone(), vc.clone()
    _, want = co.evict(w.cpu().numpy(), [n] * B, budget, 2, 20)
    for b in range(B):
        for h in range(Hkv):
            for r, j in enumerate(want[b, h]):
                src, to = int(table[b, j // page]), int(dst[b, r // page])
                for c, old in ((want_k, kc), (want_v, vc)):
                    c[to, r % page, h] = old[src, j % page, h] if 0 <= src < 20 else 0
    new_lens, _, kept = F.evict_cache(w, kc, vc, torch.full((B,), n, dtype=torch.int32, device="cuda"), table, dst, budget, sinks=2, recent=20, max_seq_len=n)
    assert np.array_equal(kept.cpu().numpy(), want) and new_lens.tolist() == [budget] * B
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)
