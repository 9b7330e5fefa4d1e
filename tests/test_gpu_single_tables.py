"""Block tables of one sequence: the stride of an axis of size one says nothing, whatever view it comes from."""
import pytest
import torch

from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def test_a_table_out_of_a_column():
    H, Hkv, D, n = 4, 2, 64, 150
    torch.manual_seed(0)
    kc, vc = (torch.randn(20, 16, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    q, w, sl = torch.randn(1, H, 3, D, device="cuda").bfloat16(), torch.rand(1, Hkv, 160, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    rows = torch.randperm(20, device="cuda").int().reshape(1, 20).clone()
    column = rows.reshape(20, 1).t()                       # [1, 20] with the strides (1, 1)
    assert column.stride() == (1, 1)
    pos, inv = torch.arange(3, dtype=torch.int32, device="cuda").reshape(1, 3, 1), torch.rand(32, device="cuda")
    results = []
    for t in (rows, column):
        k, v, x = kc.clone(), vc.clone(), w.clone()
        table, dst = t[:, :10], t[:, 10:]
        got = [F.rotary_append(q, q[:, :Hkv], q[:, :Hkv], pos, inv, k, v, sl, table), F.decode_attention(q[:, :, 0], k, v, sl, table)]
        out, lse = F.paged_prefill_attention(q, k, v, sl, table, return_lse=True)
        got += [out, F.decode_attention_weights(q, k, v, x, sl, table), F.prefill_key_weights(q, k, lse, x, sl, table)]
        got += [*F.evict_cache(x, k, v, sl, table, dst, 70, sinks=2, recent=9), k, v]
        results.append(got)
    assert all(torch.equal(a, b) for a, b in zip(*results))
