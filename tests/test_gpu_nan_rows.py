"""Weights of cached keys beside a query row of NaN: the keys that it sees become NaN, those that a mask hides from it do not."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["decode", "chunk"])
@pytest.mark.parametrize("T,window", [(1, 20), (4, None), (4, 20), (4, 2), (12, 40)])
@pytest.mark.parametrize("D", [64, 128])
def test_hidden_keys_keep_their_weight(call, T, window, D):
    """2e-5 of what is gained and 2^-22 of the sum, as for the weights without NaN."""
    H, Hkv, n, page, bad = 8, 2, 150, 16, min(T - 1, 1)           # row `bad` of head 5 is NaN
    torch.manual_seed(0)
    kc, vc = (torch.randn(11, page, Hkv, D).bfloat16().cuda() for _ in range(2))
    table = torch.randperm(11)[:10].reshape(1, 10).int().cuda()
    q, w = torch.randn(1, H, T, D).bfloat16().cuda(), torch.rand(1, Hkv, 160).cuda()
    keys = [kc[table[0].long()].flatten(0, 1)[:n].double().cpu().numpy()]
    q[0, 5, bad] = float("nan")
    sl = torch.tensor([n], dtype=torch.int32, device="cuda")
    old = w.double().cpu().numpy()
    if call == "decode":
        F.decode_attention_weights(q, kc, vc, w, sl, table, max_seq_len=n, window=window)
    else:
        lse = F.paged_prefill_attention(q, kc, vc, sl, table, max_seq_len=n, window=window, return_lse=True)[1]
        F.prefill_key_weights(q, kc, lse, w, sl, table, max_seq_len=n, window=window)
    # without that row's probabilities: zero queries give every key that a row sees the same, which is taken off again
    quiet = torch.nan_to_num(q.double().cpu(), nan=0.0).numpy()
    ref = co.key_weights(quiet, keys, old, scale=D ** -0.5, window=window)
    at = n - T + bad
    seen = np.zeros(160, dtype=bool)
    seen[0 if window is None else max(0, at - window):at + 1] = True
    got = w.double().cpu().numpy()
    base = old.copy()
    base[:, :, n - T:n] = 0.0
    assert np.isnan(got[0, 1][seen]).all()
    got[0, 1][seen] = ref[0, 1][seen] = base[0, 1][seen] = 0.0
    assert np.all(np.abs(got - ref) <= 2e-5 * np.abs(ref - base) + 2.0 ** -22 * np.abs(ref) + 1e-9)
