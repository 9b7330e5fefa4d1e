"""Weights that a chunk gives under soft-caps of any size, from log-sum-exps that the fp64 oracle has formed.

Tolerance of a probability, in units of 2^-24: a score's sum of up to 128 products (statistically eight roundings of its size) and its cap (four),
both relative to the largest score; the log-sum-exp's own rounding and the subtraction (two of its size); the exponential and the sum (16).  It does not
grow with the cap.
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [1e-38, 0.5, 5.0, 30.0, 50.0, 300.0, 1000.0, 3e4, 1e30, 3e38])
@pytest.mark.parametrize("D,size", [(32, 1.0), (64, 1.0), (128, 1.0), (128, 12.0)])
def test_soft_cap(cap, D, size):
    H, T, n, page = 2, 3, 200, 16
    torch.manual_seed(0)
    q = (size * torch.randn(1, H, T, D)).bfloat16()
    kc = torch.randn(14, page, H, D).bfloat16()
    table = torch.randperm(14)[:13].reshape(1, 13).int()
    keys = kc[table[0].long()].flatten(0, 1)[:n].double().numpy()
    lse, largest = np.zeros((1, H, T)), 0.0
    for h in range(H):
        s = D ** -0.5 * (q[0, h].double().numpy() @ keys[:, h].T)
        s = cap * np.tanh(s / cap)
        for t in range(T):
            row = s[t, :n - T + t + 1]
            lse[0, h, t] = row.max() + np.log(np.exp(row - row.max()).sum())
            largest = max(largest, float(np.abs(row).max()))
    w = torch.zeros(1, H, 208, device="cuda")
    F.prefill_key_weights(q.cuda(), kc.cuda(), torch.from_numpy(lse).float().cuda(), w, torch.tensor([n], dtype=torch.int32, device="cuda"), table.cuda(), max_seq_len=n, softcap=cap)
    ref = co.key_weights(q.double().numpy(), [keys], np.zeros((1, H, 208)), scale=D ** -0.5, softcap=cap)
    got = w.double().cpu().numpy()
    bound = 2.0 ** -24 * (12 * largest + 2 * float(np.abs(lse).max()) + 16)
    worst = float(np.max(np.abs(got - ref)[ref > 0] / ref[ref > 0]))
    print(f"cap={cap} D={D} size={size}: largest score {largest:.3g}, worst {worst:.2e} of {bound:.2e}", flush=True)
    assert np.all(np.abs(got - ref) <= bound * ref + 1e-12)
