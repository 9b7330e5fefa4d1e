"""The cache's calls where a page starts more than 2^31 elements into it: what they do there is what they do on the same pages near the start."""
import pytest
import torch

from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def test_far_pages():
    page, Hkv, H, D, n = 16, 8, 16, 128, 200
    per, pages = -(-n // page), (1 << 31) // (16 * 8 * 128) + 64
    far_k, far_v = (torch.zeros(pages, page, Hkv, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    near_k, near_v = (torch.zeros(64, page, Hkv, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.randperm(64)[:2 * per].reshape(1, -1).int().cuda()
    src, dst, shift = table[:, :per], table[:, per:], pages - 64
    pos, inv = torch.arange(n, device="cuda", dtype=torch.int32).reshape(1, n, 1), torch.rand(D // 2, device="cuda")
    q, k, v = (torch.randn(1, h, n, D, device="cuda").bfloat16() for h in (H, Hkv, Hkv))
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    results = []
    for kc, vc, by in ((near_k, near_v, 0), (far_k, far_v, shift)):
        s, d = (src + by).contiguous(), (dst + by).contiguous()
        turned = F.rotary_append(q, k, v, pos, inv, kc, vc, lens, s)
        out, lse = F.paged_prefill_attention(turned, kc, vc, lens, s, max_seq_len=n, return_lse=True)
        w = torch.zeros(1, Hkv, n, device="cuda")
        F.prefill_key_weights(turned, kc, lse, w, lens, s, max_seq_len=n)
        one = F.decode_attention_weights(turned[:, :, -1].contiguous(), kc, vc, w, lens, s, max_seq_len=n)
        new_lens, new_w, kept = F.evict_cache(w, kc, vc, lens, s, d, 100, sinks=2, recent=20, max_seq_len=n)
        after = F.decode_attention_weights(turned[:, :, -1].contiguous(), kc, vc, new_w, new_lens, d, max_seq_len=100)
        results.append((turned, out, lse, w, one, new_lens, new_w, kept, after))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert torch.equal(far_k[shift:], near_k) and torch.equal(far_v[shift:], near_v)
    assert not far_k[:64].any()
