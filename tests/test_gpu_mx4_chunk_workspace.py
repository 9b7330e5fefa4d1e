"""What a chunk over the 4-bit cache needs of a workspace, and that nothing of what it held before is read."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2511_02043_amd import binding as fb
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def pool(B, Hkv, D, page, per):
    r = np.random.default_rng(0)
    n = B * per
    k, v = (torch.from_numpy(mo.pages_of(r.integers(0, 16, (n, Hkv, page, D)).astype(np.uint8), r.integers(118, 130, (n, Hkv, page, D // 32)).astype(np.uint8))).cuda()
            for _ in range(2))
    return k, v, torch.from_numpy(r.permutation(n).reshape(B, per).astype(np.int32)).cuda()


def test_a_short_chunk_under_a_large_bound_takes_little_memory():
    """64 sequences, 17 rows of four heads a kv head (more than a decode step takes), tables for 131072 tokens each, as they are without max_seq_len:
    dense copies of that would be 34 GB, and the rows go through the decode kernels, which need none."""
    B, H, Hkv, D, page, rows = 64, 32, 8, 128, 16, 17
    kc, vc, few = pool(B, Hkv, D, page, 4)
    table = torch.zeros(B, 131072 // page, dtype=torch.int32, device="cuda")
    table[:, :4] = few
    lens = ints([17 + n % 48 for n in range(B)])
    q = torch.randn(B, H, rows, D, device="cuda").bfloat16()
    want = F.paged_prefill_attention_mx4(q, kc, vc, lens, few)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    got = F.paged_prefill_attention_mx4(q, kc, vc, lens, table)
    assert torch.cuda.max_memory_allocated() - before < 100 << 20
    assert torch.equal(got, want)
    assert torch.equal(F.paged_prefill_attention_mx4(q, kc, vc, lens, table, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), want)


@pytest.mark.parametrize("window", [None, 100])
@pytest.mark.parametrize("B,H,Hkv,rows,D,n", [(1, 32, 8, 64, 128, 8000), (2, 8, 2, 20, 64, 5000), (2, 4, 2, 700, 64, 700), (1, 4, 4, 600, 128, 900), (1, 8, 2, 5, 64, 3000)])
def test_the_least_workspace_is_enough(B, H, Hkv, rows, D, n, window):
    """As many bytes as the size for this call says, with guards behind them that stay; one fewer is refused."""
    kc, vc, table = pool(B, Hkv, D, 16, -(-n // 16))
    q = torch.randn(B, H, rows, D, device="cuda").bfloat16()
    lens, how = ints([n - 3 * b for b in range(B)]), dict(max_seq_len=n, window=window, return_lse=True)
    need = fb.fl_attn_prefill_mx4_workspace_size_for(fb.tensor_desc(q[:, None]), fb.mx4_desc(kc, 16, D), fb.paged_kv(block_table=table, seq_lens=lens, page_size=16, max_seq_len=n),
                                                     fb.variant_desc(scale=D ** -0.5, mask=fb.FL_MASK_CAUSAL if window is None else fb.FL_MASK_WINDOW, window=window or 0))
    need = max(need, 16)
    want = F.paged_prefill_attention_mx4(q, kc, vc, lens, table, **how)
    held = torch.full((need + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    got = F.paged_prefill_attention_mx4(q, kc, vc, lens, table, workspace=held[:need], **how)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool((held[need:] == 0x5A).all())
    with pytest.raises(ValueError, match=f"{need} needed"):
        F.paged_prefill_attention_mx4(q, kc, vc, lens, table, workspace=held[:need - 1], **how)


@pytest.mark.parametrize("way", ["as sent", "unpacked"])
@pytest.mark.parametrize("window", [None, 0, 1, 127, 128, 300])
@pytest.mark.parametrize("D", [64, 128])
def test_a_workspace_of_nan(D, window, way):
    """Lengths on and next to the borders of unpacked blocks and of the forward kernel's tiles, one sequence shorter than the chunk, one empty."""
    lens, page, H, Hkv, rows = [640, 639, 513, 512, 511, 385, 100, 0], 16, 4, 2, 129
    kc, vc, table = pool(len(lens), Hkv, D, page, 40)
    q = torch.randn(len(lens), H, rows, D, device="cuda").bfloat16()
    fb.check(fb.fl_set_tuning("prefill_gather", 0 if way == "as sent" else 1))
    try:
        room = fb.fl_attn_prefill_mx4_workspace_size(fb.tensor_desc(q[:, None]), fb.mx4_desc(kc, page, D), fb.paged_kv(block_table=table, seq_lens=ints(lens), page_size=page, max_seq_len=640))
        assert room > 0
        results = []
        for fill in (0x00, 0xFF):                          # (bf16 and fp32 numbers of ones alone are NaN)
            ws = torch.full((room,), fill, dtype=torch.uint8, device="cuda")
            results.append(F.paged_prefill_attention_mx4(q, kc, vc, ints(lens), table, window=window, workspace=ws, return_lse=True))
        (a, a_lse), (b, b_lse) = results
        assert torch.equal(a, b) and torch.equal(a_lse, b_lse) and not b.isnan().any() and not b_lse.isnan().any()
        assert not b[7].any() and not b[6, :, :29].any() and bool(b[6, :, 29:].any(-1).all())
    finally:
        fb.check(fb.fl_set_tuning("prefill_gather", 0))
