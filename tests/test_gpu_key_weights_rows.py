"""Weights of cached keys: several rows per sequence against the step without weights, pages that sequences share, many splits, and the slots behind
a sequence.

Tolerances.  A probability within 2e-5 of itself (scores up to some 30 and their log-sum-exps, a few roundings of 2^-24 each), so a row's
log-sum-exp within 2e-5 and its own rounding; a sum of them joins the old weight with one more rounding.
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from oracle import decode_oracle as do
from paper_2511_02043_amd import binding as fb
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def setup(lens, H, Hkv, T, D, page=16, seed=0):
    g = torch.Generator().manual_seed(seed)
    B, per = len(lens), max(1, -(-max(lens) // page))
    kc, vc = (torch.randn(B * per + 2, page, Hkv, D, generator=g).bfloat16().cuda() for _ in range(2))
    table = torch.randperm(B * per + 2, generator=g)[:B * per].reshape(B, per).int().cuda()
    q = torch.randn(B, H, T, D, generator=g).bfloat16().cuda()
    return q, kc, vc, torch.rand(B, Hkv, per * page, generator=g).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), table


def keys_of(kc, table, lens):
    return [kc[row.long()].flatten(0, 1)[:n].double().cpu().numpy() for row, n in zip(table, lens)]


def close(got, ref, old, lens, T):
    base = old.copy()
    for b, n in enumerate(lens):
        base[b, :, max(0, n - T):n] = 0.0
    assert np.all(np.abs(got.double().cpu().numpy() - ref) <= 2e-5 * np.abs(ref - base) + 2.0 ** -22 * np.abs(ref) + 1e-9)


VARIANTS = {"plain": {}, "window": dict(window=20), "softcap": dict(softcap=5.0), "alibi": dict(slopes=True)}


def plain_step(q, kc, vc, sl, table, bound, variant, slopes):
    """fl_attn_decode with the same rows: out and lse."""
    B, H, T, D = q.shape
    out, lse = torch.empty_like(q), torch.empty(B, H, T, device="cuda")
    mask = (fb.FL_MASK_WINDOW | fb.FL_MASK_CAUSAL) if variant == "window" else fb.FL_MASK_CAUSAL
    mod = {"softcap": fb.FL_MOD_SOFTCAP, "alibi": fb.FL_MOD_ALIBI}.get(variant, fb.FL_MOD_NONE)
    d = fb.variant_desc(scale=D ** -0.5, score_mod=mod, softcap=5.0 if variant == "softcap" else 0.0, mask=mask, window=20 if variant == "window" else 0)
    tq, cache = fb.tensor_desc(q[:, None]), [fb.tensor_desc(c.transpose(1, 2)[:, None]) for c in (kc, vc)]
    kv = fb.paged_kv(block_table=table, page_size=kc.shape[1], seq_lens=sl, max_seq_len=bound)
    ws = torch.empty(max(16, fb.fl_attn_decode_workspace_size(tq, cache[0], kv)), dtype=torch.uint8, device="cuda")
    a = fb.fl_aux()
    a.struct_size, a.workspace, a.workspace_bytes = fb.C.sizeof(fb.fl_aux), ws.data_ptr(), ws.numel()
    if slopes is not None:
        a.alibi_slopes = slopes.data_ptr()
    fb.check(fb.fl_attn_decode(tq, *cache, kv, d, a, fb.tensor_desc(out[:, None]), fb.tensor_desc(lse[:, None, :, :, None]), torch.cuda.current_stream().cuda_stream))
    return out, lse


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("lens,H,Hkv,T,D,page", [([40, 3, 1], 8, 2, 4, 64, 8), ([300, 31], 16, 2, 4, 128, 64), ([500], 16, 2, 8, 128, 16), ([90, 200, 0], 16, 1, 3, 64, 16),
                                                 ([2500], 4, 4, 2, 128, 16), ([70] * 20, 16, 2, 4, 64, 16)])
def test_rows_are_those_of_the_step_without_weights(lens, H, Hkv, T, D, page, variant):
    q, kc, vc, w, sl, table = setup(lens, H, Hkv, T, D, page)
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda") if variant == "alibi" else None
    kw = {"window": dict(window=20), "softcap": dict(softcap=5.0), "alibi": dict(alibi_slopes=slopes)}.get(variant, {})
    out, lse = F.decode_attention_weights(q, kc, vc, w, sl, table, max_seq_len=max(lens), return_lse=True, **kw)
    want, want_lse = plain_step(q, kc, vc, sl, table, max(lens), variant, slopes)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    theirs = dict(window=kw.get("window"), softcap_value=kw.get("softcap"), alibi_slopes=None if slopes is None else slopes.cpu().numpy())
    _, ref = do.prefill_attention(q.double().cpu().numpy(), kc.double().cpu().numpy(), vc.double().cpu().numpy(), table.cpu().numpy(), np.array(lens), scale=D ** -0.5,
                                  **{n: x for n, x in theirs.items() if x is not None})
    got, ref = lse.double().cpu().numpy(), np.asarray(ref).reshape(lse.shape)
    empty = np.isneginf(ref)
    assert np.array_equal(np.isneginf(got), empty)
    assert np.all(np.abs(got - ref)[~empty] <= 2e-5 + 2.0 ** -22 * np.abs(ref[~empty]))


@pytest.mark.parametrize("call", ["decode", "chunk"])
def test_sequences_that_share_pages_keep_their_own_weights(call):
    lens, H, Hkv, T, D, page = [200, 170, 96], 8, 2, 4, 128, 16
    q, kc, vc, w, sl, table = setup(lens, H, Hkv, T, D, page)
    table[1, :6] = table[2, :6] = table[0, :6]             # a common prefix of 96 tokens
    old = w.double().cpu().numpy()
    if call == "decode":
        F.decode_attention_weights(q, kc, vc, w, sl, table, max_seq_len=200)
    else:
        lse = F.paged_prefill_attention(q, kc, vc, sl, table, max_seq_len=200, return_lse=True)[1]
        F.prefill_key_weights(q, kc, lse, w, sl, table, max_seq_len=200)
    close(w, co.key_weights(q.double().cpu().numpy(), keys_of(kc, table, lens), old, scale=D ** -0.5), old, lens, T)


@pytest.mark.parametrize("splits", [1, 5, 9, 17, 33, 64, 65, 100, 160])
@pytest.mark.parametrize("T,H,Hkv,window", [(1, 8, 2, None), (4, 16, 1, None), (1, 4, 4, 900)])
def test_any_number_of_splits(splits, T, H, Hkv, window):
    lens, D = [5000, 33, 2100], 64
    q, kc, vc, w, sl, table = setup(lens, H, Hkv, T, D)
    old = w.double().cpu().numpy()
    try:
        fb.check(fb.fl_set_tuning("decode_splits", splits))
        F.decode_attention_weights(q, kc, vc, w, sl, table, max_seq_len=5000, window=window)
    finally:
        fb.fl_set_tuning("decode_splits", 0)
    close(w, co.key_weights(q.double().cpu().numpy(), keys_of(kc, table, lens), old, scale=D ** -0.5, window=window), old, lens, T)


def test_slots_behind_a_sequence_are_left_alone():
    lens, H, Hkv, T, D = [150, 40, 0], 4, 2, 20, 64
    q, kc, vc, w, sl, table = setup(lens, H, Hkv, T, D)
    before = w.clone()
    lse = F.paged_prefill_attention(q, kc, vc, sl, table, return_lse=True)[1]
    F.prefill_key_weights(q, kc, lse, w, sl, table)
    F.decode_attention_weights(q[:, :, 0].contiguous(), kc, vc, w, sl, table)
    for b, n in enumerate(lens):
        assert torch.equal(w[b, :, n:], before[b, :, n:]) and (n == 0 or not torch.equal(w[b, :, :n], before[b, :, :n]))
