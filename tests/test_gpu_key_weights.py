"""Accumulated weights of cached keys on the GPU against the fp64 oracle: decode steps and prompt chunks.

Tolerances.  A probability is exp of a score minus its row's log-sum-exp: both carry a few roundings of 2^-24 of numbers up to some 30
(scores of N(0, 1) rows under 1/sqrt(D), soft-caps and slopes as given here), so below 2e-5 of the probability; all terms are positive, so
the sum keeps that, and joins the old weight with one more rounding.  Outputs of the decode step as in its own tests.
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from oracle import decode_oracle as do
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def setup(lens, H, Hkv, T, D, page=16, seed=0, cap=None, garbage=True):
    g = torch.Generator().manual_seed(seed)
    B, per = len(lens), max(1, -(-max(lens) // page))
    kc, vc = (torch.randn(B * per + 2, page, Hkv, D, generator=g).bfloat16() for _ in range(2))
    table = torch.randperm(B * per + 2, generator=g)[:B * per].reshape(B, per).int()
    if garbage:                                    # what no token of a sequence lies in holds anything
        live = torch.zeros(B * per + 2, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(n):
                live[table[b, j // page], j % page] = True
        for c in (kc, vc):
            c[~live] = float("nan")
    q = torch.randn(B, H, T, D, generator=g).bfloat16()
    w = torch.rand(B, Hkv, cap or per * page, generator=g)
    keys = [torch.stack([kc[table[b, j // page], j % page] for j in range(n)]).double().numpy() if n else np.zeros((0, Hkv, D)) for b, n in enumerate(lens)]
    up = lambda *x: [y.cuda() for y in x]
    return up(q, kc, vc, w, torch.tensor(lens, dtype=torch.int32), table), keys


def variants(H):
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32)
    return {"plain": {}, "window": dict(window=20), "softcap": dict(softcap=5.0), "alibi": dict(alibi_slopes=slopes)}


def split(kw):
    ours = {n: (x.cuda() if torch.is_tensor(x) else x) for n, x in kw.items()}
    theirs = dict(kw)
    if "alibi_slopes" in theirs:
        theirs["slopes"] = theirs.pop("alibi_slopes").numpy()
    return ours, theirs


def close(got, ref, old):
    got = got.double().cpu().numpy()
    bound = 2e-5 * np.abs(ref - old) + 2.0 ** -22 * np.abs(ref) + 1e-9
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], ref[bad][:5])


def base(old, lens, T):
    """The old weights that stay: zero in the newest slots."""
    old = old.copy()
    for b, n in enumerate(lens):
        old[b, :, max(0, n - T):n] = 0.0
    return old


DECODE = [
    ([1], 4, 4, 1, 64, 16), ([5, 0, 32, 33, 257], 8, 2, 1, 128, 16), ([700, 64], 32, 8, 1, 128, 16), ([2000], 32, 8, 1, 64, 32), ([40, 3, 1], 8, 2, 4, 64, 8),
    ([300, 31], 16, 2, 4, 128, 64), ([500], 16, 2, 8, 128, 16), ([90, 200], 16, 1, 3, 64, 16), ([6000], 8, 8, 1, 128, 16), ([63] * 40, 32, 8, 1, 128, 16),
]


@pytest.mark.parametrize("variant", ["plain", "window", "softcap", "alibi"])
@pytest.mark.parametrize("lens,H,Hkv,T,D,page", DECODE)
def test_decode(lens, H, Hkv, T, D, page, variant):
    (q, kc, vc, w, sl, table), keys = setup(lens, H, Hkv, T, D, page)
    ours, theirs = split(variants(H)[variant])
    old = w.double().cpu().numpy()
    out, lse = F.decode_attention_weights(q if T > 1 else q[:, :, 0], kc, vc, w, sl, table, max_seq_len=max(lens), return_lse=True, **ours)
    ref = co.key_weights(q.double().cpu().numpy(), keys, old, scale=D ** -0.5, **theirs)
    close(w, ref, base(old, lens, T))
    # out and lse are those of the call without weights, to the bit
    plain = F.paged_prefill_attention if T > 1 else F.decode_attention
    if T == 1:
        out2, lse2 = plain(q[:, :, 0], kc, vc, sl, table, max_seq_len=max(lens), return_lse=True, **ours)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
    clean_k, clean_v = torch.nan_to_num(kc).double().cpu().numpy(), torch.nan_to_num(vc).double().cpu().numpy()
    kw = dict(theirs, softcap_value=theirs.get("softcap"), alibi_slopes=theirs.get("slopes"))
    kw.pop("softcap", None), kw.pop("slopes", None)
    ref_out, _ = do.prefill_attention(q.double().cpu().numpy(), clean_k, clean_v, table.cpu().numpy(), np.array(lens), scale=D ** -0.5, **kw)
    got = out.double().cpu().numpy().reshape(ref_out.shape)
    assert np.all(np.abs(got - ref_out) <= 1e-2 + 2.0 ** -8 * np.abs(ref_out))


CHUNK = [
    ([1], 2, 2, 1, 64, 16), ([16], 4, 1, 16, 32, 16), ([70, 130, 0, 5], 8, 2, 37, 128, 16), ([300], 4, 4, 300, 64, 8), ([512, 256, 255, 257], 4, 2, 64, 128, 32),
    ([1100, 90], 8, 2, 100, 128, 16), ([600], 16, 2, 129, 64, 64), ([40, 900], 4, 4, 200, 32, 16),
]


@pytest.mark.parametrize("variant", ["plain", "window", "softcap", "alibi"])
@pytest.mark.parametrize("lens,H,Hkv,Sq,D,page", CHUNK)
def test_chunk(lens, H, Hkv, Sq, D, page, variant):
    (q, kc, vc, w, sl, table), keys = setup(lens, H, Hkv, Sq, D, page)
    ours, theirs = split(variants(H)[variant])
    old = w.double().cpu().numpy()
    lse = F.paged_prefill_attention(q, torch.nan_to_num(kc), torch.nan_to_num(vc), sl, table, max_seq_len=max(lens), return_lse=True, **ours)[1]
    assert F.prefill_key_weights(q, kc, lse, w, sl, table, max_seq_len=max(lens), **ours) is w
    ref = co.key_weights(q.double().cpu().numpy(), keys, old, scale=D ** -0.5, **theirs)
    close(w, ref, base(old, lens, Sq))


def test_chunk_by_chunk_is_the_whole_prompt():
    """Weights after a prompt in one piece, in pieces, and token by token through the decode step."""
    n, H, Hkv, D, page = 150, 4, 2, 64, 16
    (q, kc, vc, w, sl, table), keys = setup([n], H, Hkv, n, D, page)
    ref = co.key_weights(q.double().cpu().numpy(), keys, w.double().cpu().numpy(), scale=D ** -0.5)
    tail = w[:, :, n:].clone()
    for step in (150, 64, 7, 1):
        w = torch.full_like(w, float("nan"))       # nothing has to be cleared
        for end in list(range(step, n, step)) + [n]:
            begin = max(0, end - step) if end % step == 0 else end - end % step
            rows, now = q[:, :, begin:end].contiguous(), torch.tensor([end], dtype=torch.int32, device="cuda")
            if end - begin == 1:
                F.decode_attention_weights(rows[:, :, 0], kc, vc, w, now, table)
            else:
                lse = F.paged_prefill_attention(rows, torch.nan_to_num(kc), torch.nan_to_num(vc), now, table, return_lse=True)[1]
                F.prefill_key_weights(rows, kc, lse, w, now, table)
        got = w[:, :, :n].double().cpu().numpy()
        assert np.all(np.abs(got - ref[:, :, :n]) <= 5e-5 * ref[:, :, :n]), step
    assert tail.shape[-1] == table.shape[1] * page - n


def test_values_at_infinity_and_nan():
    """A NaN key makes its rows' probabilities NaN; sequences and heads beside it keep theirs."""
    (q, kc, vc, w, sl, table), _ = setup([40, 40], 4, 2, 1, 64, 16)
    clean = w.clone()
    F.decode_attention_weights(q[:, :, 0], kc, vc, clean, sl, table)
    kc[table[0, 1], 3, 1] = float("nan")
    F.decode_attention_weights(q[:, :, 0], kc, vc, w, sl, table)
    assert torch.isnan(w[0, 1, :40]).all()
    assert torch.equal(w[0, 0], clean[0, 0]) and torch.equal(w[1], clean[1])


def test_strided_inputs_and_spare_capacity():
    lens, H, Hkv, D, page = [77, 140], 8, 2, 128, 16
    (q, kc, vc, w, sl, table), keys = setup(lens, H, Hkv, 1, D, page)
    wide = torch.rand(2, Hkv + 1, 401, device="cuda")
    view = wide[:, 1:, :333]                       # rows that do not start 16-byte aligned
    before = wide.clone()
    old = view.double().cpu().numpy()
    kt, vt = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kc, vc))    # [pages, Hkv, page, D] in memory
    qs = torch.randn(2, 3 * H, D, device="cuda").bfloat16()[:, H:2 * H].copy_(q[:, :, 0])
    F.decode_attention_weights(qs, kt, vt, view, sl, table)
    ref = co.key_weights(q.double().cpu().numpy(), keys, old, scale=D ** -0.5)
    close(view, ref, base(old, lens, 1))
    assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, :, 333:], before[:, :, 333:]) and torch.equal(view[0, :, 77:], before[0, 1:, 77:333])
    lse = torch.empty(2, H, 2, 5, device="cuda")   # a strided lse, a contiguous cache without a table
    n = 90
    qc = torch.randn(2, H, 5, D, device="cuda").bfloat16()
    dense_k, dense_v = (torch.randn(2, 128, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    now = torch.full((2,), n, dtype=torch.int32, device="cuda")
    lse[:, :, 1] = F.paged_prefill_attention(qc, dense_k, dense_v, now, max_seq_len=n, return_lse=True)[1]
    w2 = torch.zeros(2, Hkv, n, device="cuda")
    F.prefill_key_weights(qc, dense_k, lse[:, :, 1], w2, now, max_seq_len=n)
    ref = co.key_weights(qc.double().cpu().numpy(), [dense_k[b, :n].double().cpu().numpy() for b in range(2)], np.zeros((2, Hkv, n)), scale=D ** -0.5)
    close(w2, ref, np.zeros((2, Hkv, n)))


def test_lengths_past_the_bound_are_cut():
    (q, kc, vc, w, sl, table), keys = setup([64], 4, 2, 1, 64, 16)
    old = w.clone()
    F.decode_attention_weights(q[:, :, 0], kc, vc, w, torch.tensor([1000], dtype=torch.int32, device="cuda"), table, max_seq_len=64)
    close(w, co.key_weights(q.double().cpu().numpy(), keys, old.double().cpu().numpy(), scale=0.125), base(old.double().cpu().numpy(), [64], 1))


def test_bitwise_repeatable_and_with_a_workspace():
    (q, kc, vc, w, sl, table), _ = setup([900, 500], 8, 2, 90, 128, 16, garbage=False)
    lse = F.paged_prefill_attention(q, kc, vc, sl, table, return_lse=True)[1]
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda").fill_(255)
    results = [F.prefill_key_weights(q, kc, lse, w.clone(), sl, table, workspace=x) for x in (None, ws, ws)]
    assert torch.equal(results[0], results[1]) and torch.equal(results[0], results[2])
    one = [w.clone() for _ in range(2)]
    outs = [F.decode_attention_weights(q[:, :, 0].contiguous(), kc, vc, x, sl, table, workspace=ws) for x in one]
    assert torch.equal(one[0], one[1]) and torch.equal(outs[0], outs[1])


def test_graph_replays():
    """Captured, a decode step goes on accumulating at every replay."""
    (q, kc, vc, w, sl, table), _ = setup([400, 31], 8, 2, 1, 128, 16, garbage=False)
    q = q[:, :, 0].contiguous()
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    eager = w.clone()
    call = lambda x: F.decode_attention_weights(q, kc, vc, x, sl, table, workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(w.clone())
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    held = w.clone()
    with torch.cuda.graph(graph):
        out = call(held)
    held.copy_(w)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = call(eager)
        assert torch.equal(held, eager) and torch.equal(out, want)
