"""The 4-bit cache on the GPU against the fp64 oracles: what enters it, and attention over it.

Tolerances.  A key's code is the exact key's: equal bytes but where the exact value lies within 1e-9 of a border (fp64 arithmetic is off by some 1e-13; the
oracle says where).  Values are codes of what they were: equal bytes.  Attention: the scores are fp32 sums of D <= 128 exact products, off by at most 64 * 2^-24
of the sum of their sizes, which stays below 2^6 here: 2.5e-4 in a probability and in the log-sum-exp, with the machine's exponential and logarithm
2^-11; P enters the second contraction as bf16 (2^-8 of it), the result is rounded to bf16 (2^-8): |error| <= (2^-8 + 2^-10) sum_j P_j |v_j| + 2^-8 |result|.
"""
import threading

import numpy as np
import pytest
import torch

from oracle import decode_oracle as do
from oracle import mx4_oracle as mo
from paper_2511_02043_amd import binding as fb
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu
EPS = 1e-6


def f64(x):
    return x.detach().double().cpu().numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def pool(B, Hkv, D, page, per, seed=0, scales=(118, 130)):
    """Caches of arbitrary rows, more pages than are used, and a table."""
    r = np.random.default_rng(seed)
    n = B * per + 3
    caches = []
    for _ in range(2):
        codes, e = r.integers(0, 16, (n, Hkv, page, D)).astype(np.uint8), r.integers(*scales, (n, Hkv, page, D // 32)).astype(np.uint8)
        caches.append(torch.from_numpy(mo.pages_of(codes, e)).cuda())
    return caches[0], caches[1], torch.from_numpy(r.permutation(n)[:B * per].reshape(B, per).astype(np.int32)).cuda()


# ---- what enters ----

def append_inputs(B, H, Hkv, T, D, sections, seed=0):
    g = torch.Generator().manual_seed(seed)
    proj = torch.randn(B, T, H + 2 * Hkv, D, generator=g) * torch.exp(torch.randn(B, T, H + 2 * Hkv, 1, generator=g))
    proj = proj.bfloat16().cuda().transpose(1, 2)
    n = sum(sections)
    inv = (10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)).float().cuda()
    pos = torch.randint(-100, 100000, (B, T, len(sections)), generator=g).int().cuda()
    qw, kw = (torch.exp(0.5 * torch.randn(D, generator=g)).cuda() for _ in range(2))
    return proj[:, :H], proj[:, H:H + Hkv], proj[:, H + Hkv:], pos, inv, qw, kw


def expected(cache, x, lens, table, page, T, max_len):
    """The cache after rows x [B, Hkv, T, D] have entered, which of its bytes are near a border, and the rows as they are held."""
    codes, scales, gap = mo.hold(x)
    gap[f64(torch.from_numpy(x).bfloat16()) == x] = 1     # what came in as a bf16 number and was not computed on may lie on a border itself
    have = mo.rows_of(cache, page, x.shape[-1])
    near = [np.zeros(a.shape, dtype=bool) for a in have]
    for b, n in enumerate(lens):
        for t in range(T):
            slot = n - T + t
            if not 0 <= slot < max_len:
                continue
            p, at = (int(table[b, slot // page]), slot % page) if table is not None else (b, slot)
            if not 0 <= p < cache.shape[0]:
                continue
            have[0][p, :, at], have[1][p, :, at] = codes[b, :, t], scales[b, :, t]
            near[0][p, :, at], near[1][p, :, at] = gap[b, :, t] < 1e-9, (gap[b, :, t].reshape(gap.shape[1], -1, 32) < 1e-9).any(-1)
    return mo.pages_of(*have), mo.pages_of(near[0].astype(np.uint8), near[1].astype(np.uint8)) > 0, mo.values(codes, scales), gap < 1e-9


def same(a, b):
    return bool(torch.equal(a, b))


def turned_alone(got, x, pos, inv, sections, interleaved=False):
    """Rows that are turned and not normalised: sine and cosine 2^-14 of a pair's length, the rounding 2^-8 of the result."""
    ref = mo.norm_rotary(f64(x), None, pos.cpu().numpy(), f64(inv), sections, eps=0, interleaved=interleaved, norm=False)
    bad = ~(np.abs(f64(got) - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -14 + 2e-6) * mo.pair_lengths(f64(x), sections, interleaved))
    assert not bad.any(), (np.argwhere(bad)[:4], f64(got)[bad][:4], ref[bad][:4])


CASES = [
    (1, [1, 17, 64], 16, 128, (16, 24, 24), 4, 2, False), (5, [5, 3, 0, 40], 8, 64, (32,), 4, 2, True), (70, [70, 129, 12], 64, 64, (10, 6), 2, 1, False),
    (3, [9, 30], 32, 128, (20, 20), 3, 3, True), (1, [2], 16, 64, (3,), 8, 1, False), (33, [33, 40], 16, 128, (1,), 2, 2, True),
    (520, [600], 16, 128, (64,), 8, 8, False), (1, [5] * 40, 8, 64, (8, 8, 8, 8), 16, 2, False), (2, [1, 2, 3], 8, 128, (31, 30), 1, 1, False),
]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("T,lens,page,D,sections,H,Hkv,interleaved", CASES)
def test_append(T, lens, page, D, sections, H, Hkv, interleaved, norm):
    B = len(lens)
    q, k, v, pos, inv, qw, kw = append_inputs(B, H, Hkv, T, D, sections)
    kc, vc, table = pool(B, Hkv, D, page, -(-max(lens) // page))
    how = dict(sections=sections, interleaved=interleaved)
    key = mo.norm_rotary(f64(k), f64(kw) if norm else None, pos.cpu().numpy(), f64(inv), sections, eps=EPS, interleaved=interleaved, norm=norm)
    want = [expected(c.cpu().numpy(), x, lens, table.cpu().numpy(), page, T, 1 << 30) for c, x in ((kc, key), (vc, f64(v)))]
    args = (pos, inv, kc, vc, ints(lens), table) + ((qw, kw) if norm else ())
    rows = (q, k, v) if T > 1 else tuple(x[:, :, 0] for x in (q, k, v))
    got, k_held, v_held = F.norm_rotary_append(*rows, *args, eps=EPS if norm else None, return_held=True, **how)
    if norm:
        assert same(got, F.norm_rotary(q, k, pos, inv, qw, kw, eps=EPS, **how)[0].reshape(got.shape))
    else:
        turned_alone(got.reshape(q.shape), q, pos, inv, sections, interleaved)
    for cache, held, (bytes_, near, values, near_value) in ((kc, k_held, want[0]), (vc, v_held, want[1])):
        assert (near.mean() < 1e-4) and ((cache.cpu().numpy() == bytes_) | near).all()
        assert ((f64(held).reshape(values.shape) == values) | near_value).all()
    # without the rows as they are held: the same cache
    kc2, vc2, _ = pool(B, Hkv, D, page, -(-max(lens) // page))
    alone = F.norm_rotary_append(*rows, pos, inv, kc2, vc2, *args[4:], eps=EPS if norm else None, **how)
    assert same(alone, got) and same(kc2, kc) and same(vc2, vc)


def test_a_chunk_holds_what_its_tokens_alone_do():
    q, k, v, pos, inv, qw, kw = append_inputs(2, 4, 2, 50, 128, (16, 24, 24))
    caches = [pool(2, 2, 128, 16, 4) for _ in range(2)]
    F.norm_rotary_append(q, k, v, pos, inv, *caches[0][:2], ints([50, 64]), caches[0][2], qw, kw, sections=(16, 24, 24))
    for t in range(50):
        F.norm_rotary_append(q[:, :, t], k[:, :, t], v[:, :, t], pos[:, t:t + 1], inv, *caches[1][:2], ints([t + 1, t + 15]), caches[1][2], qw, kw,
                             sections=(16, 24, 24))
    assert same(caches[0][0], caches[1][0]) and same(caches[0][1], caches[1][1])


def test_every_code_border_and_what_is_not_finite():
    """Values on the borders of codes and scales, subnormal, infinite and NaN ones, each with its neighbours among the bf16 numbers."""
    base = [0.0, -0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 6.5, 6.96875, 7.0, 7.5, 8.0, 2.0 ** -126, 2.0 ** -133, 3.3e38]
    bits = torch.tensor(base, dtype=torch.bfloat16).view(torch.int16).int()
    near = torch.cat([(bits + d).clamp(0, 0x7f7f) for d in (-1, 0, 1)] + [torch.tensor([0x7f80, 0x7fc0, 0x7f81])]).to(torch.int16).view(torch.bfloat16)
    near = torch.cat([near, -near])
    g = torch.Generator().manual_seed(0)
    Hkv, T, D = 2, 800, 64
    v = near[torch.randint(0, len(near), (1, Hkv, T, D), generator=g)]
    v[..., :16] = torch.tensor(base[2:18]).bfloat16() * (2.0 ** torch.randint(-140, 127, (1, Hkv, T, 1), generator=g).float()).bfloat16()
    v[:, :, :300, 32:] = torch.randn(1, Hkv, 300, 32, generator=g).bfloat16()      # blocks of the first are finite here and there
    v[:, :, :500, 16:32] = torch.where(v[:, :, :500, 16:32].float().abs() < 100, v[:, :, :500, 16:32], torch.ones(()).bfloat16())
    v = v.cuda()
    q, k = torch.ones(1, 2, T, D, device="cuda").bfloat16(), torch.ones(1, Hkv, T, D, device="cuda").bfloat16()
    kc, vc, table = pool(1, Hkv, D, 16, T // 16)
    want, _, values, _ = expected(vc.cpu().numpy(), f64(v), [T], table.cpu().numpy(), 16, T, T)
    pos, inv = torch.zeros(1, T, 1, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")
    _, _, held = F.norm_rotary_append(q, k, v, pos, inv, kc, vc, ints([T]), table, eps=None, return_held=True)
    have, ref = mo.rows_of(vc.cpu().numpy(), 16, D), mo.rows_of(want, 16, D)
    assert np.array_equal(have[1], ref[1])
    assert np.array_equal(have[0], ref[0])
    big = np.abs(values) >= 2.0 ** -126            # below them bf16 numbers are subnormal, which a conversion may flush
    assert np.array_equal(f64(held)[big], values[big]) and np.isfinite(f64(held)).all()
    # as a key, turned by nothing: the same codes by way of 64 bits
    kc2, vc2, _ = pool(1, Hkv, D, 16, T // 16)
    F.norm_rotary_append(q, v, v, pos, inv, kc2, vc2, ints([T]), table, eps=None)
    key = mo.norm_rotary(np.where(np.isfinite(f64(v)), f64(v), 0), None, pos.cpu().numpy(), f64(inv), (32,), eps=0, norm=False)
    rows = np.isfinite(f64(v)).all(-1)
    codes, scales, _ = mo.hold(key)
    back = [a.transpose(1, 0, 2, 3).reshape(Hkv, -1, a.shape[-1])[None, :, :T] for a in (x[table[0].cpu().numpy()] for x in mo.rows_of(kc2.cpu().numpy(), 16, D))]
    assert np.array_equal(back[1][rows], scales[rows]) and np.array_equal((back[0] & 7)[rows], (codes & 7)[rows])


@pytest.mark.parametrize("mx4", [True, False])
def test_append_passes_over_what_has_no_slot(mx4):
    """Negative slots, slots from the bound on (from the true length) and entries that name no page: the rest is as without them."""
    B, H, Hkv, T, D, page = 4, 2, 2, 6, 64, 8
    q, k, v, pos, inv, qw, kw = append_inputs(B, H, Hkv, T, D, (32,))
    kc, vc, table = pool(B, Hkv, D, page, 4)
    if not mx4:
        kc, vc = (torch.randn(kc.shape[0], page, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    lens = [3, 30, 20, -5]
    table[2, 1], table[2, 2] = -1, kc.shape[0]
    before = kc.clone(), vc.clone()
    got = F.norm_rotary_append(q, k, v, pos, inv, kc, vc, ints(lens), table, qw, kw, eps=EPS, max_seq_len=26)
    turned_q, turned_k = F.norm_rotary(q, k, pos, inv, qw, kw, eps=EPS)
    assert same(got, turned_q)
    t = table.cpu().numpy()
    if mx4:
        key = mo.norm_rotary(f64(k), f64(kw), pos.cpu().numpy(), f64(inv), (32,), eps=EPS)
        for cache, x, old in ((kc, key, before[0]), (vc, f64(v), before[1])):
            want, near, _, _ = expected(old.cpu().numpy(), x, lens, t, page, T, 26)
            assert ((cache.cpu().numpy() == want) | near).all()
        return
    for cache, x, old in ((kc, turned_k, before[0]), (vc, v, before[1])):
        for b, n in enumerate(lens):
            for i in range(T):
                slot = n - T + i
                if 0 <= slot < 26 and 0 <= t[b, slot // page] < kc.shape[0]:
                    old[t[b, slot // page], slot % page] = x[b, :, i]
        assert same(cache, old)


@pytest.mark.parametrize("D,sections,H,Hkv,T", [(128, (64,), 4, 2, 1), (80, (40,), 3, 1, 20), (40, (3, 4), 2, 2, 5), (256, (100,), 2, 1, 3), (64, (16, 8), 8, 8, 130)])
@pytest.mark.parametrize("norm", [True, False])
def test_append_to_a_bf16_cache(D, sections, H, Hkv, T, norm):
    B, page = 3, 16
    q, k, v, pos, inv, qw, kw = append_inputs(B, H, Hkv, T, D, sections)
    lens, per = [T, T + 7, max(0, T - 2)], -(-(T + 7) // page)
    table = torch.randperm(B * per + 2)[:B * per].reshape(B, per).int().cuda()
    kc, vc = (torch.randn(B * per + 2, page, Hkv, D, device="cuda").bfloat16() for _ in range(2))
    want = kc.clone(), vc.clone()
    w = (qw, kw) if norm else ()
    got = F.norm_rotary_append(q, k, v, pos, inv, kc, vc, ints(lens), table, *w, eps=EPS if norm else None, sections=sections)
    if norm:
        turned = F.norm_rotary(q, k, pos, inv, *w, eps=EPS, sections=sections)
        assert same(got, turned[0])
    else:
        turned_alone(got, q, pos, inv, sections)
        turned = None, k.clone()
    for b, n in enumerate(lens):
        for t in range(T):
            if n - T + t >= 0:
                at = table[b, (n - T + t) // page], (n - T + t) % page
                want[1][at] = v[b, :, t]
                if norm:
                    want[0][at] = turned[1][b, :, t]
                else:                              # what is there, to be looked at by itself
                    turned[1][b, :, t] = want[0][at] = kc[at]
            elif not norm:
                turned[1][b, :, t] = F.rotary(k[b:b + 1, :, t:t + 1], None, pos[b:b + 1, t:t + 1], inv, sections=sections)[0][0, :, 0]
    assert same(kc, want[0]) and same(vc, want[1])
    if not norm:
        turned_alone(turned[1], k, pos, inv, sections)


# ---- attention over it ----

def check_attention(got, lse, q, kc, vc, lens, table, page, *, scale, window=None, softcap=None, slopes=None):
    q = f64(q)
    single = q.ndim == 3
    if single:
        q, got, lse = q[:, :, None], got[:, :, None], lse[:, :, None]
    D = q.shape[-1]
    k, v = (mo.dense(c.cpu().numpy(), page, D) for c in (kc, vc))
    if table is None:
        t = np.arange(q.shape[0])[:, None]
    else:
        t = np.clip(table.cpu().numpy(), 0, k.shape[0] - 1)
    lens = np.clip(np.asarray(lens), 0, t.shape[1] * page)
    kw = dict(scale=scale, window=window, softcap_value=softcap, alibi_slopes=None if slopes is None else f64(slopes))
    ref, ref_lse = do.prefill_attention(q, k, v, t, lens, **kw)
    size, _ = do.prefill_attention(q, k, np.abs(v), t, lens, **kw)
    got, lse = f64(got), f64(lse)
    bad = ~(np.abs(got - ref) <= (2.0 ** -8 + 2.0 ** -10) * size + 2.0 ** -8 * np.abs(ref))
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])
    empty = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(lse), empty)
    assert (np.abs(lse[~empty] - ref_lse[~empty]) <= 2.0 ** -11).all()


VARIANTS = dict(plain={}, softcap=dict(softcap=5.0), alibi=dict(alibi=True), window=dict(window=20), both=dict(window=9, softcap=30.0))


def variant(name, H):
    kw = dict(VARIANTS[name])
    if kw.pop("alibi", False):
        kw["alibi_slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda")
    return kw


def attend(call, q, kc, vc, lens, table, page, name="plain", **more):
    H = q.shape[1]
    kw = variant(name, H)
    scale = 0.3 * q.shape[-1] ** -0.5
    out, lse = call(q, kc, vc, ints(lens), table, scale=scale, return_lse=True, **kw, **more)
    assert out.shape == q.shape and lse.shape == q.shape[:-1]
    check_attention(out, lse, q, kc, vc, lens, table, page, scale=scale, window=kw.get("window"), softcap=kw.get("softcap"), slopes=kw.get("alibi_slopes"))
    return out, lse


@pytest.mark.parametrize("name", VARIANTS)
@pytest.mark.parametrize("D,page,H,Hkv,T,lens", [
    (128, 16, 8, 2, 1, [1, 45, 700, 0, 32]), (64, 8, 8, 8, 1, [7, 8, 9, 31, 33, 500]), (128, 64, 4, 1, 4, [3, 1, 260, 64]), (64, 32, 32, 2, 1, [100, 31]),
    (128, 8, 12, 2, 5, [5, 150, 33]), (64, 16, 8, 1, 8, [8, 9, 1000]), (128, 16, 64, 1, 1, [129, 2]), (64, 16, 6, 2, 3, [0, 0])])
def test_decode(D, page, H, Hkv, T, lens, name):
    B = len(lens)
    kc, vc, table = pool(B, Hkv, D, page, max(1, -(-max(lens) // page)))
    q = torch.randn(B, H, T, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    attend(F.decode_attention_mx4, q if T > 1 else q[:, :, 0], kc, vc, lens, table, page, name)


def test_decode_of_one_long_sequence_and_of_many_short_ones():
    for lens, page, D in (([9001], 16, 128), ([20011], 64, 64), ([(n * 37) % 130 for n in range(200)], 16, 128)):
        kc, vc, table = pool(len(lens), 2, D, page, -(-max(lens) // page))
        q = torch.randn(len(lens), 4, D, device="cuda").bfloat16()
        out, lse = attend(F.decode_attention_mx4, q, kc, vc, lens, table, page)
        again = F.decode_attention_mx4(q, kc, vc, ints(lens), table, scale=0.3 * D ** -0.5, return_lse=True)
        assert same(out, again[0]) and same(lse, again[1])


@pytest.fixture(params=["rows", "unpacked"])
def way(request):
    """Chunks as the library sends them (all that are here: through the decode kernels), and unpacked for the forward kernel."""
    fb.check(fb.fl_set_tuning("prefill_gather", 0 if request.param == "rows" else 1))
    yield request.param
    fb.check(fb.fl_set_tuning("prefill_gather", 0))


@pytest.mark.parametrize("name", VARIANTS)
@pytest.mark.parametrize("D,page,H,Hkv,Sq,lens", [(128, 16, 4, 2, 40, [40, 100, 7]), (64, 8, 2, 2, 77, [200, 77]), (128, 64, 8, 1, 9, [9, 60]), (64, 16, 2, 1, 130, [131, 0, 129]),
                                                  (128, 8, 4, 4, 12, [300]), (64, 32, 6, 2, 33, [33, 1000, 34, 32, 1]), (128, 16, 16, 2, 45, [700, 44])])
def test_prefill(D, page, H, Hkv, Sq, lens, name, way):
    B = len(lens)
    kc, vc, table = pool(B, Hkv, D, page, -(-max(lens) // page))
    q = torch.randn(B, H, Sq, D, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    attend(F.paged_prefill_attention_mx4, q, kc, vc, lens, table, page, name)


@pytest.mark.parametrize("name", VARIANTS)
@pytest.mark.parametrize("D", [64, 128])
def test_a_chunk_whose_rows_are_split_among_workgroups(D, name):
    """Blocks of rows whose keys end, and under a window begin, in other tiles than the chunk's."""
    lens, page, H, Hkv, Sq = [2500, 2049, 70], 16, 6, 2, 50
    kc, vc, table = pool(3, Hkv, D, page, -(-max(lens) // page))
    q = torch.randn(3, H, Sq, D, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    for splits in (0, 1, 5, 64):
        fb.check(fb.fl_set_tuning("decode_splits", splits))
        try:
            attend(F.paged_prefill_attention_mx4, q, kc, vc, lens, table, page, name)
        finally:
            fb.check(fb.fl_set_tuning("decode_splits", 0))


def test_many_rows_of_long_prompts():
    """Prompts that the library unpacks by itself, on some of their rows: those of a chunk that ends there."""
    B, H, Hkv, D, page, n = 2, 16, 2, 64, 16, 3000
    kc, vc, table = pool(B, Hkv, D, page, -(-n // page))
    q = torch.randn(B, H, n, D, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    scale = 0.3 * D ** -0.5
    out, lse = F.paged_prefill_attention_mx4(q, kc, vc, ints([n, n - 7]), table, scale=scale, return_lse=True)
    for first, rows in ((0, 40), (1500, 9), (2990, 10)):
        end = first + rows
        check_attention(out[:, :, first:end], lse[:, :, first:end], q[:, :, first:end], kc, vc, [end, end - 7], table, page, scale=scale)
    assert not out[1, :, :7].any() and bool(torch.isneginf(lse[1, :, :7]).all())


def test_without_a_table_and_with_other_strides(way):
    """A page per sequence of a size that is no power of two; caches that lie head by head."""
    for D in (64, 128):
        B, H, Hkv, size = 3, 4, 2, 72
        token = D // 2 + D // 32
        kc, vc, _ = pool(B, Hkv, D, size, 1)
        wide = [torch.zeros(Hkv, kc.shape[0], size * token + 16 * n, device="cuda", dtype=torch.uint8) for n in (1, 3)]
        views = [w.transpose(0, 1)[..., :size * token] for w in wide]
        for to, c in zip(views, (kc, vc)):
            to.copy_(c)
        q = torch.randn(B, H, 3, D, device="cuda").bfloat16()
        lens = [72, 1, 50]
        a = attend(F.decode_attention_mx4, q, kc, vc, lens, None, size)
        b = attend(F.decode_attention_mx4, q, *views, lens, None, size)
        assert same(a[0], b[0]) and same(a[1], b[1])
        chunk = torch.randn(B, H, 70, D, device="cuda").bfloat16()
        a = attend(F.paged_prefill_attention_mx4, chunk, kc, vc, lens, None, size)
        b = attend(F.paged_prefill_attention_mx4, chunk, *views, lens, None, size)
        assert same(a[0], b[0]) and same(a[1], b[1])
        x, k, v, pos, inv, qw, kw = append_inputs(B, H, Hkv, 5, D, (D // 2,))
        F.norm_rotary_append(x, k, v, pos, inv, kc, vc, ints(lens), None, qw, kw)
        F.norm_rotary_append(x, k, v, pos, inv, *views, ints(lens), None, qw, kw)
        assert same(views[0], kc) and same(views[1], vc)
        assert not any(w[..., size * token:].any() for w in wide)


@pytest.mark.parametrize("call,rows", [(F.decode_attention_mx4, 2), (F.paged_prefill_attention_mx4, 40)])
def test_what_lies_behind_a_sequence_is_not_seen(call, rows, way):
    """Any bytes behind the last token of its last page and in pages behind it: scales of NaN, infinity and zero among them."""
    lens, page, D, Hkv = [77, 40, 129], 16, 128, 2
    kc, vc, table = pool(3, Hkv, D, page, 12)
    q = torch.randn(3, 4, rows, D, device="cuda").bfloat16()
    want = call(q, kc, vc, ints(lens), table, return_lse=True)
    for fill in (0xFF, 0x00, 0xFE):
        k2, v2 = kc.clone(), vc.clone()
        for c in (k2, v2):
            codes, scales = c[..., :page * D // 2].unflatten(-1, (page, D // 2)), c[..., page * D // 2:].unflatten(-1, (D // 32, page))
            for b, n in enumerate(lens):
                for slot in range(n, 12 * page):
                    codes[table[b, slot // page], :, slot % page] = fill
                    scales[table[b, slot // page], :, :, slot % page] = fill
        got = call(q, k2, v2, ints(lens), table, return_lse=True)
        assert same(got[0], want[0]) and same(got[1], want[1]), fill


def test_lengths_and_entries_outside_their_bounds_are_cut(way):
    page, D = 16, 64
    kc, vc, table = pool(3, 2, D, page, 4)
    q = torch.randn(3, 4, D, device="cuda").bfloat16()
    got = F.decode_attention_mx4(q, kc, vc, ints([100, -7, 1 << 30]), table, max_seq_len=50, return_lse=True)
    want = F.decode_attention_mx4(q, kc, vc, ints([50, 0, 50]), table, max_seq_len=50, return_lse=True)
    assert same(got[0], want[0]) and same(got[1], want[1]) and not got[0][1].any() and bool(torch.isneginf(got[1][1]).all())
    wild, cut = table.clone(), table.clone()
    wild[0, 1], wild[1, 0], wild[2, 2] = -3, 1 << 30, kc.shape[0]
    cut[0, 1], cut[1, 0], cut[2, 2] = 0, kc.shape[0] - 1, kc.shape[0] - 1
    chunk = torch.randn(3, 4, 40, D, device="cuda").bfloat16()
    for call, x in ((F.decode_attention_mx4, q), (F.paged_prefill_attention_mx4, chunk)):
        assert same(call(x, kc, vc, ints([60, 60, 60]), wild), call(x, kc, vc, ints([60, 60, 60]), cut))


def test_nothing_cached_at_all(way):
    kc, vc = F.mx4_cache(4, 16, 2, 64)
    table = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    for rows, call in ((1, F.decode_attention_mx4), (50, F.paged_prefill_attention_mx4)):
        q = torch.randn(2, 4, rows, 64, device="cuda").bfloat16()
        out, lse = call(q, kc, vc, ints([0, 0]), table, return_lse=True)
        assert not out.any() and bool(torch.isneginf(lse).all())
        assert call(q[:0], kc, vc, ints([]), table[:0]).shape == (0, 4, rows, 64)


def test_scores_far_up_and_down():
    """Rows whose maximum rises from tile to tile by more than a factor of 2^8, and rows far below zero."""
    D, page, n = 64, 16, 640
    kc, vc, table = pool(1, 1, D, page, n // page, scales=(126, 127))
    r = np.random.default_rng(3)
    codes, scales, _ = mo.hold(np.ones((1, 1, n, D)) * np.linspace(-4, 4, n)[None, None, :, None])
    lines = mo.pages_of(codes.reshape(1, 1, n, D).reshape(n // page, 1, page, D), scales.reshape(n // page, 1, page, D // 32))
    kc[table[0].long()] = torch.from_numpy(lines).cuda()
    q = torch.from_numpy(np.stack([np.full(D, s) for s in (4.0, -4.0, 0.5, 30.0)])).bfloat16().cuda()[None]
    out, lse = F.decode_attention_mx4(q, kc, vc, ints([n]), table, scale=0.125, return_lse=True)
    # the sums of the scores' sizes reach 960 here: 64 * 2^-24 of them 4e-3 in a probability, and in the log-sum-exp
    k, v = (mo.dense(c.cpu().numpy(), page, D) for c in (kc, vc))
    ref, ref_lse = do.decode_attention(f64(q), k, v, table.cpu().numpy(), [n], scale=0.125)
    size, _ = do.decode_attention(f64(q), k, np.abs(v), table.cpu().numpy(), [n], scale=0.125)
    assert (np.abs(f64(out) - ref) <= (2.0 ** -8 + 8e-3) * size + 2.0 ** -8 * np.abs(ref)).all()
    assert (np.abs(f64(lse) - ref_lse) <= 5e-3).all()


@pytest.mark.parametrize("call,rows,H", [(F.decode_attention_mx4, 1, 8), (F.decode_attention_mx4, 7, 4), (F.paged_prefill_attention_mx4, 45, 4)])
def test_a_query_row_that_is_not_finite_stays_alone(call, rows, H):
    lens, page, D, Hkv = [300, 64], 16, 128, 2
    kc, vc, table = pool(2, Hkv, D, page, 20)
    q = torch.randn(2, H, rows, D, device="cuda").bfloat16()
    want, want_lse = call(q, kc, vc, ints(lens), table, return_lse=True)
    bad = q.clone()
    bad[0, 1, rows // 2, 3], bad[1, 0, 0, 70] = float("nan"), float("inf")
    got, lse = call(bad, kc, vc, ints(lens), table, return_lse=True)
    assert bool(got[0, 1, rows // 2].isnan().all())                  # (its lse says nothing: -inf, as fl_attn_decode's)
    for x in (got, want, lse, want_lse):
        x[0, 1, rows // 2], x[1, 0, 0] = 0, 0
    assert same(got, want) and same(lse, want_lse)


def test_weights_that_begin_anywhere():
    """Weights that are aligned to their four bytes alone."""
    D, page = 128, 16
    q, k, v, pos, inv, qw, kw = append_inputs(2, 4, 2, 5, D, (64,))
    odd = [torch.cat([w.new_zeros(1), w])[1:] for w in (qw, kw)]
    for a, b in zip(F.norm_rotary(q, k, pos, inv, qw, kw), F.norm_rotary(q, k, pos, inv, *odd)):
        assert same(a, b)
    held = []
    for w in ((qw, kw), odd):
        kc, vc, table = pool(2, 2, D, page, 3)
        held.append((F.norm_rotary_append(q, k, v, pos, inv, kc, vc, ints([40, 9]), table, *w), kc, vc))
    assert all(same(a, b) for a, b in zip(*held))


def test_far_pages(way):
    """Pages more than 2^32 bytes into the caches."""
    page, Hkv, H, D, n = 16, 8, 16, 128, 200
    per, each = -(-n // page), 16 * 68 * 8
    pages = (1 << 32) // each + 64
    far_k, far_v = F.mx4_cache(pages, page, Hkv, D)
    near_k, near_v = F.mx4_cache(64, page, Hkv, D)
    table = torch.randperm(64)[:per].reshape(1, -1).int().cuda()
    q, k, v, pos, inv, qw, kw = append_inputs(1, H, Hkv, n, D, (64,))
    results = []
    for kc, vc, by in ((near_k, near_v, 0), (far_k, far_v, pages - 64)):
        t = (table + by).contiguous()
        turned = F.norm_rotary_append(q, k, v, pos, inv, kc, vc, ints([n]), t, qw, kw)
        results.append((turned, F.paged_prefill_attention_mx4(turned, kc, vc, ints([n]), t), F.decode_attention_mx4(turned[:, :, -1].contiguous(), kc, vc, ints([n]), t)))
    for a, b in zip(*results):
        assert same(a, b)
    assert same(far_k[-64:], near_k) and same(far_v[-64:], near_v) and not far_k[:64].any()


def test_fp32_results_and_workspaces_through_the_abi():
    B, H, Hkv, D, page, lens = 2, 8, 2, 128, 16, [6000, 33]
    kc, vc, table = pool(B, Hkv, D, page, 400)
    q = torch.randn(B, H, 1, D, device="cuda").bfloat16()
    want, want_lse = F.decode_attention_mx4(q[:, :, 0], kc, vc, ints(lens), table, return_lse=True)
    out, lse = torch.zeros(B, H, 1, D, device="cuda"), torch.zeros(B, H, 1, 1, device="cuda")
    seq = ints(lens)
    kv = fb.paged_kv(block_table=table, page_size=page, seq_lens=seq, max_seq_len=400 * page)
    tq, tk, tv = fb.tensor_desc(q[:, None]), fb.mx4_desc(kc, page, D), fb.mx4_desc(vc, page, D)
    need = fb.fl_attn_decode_mx4_workspace_size(tq, tk, kv)
    assert need > 0
    ws = torch.full((need + 64,), 0x7F, dtype=torch.uint8, device="cuda")
    aux = fb.aux_desc(workspace=ws[:need])
    d = fb.variant_desc(scale=D ** -0.5)
    fb.check(fb.fl_attn_decode_mx4(tq, tk, tv, kv, d, aux, fb.tensor_desc(out[:, None]), fb.tensor_desc(lse[:, None]), torch.cuda.current_stream().cuda_stream))
    assert same(out[:, :, 0].bfloat16(), want) and same(lse[:, :, 0, 0], want_lse) and bool((ws[need:] == 0x7F).all())
    for call, x in ((F.decode_attention_mx4, q[:, :, 0]), (F.paged_prefill_attention_mx4, torch.randn(B, H, 40, D, device="cuda").bfloat16())):
        with pytest.raises(ValueError, match="workspace holds 16 bytes"):
            call(x, kc, vc, seq, table, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
        room = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
        assert same(call(x, kc, vc, seq, table, workspace=room), call(x, kc, vc, seq, table))


def test_serving_replays_from_a_graph_while_sequences_grow():
    """Append and decode step captured together; every replay against the eager calls on caches of their own."""
    B, H, Hkv, D, page, sections = 3, 8, 2, 128, 16, (16, 24, 24)
    caches = [pool(B, Hkv, D, page, 10) for _ in range(2)]
    table = caches[0][2]
    q, k, v, pos, inv, qw, kw = append_inputs(B, H, Hkv, 1, D, sections)
    lens = ints([5, 60, 100])
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def step(kc, vc):
        turned = F.norm_rotary_append(q, k, v, pos, inv, kc, vc, lens, table, qw, kw, sections=sections)
        return turned, F.decode_attention_mx4(turned, kc, vc, lens, table, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*caches[1][:2])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(*caches[1][:2])
    for c, old in zip(caches[1][:2], caches[0][:2]):
        c.copy_(old)
    for n in range(5):
        lens += 1
        pos.add_(1)
        for x in (q, k, v):
            x.copy_(torch.randn_like(x))
        want = step(*caches[0][:2])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(held[0], want[0]) and same(held[1], want[1]), n
        assert same(caches[0][0], caches[1][0]) and same(caches[0][1], caches[1][1])


def test_chunks_replay_from_a_graph_while_sequences_grow(way):
    """A chunk's append and attention captured together, its sequences longer at every replay; rows split among workgroups and not."""
    B, H, Hkv, D, page, T = 2, 8, 2, 64, 16, 24
    for per in (8, 200):
        caches = [pool(B, Hkv, D, page, per) for _ in range(2)]
        table = caches[0][2]
        q, k, v, pos, inv, qw, kw = append_inputs(B, H, Hkv, T, D, (32,))
        lens = ints([T - 5, T])

        def step(kc, vc):
            turned = F.norm_rotary_append(q, k, v, pos, inv, kc, vc, lens, table, qw, kw)
            return (turned,) + F.paged_prefill_attention_mx4(turned, kc, vc, lens, table, return_lse=True)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(*caches[1][:2])
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step(*caches[1][:2])
        for c, old in zip(caches[1][:2], caches[0][:2]):
            c.copy_(old)
        for n in range(4):
            lens += T * (per // 8)
            pos.add_(T)
            for x in (q, k, v):
                x.copy_(torch.randn_like(x))
            want = step(*caches[0][:2])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(same(a, b) for a, b in zip(held, want)), (per, n)
            assert same(caches[0][0], caches[1][0]) and same(caches[0][1], caches[1][1])


def test_calls_of_two_threads():
    """Each on a stream of its own, several times: what either gives is what it gives alone."""
    lens, page = [900, 333, 1], 16
    work = []
    for D, rows in ((64, 1), (128, 30)):
        kc, vc, table = pool(3, 2, D, page, 60)
        q = torch.randn(3, 8, rows, D, device="cuda").bfloat16()
        call = F.decode_attention_mx4 if rows == 1 else F.paged_prefill_attention_mx4
        work.append((call, q, kc, vc, ints(lens), table, call(q, kc, vc, ints(lens), table)))
    torch.cuda.synchronize()
    wrong = []

    def run(call, q, kc, vc, seq, table, want):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = [call(q, kc, vc, seq, table) for _ in range(20)]
            torch.cuda.current_stream().synchronize()
        wrong.extend(n for n, g in enumerate(got) if not same(g, want))

    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_another_stream(way):
    lens, page, D = [3000, 2000], 16, 128
    kc, vc, table = pool(2, 4, D, page, 188)
    q = torch.randn(2, 8, 50, D, device="cuda").bfloat16()
    want = F.decode_attention_mx4(q[:, :, 0], kc, vc, ints(lens), table), F.paged_prefill_attention_mx4(q, kc, vc, ints(lens), table)
    side, seq = torch.cuda.Stream(), ints(lens)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = F.decode_attention_mx4(q[:, :, 0], kc, vc, seq, table), F.paged_prefill_attention_mx4(q, kc, vc, seq, table)
    torch.cuda.current_stream().wait_stream(side)
    assert same(got[0], want[0]) and same(got[1], want[1])


@pytest.mark.parametrize("T", [1, 3])
def test_a_prompt_then_tokens(T):
    """A prompt in two chunks, then steps of T tokens: every row's attention is that over the keys as the cache holds them."""
    B, H, Hkv, D, page, sections = 2, 8, 2, 64, 16, (16, 16)
    kc, vc = F.mx4_cache(40, page, Hkv, D)
    table = torch.randperm(40)[:B * 12].reshape(B, 12).int().cuda()
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    held, done = [], 0
    for n in (90, 37) + (T,) * 4:
        q, k, v, _, inv, qw, kw = append_inputs(B, H, Hkv, n, D, sections, seed=done)
        pos = (torch.arange(done, done + n, device="cuda", dtype=torch.int32))[None, :, None].expand(1, n, 2)
        lens += n
        rows = (q, k, v) if n > 1 else tuple(x[:, :, 0] for x in (q, k, v))
        turned, k_held, v_held = F.norm_rotary_append(*rows, pos, inv, kc, vc, lens, table, qw, kw, sections=sections, return_held=True)
        held.append([x.reshape(B, Hkv, n, D) for x in (k_held, v_held)])
        call = F.decode_attention_mx4 if n <= 3 else F.paged_prefill_attention_mx4
        out = call(turned, kc, vc, lens, table).reshape(B, H, n, D)
        done += n
        k_all, v_all = (torch.cat([h[i] for h in held], 2) for i in range(2))
        dense = F.attention(turned.reshape(B, H, n, D), k_all, v_all, causal=True, q_offset=done - n)
        # both within (2^-8 + 2^-10) sum P |v| + 2^-8 |result| of the exact result
        size = F.attention(turned.reshape(B, H, n, D), k_all, v_all.abs(), causal=True, q_offset=done - n).double()
        assert ((out.double() - dense.double()).abs() <= 2 * (2.0 ** -8 + 2.0 ** -10) * 1.01 * size + 2.0 ** -7 * dense.double().abs()).all()
