"""CPU tests of the refusals of the calls that normalise and turn heads and of those around a 4-bit cache: through the C ABI (before any HIP call) and the
PyTorch entry points."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2511_02043_amd import binding as fb
from paper_2511_02043_amd import functional as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20                                     # an aligned address that no call gets as far as reading


def tensor(*size, dtype=fb.FL_BF16, ptr=FAKE, stride=None):
    t = fb.fl_tensor()
    t.ptr, t.dtype = ptr, dtype
    t.size[:] = size
    step = 1
    for a in range(4, -1, -1):
        t.stride[a] = step
        step *= max(size[a], 1)
    for a, s in (stride or {}).items():
        t.stride[a] = s
    return t


def pages(n=20, Hkv=2, page=16, D=64, dtype=fb.FL_MX4, ptr=FAKE, stride=None):
    each = page * (D // 2 + D // 32)
    t = tensor(n, 1, Hkv, page, D, dtype=dtype, ptr=ptr)
    t.stride[:] = [Hkv * each, 0, each, 0, 1]
    for a, s in (stride or {}).items():
        t.stride[a] = s
    return t


def rotary(axes=1, sections=(32, 0, 0, 0), **kw):
    r = fb.fl_rotary()
    r.struct_size, r.axes = ctypes.sizeof(fb.fl_rotary), axes
    r.sections[:] = sections
    r.positions, r.inv_freq = FAKE, FAKE
    for n, x in kw.items():
        setattr(r, n, x)
    return r


def norm(eps=1e-6, **kw):
    n = fb.fl_head_norm()
    n.struct_size, n.eps, n.q_weight, n.k_weight = ctypes.sizeof(fb.fl_head_norm), eps, FAKE, FAKE
    for name, x in kw.items():
        setattr(n, name, x)
    return n


def paged(page=16, max_len=64, table=FAKE, stride=4, lens=FAKE, **kw):
    kv = fb.fl_paged_kv()
    kv.struct_size = ctypes.sizeof(fb.fl_paged_kv)
    kv.block_table, kv.table_stride, kv.page_size, kv.seq_lens, kv.max_seq_len = table, stride, page, lens, max_len
    for name, x in kw.items():
        setattr(kv, name, x)
    return kv


def aux(ws=FAKE, size=1 << 40, slopes=None):
    a = fb.fl_aux()
    a.struct_size, a.workspace, a.workspace_bytes, a.alibi_slopes = ctypes.sizeof(fb.fl_aux), ws or None, size, slopes
    return a


def test_struct_layout_matches_the_header(tmp_path):
    src = tmp_path / "sz.c"
    src.write_text('''#include <stdio.h>
#include <stddef.h>
#include "fl_attn.h"
int main(void) {
  printf("%zu %zu %zu %zu %d\\n", sizeof(fl_head_norm), offsetof(fl_head_norm, eps), offsetof(fl_head_norm, q_weight), offsetof(fl_head_norm, k_weight), FL_MX4);
  return 0;
}''')
    exe = tmp_path / "sz"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    N = fb.fl_head_norm
    assert got == [ctypes.sizeof(N), N.eps.offset, N.q_weight.offset, N.k_weight.offset, fb.FL_MX4]


Q, K = (2, 1, 4, 8, 64), (2, 1, 2, 8, 64)
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("want,change", [
    (fb.FL_ERR_NULL, dict(n=None)), (fb.FL_ERR_NULL, dict(r=None)), (fb.FL_ERR_NULL, dict(q=None, k=None, qo=None, ko=None)), (fb.FL_ERR_NULL, dict(q=None)),
    (fb.FL_ERR_NULL, dict(ko=None)), (fb.FL_ERR_NULL, dict(k=tensor(*K, ptr=0))), (fb.FL_ERR_NULL, dict(r=rotary(positions=None))),
    (fb.FL_ERR_DESC, dict(n=norm(struct_size=8))), (fb.FL_ERR_DESC, dict(n=norm(-1e-6))), (fb.FL_ERR_DESC, dict(n=norm(INF))), (fb.FL_ERR_DESC, dict(n=norm(NAN))),
    (fb.FL_ERR_DESC, dict(r=rotary(inverse=1))), (fb.FL_ERR_DESC, dict(r=rotary(axes=5))), (fb.FL_ERR_SHAPE, dict(r=rotary(sections=(33, 0, 0, 0)))),
    (fb.FL_ERR_UNSUPPORTED, dict(q=tensor(2, 1, 4, 8, 1032), qo=tensor(2, 1, 4, 8, 1032), k=None, ko=None)), (fb.FL_ERR_DTYPE, dict(q=tensor(*Q, dtype=fb.FL_MX4))),
    (fb.FL_ERR_DTYPE, dict(k=tensor(*K, dtype=fb.FL_F32))), (fb.FL_ERR_DTYPE, dict(qo=tensor(*Q, dtype=fb.FL_F32))), (fb.FL_ERR_SHAPE, dict(k=tensor(2, 1, 2, 7, 64))),
    (fb.FL_ERR_SHAPE, dict(q=tensor(2, 2, 4, 8, 64))), (fb.FL_ERR_SHAPE, dict(q=tensor(2, 1, -4, 8, 64))), (fb.FL_ERR_SHAPE, dict(ko=tensor(2, 1, 2, 8, 32))),
    (fb.FL_ERR_SHAPE, dict(q=tensor(2, 1, 20000, 8, 64))), (fb.FL_ERR_SHAPE, dict(q=tensor(1 << 16, 1, 4, 1 << 16, 64), k=None, ko=None)),
    (fb.FL_ERR_STRIDE, dict(q=tensor(*Q, stride={4: 2}))), (fb.FL_ERR_STRIDE, dict(q=tensor(*Q, stride={2: 0}))), (fb.FL_ERR_ALIGN, dict(k=tensor(*K, stride={3: 68}))),
    (fb.FL_ERR_ALIGN, dict(qo=tensor(*Q, ptr=FAKE + 2))),
])
def test_norm_refusals(want, change):
    a = dict(q=tensor(*Q), k=tensor(*K), r=rotary(), n=norm(), qo=tensor(*Q), ko=tensor(*K))
    a.update(change)
    assert fb.fl_norm_rotary(a["q"], a["k"], a["r"], a["n"], a["qo"], a["ko"]) == want, fb.fl_last_error_detail()
    assert fb.fl_last_error_detail()
    # the gradient reads its inputs as the call itself, with the outputs as what arrives
    assert fb.fl_norm_rotary_bwd(a["q"], a["k"], a["qo"], a["ko"], a["r"], a["n"], tensor(*Q) if a["q"] is not None else None,
                                 tensor(*K) if a["k"] is not None else None, FAKE if a["q"] is not None else None, None, FAKE, 1 << 40) == want
    assert fb.fl_last_error_detail()


@pytest.mark.parametrize("want,change", [
    (fb.FL_ERR_NULL, dict(q=None, dy=None)), (fb.FL_ERR_NULL, dict(k=None, dyk=None)), (fb.FL_ERR_NULL, dict(k=None, dyk=None, dk=None)),
    (fb.FL_ERR_DTYPE, dict(dq=tensor(*Q, dtype=fb.FL_F32))), (fb.FL_ERR_SHAPE, dict(dk=tensor(*Q))), (fb.FL_ERR_NULL, dict(dk=tensor(*K, ptr=0))),
    (fb.FL_ERR_WORKSPACE, dict(ws=None)), (fb.FL_ERR_WORKSPACE, dict(less=1)), (fb.FL_ERR_ALIGN, dict(ws=FAKE + 8)),
])
def test_gradient_refusals(want, change):
    a = dict(q=tensor(*Q), k=tensor(*K), dy=tensor(*Q), dyk=tensor(*K), dq=tensor(*Q), dk=tensor(*K), ws=FAKE, less=0)
    a.update(change)
    need = fb.fl_norm_rotary_bwd_workspace_size(tensor(*Q), tensor(*K), rotary())
    assert need >= 2 * 64 * 4 and need % 256 == 0
    assert fb.fl_norm_rotary_bwd(a["q"], a["k"], a["dy"], a["dyk"], rotary(), norm(), a["dq"], a["dk"], FAKE, FAKE, a["ws"], need - a["less"]) == want
    assert fb.fl_last_error_detail()


def test_gradient_workspace():
    """Bounded however many tokens there are; nothing where the call would refuse."""
    big = lambda S, H, D: fb.fl_norm_rotary_bwd_workspace_size(tensor(1, 1, H, S, D), tensor(1, 1, 1, S, D), rotary())
    assert big(1, 1, 64) <= big(100, 8, 64) <= 2048 * 64 * 4 + 4096 * 64 * 4 and big(1 << 20, 8, 64) <= 4096 * 64 * 4
    assert fb.fl_norm_rotary_bwd_workspace_size(None, None, rotary()) == 0 and fb.fl_norm_rotary_bwd_workspace_size(tensor(*Q), None, None) == 0
    assert big(0, 4, 64) == 0 and big(8, 4, 1032) == 0 and big(-1, 4, 64) == 0
    assert fb.fl_norm_rotary_bwd_workspace_size(tensor(*Q), None, rotary(inverse=1)) == 0


T = dict(q=(2, 1, 4, 3, 64), k=(2, 1, 2, 3, 64))


@pytest.mark.parametrize("want,change", [
    (fb.FL_ERR_NULL, dict(v=None)), (fb.FL_ERR_NULL, dict(q=None)), (fb.FL_ERR_NULL, dict(qo=None)), (fb.FL_ERR_NULL, dict(kv=None)), (fb.FL_ERR_NULL, dict(vc=None)),
    (fb.FL_ERR_NULL, dict(kv=paged(lens=None))), (fb.FL_ERR_NULL, dict(kc=pages(ptr=0))), (fb.FL_ERR_NULL, dict(r=None)), (fb.FL_ERR_NULL, dict(kh=tensor(*T["k"], ptr=0))),
    (fb.FL_ERR_DESC, dict(r=rotary(inverse=1))), (fb.FL_ERR_DESC, dict(n=norm(NAN))), (fb.FL_ERR_DESC, dict(kv=paged(struct_size=4))),
    (fb.FL_ERR_DTYPE, dict(kc=tensor(20, 1, 2, 16, 64))), (fb.FL_ERR_DTYPE, dict(vc=tensor(20, 1, 2, 16, 64, dtype=fb.FL_F32))),
    (fb.FL_ERR_DTYPE, dict(kc=tensor(20, 1, 2, 16, 64, dtype=fb.FL_F32), vc=tensor(20, 1, 2, 16, 64, dtype=fb.FL_F32))), (fb.FL_ERR_DTYPE, dict(q=tensor(*T["q"], dtype=fb.FL_F32))),
    (fb.FL_ERR_DTYPE, dict(v=tensor(*T["k"], dtype=fb.FL_F32))), (fb.FL_ERR_DTYPE, dict(vh=tensor(*T["k"], dtype=fb.FL_F32))),
    (fb.FL_ERR_DESC, dict(kc=tensor(20, 1, 2, 16, 64), vc=tensor(20, 1, 2, 16, 64), kh=tensor(*T["k"]))),
    (fb.FL_ERR_UNSUPPORTED, dict(q=tensor(2, 1, 4, 3, 96), qo=tensor(2, 1, 4, 3, 96), k=tensor(2, 1, 2, 3, 96), v=tensor(2, 1, 2, 3, 96), kc=pages(D=96), vc=pages(D=96))),
    (fb.FL_ERR_SHAPE, dict(kh=tensor(2, 1, 2, 2, 64))), (fb.FL_ERR_SHAPE, dict(k=tensor(2, 1, 4, 3, 64))), (fb.FL_ERR_SHAPE, dict(vc=pages(n=19))),
    (fb.FL_ERR_SHAPE, dict(kv=paged(page=8))), (fb.FL_ERR_SHAPE, dict(kv=paged(stride=3))), (fb.FL_ERR_SHAPE, dict(kv=paged(max_len=-1))), (fb.FL_ERR_SHAPE, dict(kc=pages(n=0), vc=pages(n=0))),
    (fb.FL_ERR_SHAPE, dict(kc=pages(page=4), vc=pages(page=4), kv=paged(page=4, max_len=16))), (fb.FL_ERR_SHAPE, dict(kc=pages(page=24), vc=pages(page=24), kv=paged(page=24))),
    (fb.FL_ERR_SHAPE, dict(kc=pages(page=20), vc=pages(page=20), kv=paged(page=20, max_len=20, table=None))),
    (fb.FL_ERR_SHAPE, dict(kc=pages(n=1), vc=pages(n=1), kv=paged(table=None, max_len=16))), (fb.FL_ERR_SHAPE, dict(kv=paged(table=None))),
    (fb.FL_ERR_SHAPE, dict(kc=pages(page=1 << 25), vc=pages(page=1 << 25), kv=paged(page=1 << 25))),
    (fb.FL_ERR_ALIGN, dict(kc=pages(ptr=FAKE + 8))), (fb.FL_ERR_ALIGN, dict(vc=pages(stride={0: 2 * 544 + 8}))), (fb.FL_ERR_STRIDE, dict(kc=pages(stride={2: 528}))),
    (fb.FL_ERR_STRIDE, dict(kc=pages(stride={0: 544}))), (fb.FL_ERR_STRIDE, dict(vc=pages(stride={0: 1 << 32}))), (fb.FL_ERR_STRIDE, dict(kc=pages(stride={2: 0}))),
    (fb.FL_ERR_SHAPE, dict(q=tensor(2, 1, 20000, 3, 64), qo=tensor(2, 1, 20000, 3, 64))),
])
def test_append_refusals(want, change):
    a = dict(q=tensor(*T["q"]), k=tensor(*T["k"]), v=tensor(*T["k"]), r=rotary(), n=norm(), kv=paged(), qo=tensor(*T["q"]), kc=pages(), vc=pages(), kh=None, vh=None)
    a.update(change)
    assert fb.fl_norm_rotary_append(*a.values()) == want, fb.fl_last_error_detail()
    assert fb.fl_last_error_detail()


CALLS = [fb.fl_attn_decode_mx4, fb.fl_attn_prefill_mx4]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("want,change", [
    (fb.FL_ERR_NULL, dict(q=None)), (fb.FL_ERR_NULL, dict(kc=None)), (fb.FL_ERR_NULL, dict(vc=None)), (fb.FL_ERR_NULL, dict(kv=None)), (fb.FL_ERR_NULL, dict(out=None)),
    (fb.FL_ERR_NULL, dict(d=None)), (fb.FL_ERR_NULL, dict(vc=pages(ptr=0))), (fb.FL_ERR_NULL, dict(kv=paged(lens=None))),
    (fb.FL_ERR_DESC, dict(d=fb.variant_desc(scale=0.0))), (fb.FL_ERR_AUX_MISSING, dict(a=None)), (fb.FL_ERR_AUX_MISSING, dict(d=fb.variant_desc(scale=1.0, score_mod=fb.FL_MOD_ALIBI))),
    (fb.FL_ERR_UNSUPPORTED, dict(d=fb.variant_desc(scale=1.0, mask=fb.FL_MASK_DOC))), (fb.FL_ERR_UNSUPPORTED, dict(d=fb.variant_desc(scale=1.0, mask=fb.FL_MASK_PREFIX))),
    (fb.FL_ERR_UNSUPPORTED, dict(d=fb.variant_desc(scale=1.0, q_offset=1))), (fb.FL_ERR_UNSUPPORTED, dict(q=tensor(2, 1, 4, 3, 96), out=tensor(2, 1, 4, 3, 96), kc=pages(D=96), vc=pages(D=96))),
    (fb.FL_ERR_DTYPE, dict(q=tensor(*T["q"], dtype=fb.FL_F32))), (fb.FL_ERR_DTYPE, dict(kc=tensor(20, 1, 2, 16, 64))), (fb.FL_ERR_DTYPE, dict(out=tensor(*T["q"], dtype=fb.FL_I32))),
    (fb.FL_ERR_DTYPE, dict(lse=tensor(2, 1, 4, 3, 1))), (fb.FL_ERR_SHAPE, dict(lse=tensor(2, 1, 4, 2, 1, dtype=fb.FL_F32))), (fb.FL_ERR_SHAPE, dict(out=tensor(2, 1, 4, 3, 32))),
    (fb.FL_ERR_SHAPE, dict(q=tensor(2, 1, 3, 3, 64), out=tensor(2, 1, 3, 3, 64))), (fb.FL_ERR_SHAPE, dict(q=tensor(2, 2, 4, 3, 64))), (fb.FL_ERR_SHAPE, dict(vc=pages(n=19))),
    (fb.FL_ERR_SHAPE, dict(kc=pages(page=4), vc=pages(page=4), kv=paged(page=4, max_len=16))), (fb.FL_ERR_SHAPE, dict(kv=paged(stride=2))),
    (fb.FL_ERR_SHAPE, dict(q=tensor(2, 1, 4, 1 << 31, 64))), (fb.FL_ERR_STRIDE, dict(kc=pages(stride={0: 1 << 32}))), (fb.FL_ERR_STRIDE, dict(vc=pages(stride={0: 544}))),
    (fb.FL_ERR_ALIGN, dict(vc=pages(stride={0: 1096}))), (fb.FL_ERR_ALIGN, dict(kc=pages(ptr=FAKE + 8))), (fb.FL_ERR_ALIGN, dict(a=aux(FAKE + 8), kv=paged(max_len=1 << 16, stride=1 << 12))),
    (fb.FL_ERR_WORKSPACE, dict(a=aux(0), kv=paged(max_len=1 << 16, stride=1 << 12))),
])
def test_attention_refusals(call, want, change):
    a = dict(q=tensor(*T["q"]), kc=pages(), vc=pages(), kv=paged(), d=fb.variant_desc(scale=0.125), a=aux(), out=tensor(*T["q"]), lse=None)
    a.update(change)
    assert call(*a.values()) == want, fb.fl_last_error_detail()
    assert fb.fl_last_error_detail()


def test_attention_workspaces():
    q, c, d = tensor(*T["q"]), pages(), fb.variant_desc(scale=0.125)
    decode, prefill = fb.fl_attn_decode_mx4_workspace_size, fb.fl_attn_prefill_mx4_workspace_size
    assert decode(q, c, paged()) == prefill(q, c, paged()) == 0                 # one split: no partial results
    long = paged(max_len=1 << 20, stride=1 << 16)
    need = decode(q, c, long)
    assert need == prefill(q, c, long) == 64 * 2 * 3 * 4 * 66 * 4
    for call in CALLS:
        assert call(q, c, c, long, d, aux(size=need - 1), q, None) == fb.FL_ERR_WORKSPACE
    assert fb.fl_set_tuning("decode_splits", 3) == fb.FL_OK
    assert decode(q, c, long) == 3 * 2 * 3 * 4 * 66 * 4
    assert fb.fl_set_tuning("decode_splits", 0) == fb.FL_OK
    assert decode(q, c, long) == need
    rows = tensor(2, 1, 4, 33, 64)                                              # 66 pairs of a kv head
    assert fb.fl_attn_decode_mx4(rows, c, c, paged(), d, aux(), rows, None) == fb.FL_ERR_SHAPE and "pairs" in fb.fl_last_error_detail()
    # more rows: room for either way, which the call chooses with the mask known
    assert prefill(rows, c, paged()) == 2 * 2 * 2 * 64 * 64 * 2 and prefill(rows, c, long) >= decode(rows, c, long) > 0
    many = tensor(64, 1, 4, 4000, 64)
    need = prefill(many, c, paged(max_len=4096, stride=256))
    assert need == 2 * 64 * 2 * 4096 * 64 * 2
    assert fb.fl_attn_prefill_mx4(many, c, c, paged(max_len=4096, stride=256), d, aux(size=need - 1), many, None) == fb.FL_ERR_WORKSPACE
    for size in (decode, prefill):
        assert size(None, c, long) == 0 and size(q, None, long) == 0 and size(q, c, None) == 0


def test_empty_calls_are_fine():
    d, none = fb.variant_desc(scale=0.125), tensor(0, 1, 4, 8, 64)
    assert fb.fl_norm_rotary(none, tensor(0, 1, 2, 8, 64), rotary(), norm(), none, tensor(0, 1, 2, 8, 64)) == fb.FL_OK
    assert fb.fl_norm_rotary_bwd(none, None, none, None, rotary(), norm(), none, None) == fb.FL_OK
    assert fb.fl_norm_rotary_bwd(tensor(*Q), None, tensor(*Q), None, rotary(), norm(), None, None) == fb.FL_OK           # nothing is wanted
    no_tokens = tensor(2, 1, 4, 0, 64)
    assert fb.fl_norm_rotary_append(no_tokens, tensor(2, 1, 2, 0, 64), tensor(2, 1, 2, 0, 64), rotary(), norm(), paged(), no_tokens, pages(), pages()) == fb.FL_OK
    for call in CALLS:
        assert call(no_tokens, pages(), pages(), paged(), d, None, no_tokens, None) == fb.FL_OK
        assert call(tensor(0, 1, 4, 3, 64), pages(), pages(), paged(lens=None), d, None, tensor(0, 1, 4, 3, 64), None) == fb.FL_OK


# ---- the PyTorch entry points ----


def test_entry_points_refuse_cpu_tensors():
    q, n = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    kc, vc = F.mx4_cache(2, 16, 2, 64, device="cpu")
    pos, inv = torch.zeros(1, 8, 1, dtype=torch.int32), torch.ones(32)
    for call in (lambda: F.norm_rotary(q, q, pos, inv), lambda: F.norm_rotary_append(q, q, q, pos, inv, kc, vc, n), lambda: F.decode_attention_mx4(q, kc, vc, n),
                 lambda: F.paged_prefill_attention_mx4(q, kc, vc, n)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_pages():
    k, v = F.mx4_cache(5, 24, 3, 128, device="cpu")
    assert k.shape == v.shape == (5, 3, 24 * 68) and k.dtype == torch.uint8 and not k.any() and k.data_ptr() != v.data_ptr()
    assert F.mx4_cache(0, 8, 1, 64, device="cpu")[0].shape == (0, 1, 8 * 34)
    for page, D in ((16, 96), (16, 0), (4, 64), (12, 64), (0, 64), (-8, 64)):
        with pytest.raises(ValueError):
            F.mx4_cache(5, page, 3, D, device="cpu")


U8 = torch.uint8


@pytest.mark.parametrize("change", [
    dict(k=torch.zeros(9, 2, 544)), dict(k=torch.zeros(9, 2, 16, 34, dtype=U8)), dict(v=torch.zeros(8, 2, 544, dtype=U8)), dict(v=torch.zeros(9, 2, 1088, dtype=U8)[..., ::2]),
    dict(k=torch.zeros(9, 2, 545, dtype=U8), v=torch.zeros(9, 2, 545, dtype=U8)), dict(k=torch.zeros(9, 2, 34 * 12, dtype=U8), v=torch.zeros(9, 2, 34 * 12, dtype=U8)),
    dict(k=torch.zeros(9, 2, 0, dtype=U8), v=torch.zeros(9, 2, 0, dtype=U8)), dict(q=torch.zeros(2, 4, 96)), dict(lens=torch.zeros(2, dtype=torch.int64)),
    dict(lens=torch.zeros(3, dtype=torch.int32)), dict(lens=None), dict(table=torch.zeros(2, 4, dtype=torch.int64)), dict(table=torch.zeros(8, dtype=torch.int32)),
    dict(table=torch.zeros(1, 4, dtype=torch.int32)), dict(bound=65), dict(bound=-1)])
def test_caches_that_no_call_takes(change):
    a = dict(q=torch.zeros(2, 4, 64), k=torch.zeros(9, 2, 544, dtype=U8), v=torch.zeros(9, 2, 544, dtype=U8), lens=torch.zeros(2, dtype=torch.int32),
             table=torch.zeros(2, 4, dtype=torch.int32), bound=None)
    assert F._check_cache_mx4(*a.values()) == (16, 64)
    assert F._check_cache_mx4(*dict(a, table=None, bound=7).values()) == (16, 7) and F._check_cache_mx4(*dict(a, table=None).values()) == (16, 16)
    a.update(change)
    with pytest.raises(ValueError):
        F._check_cache_mx4(*a.values())
