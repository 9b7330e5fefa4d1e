"""CPU tests of the refusals of the calls around a bounded key/value cache: through the C ABI (before any HIP call) and the PyTorch entry points."""
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
        step *= size[a]
    if stride is not None:
        for a, s in stride.items():
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


def paged(page=16, max_len=64, table=FAKE, stride=4, lens=FAKE):
    kv = fb.fl_paged_kv()
    kv.struct_size = ctypes.sizeof(fb.fl_paged_kv)
    kv.block_table, kv.table_stride, kv.page_size, kv.seq_lens, kv.max_seq_len = table, stride, page, lens, max_len
    return kv


def evict(budget=32, sinks=2, recent=4, stride=2, **kw):
    e = fb.fl_evict()
    e.struct_size, e.budget, e.sinks, e.recent, e.dst_stride = ctypes.sizeof(fb.fl_evict), budget, sinks, recent, stride
    e.dst_table = e.new_lens = e.kept = FAKE
    for n, x in kw.items():
        setattr(e, n, x)
    return e


def aux(ws=0, size=0, slopes=None):
    a = fb.fl_aux()
    a.struct_size, a.workspace, a.workspace_bytes, a.alibi_slopes = ctypes.sizeof(fb.fl_aux), ws or None, size, slopes
    return a


def test_struct_layouts_match_the_header(tmp_path):
    src = tmp_path / "sz.c"
    src.write_text('''#include <stdio.h>
#include <stddef.h>
#include "fl_attn.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(fl_rotary), offsetof(fl_rotary, positions), offsetof(fl_rotary, inv_freq), sizeof(fl_evict),
         offsetof(fl_evict, dst_table), offsetof(fl_evict, kept));
  return 0;
}''')
    exe = tmp_path / "sz"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert got == [ctypes.sizeof(fb.fl_rotary), fb.fl_rotary.positions.offset, fb.fl_rotary.inv_freq.offset, ctypes.sizeof(fb.fl_evict),
                   fb.fl_evict.dst_table.offset, fb.fl_evict.kept.offset]


Q, K = (2, 1, 4, 8, 64), (2, 1, 2, 8, 64)


@pytest.mark.parametrize("want,change", [
    (fb.FL_ERR_DESC, dict(r=rotary(struct_size=4))), (fb.FL_ERR_DESC, dict(r=rotary(axes=0))), (fb.FL_ERR_DESC, dict(r=rotary(axes=5))),
    (fb.FL_ERR_DESC, dict(r=rotary(axes=2, sections=(33, -1, 0, 0)))), (fb.FL_ERR_DESC, dict(r=rotary(inverse=2))), (fb.FL_ERR_DESC, dict(r=rotary(interleaved=7))),
    (fb.FL_ERR_SHAPE, dict(r=rotary(sections=(33, 0, 0, 0)))), (fb.FL_ERR_SHAPE, dict(r=rotary(sections=(0, 0, 0, 0)))),
    (fb.FL_ERR_SHAPE, dict(r=rotary(axes=2, sections=(2147483647, 2147483647, 0, 0)))),
    (fb.FL_ERR_NULL, dict(r=None)), (fb.FL_ERR_NULL, dict(r=rotary(positions=None))), (fb.FL_ERR_NULL, dict(r=rotary(inv_freq=None))),
    (fb.FL_ERR_NULL, dict(qo=None)), (fb.FL_ERR_NULL, dict(q=None, k=None, qo=None, ko=None)), (fb.FL_ERR_NULL, dict(q=tensor(*Q, ptr=0))),
    (fb.FL_ERR_DTYPE, dict(q=tensor(*Q, dtype=fb.FL_I32))), (fb.FL_ERR_DTYPE, dict(k=tensor(*K, dtype=fb.FL_F32))), (fb.FL_ERR_DTYPE, dict(qo=tensor(*Q, dtype=fb.FL_F32))),
    (fb.FL_ERR_SHAPE, dict(k=tensor(2, 1, 2, 7, 64))), (fb.FL_ERR_SHAPE, dict(qo=tensor(2, 1, 4, 8, 32))), (fb.FL_ERR_SHAPE, dict(q=tensor(2, 2, 4, 8, 64))),
    (fb.FL_ERR_SHAPE, dict(q=tensor(2, 1, -4, 8, 64))), (fb.FL_ERR_STRIDE, dict(q=tensor(*Q, stride={4: 2}))), (fb.FL_ERR_STRIDE, dict(q=tensor(*Q, stride={2: 0}))),
    (fb.FL_ERR_STRIDE, dict(q=tensor(*Q, stride={0: -64}))), (fb.FL_ERR_ALIGN, dict(q=tensor(*Q, ptr=FAKE + 2))), (fb.FL_ERR_ALIGN, dict(ko=tensor(*K, stride={3: 68}))),
    (fb.FL_ERR_SHAPE, dict(q=tensor(1 << 16, 1, 4, 1 << 16, 64), k=None, ko=None)), (fb.FL_ERR_SHAPE, dict(q=tensor(2, 1, 20000, 8, 64))),
])
def test_rotary_refusals(want, change):
    a = dict(q=tensor(*Q), k=tensor(*K), r=rotary(), qo=tensor(*Q), ko=tensor(*K))
    a.update(change)
    assert fb.fl_rotary_embed(a["q"], a["k"], a["r"], a["qo"], a["ko"]) == want, fb.fl_last_error_detail()
    assert fb.fl_last_error_detail()


CACHE = (20, 1, 2, 16, 64)
T = dict(q=(2, 1, 4, 3, 64), k=(2, 1, 2, 3, 64))


@pytest.mark.parametrize("want,change", [
    (fb.FL_ERR_NULL, dict(v=None)), (fb.FL_ERR_NULL, dict(kv=None)), (fb.FL_ERR_NULL, dict(kv=paged(lens=None))), (fb.FL_ERR_DESC, dict(r=rotary(inverse=1))),
    (fb.FL_ERR_SHAPE, dict(kv=paged(page=8))), (fb.FL_ERR_SHAPE, dict(kv=paged(stride=3))), (fb.FL_ERR_SHAPE, dict(kv=paged(table=None))),
    (fb.FL_ERR_SHAPE, dict(kv=paged(max_len=-1))), (fb.FL_ERR_SHAPE, dict(kc=tensor(20, 1, 2, 12, 64), kv=paged(page=12))),
    (fb.FL_ERR_SHAPE, dict(vc=tensor(20, 1, 2, 16, 32))), (fb.FL_ERR_DTYPE, dict(kc=tensor(*CACHE, dtype=fb.FL_F32))),
    (fb.FL_ERR_SHAPE, dict(k=tensor(2, 1, 4, 3, 64))), (fb.FL_ERR_DTYPE, dict(v=tensor(*T["k"], dtype=fb.FL_F32))), (fb.FL_ERR_SHAPE, dict(kc=tensor(0, 1, 2, 16, 64))),
])
def test_append_refusals(want, change):
    a = dict(q=tensor(*T["q"]), k=tensor(*T["k"]), v=tensor(*T["k"]), r=rotary(), kv=paged(), qo=tensor(*T["q"]), kc=tensor(*CACHE), vc=tensor(*CACHE))
    a.update(change)
    assert fb.fl_rotary_append(a["q"], a["k"], a["v"], a["r"], a["kv"], a["qo"], a["kc"], a["vc"]) == want, fb.fl_last_error_detail()


W = (2, 1, 2, 1, 64)


@pytest.mark.parametrize("want,w", [
    (fb.FL_ERR_NULL, None), (fb.FL_ERR_NULL, tensor(*W, dtype=fb.FL_F32, ptr=0)), (fb.FL_ERR_DTYPE, tensor(*W)), (fb.FL_ERR_SHAPE, tensor(2, 1, 2, 1, 63, dtype=fb.FL_F32)),
    (fb.FL_ERR_SHAPE, tensor(2, 1, 4, 1, 64, dtype=fb.FL_F32)), (fb.FL_ERR_STRIDE, tensor(*W, dtype=fb.FL_F32, stride={4: 2})),
    (fb.FL_ERR_STRIDE, tensor(*W, dtype=fb.FL_F32, stride={2: 0})), (fb.FL_ERR_STRIDE, tensor(*W, dtype=fb.FL_F32, stride={0: 32})),
    (fb.FL_ERR_ALIGN, tensor(*W, dtype=fb.FL_F32, ptr=FAKE + 2)),
])
def test_weights_that_no_call_takes(want, w):
    q, c, lse = tensor(2, 1, 4, 1, 64), tensor(*CACHE), tensor(2, 1, 4, 1, 1, dtype=fb.FL_F32)
    d = fb.variant_desc(scale=0.125)
    assert fb.fl_attn_decode_weights(q, c, c, paged(), d, aux(FAKE, 1 << 30), tensor(2, 1, 4, 1, 64), None, w) == want, fb.fl_last_error_detail()
    assert fb.fl_key_weights(q, c, lse, paged(), d, aux(FAKE, 1 << 30), w) == want, fb.fl_last_error_detail()
    assert fb.fl_cache_evict(w, c, c, paged(), evict(), tensor(2, 1, 2, 1, 40, dtype=fb.FL_F32, ptr=2 * FAKE)) == (want if w is None or w.size[2] == 2 else want)


@pytest.mark.parametrize("want,change", [
    (fb.FL_ERR_DESC, dict(d=fb.variant_desc(scale=0.0))), (fb.FL_ERR_UNSUPPORTED, dict(d=fb.variant_desc(scale=1.0, mask=fb.FL_MASK_DOC))),
    (fb.FL_ERR_UNSUPPORTED, dict(d=fb.variant_desc(scale=1.0, mask=fb.FL_MASK_PREFIX))), (fb.FL_ERR_UNSUPPORTED, dict(d=fb.variant_desc(scale=1.0, q_offset=1))),
    (fb.FL_ERR_AUX_MISSING, dict(d=fb.variant_desc(scale=1.0, score_mod=fb.FL_MOD_ALIBI))), (fb.FL_ERR_NULL, dict(lse=None)),
    (fb.FL_ERR_NULL, dict(lse=tensor(2, 1, 4, 300, 1, dtype=fb.FL_F32, ptr=0))), (fb.FL_ERR_DTYPE, dict(lse=tensor(2, 1, 4, 300, 1))),
    (fb.FL_ERR_SHAPE, dict(lse=tensor(2, 1, 4, 299, 1, dtype=fb.FL_F32))), (fb.FL_ERR_UNSUPPORTED, dict(q=tensor(2, 1, 4, 300, 96))),
    (fb.FL_ERR_SHAPE, dict(q=tensor(2, 1, 3, 300, 64))), (fb.FL_ERR_DTYPE, dict(q=tensor(2, 1, 4, 300, 64, dtype=fb.FL_F32))),
    (fb.FL_ERR_WORKSPACE, dict(a=aux())), (fb.FL_ERR_WORKSPACE, dict(a=None)), (fb.FL_ERR_ALIGN, dict(a=aux(FAKE + 8, 1 << 30))),
    (fb.FL_ERR_SHAPE, dict(kv=paged(stride=2))),
])
def test_key_weight_refusals(want, change):
    a = dict(q=tensor(2, 1, 4, 300, 64), c=tensor(*CACHE), lse=tensor(2, 1, 4, 300, 1, dtype=fb.FL_F32), kv=paged(), d=fb.variant_desc(scale=0.125),
             a=aux(FAKE, 1 << 30), w=tensor(*W, dtype=fb.FL_F32))
    a.update(change)
    assert fb.fl_key_weights(a["q"], a["c"], a["lse"], a["kv"], a["d"], a["a"], a["w"]) == want, fb.fl_last_error_detail()


def test_decode_weights_need_their_workspace():
    q, c, w = tensor(2, 1, 4, 1, 64), tensor(*CACHE), tensor(*W, dtype=fb.FL_F32)
    need = fb.fl_attn_decode_weights_workspace_size(q, c, paged())
    assert need >= fb.fl_attn_decode_workspace_size(q, c, paged()) + 2 * 4 * 64 * 4
    d = fb.variant_desc(scale=0.125)
    call = lambda a: fb.fl_attn_decode_weights(q, c, c, paged(), d, a, tensor(2, 1, 4, 1, 64), None, w)
    assert call(aux(FAKE, need - 1)) == fb.FL_ERR_WORKSPACE and call(None) == fb.FL_ERR_AUX_MISSING
    assert fb.fl_attn_decode_weights_workspace_size(None, c, paged()) == 0 and fb.fl_key_weights_workspace_size(q, None, paged()) == 0


@pytest.mark.parametrize("want,change", [
    (fb.FL_ERR_DESC, dict(e=evict(budget=0))), (fb.FL_ERR_DESC, dict(e=evict(sinks=-1))), (fb.FL_ERR_DESC, dict(e=evict(recent=-1))),
    (fb.FL_ERR_DESC, dict(e=evict(sinks=30, recent=3))), (fb.FL_ERR_DESC, dict(e=evict(sinks=2147483647, recent=2147483647))), (fb.FL_ERR_DESC, dict(e=evict(struct_size=8))),
    (fb.FL_ERR_SHAPE, dict(e=evict(stride=1))), (fb.FL_ERR_NULL, dict(e=evict(dst_table=None))), (fb.FL_ERR_NULL, dict(e=evict(kept=None))),
    (fb.FL_ERR_NULL, dict(e=evict(new_lens=None))), (fb.FL_ERR_NULL, dict(e=None)), (fb.FL_ERR_NULL, dict(vc=None)),
    (fb.FL_ERR_SHAPE, dict(nw=tensor(2, 1, 2, 1, 31, dtype=fb.FL_F32))), (fb.FL_ERR_DESC, dict(nw=tensor(*W, dtype=fb.FL_F32))),
    (fb.FL_ERR_UNSUPPORTED, dict(c=tensor(20, 1, 2, 16, 60))), (fb.FL_ERR_SHAPE, dict(c=tensor(20, 1, 2, 20, 64), vc=tensor(20, 1, 2, 20, 64), kv=paged(page=20, max_len=20, table=None))),
    (fb.FL_ERR_SHAPE, dict(vc=tensor(20, 1, 3, 16, 64))),
])
def test_evict_refusals(want, change):
    a = dict(w=tensor(*W, dtype=fb.FL_F32), c=tensor(*CACHE), vc=tensor(*CACHE), kv=paged(), e=evict(), nw=tensor(2, 1, 2, 1, 40, dtype=fb.FL_F32, ptr=2 * FAKE))
    a.update(change)
    assert fb.fl_cache_evict(a["w"], a["c"], a["vc"], a["kv"], a["e"], a["nw"]) == want, fb.fl_last_error_detail()


def test_empty_calls_are_fine():
    d = fb.variant_desc(scale=0.125)
    assert fb.fl_rotary_embed(tensor(0, 1, 4, 8, 64), tensor(0, 1, 2, 8, 64), rotary(), tensor(0, 1, 4, 8, 64), tensor(0, 1, 2, 8, 64)) == fb.FL_OK
    assert fb.fl_rotary_append(tensor(2, 1, 4, 0, 64), tensor(2, 1, 2, 0, 64), tensor(2, 1, 2, 0, 64), rotary(), paged(), tensor(2, 1, 4, 0, 64), tensor(*CACHE),
                               tensor(*CACHE)) == fb.FL_OK
    assert fb.fl_key_weights(tensor(2, 1, 4, 0, 64), tensor(*CACHE), tensor(2, 1, 4, 0, 1, dtype=fb.FL_F32), paged(), d, None, tensor(*W, dtype=fb.FL_F32)) == fb.FL_OK
    assert fb.fl_cache_evict(tensor(0, 1, 2, 1, 64, dtype=fb.FL_F32), tensor(*CACHE), tensor(*CACHE), paged(), evict(), tensor(0, 1, 2, 1, 40, dtype=fb.FL_F32)) == fb.FL_OK


def test_entry_points_refuse_cpu_tensors():
    q, w, n = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 16), torch.zeros(1, dtype=torch.int32)
    c = torch.zeros(1, 16, 2, 64, dtype=torch.bfloat16)
    pos, inv = torch.zeros(1, 8, 1, dtype=torch.int32), torch.ones(32)
    for call in (lambda: F.rotary(q, q, pos, inv), lambda: F.rotary_append(q, q, q, pos, inv, c, c, n), lambda: F.decode_attention_weights(q, c, c, w, n),
                 lambda: F.prefill_key_weights(q, c, w, w, n), lambda: F.evict_cache(w, c, c, n, None, n[None], 8)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("change", [dict(positions=torch.zeros(2, 8, 1)), dict(positions=torch.zeros(2, 8, dtype=torch.int32)), dict(positions=torch.zeros(2, 7, 1, dtype=torch.int32)),
                                    dict(positions=torch.zeros(3, 8, 1, dtype=torch.int32)), dict(inv_freq=torch.ones(32, dtype=torch.float64)), dict(inv_freq=torch.ones(64)[::2]),
                                    dict(sections=(16, 16)), dict(sections=(31,)), dict(sections=(33, -1), positions=torch.zeros(2, 8, 2, dtype=torch.int32)),
                                    dict(k=torch.zeros(2, 1, 7, 64)), dict(k=torch.zeros(2, 1, 8, 64, dtype=torch.bfloat16)), dict(inv_freq=None), dict(positions=None)])
def test_positions_that_rotary_refuses(change):
    a = dict(q=torch.zeros(2, 4, 8, 64), k=torch.zeros(2, 1, 8, 64), positions=torch.zeros(2, 8, 1, dtype=torch.int32), inv_freq=torch.ones(32), sections=None)
    assert F._check_rotary(*a.values(), 2, 8)[1] == (32,)
    assert F._check_rotary(a["q"], None, a["positions"][:1], a["inv_freq"], None, 2, 8)[0].shape == (2, 8, 1)
    a.update(change)
    with pytest.raises(ValueError):
        F._check_rotary(*a.values(), 2, 8)


@pytest.mark.parametrize("change", [dict(k=torch.zeros(9, 16, 2, 64)), dict(v=torch.zeros(9, 16, 1, 64, dtype=torch.bfloat16)), dict(lens=torch.zeros(2, dtype=torch.int64)),
                                    dict(table=torch.zeros(2, 4, dtype=torch.int64)), dict(table=torch.zeros(8, dtype=torch.int32)), dict(bound=65)])
def test_caches_that_no_call_takes(change):
    a = dict(q=torch.zeros(2, 4, 64), k=torch.zeros(9, 16, 2, 64, dtype=torch.bfloat16), v=torch.zeros(9, 16, 2, 64, dtype=torch.bfloat16), lens=torch.zeros(2, dtype=torch.int32),
             table=torch.zeros(2, 4, dtype=torch.int32), bound=None)
    assert F._check_cache(*a.values()) == 64
    a.update(change)
    with pytest.raises(ValueError):
        F._check_cache(*a.values())
