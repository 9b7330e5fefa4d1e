"""CPU tests of the workspace that a chunk over the 4-bit cache needs: that of the way which its rows take, and no call takes less (before any HIP call)."""
import ctypes

import pytest

from paper_2511_02043_amd import binding as fb

FAKE = 1 << 20                                     # an aligned address that no call gets as far as reading
size_for, size_any = fb.fl_attn_prefill_mx4_workspace_size_for, fb.fl_attn_prefill_mx4_workspace_size


def tensor(*size, dtype=fb.FL_BF16):
    t = fb.fl_tensor()
    t.ptr, t.dtype = FAKE, dtype
    t.size[:] = size
    step = 1
    for a in range(4, -1, -1):
        t.stride[a] = step
        step *= max(size[a], 1)
    return t


def pages(n, Hkv, page, D):
    each = page * (D // 2 + D // 32)
    t = tensor(n, 1, Hkv, page, D, dtype=fb.FL_MX4)
    t.stride[:] = [Hkv * each, 0, each, 0, 1]
    return t


def paged(max_len, page=16):
    kv = fb.fl_paged_kv()
    kv.struct_size = ctypes.sizeof(fb.fl_paged_kv)
    kv.block_table, kv.table_stride, kv.page_size, kv.seq_lens, kv.max_seq_len = FAKE, -(-max_len // page), page, FAKE, max_len
    return kv


def aux(size):
    a = fb.fl_aux()
    a.struct_size, a.workspace, a.workspace_bytes = ctypes.sizeof(fb.fl_aux), FAKE, size
    return a


def desc(window=None, **kw):
    return fb.variant_desc(scale=0.125, mask=fb.FL_MASK_CAUSAL if window is None else fb.FL_MASK_WINDOW, window=window or 0, **kw)


def test_rows_that_go_through_the_decode_kernels_need_no_dense_copies():
    """64 sequences of 64 rows under a bound of 131072 tokens, as a wide table has without max_seq_len."""
    q, c, kv = tensor(64, 1, 32, 64, 128), pages(4096, 8, 16, 128), paged(131072)
    assert size_any(q, c, kv) == 2 * 64 * 8 * 131072 * 128 * 2
    for d in (desc(), desc(window=512), desc(score_mod=fb.FL_MOD_SOFTCAP, softcap=30.0)):
        assert size_for(q, c, kv, d) < 64 << 20


CASES = [(B, H, Hkv, T, D, L) for B in (1, 3, 64) for H, Hkv in ((8, 8), (16, 2), (32, 8)) for T in (1, 8, 17, 64, 500, 4000) for D in (64, 128) for L in (8, 700, 9000, 131072)]


@pytest.mark.parametrize("splits,gather", [(0, 0), (0, 1), (3, 0), (64, 0)])
def test_it_is_what_the_call_asks_for(splits, gather):
    """Never more than the size for any mask; one byte less is refused, as is none at all."""
    assert fb.fl_set_tuning("decode_splits", splits) == fb.fl_set_tuning("prefill_gather", gather) == fb.FL_OK
    try:
        ways = set()
        for B, H, Hkv, T, D, L in CASES:
            q, c, kv = tensor(B, 1, H, T, D), pages(B * -(-L // 16), Hkv, 16, D), paged(L)
            most = size_any(q, c, kv)
            for d in (desc(), desc(window=0), desc(window=512), desc(window=(1 << 31) - 1)):
                need = size_for(q, c, kv, d)
                assert 0 <= need <= most, (B, H, Hkv, T, D, L, d.window)
                if need > 0:
                    assert fb.fl_attn_prefill_mx4(q, c, c, kv, d, aux(need - 1), q, None) == fb.FL_ERR_WORKSPACE
                    assert f"needs {need} bytes" in fb.fl_last_error_detail()
                ways.add("none" if need == 0 else "copies" if need == 2 * ((B * Hkv * L * D * 2 + 255) // 256 * 256) else "partial results")
        assert ways == ({"copies"} if gather else {"none", "copies", "partial results"})
    finally:
        assert fb.fl_set_tuning("decode_splits", 0) == fb.fl_set_tuning("prefill_gather", 0) == fb.FL_OK


def test_nothing_for_calls_that_are_refused_or_have_nothing_to_do():
    q, c, kv = tensor(8, 1, 32, 4000, 64), pages(2000, 8, 16, 64), paged(4000)
    assert size_for(q, c, kv, desc()) > 0
    for args in ((None, c, kv, desc()), (q, None, kv, desc()), (q, c, None, desc()), (q, c, kv, None), (q, c, kv, fb.variant_desc(scale=0.0)), (q, c, kv, desc(window=-1)),
                 (q, c, paged(-1), desc()), (q, pages(2000, 0, 16, 64), kv, desc())):
        assert size_for(*args) == 0 and not fb.fl_last_error_detail()
    for axis, n in ((0, 0), (0, -1), (2, 0), (3, 0), (3, -5), (4, 0)):
        x = tensor(8, 1, 32, 4000, 64)
        x.size[axis] = n
        assert size_for(x, c, kv, desc()) == 0
