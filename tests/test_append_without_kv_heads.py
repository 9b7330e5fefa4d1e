"""CPU test: fl_rotary_append with queries alone.  The kernel reads the lengths for them too, so a NULL is refused before any HIP call."""
import ctypes

from paper_2511_02043_amd import binding as fb

FAKE = 1 << 20


def tensor(*size):
    t = fb.fl_tensor()
    t.ptr, t.dtype = FAKE, fb.FL_BF16
    t.size[:] = size
    step = 1
    for a in range(4, -1, -1):
        t.stride[a] = step
        step *= max(size[a], 1)
    return t


def test_lengths_are_needed():
    r, kv = fb.fl_rotary(), fb.fl_paged_kv()
    r.struct_size, r.axes, r.positions, r.inv_freq = ctypes.sizeof(fb.fl_rotary), 1, FAKE, FAKE
    r.sections[:] = (32, 0, 0, 0)
    kv.struct_size, kv.block_table, kv.table_stride, kv.page_size, kv.max_seq_len = ctypes.sizeof(fb.fl_paged_kv), FAKE, 4, 16, 64
    q, new, cache = tensor(2, 1, 4, 3, 64), tensor(2, 1, 0, 3, 64), tensor(20, 1, 0, 16, 64)
    assert kv.seq_lens is None
    assert fb.fl_rotary_append(q, new, new, r, kv, q, cache, cache) == fb.FL_ERR_NULL
    assert "seq_lens" in fb.fl_last_error_detail()
