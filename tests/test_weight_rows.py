"""CPU tests: weights whose rows lie over each other, which workgroups would add to at the same time, are refused before any HIP call; the rule,
compiled for the host, against sets of elements."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2511_02043_amd import binding as fb

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_02043_amd", "csrc")
AT = 1 << 20


def tensor(size, dtype=fb.FL_BF16, at=AT, stride=None):
    t = fb.fl_tensor()
    t.ptr, t.dtype = at, dtype
    t.size[:] = size
    step = 1
    for a in range(4, -1, -1):
        t.stride[a] = step
        step *= size[a]
    for a, s in (stride or {}).items():
        t.stride[a] = s
    return t


# 3 sequences, 4 kv heads, rows of 64: the rows (0, 1) and (1, 0), (0, 3) and (2, 0), (1, 2) and (2, 0)
@pytest.mark.parametrize("stride", [{0: 64, 2: 64}, {0: 96, 2: 64}, {0: 127, 2: 64}, {0: 64, 2: 128}])
def test_rows_that_overlap(stride):
    kv, a, e = fb.fl_paged_kv(), fb.fl_aux(), fb.fl_evict()
    kv.struct_size, kv.block_table, kv.table_stride, kv.page_size, kv.seq_lens, kv.max_seq_len = ctypes.sizeof(fb.fl_paged_kv), AT, 4, 16, AT, 64
    a.struct_size, a.workspace, a.workspace_bytes = ctypes.sizeof(fb.fl_aux), AT, 1 << 30
    e.struct_size, e.budget, e.dst_table, e.dst_stride, e.new_lens, e.kept = ctypes.sizeof(fb.fl_evict), 64, 2 * AT, 4, 3 * AT, 4 * AT
    q, c, d = tensor((3, 1, 8, 1, 64)), tensor((20, 1, 4, 16, 64)), fb.variant_desc(scale=0.125)
    w, apart = tensor((3, 1, 4, 1, 64), fb.FL_F32, 5 * AT, stride), tensor((3, 1, 4, 1, 64), fb.FL_F32, 6 * AT)
    for call in (lambda: fb.fl_attn_decode_weights(q, c, c, kv, d, a, q, None, w), lambda: fb.fl_key_weights(q, c, tensor((3, 1, 8, 1, 1), fb.FL_F32), kv, d, a, w),
                 lambda: fb.fl_cache_evict(apart, c, c, kv, e, w)):
        assert call() == fb.FL_ERR_STRIDE
        assert "rows overlap" in fb.fl_last_error_detail()


SOURCE = r"""
#include <cstdio>
#include <random>
#include "fl_host.hpp"
int main() {
  std::mt19937 rng(1);
  for (int n = 0; n < 300000; ++n) {
    const int n0 = 1 + rng() % 5, n1 = 1 + rng() % 5, len = 1 + rng() % 6, s0 = len + rng() % 40, s1 = len + rng() % 40;
    int count[600] = {};
    bool want = false;
    for (int i = 0; i < n0; ++i)
      for (int j = 0; j < n1; ++j)
        for (int u = 0; u < len; ++u) want = ++count[i * s0 + j * s1 + u] > 1 || want;
    if (fl::host::rows_overlap(n0, s0, n1, s1, len) != want) {
      std::printf("%d x %d rows of %d, %d and %d apart\n", n0, n1, len, s0, s1);
      return 1;
    }
  }
  return fl::host::rows_overlap(2, INT64_MAX, 3, INT64_MAX, 4) ? 0 : 1;
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_rows_against_sets_of_elements(tmp_path):
    src, exe = tmp_path / "rows.hip", tmp_path / "rows"
    src.write_text(SOURCE)
    subprocess.check_call(["hipcc", "-std=c++17", "-O2", "--cuda-host-only", "-I" + CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)]).returncode == 0
