"""CPU tests: memory that two arguments of a call over the bounded cache share, where workgroups would read what others write.  The calls return before
any HIP call; the comparison of strided rows, compiled for the host, against sets of bytes."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2511_02043_amd import binding as fb

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_02043_amd", "csrc")
PART = 1 << 20                                     # the arguments, far apart; no call gets as far as reading them
NAMES = ["lens", "table", "dst", "new_lens", "kept", "weights", "new_weights", "k", "v"]
B, HKV, D, PAGE, MAX_LEN, BUDGET = 2, 2, 64, 16, 64, 32


def tensor(ptr, size, dtype, stride=None):
    t = fb.fl_tensor()
    t.ptr, t.dtype = ptr, dtype
    t.size[:] = size
    step = 1
    for a in range(4, -1, -1):
        t.stride[a] = step
        step *= size[a]
    for a, s in (stride or {}).items():
        t.stride[a] = s
    return t


def evict(weights_stride=None, new_stride=None, capacity=40, **moved):
    at = {n: (i + 1) * PART for i, n in enumerate(NAMES)}
    at.update(moved)
    kv = fb.fl_paged_kv()
    kv.struct_size = ctypes.sizeof(fb.fl_paged_kv)
    kv.block_table, kv.table_stride, kv.page_size, kv.seq_lens, kv.max_seq_len = at["table"], 8, PAGE, at["lens"], MAX_LEN
    e = fb.fl_evict()
    e.struct_size, e.budget, e.sinks, e.recent, e.dst_table, e.dst_stride = ctypes.sizeof(fb.fl_evict), BUDGET, 2, 4, at["dst"], 8
    e.new_lens, e.kept = at["new_lens"], at["kept"]
    cache = (20, 1, HKV, PAGE, D)
    return fb.fl_cache_evict(tensor(at["weights"], (B, 1, HKV, 1, MAX_LEN), fb.FL_F32, weights_stride), tensor(at["k"], cache, fb.FL_BF16),
                             tensor(at["v"], cache, fb.FL_BF16), kv, e, tensor(at["new_weights"], (B, 1, HKV, 1, capacity), fb.FL_F32, new_stride))


LENS, TABLE, DST, NEW_LENS, KEPT, WEIGHTS, NEW_WEIGHTS = (PART * (i + 1) for i in range(7))


@pytest.mark.parametrize("names,moved", [
    ("new_lens and seq_lens", dict(new_lens=LENS)), ("new_lens and seq_lens", dict(new_lens=LENS - 4)), ("new_lens and seq_lens", dict(lens=NEW_LENS - 4)),
    ("kept and seq_lens", dict(lens=KEPT + 4 * B * HKV * BUDGET - 4)), ("new_lens and kept", dict(new_lens=KEPT + 8)),
    ("new_lens and block_table", dict(new_lens=TABLE + 4 * 3)), ("new_lens and block_table", dict(new_lens=TABLE + 4 * 10)),
    ("new_lens and dst_table", dict(new_lens=DST)), ("kept and new_weights", dict(kept=NEW_WEIGHTS)), ("new_weights and weights", dict(new_weights=WEIGHTS + 4)),
    ("new_weights and weights", dict(new_weights=WEIGHTS - 4 * 40)), ("new_weights and weights", dict(new_weights=WEIGHTS + 4 * (B * HKV * MAX_LEN - 1))),
    ("new_weights and weights", dict(weights_stride={0: 208, 2: 104}, new_stride={0: 208, 2: 104}, new_weights=WEIGHTS + 4 * 63)),
    ("new_weights and seq_lens", dict(lens=NEW_WEIGHTS)),
])
def test_arguments_that_share_memory(names, moved):
    assert evict(**moved) == fb.FL_ERR_DESC
    assert names in fb.fl_last_error_detail()


SOURCE = r"""
#include <cstdio>
#include <random>
#include "fl_host.hpp"
using namespace fl::host;
int main() {
  std::mt19937 rng(1);
  for (int n = 0; n < 300000; ++n) {
    bool in[2][400] = {};
    Rows rows[2];
    for (int k = 0; k < 2; ++k) {
      Rows& r = rows[k];
      r.at = 1000 + rng() % 60;
      r.n0 = 1 + rng() % 4, r.n1 = 1 + rng() % 4, r.bytes = 1 + rng() % 6;
      r.s0 = r.n0 == 1 && rng() % 2 ? 0 : r.bytes + rng() % 30;
      r.s1 = r.n1 == 1 && rng() % 2 ? 0 : r.bytes + rng() % 30;
      for (int i = 0; i < r.n0; ++i)
        for (int j = 0; j < r.n1; ++j)
          for (int u = 0; u < r.bytes; ++u) in[k][r.at - 1000 + i * r.s0 + j * r.s1 + u] = true;
    }
    bool want = false;
    for (int i = 0; i < 400; ++i) want = want || (in[0][i] && in[1][i]);
    if (rows_meet(rows[0], rows[1]) != want) {
      std::printf("case %d\n", n);
      return 1;
    }
  }
  const Rows far = {1000, 2, INT64_MAX, 2, INT64_MAX, 4}, none = {1000, 0, 8, 1, 0, 4};
  return rows_meet(far, flat_rows((void*)8, 4)) && !rows_meet(none, flat_rows((void*)1000, 4)) ? 0 : 1;
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_rows_against_sets_of_bytes(tmp_path):
    src, exe = tmp_path / "rows.hip", tmp_path / "rows"
    src.write_text(SOURCE)
    subprocess.check_call(["hipcc", "-std=c++17", "-O2", "--cuda-host-only", "-I" + CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)]).returncode == 0
