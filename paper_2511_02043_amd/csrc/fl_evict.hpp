// Eviction from a paged key/value cache by accumulated attention weight, for gfx950.
//
// Of every (sequence, kv head) the first `sinks` slots, the newest `recent`, and of the others the heaviest stay, `budget` in all:
//   * evict_select_kernel, a workgroup per (sequence, kv head), finds the weight T at which the count is reached by a radix selection
//     (four histograms of eight bits, on a key that orders floats as whole numbers), then walks the slots in order: what is above T stays,
//     what equals T stays while it is needed, which leaves ties to the lower slots, and two prefix sums give each its place in the result;
//   * evict_move_kernel copies the rows that stay: no row has two readers or two writers, pages of the result are pages that nothing is
//     read from, so the copy needs no order and runs over all of them at once.
// Bound by the copy: 8 D bytes read and written per row and kv head beside the 4 bytes of a weight.
#pragma once
#include "fl_params.hpp"

namespace fl {

struct EvictParams {
  const float* weights;            // [B, Hkv, C]
  int64_t w_sb, w_sh;
  float* new_weights;              // [B, Hkv, C2]
  int64_t nw_sb, nw_sh;
  int32_t* kept;                   // [B, Hkv, budget]
  int32_t* new_lens;               // [B]
  uint16_t* k_cache;               // page, token in page, kv head strides in elements
  uint16_t* v_cache;
  int64_t k_sp, k_st, k_sh, v_sp, v_st, v_sh;
  const int32_t* block_table;      // [B, table_stride], or null: sequence b is page b
  const int32_t* dst_table;        // [B, dst_stride]
  int32_t table_stride, dst_stride, page_shift, num_pages, max_len;
  const int32_t* seq_lens;
  int32_t B, Hkv, D, budget, sinks, recent, capacity;
  int32_t pieces;                  // 16-byte pieces of a row
  Divisor by_hkv, by_groups, by_pieces;   // Hkv; workgroups of a (sequence, kv head); pieces
  int32_t rows_per_block;
};

// Whole numbers in the order of the weights: NaN below -inf, both zeros alike.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int kSelectThreads = 1024;

__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const EvictParams p) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t wave_sum[2][kSelectThreads / 64];
  __shared__ uint32_t chosen[2];                   // digit, count above it
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int b, h;
  p.by_hkv.split(blockIdx.x, b, h);
  const int len = min(max(p.seq_lens[b], 0), p.max_len);
  const int n_keep = min(len, p.budget);
  const float* w = p.weights + b * p.w_sb + h * p.w_sh;
  float* nw = p.new_weights + b * p.nw_sb + h * p.nw_sh;
  int32_t* kept = p.kept + ((int64_t)b * p.Hkv + h) * p.budget;
  if (h == 0 && tid == 0) p.new_lens[b] = n_keep;
  for (int r = n_keep + tid; r < p.capacity; r += kSelectThreads) nw[r] = 0.f;
  for (int r = n_keep + tid; r < p.budget; r += kSelectThreads) kept[r] = -1;
  if (len <= p.budget) {                           // everything stays where it is in the order
    for (int j = tid; j < len; j += kSelectThreads) {
      kept[j] = j;
      nw[j] = w[j];
    }
    return;
  }
  // slots [lo, hi) compete for `need` places (sinks + recent <= budget < len)
  const int lo = p.sinks, hi = len - p.recent;
  int need = p.budget - p.sinks - p.recent;
  uint32_t prefix = 0;
  int more = need;                                 // places left for keys that agree with `prefix` in the digits seen
  for (int shift = 24; shift >= 0 && need > 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
    for (int j = lo + tid; j < hi; j += kSelectThreads) {
      const uint32_t key = weight_key(w[j]);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid < 64) {                                // digit d: lane 63 - d / 4, so that a prefix sum over lanes counts from the top
      const int d0 = 4 * (63 - lane);
      const uint32_t c3 = hist[d0 + 3], c2 = hist[d0 + 2], c1 = hist[d0 + 1], c0 = hist[d0];
      uint32_t above = c0 + c1 + c2 + c3;
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(above, o);
        if (lane >= o) above += x;
      }
      above -= c0 + c1 + c2 + c3;                  // keys in higher lanes' digits
      const uint32_t want = (uint32_t)more;
      uint32_t a = above;
      const uint32_t c[4] = {c3, c2, c1, c0};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (a < want && a + c[u] >= want) {
          chosen[0] = (uint32_t)(d0 + 3 - u);
          chosen[1] = a;
        }
        a += c[u];
      }
    }
    __syncthreads();
    prefix |= chosen[0] << shift;
    more -= (int)chosen[1];
    __syncthreads();
  }
  // `prefix` is T; `more` of the keys that equal it stay
  uint32_t ties_before = 0, kept_before = 0;
  for (int j0 = 0; j0 < len; j0 += kSelectThreads) {
    const int j = j0 + tid;
    const bool in = j < len;
    const float x = in ? w[j] : 0.f;
    const bool competes = in && j >= lo && j < hi;
    const uint32_t key = weight_key(x);
    const bool tie = competes && need > 0 && key == prefix;
    const uint64_t tie_mask = __ballot(tie);
    if (lane == 0) wave_sum[0][wave] = __popcll(tie_mask);
    __syncthreads();
    uint32_t before = ties_before, all = 0;
    for (int u = 0; u < kSelectThreads / 64; ++u) {
      if (u < wave) before += wave_sum[0][u];
      all += wave_sum[0][u];
    }
    before += __popcll(tie_mask & ((1ull << lane) - 1));
    ties_before += all;
    const bool stays = in && (!competes || (need > 0 && key > prefix) || (tie && before < (uint32_t)more));
    const uint64_t stay_mask = __ballot(stays);
    if (lane == 0) wave_sum[1][wave] = __popcll(stay_mask);
    __syncthreads();
    uint32_t at = kept_before, sum = 0;
    for (int u = 0; u < kSelectThreads / 64; ++u) {
      if (u < wave) at += wave_sum[1][u];
      sum += wave_sum[1][u];
    }
    at += __popcll(stay_mask & ((1ull << lane) - 1));
    kept_before += sum;
    if (stays) {
      kept[at] = j;
      nw[at] = x;
    }
  }
}

// 16 bytes of a key row and of a value row per thread and step.
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictParams p) {
  int bh, group, b, h;
  p.by_groups.split(blockIdx.x, bh, group);
  p.by_hkv.split(bh, b, h);
  const int len = min(max(p.seq_lens[b], 0), p.max_len);
  const int n_keep = min(len, p.budget);
  const int r0 = group * p.rows_per_block, r1 = min(n_keep, r0 + p.rows_per_block);
  const int32_t* kept = p.kept + (int64_t)bh * p.budget;
  const int in_page = (1 << p.page_shift) - 1;
  for (int e = threadIdx.x; e < (r1 - r0) * p.pieces; e += 256) {
    int row, piece;
    p.by_pieces.split(e, row, piece);
    const int r = r0 + row;
    const int j = kept[r];
    int64_t page = b, off = j;
    if (p.block_table != nullptr) {
      page = min(max(p.block_table[(int64_t)b * p.table_stride + (j >> p.page_shift)], 0), p.num_pages - 1);
      off = j & in_page;
    }
    const int to = p.dst_table[(int64_t)b * p.dst_stride + (r >> p.page_shift)];
    if (to < 0 || to >= p.num_pages) continue;
    const uint4 x = *(const uint4*)(p.k_cache + page * p.k_sp + off * p.k_st + h * p.k_sh + piece * 8);
    const uint4 y = *(const uint4*)(p.v_cache + page * p.v_sp + off * p.v_st + h * p.v_sh + piece * 8);
    *(uint4*)(p.k_cache + (int64_t)to * p.k_sp + (int64_t)(r & in_page) * p.k_st + h * p.k_sh + piece * 8) = x;
    *(uint4*)(p.v_cache + (int64_t)to * p.v_sp + (int64_t)(r & in_page) * p.v_st + h * p.v_sh + piece * 8) = y;
  }
}

}  // namespace fl
