// Eviction from a paged key/value cache by accumulated attention weight, for gfx950.
//
// Of every (sequence, kv head) the first `sinks` slots, the newest `recent`, and of the others the heaviest stay, `budget` in all:
//   * evict_select_kernel, a workgroup per (sequence, kv head), finds the weight T at which the count is reached by a radix selection
//     (three histograms of up to eleven bits, on a key that orders floats as whole numbers: the first digit has two bits of mantissa,
//     since accumulated weights share few exponents and a wave's additions to one bin go one after the other), then walks the slots in
//     order: what is above T stays, what equals T stays while it is needed, which leaves ties to the lower slots.  The weights are read once
//     and wait in LDS;
//   * evict_move_kernel copies the rows that stay: no row has two readers or two writers, pages of the result are pages that nothing is
//     read from, so the copy needs no order and runs over all of them at once.
// The copy moves 8 D bytes per row and kv head, beside the 4 bytes of a weight: at D = 128 64 sequences x 8 heads x 2048 rows in 220 us (4.9 TB/s, what a
// large copy reaches), 8 x 8 x 2048 in 24.  The selection has a compute unit per (sequence, kv head): 12 us for 64 x 8 of 2049 - 2304 slots,
// 28 for 8 x 8 of 16k - 32k, 7 for one short sequence, which is its chain of loads and barriers.  (Three copies of the first histogram, one per
// lane modulo three, changed nothing: additions to one bin are not what holds it.)
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

constexpr int kSelectBins = 2048;                  // digits of 11, 11 and 10 bits
constexpr int kSelectHeld = 32768;                 // slots whose weights fit into LDS beside the histograms

struct SelectShared {                              // in front of the weights that wait in LDS
  uint32_t hist[3][kSelectBins];
  uint32_t wave_sum[3][16], wave_ties[16], wave_sures[16];
  uint32_t chosen[3][2];                           // digit, keys above it
};

__device__ __forceinline__ float weight_of_key(uint32_t key) {
  return key == 0u ? __uint_as_float(0x7fc00000u) : __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

// Inclusive prefix sum over a wave, by the data paths between lanes (no trip through LDS).
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);   // from 1, 2, 4, 8 lanes below in a row of 16
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);   // row 0 -> 1, 2 -> 3: their last lane
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);   // rows 0, 1 -> 2, 3
  return x;
}

// HELD: the keys wait in LDS between the walks over them, else the weights are read again.  A wave owns a run of the competing slots and walks it
// 64 at a time, so that an order over the workgroup is an order over waves: counts in a wave are popcounts of a ballot, and only wave totals
// cross it.  A walk is bound by instructions (64 slots of a wave are four cycles each), so its steps are short: slots that compete are a
// range of their own, keys are formed once, and only a run's last step looks where the run ends.
template <int THREADS, bool HELD>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(const EvictParams p) {
  constexpr int WAVES = THREADS / 64, BPT = kSelectBins / THREADS;             // bins per thread
  extern __shared__ __attribute__((aligned(16))) unsigned char select_lds[];
  SelectShared& sh = *(SelectShared*)select_lds;
  uint32_t* const held = (uint32_t*)(select_lds + sizeof(SelectShared));
  static_assert(WAVES <= 16 && sizeof(SelectShared) + kSelectHeld * sizeof(uint32_t) <= 160 * 1024, "LDS of the selection");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int b, h;
  p.by_hkv.split(blockIdx.x, b, h);
  const int len = min(max(p.seq_lens[b], 0), p.max_len);
  const int n_keep = min(len, p.budget);
  const float* w = p.weights + b * p.w_sb + h * p.w_sh;
  float* nw = p.new_weights + b * p.nw_sb + h * p.nw_sh;
  int32_t* kept = p.kept + ((int64_t)b * p.Hkv + h) * p.budget;
  // sinks + recent <= budget; a sequence within its budget has no slot that competes
  const int lo = len > p.budget ? p.sinks : len, m = len > p.budget ? len - p.recent - lo : 0;
  const uint32_t need = len > p.budget ? (uint32_t)(p.budget - p.sinks - p.recent) : 0u;
  const int steps = ((m + 63) / 64 + WAVES - 1) / WAVES;                       // of 64 slots, per wave
  const int i0 = wave * steps * 64, count = min(max(m - i0, 0), steps * 64);   // this wave's run of competing slots
  // f(index of a competing slot, its key), 64 together
  auto walk = [&](auto&& f) __attribute__((always_inline)) {
    auto key_at = [&](int i) __attribute__((always_inline)) { return HELD ? held[i] : weight_key(w[lo + i]); };
    int i = i0 + lane;
    const int whole = i0 + (count & ~63) + lane;
#pragma unroll 4
    for (; i < whole; i += 64) f(i, key_at(i));
    if (i < i0 + count) f(i, key_at(i));
  };
  if constexpr (HELD) {                            // (a thread reads back what it has written itself)
    constexpr int BATCH = THREADS == 256 ? 8 : 16;  // loads under way together: a trip to memory is longer than all the rest of a step
    for (int at = 0; at < count; at += 64 * BATCH) {
      float v[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) v[u] = at + 64 * u + lane < count ? w[lo + i0 + at + 64 * u + lane] : 0.f;
#pragma unroll
      for (int u = 0; u < BATCH; ++u)
        if (at + 64 * u + lane < count) held[i0 + at + 64 * u + lane] = weight_key(v[u]);
    }
  }
  for (int i = tid; i < 3 * kSelectBins / 4; i += THREADS) ((uint4*)&sh.hist[0][0])[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();

  uint32_t top = 0, more = need;                   // the digits of T found so far; places left for keys that agree with them
  if (need > 0) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
      const uint32_t seen = pass == 0 ? 0u : (pass == 1 ? ~0u << 21 : ~0u << 10);
      walk([&](int, uint32_t key) __attribute__((always_inline)) {
        if (pass == 0 || (key & seen) == top) atomicAdd(&sh.hist[pass][(key >> shift) & (kSelectBins - 1)], 1u);
      });
      __syncthreads();
      // thread t has the bins BPT (THREADS - 1 - t) and following, so that a prefix sum over threads counts from the top
      const int d = BPT * (THREADS - 1 - tid);
      uint32_t c[BPT], sum = 0;
#pragma unroll
      for (int u = 0; u < BPT; ++u) sum += c[u] = sh.hist[pass][d + u];
      const uint32_t upto = wave_prefix(sum);
      if (lane == 63) sh.wave_sum[pass][wave] = upto;
      __syncthreads();
      uint32_t above = upto - sum;
#pragma unroll
      for (int u = 0; u < WAVES; ++u)
        if (u < wave) above += sh.wave_sum[pass][u];
#pragma unroll
      for (int u = BPT - 1; u >= 0; --u) {
        if (above < more && above + c[u] >= more) sh.chosen[pass][0] = (uint32_t)(d + u), sh.chosen[pass][1] = above;
        above += c[u];
      }
      __syncthreads();
      top |= sh.chosen[pass][0] << shift;
      more -= sh.chosen[pass][1];
    }
  }
  // `top` is T now, and `more` of the keys that equal it stay: those in the lowest slots
  if (need > 0) {
    uint32_t ties = 0, sures = 0;                  // of this wave
    walk([&](int, uint32_t key) __attribute__((always_inline)) {
      ties += __popcll(__ballot(key == top));
      sures += __popcll(__ballot(key > top));
    });
    // (the last step's lanes past the run have not counted along)
    ties = __builtin_amdgcn_readfirstlane(ties);
    sures = __builtin_amdgcn_readfirstlane(sures);
    if (lane == 0) sh.wave_ties[wave] = ties, sh.wave_sures[wave] = sures;
    __syncthreads();
    uint32_t tie = 0, at = 0;                      // ties before this wave, and slots that stay
#pragma unroll
    for (int u = 0; u < WAVES; ++u)
      if (u < wave) tie += sh.wave_ties[u], at += sh.wave_sures[u];
    at += (uint32_t)lo + min(tie, more);
    const uint64_t below = (1ull << lane) - 1;
    walk([&](int i, uint32_t key) __attribute__((always_inline)) {
      const uint64_t tie_mask = __ballot(key == top);
      const bool stays = key > top || (key == top && tie + (uint32_t)__popcll(tie_mask & below) < more);
      const uint64_t stay_mask = __ballot(stays);
      if (stays) {
        const uint32_t r = at + (uint32_t)__popcll(stay_mask & below);
        kept[r] = lo + i;
        nw[r] = weight_of_key(key);
      }
      tie += __popcll(tie_mask);
      at += __popcll(stay_mask);
    });
  }
  // what stays whatever its weight: the first slots (all, within the budget) and the newest
  if (h == 0 && tid == 0) p.new_lens[b] = n_keep;
  for (int j = tid; j < lo; j += THREADS) {
    kept[j] = j;
    nw[j] = w[j];
  }
  for (int r = lo + (int)need + tid; r < n_keep; r += THREADS) {
    const int j = len - n_keep + r;
    kept[r] = j;
    nw[r] = w[j];
  }
  for (int r = n_keep + tid; r < p.budget; r += THREADS) kept[r] = -1;
  for (int r = n_keep + tid; r < p.capacity; r += THREADS) nw[r] = 0.f;
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
      page = p.block_table[(int64_t)b * p.table_stride + (j >> p.page_shift)];
      off = j & in_page;
    }
    const int to = p.dst_table[(int64_t)b * p.dst_stride + (r >> p.page_shift)];
    if (to < 0 || to >= p.num_pages) continue;
    uint4 x = make_uint4(0, 0, 0, 0), y = x;       // a token whose entry names no page has no row: not one of another page's
    if (page >= 0 && page < p.num_pages) {
      x = *(const uint4*)(p.k_cache + page * p.k_sp + off * p.k_st + h * p.k_sh + piece * 8);
      y = *(const uint4*)(p.v_cache + page * p.v_sp + off * p.v_st + h * p.v_sh + piece * 8);
    }
    *(uint4*)(p.k_cache + (int64_t)to * p.k_sp + (int64_t)(r & in_page) * p.k_st + h * p.k_sh + piece * 8) = x;
    *(uint4*)(p.v_cache + (int64_t)to * p.v_sp + (int64_t)(r & in_page) * p.v_st + h * p.v_sh + piece * 8) = y;
  }
}

}  // namespace fl
