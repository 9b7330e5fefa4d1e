// Attention over a paged cache in 4 bits for gfx950: the decode step, and the unpacked copy that a long chunk of queries reads.
//
// What bounds the step: reading D/2 + D/32 bytes for a key and as many for its value.  Every code has to be converted too, two a lane and instruction, for
// one query row of a group of heads as for sixteen: 64 sequences of 4k - 8k tokens, 32 / 8 heads, D = 128, take 85 us (5.0 TB/s), with the loads alone 82 - 86,
// with the arithmetic alone 60 - 65, and 69 at the rate of a large read.  Loads therefore need no registers and no instruction slots beyond their own (rings in LDS, tiles ahead:
// 104 -> 87 us), and as many waves share a SIMD as the registers allow.
#pragma once
#include "fl_decode_bf16.hpp"
#include "fl_mx4.hpp"

namespace fl {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;

// Every sequence's cached rows as dense bf16 tensors [B, Hkv, L, D], row j token j, for the forward kernel that a long chunk of queries runs through.
// Rows from a sequence's length on are left as they are: that kernel is told the length.  A workgroup has 128 keys, or values, of a kv head; a thread has
// eight channels of every 16th (D = 64: 32nd) of them, all requested before the first is converted, so that a wave stores runs of 1 KB (8 sequences of 4k - 8k tokens, 8 heads,
// D = 128: 48 us, 250 MB at the rate of a copy; a row a thread 80).
constexpr int kUnpackKeys = 128;
struct Mx4UnpackParams {
  Mx4Cache cache;
  uint16_t* dst[2];
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t table_stride, page_shift, num_pages, max_len, L;
  Divisor by_blocks, by_heads, by_hkv;             // workgroups of a kv head, 2, Hkv
};
template <int D>
__global__ void __launch_bounds__(256) mx4_unpack_kernel(const Mx4UnpackParams p) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES, N = kUnpackKeys / ROWS;
  int rest, blk, which, bhk, b, hk;
  p.by_blocks.split(blockIdx.x, rest, blk);
  p.by_heads.split(rest, bhk, which);
  p.by_hkv.split(bhk, b, hk);
  const int len = min(max(p.seq_lens[b], 0), p.max_len), c = threadIdx.x % LANES, j0 = blk * kUnpackKeys + threadIdx.x / LANES;
  if (blk * kUnpackKeys >= len) return;
  const uint8_t* base = which ? p.cache.v + hk * p.cache.v_sh : p.cache.k + hk * p.cache.k_sh;
  const int64_t sp = which ? p.cache.v_sp : p.cache.k_sp, scales = (int64_t)p.cache.page_size * (D / 2) + (int64_t)(c / 4) * p.cache.page_size;
  int page[N], within[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int j = min(j0 + i * ROWS, len - 1);     // (past the end: the last key again, not stored)
    page[i] = b;
    within[i] = j;
    if (p.block_table != nullptr) {
      page[i] = p.block_table[(int64_t)b * p.table_stride + (j >> p.page_shift)];
      within[i] = j & ((1 << p.page_shift) - 1);
    }
  }
  uint32_t codes[N];
  int e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint8_t* at = base + min(max(page[i], 0), p.num_pages - 1) * sp;
    codes[i] = *(const uint32_t*)(at + (int64_t)within[i] * (D / 2) + c * 4);
    e[i] = at[scales + within[i]];
  }
  uint16_t* to = p.dst[which] + ((int64_t)bhk * p.L + j0) * D + c * 8;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (j0 + i * ROWS < len) *(uint4*)(to + (int64_t)i * ROWS * D) = mx4_bf16x8(codes[i], mx4_scale_value(e[i]));
}

// ---- the decode step over a cache in 4 bits ----

struct Mx4DecodeParams : DecodeParams {
  Mx4Cache cache;                  // in place of k, v and their strides
  Divisor by_block;                // blocks of 16 NB (query row, head) pairs of a kv head
};

// max and sum over the four lanes of a column (16 apart)
__device__ __forceinline__ float quarter_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quarter_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// A workgroup owns one (sequence, kv head, split of the key range), a wave a run of its tiles of 32 keys.  NB blocks of 16 (query row, head) pairs are the columns of the matrix products, S^T = K Q^T and O^T += V^T P^T on 16 x 16 x 32 instructions:
//   * lane = (g, m), g = lane / 16.  The order of a contraction's terms is free, so that a lane's codes of one key are a quarter of its row in
//     one load, channels D/4 g + 8 s + .. in step s, and its block's scale goes into the conversion;
//   * row m of product u = 0, 1 is key 8 (m / 4) + 4 u + m % 4 of the tile.  A lane's scores are then those of keys 8 g .. 8 g + 7 in order, which
//     is what the second contraction wants of P: no exchange between lanes;
//   * for that one, a lane has keys 8 g .. + 7 of channels D/16 m .. + D/16 - 1: the codes of two keys are converted two channels at a time, then
//     paired key by key.
// Waves of a SIMD, which are workgroups of a compute unit: what the registers of an instance leave room for.  LDS is shared out among them as rings.  (One block: four waves
// of two stages; three of three are as fast or slower.  Four blocks of 16 pairs would leave one wave: 16 rows of 4 heads 59 us, as two times two blocks 36.)
constexpr int mx4_decode_waves(int D, int NB) { return NB == 1 ? 4 : 2; }
template <int D, int NB>
struct Mx4Ring {
  static constexpr int V = 32 * (D / 2), E = 2 * V, STAGE = E + 256;             // bytes: keys, values, scales
  static constexpr int LOADS = D == 128 ? 5 : 3;                                 // of a tile
  static constexpr int ROOM = 160 * 1024 / (4 * mx4_decode_waves(D, NB)) / 16 * 16 - 512;
  static constexpr int STAGES = ROOM / STAGE < 8 ? ROOM / STAGE : 8;
  static constexpr int ENTRIES = STAGES * STAGE, BYTES = ENTRIES + 512, LDS = 4 * BYTES;
  static_assert(STAGES >= 2 && (STAGES - 1) * LOADS < 64 && 16 - STAGES >= STAGES, "a wave's ring");
  static_assert((D / 16 * 4 * 64) * 4 + 64 * 8 <= BYTES, "where a wave parks its sums");
};

template <int D, int MOD, int NB>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(mx4_decode_waves(D, NB), mx4_decode_waves(D, NB)))) mx4_decode_kernel(const Mx4DecodeParams p) {
  constexpr int KS = D / 32;                       // steps of the first contraction
  constexpr int CH = D / 16;                       // channels of a lane in the second
  typedef Mx4Ring<D, NB> R;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const int group = (int)p.by_group.d, ncol = p.T * group;
  const float c_scale = p.scale * kLog2e;
  const int64_t codes_bytes = (int64_t)p.cache.page_size * (D / 2);
  const int lane = threadIdx.x & 63, g = lane >> 4, m = lane & 15;
  // workgroups go out to the eight XCDs in turn: an XCD takes neighbours, whose kv heads share the lines of memory in which one's part of a page ends and
  // the next one's begins (64 sequences of 4k - 8k tokens, 32 / 8 heads, D = 128: 87.7 -> 86.5 us)
  const int place = (gridDim.x & 7) == 0 ? (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)) : (int)blockIdx.x;
  int rest, block, split, bhk, hk, b;
  p.by_block.split(place, rest, block);            // blocks of a split's rows side by side: they read the same keys
  p.by_split.split(rest, bhk, split);
  p.by_hkv.split(bhk, b, hk);
  const int len = min(max(p.seq_lens[b], 0), p.max_len), first_pair = block * 16 * NB, last_pair = min(first_pair + 16 * NB, ncol) - 1;
  const int pos_lo = len - p.T + p.by_group.div(first_pair), pos_hi = len - p.T + p.by_group.div(last_pair);     // of the first and last row
  const int t_lo = p.window >= 0 ? max(0, pos_lo - p.window) / 32 : 0, t_hi = pos_hi < 0 ? 0 : pos_hi / 32 + 1;
  const int per_split = p.by_split.div(max(t_hi - t_lo, 0) + p.nsplit - 1);
  const int t_begin = t_lo + split * per_split, t_end = min(t_hi, t_begin + per_split);
  int row[NB], hq[NB], pos[NB];                    // (columns behind the last pair are copies of it)
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    int head;
    p.by_group.split(min(first_pair + 16 * nb + m, last_pair), row[nb], head);
    hq[nb] = hk * group + head;
    pos[nb] = len - p.T + row[nb];
  }
  const int first_full = p.window >= 0 ? max(0, pos_hi - p.window) : 0;

  bf16x8 qf[NB][KS];
  float slope2[NB], m_run[NB], l_run[NB];
  f32x4 oacc[NB][CH];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const uint16_t* qp = p.q + b * p.q_sb + hq[nb] * p.q_sh + row[nb] * p.q_st + g * (D / 4);
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[nb][s] = *(const bf16x8*)(qp + 8 * s);
    slope2[nb] = MOD == kModAlibi ? p.alibi_slopes[hq[nb]] * kLog2e : 0.f;
    m_run[nb] = -INFINITY;
    l_run[nb] = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) oacc[nb][c] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  // The wave's tiles come through its ring in LDS, STAGES - 1 of them ahead of the one in use, by loads that need no registers.  In every one of them lane (g, m)
  // fetches from octet m / 4 of the tile's keys (an octet lies in one page; behind the sequence: its last one), so that a tile is one table entry a lane:
  //   keys     D = 128: the lane's own 16 bytes of keys m % 4 and 4 + m % 4; D = 64: the half g % 2 of key 4 (g / 2) + m % 4
  //   values   rows of D / 2 bytes, the four octets' rows of one number next to each other: eight reads without bank conflicts
  //   scales   a dword each
  // The entries come the same way, for 16 tiles at a time.
  unsigned char* const ring = lds + wave * R::BYTES;
  const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void*)ring;
  const int n_all = t_end - t_begin, n_each = (n_all + 3) / 4, t0 = t_begin + wave * n_each, n = min(n_each, n_all - wave * n_each);
  const int32_t* const table = p.block_table + (p.block_table != nullptr ? (int64_t)b * p.table_stride : 0);
  const int last_octet = (len - 1) & ~7, in_page = p.block_table != nullptr ? (1 << p.page_shift) - 1 : -1;
  const int oct8 = (m >> 2) * 8;
  const uint8_t *k_lane = p.cache.k + hk * p.cache.k_sh, *v_lane = p.cache.v + hk * p.cache.v_sh;
  const bool v_scale = lane >= 32;
  const uint8_t* const e_lane = (v_scale ? v_lane : k_lane) + codes_bytes +
                                (int64_t)((lane >> 1 & 1) + (D == 128 ? (lane >> 4 & 1) * 2 : 0)) * p.cache.page_size + (lane & 1) * 4;
  const uint32_t e_sp = (uint32_t)(v_scale ? p.cache.v_sp : p.cache.k_sp), k_sp = (uint32_t)p.cache.k_sp, v_sp = (uint32_t)p.cache.v_sp;
  k_lane += D == 128 ? (m & 3) * 64 + g * 16 : (m & 3) * 32 + (g & 1) * 16 + (g >> 1) * 128;
  v_lane += D == 128 ? g * 64 + (m & 3) * 16 : (2 * g + (m >> 1 & 1)) * 32 + (m & 1) * 16;
  auto fetch_entries = [&](int w) __attribute__((always_inline)) {               // of tiles 16 w .. of this wave
    const int j = min((t0 + 16 * w) * 32 + lane * 8, last_octet);
    __builtin_amdgcn_global_load_lds((global_cvoid*)(table + (j >> p.page_shift)), (lds_void*)(ring + R::ENTRIES + (w & 1) * 256), 4, 0, 0);
  };
  auto fetch = [&](int i, int entry) __attribute__((always_inline)) {            // tile i of this wave
    unsigned char* st = ring + i % R::STAGES * R::STAGE;
    const uint32_t page = p.block_table != nullptr ? (uint32_t)min(max(entry, 0), p.num_pages - 1) : (uint32_t)b;
    const uint32_t within = (uint32_t)(min((t0 + i) * 32 + oct8, last_octet) & in_page);
    const uint8_t* kp = k_lane + (uint64_t)page * k_sp + (uint64_t)within * (D / 2);
    const uint8_t* vp = v_lane + (uint64_t)page * v_sp + (uint64_t)within * (D / 2);
    __builtin_amdgcn_global_load_lds((global_cvoid*)kp, (lds_void*)st, 16, 0, 0);
    if (D == 128) __builtin_amdgcn_global_load_lds((global_cvoid*)kp, (lds_void*)(st + 1024 - 256), 16, 256, 0);   // (the offset counts on both sides)
    __builtin_amdgcn_global_load_lds((global_cvoid*)vp, (lds_void*)(st + R::V), 16, 0, 0);
    if (D == 128) __builtin_amdgcn_global_load_lds((global_cvoid*)vp, (lds_void*)(st + R::V + 1024 - 256), 16, 256, 0);
    __builtin_amdgcn_global_load_lds((global_cvoid*)(e_lane + (uint64_t)page * e_sp + within), (lds_void*)(st + R::E), 4, 0, 0);
  };
  struct Tile {
    i32x4 k[2];                                    // D = 64: two dwords of each
    uint32_t v[8];
    i32x2 ke, ve;                                  // scales of eight keys of the lane's block
  };
  // where in a stage this lane reads
  const uint32_t at_k = D == 128 ? lane * 16 : (g >> 1) * 256 + m * 16 + (g & 1) * 8, at_v = R::V + (D == 128 ? lane * 4 : g * 64 + m * 2);
  auto e_at = [&](int which, int block, int o) __attribute__((always_inline)) {
    return (uint32_t)(R::E + 4 * (which * 32 + (block >> 1) * 16 + o * 4 + (block & 1) * 2));
  };
  const uint32_t at_ke = e_at(0, g * (D / 4) / 32, m >> 2), at_ve = e_at(1, m * CH / 32, g);
  // Everything the products of tile i need, and the entry of tile i + STAGES: reads and their wait in one block, which the compiler takes to be
  // done where it ends (it would make any other read of the ring wait for all loads into it).
  auto take = [&](int i, Tile& x, int& entry) __attribute__((always_inline)) {
    const uint32_t st = ring_at + i % R::STAGES * R::STAGE, a = st + at_k, c = st + at_v, d = st + at_ke, e = st + at_ve;
    const uint32_t f = ring_at + R::ENTRIES + ((i + R::STAGES) & 31) * 16 + (m >> 2) * 4;
    if constexpr (D == 128) {
      asm volatile(
          "ds_read_b128 %0, %13\n\tds_read_b128 %1, %13 offset:1024\n\tds_read_b64 %2, %15\n\tds_read_b64 %3, %16\n\t"
          "ds_read_b32 %4, %14\n\tds_read_b32 %5, %14 offset:256\n\tds_read_b32 %6, %14 offset:512\n\tds_read_b32 %7, %14 offset:768\n\t"
          "ds_read_b32 %8, %14 offset:1024\n\tds_read_b32 %9, %14 offset:1280\n\tds_read_b32 %10, %14 offset:1536\n\tds_read_b32 %11, %14 offset:1792\n\t"
          "ds_read_b32 %12, %17\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(x.k[0]), "=&v"(x.k[1]), "=&v"(x.ke), "=&v"(x.ve), "=&v"(x.v[0]), "=&v"(x.v[1]), "=&v"(x.v[2]), "=&v"(x.v[3]), "=&v"(x.v[4]),
            "=&v"(x.v[5]), "=&v"(x.v[6]), "=&v"(x.v[7]), "=&v"(entry)
          : "v"(a), "v"(c), "v"(d), "v"(e), "v"(f)
          : "memory");
    } else {
      i32x2 k0, k1;
      asm volatile(
          "ds_read_b64 %0, %13\n\tds_read_b64 %1, %13 offset:512\n\tds_read_b64 %2, %15\n\tds_read_b64 %3, %16\n\t"
          "ds_read_u16 %4, %14\n\tds_read_u16 %5, %14 offset:32\n\tds_read_u16 %6, %14 offset:256\n\tds_read_u16 %7, %14 offset:288\n\t"
          "ds_read_u16 %8, %14 offset:512\n\tds_read_u16 %9, %14 offset:544\n\tds_read_u16 %10, %14 offset:768\n\tds_read_u16 %11, %14 offset:800\n\t"
          "ds_read_b32 %12, %17\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(k0), "=&v"(k1), "=&v"(x.ke), "=&v"(x.ve), "=&v"(x.v[0]), "=&v"(x.v[1]), "=&v"(x.v[2]), "=&v"(x.v[3]), "=&v"(x.v[4]),
            "=&v"(x.v[5]), "=&v"(x.v[6]), "=&v"(x.v[7]), "=&v"(entry)
          : "v"(a), "v"(c), "v"(d), "v"(e), "v"(f)
          : "memory");
      x.k[0] = (i32x4){k0[0], k0[1], 0, 0};
      x.k[1] = (i32x4){k1[0], k1[1], 0, 0};
    }
  };
  auto entry_of = [&](int i) __attribute__((always_inline)) {
    int x;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(x) : "v"(ring_at + R::ENTRIES + (i & 31) * 16 + (m >> 2) * 4) : "memory");
    return x;
  };

  auto compute = [&](int t, const Tile& tile) __attribute__((always_inline)) {
    f32x4 s[NB][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s[nb][u] = (f32x4){0.f, 0.f, 0.f, 0.f};
      const float scale = mx4_scale_value(((uint32_t)tile.ke[u] >> (8 * (m & 3))) & 255);
#pragma unroll
      for (int f = 0; f < KS; ++f) {
        const bf16x8 a = __builtin_bit_cast(bf16x8, mx4_bf16x8((uint32_t)tile.k[u][f], scale));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[nb][f], s[nb][u], 0, 0, 0);
      }
    }
    const int jb = t * 32 + 8 * g;
    const bool partial = t * 32 + 32 > pos_lo + 1 || t * 32 < first_full;       // uniform
    bf16x8 pf[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float x[8], mx = -INFINITY;                  // x: in the log2 domain, but for the plain scores their factor c_scale
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float raw = s[nb][i >> 2][i & 3];
        if constexpr (MOD == kModSoftcap) {
          const float e = fast_exp2(raw * fminf(2.f * c_scale / p.softcap, 0x1p127f));     // (finite: a raw score of 0 stays 0)
          x[i] = fmaf(fast_rcp(e + 1.f), -2.f * p.softcap * kLog2e, p.softcap * kLog2e);
        } else if constexpr (MOD == kModAlibi) {
          x[i] = fmaf(raw, c_scale, -slope2[nb] * (float)(pos[nb] - jb - i));
        } else {
          x[i] = raw;
        }
      }
      if (partial) {
        const int lo_key = p.window >= 0 ? pos[nb] - p.window : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = jb + i > pos[nb] || jb + i < lo_key ? -INFINITY : x[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = fmaxf(mx, x[i]);
      if constexpr (MOD == kModNone) mx *= c_scale;                                // (a positive factor)
      // as in the step over bf16 pages the running maximum moves only where a score exceeds it by 2^8, here before any lane has
      // looked at the column's others
      if (__builtin_amdgcn_ballot_w64(mx - m_run[nb] > kLazyMaxLog2) != 0) {
        mx = quarter_max(mx);
        const float m_new = (mx - m_run[nb] > kLazyMaxLog2) ? mx : m_run[nb];
        const float alpha = m_new != m_run[nb] ? fast_exp2(m_run[nb] - m_new) : 1.f;
        m_run[nb] = m_new;
        l_run[nb] *= alpha;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) oacc[nb][c][r] *= alpha;
      }
      const float m_safe = m_run[nb] == -INFINITY ? 0.f : m_run[nb];
      float psum = 0.f;
      uint32_t pw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = fast_exp2(MOD == kModNone ? fmaf(x[2 * i], c_scale, -m_safe) : x[2 * i] - m_safe);
        const float p1 = fast_exp2(MOD == kModNone ? fmaf(x[2 * i + 1], c_scale, -m_safe) : x[2 * i + 1] - m_safe);
        psum += p0 + p1;
        // P is rounded to bf16, 2^-8 of it at most, for the second product, as in the framework's other attention kernels; the sum that divides it is not.  (A result
        // is off by 2.1 - 2.4e-3 of its size so, 1.6 - 1.7 of which its own rounding makes; P in two parts would double the product's instructions.)
        pw[i] = pack_bf16(p0, p1);
      }
      l_run[nb] += psum;
      pf[nb] = __builtin_bit_cast(bf16x8, (i32x4){(int)pw[0], (int)pw[1], (int)pw[2], (int)pw[3]});
    }
    float vs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) vs[i] = mx4_scale_value(((uint32_t)tile.ve[i >> 2] >> (8 * (i & 3))) & 255);
    if (t * 32 + 32 > len) {
      // what lies behind the sequence's end in its last page is any bytes: finite, for P is zero there
#pragma unroll
      for (int i = 0; i < 8; ++i) vs[i] = jb + i < len ? vs[i] : 1.f;
    }
#pragma unroll
    for (int f = 0; f < CH / 2; ++f) {
      uint32_t c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        bf16x2 y;
        if (f == 0) y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(tile.v[i], vs[i], 0);
        else if (f == 1) y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(tile.v[i], vs[i], 1);
        else if (f == 2) y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(tile.v[i], vs[i], 2);
        else y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(tile.v[i], vs[i], 3);
        c[i] = __builtin_bit_cast(uint32_t, y);
      }
      i32x4 lo, hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = (int)__builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
        hi[i] = (int)__builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        oacc[nb][2 * f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), pf[nb], oacc[nb][2 * f], 0, 0, 0);
        oacc[nb][2 * f + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), pf[nb], oacc[nb][2 * f + 1], 0, 0, 0);
      }
    }
  };

  if (n > 0) {
    int entry = 0;
    if (p.block_table != nullptr) {
      fetch_entries(0);
      wait_vm<0>();
    }
#pragma unroll
    for (int i = 0; i < R::STAGES - 1; ++i) {
      entry = entry_of(i);                         // (without a table: not used)
      if (i < n) fetch(i, entry);
    }
    entry = entry_of(R::STAGES - 1);
    for (int i = 0; i < n; ++i) {
      if ((i & 15) == 0 && i + 16 < n && p.block_table != nullptr) fetch_entries(i / 16 + 1);      // (first asked for 16 - STAGES steps later)
      if (i + R::STAGES - 1 < n) {
        fetch(i + R::STAGES - 1, entry);
        wait_vm<(R::STAGES - 1) * R::LOADS>();     // all but the STAGES - 1 younger tiles has landed
      } else {
        wait_vm<0>();
      }
      Tile x;
      take(i, x, entry);
      compute(t0 + i, x);
    }
  }

  // ---- merge of the waves, a column block at a time; wave i then holds channels CH (4 g + i) .. + CH - 1 of column m
  auto park = [&](int w) __attribute__((always_inline)) { return (float*)(lds + w * R::BYTES); };
  auto park_ml = [&](int w) __attribute__((always_inline)) { return (float2*)(lds + w * R::BYTES + CH * 4 * 64 * 4); };
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    if (nb > 0) __syncthreads();                   // everyone has read what was parked before
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int r = 0; r < 4; ++r) park(wave)[(k * 4 + r) * 64 + lane] = oacc[nb][k][r];
    park_ml(wave)[lane] = make_float2(m_run[nb], quarter_sum(l_run[nb]));
    __syncthreads();
    float m_all = -INFINITY, l_all = 0.f, wgt[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) m_all = fmaxf(m_all, park_ml(u)[lane].x);
    const float m_safe = m_all == -INFINITY ? 0.f : m_all;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float2 ml = park_ml(u)[lane];
      wgt[u] = fast_exp2(ml.x - m_safe);
      l_all = fmaf(ml.y, wgt[u], l_all);
    }
    const bool result = p.nsplit == 1;             // the only split of its sequence: no partials and no merge kernel
    const float inv = result ? (l_all > 0.f ? 1.f / l_all : 0.f) : 1.f;
    float x[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      x[k] = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) x[k] = fmaf(park(u)[(k * 4 + wave) * 64 + lane], wgt[u], x[k]);
      x[k] *= inv;
    }
    if (first_pair + 16 * nb + m > last_pair) continue;
    const int64_t slot = (((int64_t)b * p.T + row[nb]) * p.H + hq[nb]) * p.nsplit + split;
    const int ch = CH * (4 * g + wave);
    if (!result || p.out_f32) {
      float* to = result ? (float*)p.out + b * p.o_sb + hq[nb] * p.o_sh + row[nb] * p.o_st + ch : p.part_o + slot * D + ch;
#pragma unroll
      for (int k = 0; k < CH; k += 4) *(float4*)(to + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
    } else {
      uint16_t* to = (uint16_t*)p.out + b * p.o_sb + hq[nb] * p.o_sh + row[nb] * p.o_st + ch;
#pragma unroll
      for (int k = 0; k < CH; k += 4) *(uint2*)(to + k) = make_uint2(pack_bf16(x[k], x[k + 1]), pack_bf16(x[k + 2], x[k + 3]));
    }
    if (wave == 0 && g == 0) {
      if (!result) *(float2*)(p.part_ml + slot * 2) = make_float2(m_all, l_all);
      else if (p.lse != nullptr)
        p.lse[b * p.lse_sb + hq[nb] * p.lse_sh + row[nb] * p.lse_st] = l_all > 0.f ? (m_all + __log2f(l_all)) * kLn2 : -INFINITY;
    }
  }
}

}  // namespace fl
