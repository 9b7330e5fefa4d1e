// Attention over a paged cache in 4 bits for gfx950: the decode step, and the unpacked copy that a long chunk of queries reads.
#pragma once
#include "fl_decode_bf16.hpp"
#include "fl_mx4.hpp"

namespace fl {

typedef __attribute__((ext_vector_type(4))) float f32x4;

// Every sequence's cached rows as dense bf16 tensors [B, Hkv, L, D], row j token j, for the forward kernel that a long chunk of queries runs through.
// Rows from a sequence's length on are left as they are: that kernel is told the length.  A thread has a block of 32 channels of a key or
// a value (blockIdx.y): 17 bytes in, 64 out.
struct Mx4UnpackParams {
  Mx4Cache cache;
  uint16_t* dst[2];
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t table_stride, page_shift, num_pages, max_len, Hkv, L, D, blocks;           // blocks = D / 32
  int64_t total;                                                                     // B * Hkv * L * blocks
};
__global__ void __launch_bounds__(256) mx4_unpack_kernel(const Mx4UnpackParams p) {
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= p.total) return;
  const int blk = (int)(idx % p.blocks);
  int64_t rest = idx / p.blocks;
  const int j = (int)(rest % p.L);
  rest /= p.L;
  const int hk = (int)(rest % p.Hkv), b = (int)(rest / p.Hkv);
  const int len = min(max(p.seq_lens[b], 0), p.max_len);
  if (j >= len) return;
  int64_t page = b;
  int within = j;
  if (p.block_table != nullptr) {
    page = min(max(p.block_table[(int64_t)b * p.table_stride + (j >> p.page_shift)], 0), p.num_pages - 1);
    within = j & ((1 << p.page_shift) - 1);
  }
  const bool values = blockIdx.y != 0;
  const uint8_t* at = values ? p.cache.v + page * p.cache.v_sp + hk * p.cache.v_sh : p.cache.k + page * p.cache.k_sp + hk * p.cache.k_sh;
  const uint4 codes = *(const uint4*)(at + (int64_t)within * (p.D / 2) + blk * 16);
  const float scale = mx4_scale_value(at[(int64_t)p.cache.page_size * (p.D / 2) + (int64_t)blk * p.cache.page_size + within]);
  uint4* to = (uint4*)(p.dst[values ? 1 : 0] + idx * 32);
  to[0] = mx4_bf16x8(codes.x, scale);
  to[1] = mx4_bf16x8(codes.y, scale);
  to[2] = mx4_bf16x8(codes.z, scale);
  to[3] = mx4_bf16x8(codes.w, scale);
}

// ---- the decode step over a cache in 4 bits ----

struct Mx4DecodeParams : DecodeParams {
  Mx4Cache cache;                  // in place of k, v and their strides
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

// A workgroup owns one (sequence, kv head, split of the key range); its four waves take tiles of 32 keys in turn.  NB blocks of 16
// (query row, head) pairs are the columns of the matrix products, S^T = K Q^T and O^T += V^T P^T on 16 x 16 x 32 instructions:
//   * lane = (g, m), g = lane / 16.  The order of a contraction's terms is free, so that a lane's codes of one key are a quarter of its row in
//     one load, channels D/4 g + 8 s + .. in step s, and its block's scale goes into the conversion;
//   * row m of product u = 0, 1 is key 8 (m / 4) + 4 u + m % 4 of the tile.  A lane's scores are then those of keys 8 g .. 8 g + 7 in order, which
//     is what the second contraction wants of P: no exchange between lanes;
//   * for that one, a lane has keys 8 g .. + 7 of channels D/16 m .. + D/16 - 1: the codes of two keys are converted two channels at a time, then
//     paired key by key.
// waves of a SIMD: what the registers of an instance leave room for
constexpr int mx4_decode_waves(int D, int NB) { return NB == 1 ? (D == 128 ? 3 : 4) : (NB == 2 ? 2 : 1); }

template <int D, int MOD, int NB>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(mx4_decode_waves(D, NB), mx4_decode_waves(D, NB)))) mx4_decode_kernel(const Mx4DecodeParams p) {
  constexpr int KS = D / 32;                       // steps of the first contraction
  constexpr int CH = D / 16;                       // channels of a lane in the second
  __shared__ float park[4][CH * 4 * 64];
  __shared__ float2 park_ml[4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, m = lane & 15;

  int split, bhk, hk, b;
  p.by_split.split(blockIdx.x, bhk, split);
  p.by_hkv.split(bhk, b, hk);
  const int group = (int)p.by_group.d, ncol = p.T * group;
  const int len = min(max(p.seq_lens[b], 0), p.max_len);
  int row[NB], hq[NB], pos[NB];
  bool live[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int c = 16 * nb + m;
    live[nb] = c < ncol;
    int head;
    p.by_group.split(live[nb] ? c : ncol - 1, row[nb], head);
    hq[nb] = hk * group + head;
    pos[nb] = len - p.T + row[nb];
  }
  const int first_key = p.window >= 0 ? max(0, len - p.T - p.window) : 0;
  const int first_full = p.window >= 0 ? max(0, len - 1 - p.window) : 0;
  const int t_lo = first_key / 32, t_hi = (len + 31) / 32;
  const int per_split = p.by_split.div(t_hi - t_lo + p.nsplit - 1);
  const int t_begin = t_lo + split * per_split, t_end = min(t_hi, t_begin + per_split);

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
  const float c_scale = p.scale * kLog2e;
  const int64_t codes_bytes = (int64_t)p.cache.page_size * (D / 2);

  // A lane's page of its eight keys of tile t in either contraction (an octet lies in one page; behind the sequence: its last one).  The entries of a
  // tile are requested two tiles ahead of its products, its codes and scales one tile ahead.  The tile behind a wave's last is the last again: a load
  // that is not there on one path would make the compiler wait for every load on the other.
  const int t_last = t_begin + wave + max(0, t_end - 1 - t_begin - wave) / 4 * 4;
  const int32_t* const table = p.block_table + (p.block_table != nullptr ? (int64_t)b * p.table_stride : 0);
  const int in_page = p.block_table != nullptr ? (1 << p.page_shift) - 1 : -1;
  struct Pages {
    int k, v;
  };
  auto octet = [&](int t, int o) __attribute__((always_inline)) { return min(min(t, t_last) * 32 + 8 * o, (len - 1) & ~7); };
  auto lookup = [&](int t) __attribute__((always_inline)) -> Pages {
    if (p.block_table == nullptr) return {b, b};
    return {table[octet(t, m >> 2) >> p.page_shift], table[octet(t, g) >> p.page_shift]};
  };
  struct Tile {
    uint32_t k[2][KS], v[8];
    uint2 ke, ve;                                  // scales of eight keys of the lane's block
  };
  const uint8_t* const k_lane = p.cache.k + hk * p.cache.k_sh + (m & 3) * (D / 2) + g * (D / 8);
  const uint8_t* const v_lane = p.cache.v + hk * p.cache.v_sh + m * (CH / 2);
  const uint8_t* const ke_lane = p.cache.k + hk * p.cache.k_sh + codes_bytes + (int64_t)(g * (D / 4) / 32) * p.cache.page_size;
  const uint8_t* const ve_lane = p.cache.v + hk * p.cache.v_sh + codes_bytes + (int64_t)(m * CH / 32) * p.cache.page_size;
  auto load = [&](int t, const Pages& pages, Tile& x) __attribute__((always_inline)) {
    const int last = p.num_pages - 1;
    const int64_t k_page = min(max(pages.k, 0), last) * p.cache.k_sp, v_page = min(max(pages.v, 0), last) * p.cache.v_sp;
    const int k_in = octet(t, m >> 2) & in_page, v_in = octet(t, g) & in_page;
    const uint8_t* kp = k_lane + k_page + (int64_t)k_in * (D / 2);
    const uint8_t* vp = v_lane + v_page + (int64_t)v_in * (D / 2);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (D == 128) {
        const uint4 y = *(const uint4*)(kp + 4 * u * (D / 2));
        x.k[u][0] = y.x; x.k[u][1] = y.y; x.k[u][2] = y.z; x.k[u][3] = y.w;
      } else {
        const uint2 y = *(const uint2*)(kp + 4 * u * (D / 2));
        x.k[u][0] = y.x; x.k[u][1] = y.y;
      }
    }
    x.ke = *(const uint2*)(ke_lane + k_page + k_in);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (D == 128) x.v[i] = *(const uint32_t*)(vp + i * (D / 2));
      else x.v[i] = *(const uint16_t*)(vp + i * (D / 2));
    }
    x.ve = *(const uint2*)(ve_lane + v_page + v_in);
  };

  auto compute = [&](int t, const Tile& tile) __attribute__((always_inline)) {
    f32x4 s[NB][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s[nb][u] = (f32x4){0.f, 0.f, 0.f, 0.f};
      const float scale = mx4_scale_value(((u ? tile.ke.y : tile.ke.x) >> (8 * (m & 3))) & 255);
#pragma unroll
      for (int f = 0; f < KS; ++f) {
        const bf16x8 a = __builtin_bit_cast(bf16x8, mx4_bf16x8(tile.k[u][f], scale));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[nb][f], s[nb][u], 0, 0, 0);
      }
    }
    const int jb = t * 32 + 8 * g;
    const bool partial = t * 32 + 32 > len - p.T + 1 || t * 32 < first_full;       // uniform
    bf16x8 pf[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float x[8], mx = -INFINITY;                  // x: in the log2 domain, but for the plain scores their factor c_scale
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float raw = s[nb][i >> 2][i & 3];
        if constexpr (MOD == kModSoftcap) {
          const float e = fast_exp2(raw * (2.f * c_scale / p.softcap));
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
        pw[i] = pack_bf16(p0, p1);
      }
      l_run[nb] += psum;
      pf[nb] = __builtin_bit_cast(bf16x8, (i32x4){(int)pw[0], (int)pw[1], (int)pw[2], (int)pw[3]});
    }
    float vs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) vs[i] = mx4_scale_value(((i < 4 ? tile.ve.x : tile.ve.y) >> (8 * (i & 3))) & 255);
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

  int t = t_begin + wave;
  if (t < t_end) {
    Tile even, odd;
    Pages ahead = lookup(t);
    load(t, ahead, even);
    ahead = lookup(t + 4);
    while (true) {
      load(t + 4, ahead, odd);
      ahead = lookup(t + 8);
      compute(t, even);
      if ((t += 4) >= t_end) break;
      load(t + 4, ahead, even);
      ahead = lookup(t + 8);
      compute(t, odd);
      if ((t += 4) >= t_end) break;
    }
  }

  // ---- merge of the waves, a column block at a time; wave i then holds channels CH (4 g + i) .. + CH - 1 of column m
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    if (nb > 0) __syncthreads();
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) park[wave][(c * 4 + r) * 64 + lane] = oacc[nb][c][r];
    park_ml[wave][lane] = make_float2(m_run[nb], quarter_sum(l_run[nb]));
    __syncthreads();
    float m_all = -INFINITY, l_all = 0.f, wgt[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) m_all = fmaxf(m_all, park_ml[u][lane].x);
    const float m_safe = m_all == -INFINITY ? 0.f : m_all;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float2 ml = park_ml[u][lane];
      wgt[u] = fast_exp2(ml.x - m_safe);
      l_all = fmaf(ml.y, wgt[u], l_all);
    }
    const bool result = p.nsplit == 1;
    const float inv = result ? (l_all > 0.f ? 1.f / l_all : 0.f) : 1.f;
    float x[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      x[c] = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) x[c] = fmaf(park[u][(c * 4 + wave) * 64 + lane], wgt[u], x[c]);
      x[c] *= inv;
    }
    const int64_t slot = (((int64_t)b * p.T + row[nb]) * p.H + hq[nb]) * p.nsplit + split;
    const int ch = CH * (4 * g + wave);
    if (live[nb]) {
      if (!result || p.out_f32) {
        float* to = result ? (float*)p.out + b * p.o_sb + hq[nb] * p.o_sh + row[nb] * p.o_st + ch : p.part_o + slot * D + ch;
#pragma unroll
        for (int c = 0; c < CH; c += 4) *(float4*)(to + c) = make_float4(x[c], x[c + 1], x[c + 2], x[c + 3]);
      } else {
        uint16_t* to = (uint16_t*)p.out + b * p.o_sb + hq[nb] * p.o_sh + row[nb] * p.o_st + ch;
#pragma unroll
        for (int c = 0; c < CH; c += 4) *(uint2*)(to + c) = make_uint2(pack_bf16(x[c], x[c + 1]), pack_bf16(x[c + 2], x[c + 3]));
      }
      if (wave == 0 && g == 0) {
        if (!result) *(float2*)(p.part_ml + slot * 2) = make_float2(m_all, l_all);
        else if (p.lse != nullptr)
          p.lse[b * p.lse_sb + hq[nb] * p.lse_sh + row[nb] * p.lse_st] = l_all > 0.f ? (m_all + __log2f(l_all)) * kLn2 : -INFINITY;
      }
    }
  }
}

}  // namespace fl
