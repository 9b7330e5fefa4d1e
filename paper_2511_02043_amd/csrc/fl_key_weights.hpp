// Weight that the rows of a prompt chunk give to each cached key, for gfx950:
//     gained[b, hkv, j] = sum over the query heads h of hkv and the rows i that see j of exp(s_ij - lse_i),
// with s the scores of the forward pass (Eq. 3, score_mod of Eq. 4) and lse what it has left behind: column sums of a matrix that is
// formed tile by tile and never stored.  One contraction of 2 D operations per score, one exponential, a multiply-add and an addition, so at
// D = 128 matrix and vector units have about as much to do, and what counts is that they do it at the same time.
//
//   * a wave owns 32 keys, held in registers as the B operand of the MFMA for the whole launch; S = Q K^T then has the key in the lane and
//     the row in the register index, so that a column sum is additions in a lane, and a half swap at the very end;
//   * the rows of the kv head's query heads stream through a ring of three LDS stages of 64 rows that the workgroup's eight waves share
//     (one barrier per stage, two stages in flight); two workgroups, four waves a SIMD, whose products and exponentials overlap.  Measured
//     against 64 keys per wave (half the LDS reads, two waves a SIMD, 264 / 326 us in the cases below), that with the products of one block
//     and the exponentials of the one before in a single instruction stream (244 / 298, but registers in scratch with ALiBi), and three
//     waves a SIMD (316 / 380): 250 / 306 us for 8 chunks of 512 rows on 4k - 8k keys and for a prompt of 8192, 32 / 8 heads, D = 128.
//     That is 0.8 - 0.9 PFLOP/s; without the exponentials 224 / 281, with one of eight products 191 / 228, without both 156 / 193.  Of the SIMDs' cycles
//     matrix units are busy in 33 % / 42 %, vector instructions issued in 51 % / 63 %, LDS is read in 25 % / 31 % of the compute units', without conflicts;
//   * sums over a tile's 16 registers are a tree, and only they meet the running sum: 16 times fewer roundings in the longest chain;
//   * where few keys leave compute units idle, the (head, row tile) sequence of a key block is cut over several workgroups, whose partial
//     sums a second kernel adds in a fixed order.
#pragma once
#include "fl_bwd_bf16.hpp"

namespace fl {

struct KeyWeightParams {
  const uint16_t* q;               // [B, H, Sq, D], strides in elements
  int64_t q_sb, q_sh, q_ss;
  const uint16_t* k;               // cache: page, token in page, kv head strides in elements
  int64_t k_sp, k_st, k_sh;
  const int32_t* block_table;      // [B, table_stride], or null: sequence b is page b
  int32_t table_stride, page_shift, num_pages;
  const int32_t* seq_lens;
  const float* lse;                // [B, H, Sq]
  int64_t lse_sb, lse_sh, lse_ss;
  float* weights;                  // [B, Hkv, C]
  int64_t w_sb, w_sh;
  float* part;                     // workspace [nsplit, B * Hkv, n_kblocks * 256], or null: one workgroup per key block
  const float* alibi_slopes;
  int32_t B, H, Hkv, Sq, group;
  int32_t max_len, n_kblocks, nsplit;
  int32_t window;                  // < 0: no window
  float scale, softcap;
  Divisor by_problems, by_hkv, by_kblocks, by_split;   // B * Hkv, Hkv, n_kblocks, nsplit
};

template <int D_, int MOD_>
struct KeyWeightCfg : BwdCfg<D_, MOD_, 0, 64, 2> {
  typedef BwdCfg<D_, MOD_, 0, 64, 2> Base;
  static constexpr int NW = 8, KEYS = NW * 32;     // waves and keys per workgroup
  static constexpr int NSTG = 3;
  static constexpr int STAGE = Base::TILE + 64 * 4;          // 64 rows, then their lse
  static constexpr int LDS = NSTG * STAGE;
  static constexpr int IPW = (Base::TILE_INSTR + NW - 1) / NW;           // row loads of a wave per stage; wave 0 loads the lse, too
};

// A capped score cap tanh(s / cap) is s tanh(z) / z with z = s / cap, and tanh(z) / z the cubic 1 + c1 z^2 + c2 z^4 + c3 z^6 to 2^-28 while z is
// below kCapNear (fitted to the largest error up to there).  Beyond, cap - 2 cap / (exp(2 z) + 1): it subtracts numbers of the cap's size, so
// that its roundings are those of scores four times as large; scores of up to 6 under a cap of 1000 would lose 10^-4 of their probabilities.  Up to a
// cap of kCapFar those roundings are about 2^-19 at most, and no block is asked.  (8 chunks of 512 rows on 4k - 8k keys, 32 / 8 heads, us: cap 30,
// D = 128 and 64, 362 and 289, with the quotient everywhere 387 and 338; cap 12, where most blocks have a score beyond, 404 and 386; cap 5 397, and
// 409 with blocks asked.)
constexpr float kCapNear = 0.25f, kCapFar = 8.f, kCap1 = -0.33333242f, kCap2 = 0.13324264f, kCap3 = -0.05143305f;

template <class C>
__global__ void __launch_bounds__(C::NW * 64) __attribute__((amdgpu_waves_per_eu(4, 4))) key_weights_kernel(const KeyWeightParams p) {
  constexpr int D = C::D, KK = C::KK, ROW = C::ROW;
  typedef BwdWave<C> W;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  W w;
  w.init(tid & 63);
  const int lane = w.lane;

  // problems fastest: the workgroups of one (b, hkv) go to one XCD where their number is a multiple of eight, and share its L2; early key
  // blocks, which more rows see, first, with all their parts
  int rest, bh, kb, split, b, hk;
  p.by_problems.split(blockIdx.x, rest, bh);
  p.by_split.split(rest, kb, split);
  p.by_hkv.split(bh, b, hk);
  const int len = min(max(p.seq_lens[b], 0), p.max_len);
  const int k0 = kb * C::KEYS;
  const int first_pos = len - p.Sq;                // position of row 0
  // rows that see a key of the block
  int i_lo = 0, i_hi = 0;
  if (k0 < len) {
    i_lo = max(0, k0 - first_pos);
    i_hi = p.Sq;
    if (p.window >= 0) i_hi = (int)min((int64_t)p.Sq, (int64_t)min(k0 + C::KEYS, len) + p.window - first_pos);
  }
  const int tiles = i_hi > i_lo ? (i_hi - i_lo + 63) / 64 : 0;
  const int items = tiles * p.group;               // (head, row tile) in order
  const int per = (items + p.nsplit - 1) / p.nsplit;
  const int it_begin = min(items, split * per), it_end = min(items, it_begin + per);

  // this wave's keys, in registers: lane = key, 8 channels a fragment; keys past the length repeat the last one
  const int kw = k0 + wave * 32, j = kw + w.col;
  bf16x8 kf[KK];
  float sum = 0.f;
  if (it_begin < it_end) {
    const int jj = min(j, len - 1);
    int64_t page = b, off = jj;
    if (p.block_table != nullptr) {
      page = min(max(p.block_table[(int64_t)b * p.table_stride + (jj >> p.page_shift)], 0), p.num_pages - 1);
      off = jj & ((1 << p.page_shift) - 1);
    }
    const uint16_t* row = p.k + page * p.k_sp + off * p.k_st + hk * p.k_sh;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) kf[kk] = *(const bf16x8*)(row + 16 * kk + 8 * w.half);
  }
  const float c_scale = p.scale * kLog2e;
  // soft-cap: where all raw scores of a block are below near_to, s * (near0 + near1 s^2 + ...) scales and caps them at once; exp2(s * far_in) is
  // exp(2 z), cap_l2 the cap in the log2 domain.  (Within the bounds both and twice them are finite; beyond them a cap changes nothing, or all scores
  // are 0.  near_to keeps the powers finite.)
  float cap_l2 = 0.f, far_in = 0.f, near_to = 0.f, near0 = 0.f, near1 = 0.f, near2 = 0.f, near3 = 0.f;
  if constexpr (C::MOD == kModSoftcap) {
    auto uniform = [](float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); };
    const float cap = fminf(fmaxf(p.softcap, 0x1p-120f), 0x1p120f), z1 = p.scale / cap, square = z1 * z1;   // z of a raw score of 1
    cap_l2 = uniform(cap * kLog2e);
    far_in = uniform(fminf(2.f * c_scale / cap, 0x1p127f));
    near0 = uniform(c_scale);
    near1 = uniform(c_scale * kCap1 * square);
    near2 = uniform(c_scale * kCap2 * square * square);
    near3 = uniform(c_scale * kCap3 * square * square * square);
    near_to = cap > kCapFar && fabsf(near3) < 0x1p100f ? uniform(fminf(kCapNear / z1, 0x1p60f)) : 0.f;
  }

  int ld_head = 0, ld_tile = 0;                    // next item to request
  // byte offsets of this lane's pieces in a whole tile: rows are below 2^23 elements apart, so 32 bits hold them
  uint32_t ld_row[C::IPW], ld_off[C::IPW];
#pragma unroll
  for (int u = 0; u < C::IPW; ++u) {
    const int r = (wave * C::IPW + u) * C::RPI + lane / (D / 8);
    ld_row[u] = (uint32_t)(((lane % (D / 8)) ^ swz_u<D>(r)) * 16);
    ld_off[u] = (uint32_t)(r * (int)p.q_ss * 2) + ld_row[u];
  }
  auto load_item = [&](int stage) __attribute__((always_inline)) {
    const int h = hk * p.group + ld_head, i0 = i_lo + ld_tile * 64;
    unsigned char* st = lds_raw + stage * C::STAGE;
    const unsigned char* base = (const unsigned char*)(p.q + b * p.q_sb + h * p.q_sh + (int64_t)i0 * p.q_ss);
    const bool whole = i0 + 64 <= p.Sq;
#pragma unroll
    for (int u = 0; u < C::IPW; ++u) {
      const int inst = wave * C::IPW + u;
      if (C::TILE_INSTR < C::NW && inst >= C::TILE_INSTR) break;   // (uniform; such a wave's count below waits for less than there is)
      uint32_t off = ld_off[u];
      if (!whole) off = (uint32_t)(min(inst * C::RPI + lane / (D / 8), p.Sq - 1 - i0) * (int)p.q_ss * 2) + ld_row[u];   // the last row again
      __builtin_amdgcn_global_load_lds((global_cvoid*)(base + off), (lds_void*)(st + inst * 1024), 16, 0, 0);
    }
    if (wave == 0) {
      const float* src = p.lse + b * p.lse_sb + h * p.lse_sh + (int64_t)min(i0 + lane, p.Sq - 1) * p.lse_ss;
      __builtin_amdgcn_global_load_lds((global_cvoid*)src, (lds_void*)(st + C::TILE), 4, 0, 0);
    }
    if (++ld_tile == tiles) {
      ld_tile = 0;
      ++ld_head;
    }
  };
  if (tiles > 0) {
    ld_head = it_begin / tiles;
    ld_tile = it_begin - ld_head * tiles;
  }
  int head = ld_head, tile = ld_tile;
  if (it_begin < it_end) load_item(0);
  if (it_begin + 1 < it_end) load_item(1);
  // how far behind a key a row may be that sees it: the window, or what is left up to the sequence's last position
  const uint32_t reach = (uint32_t)(p.window >= 0 ? min(p.window, len - 1 - j) : len - 1 - j);
  int stage = 0;
  for (int it = it_begin; it < it_end; ++it) {
    // this wave's part of the stage has landed (one younger stage may be in flight); behind the barrier everyone's has, and the
    // stage before is free
    if (it + 1 < it_end) {
      if (wave == 0) __builtin_amdgcn_s_waitcnt(((C::IPW + 1) & 15) | 0x0F70 | (((C::IPW + 1) >> 4) << 14));
      else __builtin_amdgcn_s_waitcnt((C::IPW & 15) | 0x0F70 | ((C::IPW >> 4) << 14));
    } else {
      __builtin_amdgcn_s_waitcnt(0x0F70);
    }
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (it + 2 < it_end) load_item(stage == 0 ? 2 : stage - 1);
    const uint32_t base = (uint32_t)(stage * C::STAGE);
    const int i0 = i_lo + tile * 64;
    const float slope2 = C::MOD == kModAlibi ? p.alibi_slopes[hk * p.group + head] * kLog2e : 0.f;
    uint32_t ra_b[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) ra_b[kk] = w.ra[kk] + base;
    static_for<0, 2>([&](auto rbc) __attribute__((always_inline)) {
      constexpr int rb = rbc;
      const int r0 = i0 + 32 * rb;                 // first row of the block
      const int p_lo = first_pos + r0, p_hi = first_pos + min(r0 + 31, p.Sq - 1);   // its positions
      // (uniform) a block past the last row, or whose rows see none of this wave's keys
      if (r0 >= i_hi || p_hi < kw || kw >= len || (p.window >= 0 && p_lo - p.window > min(kw + 32, len) - 1)) return;
      const bool partial = r0 + 31 >= p.Sq || p_lo < kw + 31 || kw + 32 > len || (p.window >= 0 && p_hi - p.window > kw);
      i32x4 ls[4];                                 // lse of rows 8 g + 4 half + 0 .. 3
      const uint32_t ls_at = base + (uint32_t)C::TILE + rb * 128 + 16 * w.half;
      static_for<0, 4>([&](auto g) __attribute__((always_inline)) { W::template read_b128<32 * g>(ls[g], ls_at); });
      f32x16 s = W::zero16();
      w.template row_stream_g<RowOne<rb * 32 * ROW>, KK, 2>([&](auto fc) __attribute__((always_inline)) {
        return ra_b[decltype(fc)::value];
      }, [&](auto fc, bf16x8 a) __attribute__((always_inline)) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, kf[decltype(fc)::value], s, 0, 0, 0);
      });
#pragma unroll
      for (int g = 0; g < 4; ++g) asm volatile("" : "+v"(ls[g]));              // landed: not to be used further up
      float nl[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) nl[r] = __int_as_float(ls[r >> 2][r & 3]) * -kLog2e;
      // row and key `gap` apart, register by register: visible from 0 to `reach` (keys past the length may hold anything)
      const int gap = p_lo + 4 * w.half - j;
      float x[16];
      if constexpr (C::MOD == kModSoftcap) {
        float largest = INFINITY;
        if (near_to > 0.f) {
          largest = 0.f;                           // (NaN is left out: it comes out as NaN either way)
#pragma unroll
          for (int r = 0; r < 16; ++r) largest = fmaxf(largest, fabsf(s[r]));
        }
        if (__builtin_amdgcn_ballot_w64(largest >= near_to) == 0) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float y = s[r] * s[r];
            x[r] = fast_exp2(fmaf(s[r], fmaf(y, fmaf(y, fmaf(y, near3, near2), near1), near0), nl[r]));
          }
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = fast_exp2(fmaf(__int_as_float(ls[r >> 2][r & 3]), -kLog2e, fmaf(fast_rcp(fast_exp2(s[r] * far_in) + 1.f), -2.f * cap_l2, cap_l2)));
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          x[r] = fast_exp2(fmaf(s[r], c_scale, C::MOD == kModAlibi ? fmaf(-slope2, (float)(gap + 8 * (r >> 2) + (r & 3)), nl[r]) : nl[r]));
      }
      if (partial) {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = (uint32_t)(gap + 8 * (r >> 2) + (r & 3)) <= reach ? x[r] : 0.f;
      }
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1)
#pragma unroll
        for (int r = 0; r < d; ++r) x[r] += x[r + d];
      sum += x[0];
    });
    if (++tile == tiles) {
      tile = 0;
      ++head;
    }
    stage = stage == 2 ? 0 : stage + 1;
  }

  const float gained = half_swap_sum(sum);
  if (w.half != 0) return;
  if (p.part != nullptr) {
    p.part[((int64_t)split * p.B * p.Hkv + bh) * p.n_kblocks * C::KEYS + j] = gained;
  } else if (j < len) {
    float* at = p.weights + b * p.w_sb + hk * p.w_sh + j;
    *at = (j < len - p.Sq ? *at : 0.f) + gained;
  }
}

// The partial sums of a key's workgroups, added in order, join its weight.
__global__ void __launch_bounds__(256) key_weights_join_kernel(const KeyWeightParams p) {
  int kb, bh, b, hk;
  p.by_kblocks.split(blockIdx.x, bh, kb);
  p.by_hkv.split(bh, b, hk);
  const int len = min(max(p.seq_lens[b], 0), p.max_len);
  const int j = kb * 256 + threadIdx.x;
  if (j >= len) return;
  float gained = 0.f;
  for (int s = 0; s < p.nsplit; ++s) gained += p.part[(((int64_t)s * p.B * p.Hkv + bh) * p.n_kblocks + kb) * 256 + threadIdx.x];
  float* at = p.weights + b * p.w_sb + hk * p.w_sh + j;
  *at = (j < len - p.Sq ? *at : 0.f) + gained;
}

}  // namespace fl
