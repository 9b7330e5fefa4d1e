// Weight that the rows of a prompt chunk give to each cached key, for gfx950:
//     gained[b, hkv, j] = sum over the query heads h of hkv and the rows i that see j of exp(s_ij - lse_i),
// with s the scores of the forward pass (Eq. 3, score_mod of Eq. 4) and lse what it has left behind: column sums of a matrix that is
// formed tile by tile and never stored.  One contraction of 2 D operations per score, one exponential and some five vector instructions:
// matrix and vector units have about as much to do at D = 128, the vector units more at 64.
//
//   * a wave owns 64 keys, held in registers as the B operand of the MFMA for the whole launch; S = Q K^T then has the key in the lane and
//     the row in the register index, so that a column sum is additions in a lane, and a half swap at the very end;
//   * the rows of the kv head's query heads stream through a ring of three LDS stages of 64 rows that the workgroup's four waves share
//     (one barrier per stage, two stages in flight); with 64 keys per wave a row fragment read from LDS feeds two MFMAs, which
//     halves the LDS traffic to what it can carry beside the matrix units;
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
  static constexpr int KB = 2, KEYS = 4 * 32 * KB; // 32-key blocks per wave; keys per workgroup
  static constexpr int NSTG = 3;
  static constexpr int STAGE = Base::TILE + 64 * 4;          // 64 rows, then their lse
  static constexpr int LDS = NSTG * STAGE;
  static constexpr int IPW = Base::TILE_INSTR / 4;           // row loads of a wave per stage; wave 0 loads the lse, too
};

template <class C>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) key_weights_kernel(const KeyWeightParams p) {
  constexpr int D = C::D, KK = C::KK, ROW = C::ROW, KB = C::KB;
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
    if (p.window >= 0) i_hi = min(p.Sq, capped_sum(min(k0 + C::KEYS, len) - 1, p.window) - first_pos + 1);
  }
  const int tiles = i_hi > i_lo ? (i_hi - i_lo + 63) / 64 : 0;
  const int items = tiles * p.group;               // (head, row tile) in order
  const int per = (items + p.nsplit - 1) / p.nsplit;
  const int it_begin = min(items, split * per), it_end = min(items, it_begin + per);

  // this wave's keys, in registers: lane = key, 8 channels a fragment; keys past the length repeat the last one
  const int kw = k0 + wave * 32 * KB;
  bf16x8 kf[KB][KK];
  float sum[KB];
#pragma unroll
  for (int n = 0; n < KB; ++n) sum[n] = 0.f;
  if (it_begin < it_end) {
#pragma unroll
    for (int n = 0; n < KB; ++n) {
      const int j = min(kw + 32 * n + w.col, len - 1);
      int64_t page = b, off = j;
      if (p.block_table != nullptr) {
        page = min(max(p.block_table[(int64_t)b * p.table_stride + (j >> p.page_shift)], 0), p.num_pages - 1);
        off = j & ((1 << p.page_shift) - 1);
      }
      const uint16_t* row = p.k + page * p.k_sp + off * p.k_st + hk * p.k_sh;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) kf[n][kk] = *(const bf16x8*)(row + 16 * kk + 8 * w.half);
    }
  }
  const float c_scale = p.scale * kLog2e;

  int ld_head = 0, ld_tile = 0;                    // next item to request
  auto load_item = [&](int stage) __attribute__((always_inline)) {
    const int h = hk * p.group + ld_head, i0 = i_lo + ld_tile * 64;
    unsigned char* st = lds_raw + stage * C::STAGE;
    const uint16_t* qb = p.q + b * p.q_sb + h * p.q_sh;
#pragma unroll
    for (int u = 0; u < C::IPW; ++u) {
      const int inst = wave * C::IPW + u;
      const int r = inst * C::RPI + lane / (D / 8);
      const int chunk = (lane % (D / 8)) ^ swz_u<D>(r);
      const uint16_t* src = qb + (int64_t)min(i0 + r, p.Sq - 1) * p.q_ss + chunk * 8;
      __builtin_amdgcn_global_load_lds((global_cvoid*)src, (lds_void*)(st + inst * 1024), 16, 0, 0);
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
  // A block of 32 rows against the wave's keys, in flight between its products and its exponentials.  The products of one block and the
  // exponentials of the one before are a single stream of instructions: a matrix instruction takes the unit for 32 cycles and the wave's
  // issue for four, and what follows it in the stream runs meanwhile.
  struct Block {
    f32x16 s[KB];
    i32x4 ls[4];                                   // lse of rows 8 g + 4 half + 0 .. 3
    int p_lo;                                      // position of its first row
    bool partial;                                  // some score is hidden (or all, of rows past the end among them)
    float slope2;
  };
  Block blk[2] = {};
  uint32_t reach[KB];                              // of a key: the window, and the positions that are left up to the sequence's last
#pragma unroll
  for (int n = 0; n < KB; ++n) {
    const int left = len - 1 - (kw + 32 * n + w.col);
    reach[n] = (uint32_t)(p.window >= 0 ? min(p.window, left) : left);
  }
  // exponentials of registers [R0, R1) of block o
  auto add_up = [&](const Block& o, float (&part)[KB], auto r0c, auto r1c, auto partial) __attribute__((always_inline)) {
    constexpr int R0 = r0c, R1 = r1c;
    float nl[R1 - R0];
#pragma unroll
    for (int r = R0; r < R1; ++r) nl[r - R0] = __int_as_float(o.ls[r >> 2][r & 3]) * -kLog2e;
#pragma unroll
    for (int n = 0; n < KB; ++n) {
      const int j = kw + 32 * n + w.col;
      float x[R1 - R0];
#pragma unroll
      for (int r = R0; r < R1; ++r) {
        const int pos = o.p_lo + 8 * (r >> 2) + 4 * w.half + (r & 3);
        float a;
        if constexpr (C::MOD == kModSoftcap) {
          const float e = fast_exp2(o.s[n][r] * (2.f * c_scale / p.softcap));
          a = fmaf(fast_rcp(e + 1.f), -2.f * p.softcap * kLog2e, p.softcap * kLog2e) + nl[r - R0];
        } else if constexpr (C::MOD == kModAlibi) {
          a = fmaf(o.s[n][r], c_scale, fmaf(-o.slope2, (float)(pos - j), nl[r - R0]));
        } else {
          a = fmaf(o.s[n][r], c_scale, nl[r - R0]);
        }
        x[r - R0] = fast_exp2(a);
      }
      if constexpr (partial) {
        // row and key `gap` apart: visible from 0 to reach[n] (no branches in here; keys past the length may hold anything)
        const int gap = o.p_lo + 4 * w.half - j;
#pragma unroll
        for (int r = R0; r < R1; ++r) x[r - R0] = (uint32_t)(gap + 8 * (r >> 2) + (r & 3)) <= reach[n] ? x[r - R0] : 0.f;
      }
#pragma unroll
      for (int d = (R1 - R0) / 2; d >= 1; d >>= 1)
#pragma unroll
        for (int r = 0; r < d; ++r) x[r] += x[r + d];
      part[n] += x[0];
    }
  };
  int stage = 0;
  bool pending = false;                            // blk[1] waits for its exponentials
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
    uint32_t ra_b[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) ra_b[kk] = w.ra[kk] + base;
    static_for<0, 2>([&](auto rbc) __attribute__((always_inline)) {
      constexpr int rb = rbc;
      Block& now = blk[rb];
      const Block& before = blk[rb ^ 1];
      const int r0 = i0 + 32 * rb;                 // first row of the block
      const int p_hi = first_pos + min(r0 + 31, p.Sq - 1);
      now.p_lo = first_pos + r0;
      now.partial = r0 + 31 >= p.Sq || now.p_lo < kw + 32 * KB - 1 || kw + 32 * KB > len || (p.window >= 0 && p_hi - p.window > kw);
      now.slope2 = C::MOD == kModAlibi ? p.alibi_slopes[hk * p.group + head] * kLog2e : 0.f;
      const uint32_t ls_at = base + (uint32_t)C::TILE + rb * 128 + 16 * w.half;
      static_for<0, 4>([&](auto g) __attribute__((always_inline)) { W::template read_b128<32 * g>(now.ls[g], ls_at); });
#pragma unroll
      for (int n = 0; n < KB; ++n) now.s[n] = W::zero16();
      float part[KB];
#pragma unroll
      for (int n = 0; n < KB; ++n) part[n] = 0.f;
      auto products = [&](auto partial) __attribute__((always_inline)) {
        w.template row_stream_g<RowOne<rb * 32 * ROW>, KK, 2>([&](auto fc) __attribute__((always_inline)) {
          return ra_b[decltype(fc)::value];
        }, [&](auto fc, bf16x8 a) __attribute__((always_inline)) {
          constexpr int f = decltype(fc)::value, RS = 16 / KK;
#pragma unroll
          for (int n = 0; n < KB; ++n) now.s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, kf[n][f], now.s[n], 0, 0, 0);
          add_up(before, part, std::integral_constant<int, RS * f>(), std::integral_constant<int, RS * (f + 1)>(), partial);
        });
      };
      if (before.partial) products(std::true_type());
      else products(std::false_type());
#pragma unroll
      for (int g = 0; g < 4; ++g) asm volatile("" : "+v"(now.ls[g]));          // landed: not to be used further up
      if (rb == 1 || pending) {
#pragma unroll
        for (int n = 0; n < KB; ++n) sum[n] += part[n];
      }
    });
    pending = true;
    if (++tile == tiles) {
      tile = 0;
      ++head;
    }
    stage = stage == 2 ? 0 : stage + 1;
  }
  if (pending) {
    float part[KB];
#pragma unroll
    for (int n = 0; n < KB; ++n) part[n] = 0.f;
    add_up(blk[1], part, std::integral_constant<int, 0>(), std::integral_constant<int, 16>(), std::true_type());
#pragma unroll
    for (int n = 0; n < KB; ++n) sum[n] += part[n];
  }

#pragma unroll
  for (int n = 0; n < KB; ++n) {
    const float gained = half_swap_sum(sum[n]);
    const int j = kw + 32 * n + w.col;
    if (w.half != 0) continue;
    if (p.part != nullptr) {
      p.part[((int64_t)split * p.B * p.Hkv + bh) * p.n_kblocks * C::KEYS + j] = gained;
    } else if (j < len) {
      float* at = p.weights + b * p.w_sb + hk * p.w_sh + j;
      *at = (j < len - p.Sq ? *at : 0.f) + gained;
    }
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
