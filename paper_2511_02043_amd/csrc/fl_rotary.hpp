// Rotary positions with several axes for gfx950, and the write of turned keys and of values into a paged cache.
//
// Channel pair i of a query or key turns by t = position[axis of i] * inv_freq[i]:
//     (x_a, x_b)  ->  (x_a cos t - x_b sin t,  x_b cos t + x_a sin t),
// an orthogonal map, so that its gradient is the same with -t.  Every element is read once and written once, at six operations per
// pair: the work is memory traffic.  What could outgrow it is the angle: one sine and cosine per (token, pair), with the angle reduced in
// 64 bits (a float's product with a position of 10^5 leaves 10^-2 of phase).  A thread therefore owns one token and VEC pairs, forms their
// angles once and turns several heads with them; its pieces of a head are 16-byte loads and stores, neighbouring threads continue a row.
// Measured: 2 x 8192 tokens, 32 / 8 heads, D = 128, bf16 80 us a pass (4.2 TB/s; a large copy 4.9), 8 x 512 tokens into the cache 19 - 22 (4.6 - 5.3), one
// token of 64 sequences 5, a chain of loads: length, page, row.
#pragma once
#include "fl_params.hpp"

namespace fl {

struct RotaryParams {
  View q, k, v, q_out, k_out;      // [B, 1, heads, S, D]
  const int32_t* positions;        // [B, S, axes], strides in elements
  int64_t pos_sb, pos_ss, pos_sa;
  const float* inv_freq;           // [pairs]
  int32_t ends[4];                 // pairs of the axes up to and with each; the last one is `pairs`
  int32_t axes, pairs, D;
  int32_t inverse;
  int32_t B, S, H, Hkv;
  int32_t heads_per_thread;
  int32_t units, tokens_per_block; // units: pieces of VEC pairs, then of VEC channels that stay, of a row
  Divisor by_s, by_units;
  // fl_rotary_append: where keys and values go
  uint16_t* k_cache;               // page, token in page, kv head strides in elements
  uint16_t* v_cache;
  int64_t kc_sp, kc_st, kc_sh, vc_sp, vc_st, vc_sh;
  const int32_t* block_table;      // [B, table_stride], or null: sequence b is page b
  int32_t table_stride, page_shift, num_pages, max_len;
  const int32_t* seq_lens;
};

template <class T>
struct RotaryElem;
template <>
struct RotaryElem<uint16_t> {      // bf16
  static __device__ __forceinline__ float load(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
  static __device__ __forceinline__ uint16_t store(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
  // the machine's sine and cosine (of whole turns); the tests hold a result to 2^-14 of its pair's length beside its own rounding of 2^-8
  static __device__ __forceinline__ void sincos_turns(float r, float& s, float& c) {
    s = __builtin_amdgcn_sinf(r);
    c = __builtin_amdgcn_cosf(r);
  }
};
template <>
struct RotaryElem<float> {
  static __device__ __forceinline__ float load(float x) { return x; }
  static __device__ __forceinline__ float store(float x) { return x; }
  static __device__ __forceinline__ void sincos_turns(float r, float& s, float& c) { sincospif(2.f * r, &s, &c); }
};

template <class T, int VEC>
struct alignas(VEC * sizeof(T)) RotaryPiece {
  T x[VEC];
};

// One of VEC pairs' two pieces: (i, i + pairs) are a piece each; interleaved pairs (2i, 2i + 1) fill both, one after the other.
template <class T, int VEC, bool INTERLEAVED, bool APPEND>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryParams p) {
  typedef RotaryPiece<T, VEC> Piece;
  typedef RotaryElem<T> E;
  constexpr int HU = VEC == 1 ? 2 : 4;             // heads whose loads are in flight together
  const int tid = threadIdx.x;
  int local, first_unit;
  if (p.units <= 256) p.by_units.split(tid, local, first_unit);
  else local = 0, first_unit = tid;                // a row of more pieces than threads: several each
  const int64_t token = (int64_t)blockIdx.x * p.tokens_per_block + local;
  if (local >= p.tokens_per_block || token >= (int64_t)p.B * p.S) return;
  int b, s;
  p.by_s.split((int)token, b, s);

  int32_t pos[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) pos[a] = a < p.axes ? p.positions[b * p.pos_sb + s * p.pos_ss + a * p.pos_sa] : 0;

  T* k_slot = nullptr;                             // APPEND: this token's row of kv head 0 in the caches; null: it has none
  T* v_slot = nullptr;
  if constexpr (APPEND) {
    // (from the true length: cut to the bound as in the calls that read, it would put the tokens on the slots of older ones)
    const int slot = max(p.seq_lens[b], 0) - p.S + s;
    if (slot >= 0 && slot < p.max_len) {
      int64_t page = b, in_page = slot;
      if (p.block_table != nullptr) {
        page = p.block_table[(int64_t)b * p.table_stride + (slot >> p.page_shift)];
        in_page = slot & ((1 << p.page_shift) - 1);
      }
      if (page >= 0 && page < p.num_pages) {
        k_slot = (T*)p.k_cache + page * p.kc_sp + in_page * p.kc_st;
        v_slot = (T*)p.v_cache + page * p.vc_sp + in_page * p.vc_st;
      }
    }
  }
  const T* const q_in = (const T*)p.q.ptr + b * p.q.sb + s * p.q.ss;
  const T* const k_in = (const T*)p.k.ptr + b * p.k.sb + s * p.k.ss;
  const T* const v_in = APPEND ? (const T*)p.v.ptr + b * p.v.sb + s * p.v.ss : nullptr;
  T* const q_to = (T*)p.q_out.ptr + b * p.q_out.sb + s * p.q_out.ss;
  T* const k_to = APPEND ? k_slot : (T*)p.k_out.ptr + b * p.k_out.sb + s * p.k_out.ss;
  const int64_t k_to_sh = APPEND ? p.kc_sh : p.k_out.sh;

  const int h_begin = blockIdx.y * p.heads_per_thread;
  const int h_end = min(h_begin + p.heads_per_thread, p.H + p.Hkv + (APPEND ? p.Hkv : 0));
  const int turning = p.pairs / VEC;

  for (int unit = first_unit; unit < p.units; unit += 256) {
    const bool turns = unit < turning;
    const int at0 = turns ? (INTERLEAVED ? 2 * unit * VEC : unit * VEC) : 2 * p.pairs + (unit - turning) * VEC;
    const int at1 = turns ? (INTERLEAVED ? at0 + VEC : p.pairs + at0) : at0;         // a piece that stays is read and written as both
    Piece x0[HU], x1[HU];
    auto load = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < HU; ++u) {
        const int h = h0 + u;
        if (h < h_end) {
          const T* in = h < p.H ? q_in + h * p.q.sh : (h < p.H + p.Hkv ? k_in + (h - p.H) * p.k.sh : v_in + (h - p.H - p.Hkv) * p.v.sh);
          x0[u] = *(const Piece*)(in + at0);
          x1[u] = *(const Piece*)(in + at1);
        }
      }
    };
    load(h_begin);                                 // on their way while the angles are formed
    float cs[VEC], sn[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      cs[j] = 1.f;
      sn[j] = 0.f;
    }
    if (turns) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int pair = unit * VEC + j;
        const int32_t at = pair < p.ends[0] ? pos[0] : (pair < p.ends[1] ? pos[1] : (pair < p.ends[2] ? pos[2] : pos[3]));
        const double turn = (double)at * ((double)p.inv_freq[pair] * 0.15915494309189533577);   // in whole turns
        E::sincos_turns((float)(turn - rint(turn)), sn[j], cs[j]);
        if (p.inverse) sn[j] = -sn[j];
      }
    }
    for (int h0 = h_begin; h0 < h_end; h0 += HU) {
      if (h0 > h_begin) load(h0);
#pragma unroll
      for (int u = 0; u < HU; ++u) {
        const int h = h0 + u;
        if (h < h_end) {
          T* to;
          if (h < p.H) to = q_to + h * p.q_out.sh;
          else if (h < p.H + p.Hkv) to = k_to != nullptr ? k_to + (h - p.H) * k_to_sh : nullptr;
          else to = v_slot != nullptr ? v_slot + (h - p.H - p.Hkv) * p.vc_sh : nullptr;
          if (turns && (!APPEND || h < p.H + p.Hkv)) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              T& ta = INTERLEAVED ? (2 * j < VEC ? x0[u].x[(2 * j) % VEC] : x1[u].x[(2 * j) % VEC]) : x0[u].x[j];
              T& tb = INTERLEAVED ? (2 * j + 1 < VEC ? x0[u].x[(2 * j + 1) % VEC] : x1[u].x[(2 * j + 1) % VEC]) : x1[u].x[j];
              const float a = E::load(ta), c = E::load(tb);
              ta = E::store(a * cs[j] - c * sn[j]);
              tb = E::store(c * cs[j] + a * sn[j]);
            }
          }
          if (to != nullptr) {
            *(Piece*)(to + at0) = x0[u];
            *(Piece*)(to + at1) = x1[u];
          }
        }
      }
    }
  }
}

}  // namespace fl
