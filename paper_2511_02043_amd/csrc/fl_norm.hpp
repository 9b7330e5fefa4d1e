// Heads normalised and turned for gfx950: forward pass, gradient, and the write of new tokens into a paged cache.
//
// Every row x of a query or key head (D channels) becomes
//     y = R(t) z,   z = w r x,   r = (mean_c x_c^2 + eps)^(-1/2),
// with R the turn of channel pairs by the positions' angles (fl_rotary.hpp).  Its gradient, with dz = R(-t) dy and g = w dz:
//     dx = r (g - u mean_c(u_c g_c)),  u = r x,     dw = sum over tokens and heads of u dz.
// An element is read once (the gradient: x and dy) and written once, at some twenty operations: memory traffic, if the row's sum costs no second pass and the
// angles little.  A row therefore lies in the registers of a few lanes: lane `sub` of a group of them has the row's pairs sub VEC .. (two pieces of VEC channels,
// 16 bytes each, at D = 128 eight lanes), and the sum is three exchanges between neighbours.  Forwards a workgroup has some tokens: it forms their angles
// once, one (token, pair) a thread, keeps them in LDS, and goes through the rows in the order of memory, heads of a token first, so that its waves read and
// write long runs (2 x 8192 tokens, 32 / 8 heads, D = 128, bf16: 63 - 70 us, 4.8 - 5.3 TB/s; fp32 130; lane groups that stay with a token and its angles, pieces of
// 256 bytes 12 KB apart, 81).
#pragma once
#include "fl_mx4.hpp"
#include "fl_rotary.hpp"

namespace fl {

struct NormParams : RotaryParams {
  const float* weight[2];          // of queries and keys, [D], or null: ones
  float eps;
  int32_t norm;                    // 0: turns alone (appending only)
  int32_t log_lanes;               // lanes of a row: 2^log_lanes, times UPL at least the units
  Divisor by_pairs, by_h, by_hkv;
  // gradient
  View dy[2], dx[2];
  int32_t q_chunks, k_chunks;      // workgroups along y that take queries, keys, heads_per_thread heads each
  int32_t blocks, groups;          // workgroups along x; groups of tokens_per_block tokens that they share out
  float* part;                     // [q_chunks + k_chunks][blocks][D]: sums of dw; null: not wanted
  float* dweight[2];               // [D], or null: not wanted
  // appending
  int32_t rows_per_part;           // of the keys', queries' and values' rows of its tokens that a workgroup of a column takes
  Mx4Cache mx4;
  View k_held, v_held;             // what a cache in 4 bits holds for the new tokens; ptr null: not wanted
};

// Sums over the `lanes` lanes of each group, N of them at once.
template <int N>
__device__ __forceinline__ void group_sum(float (&x)[N], int lanes) {
  auto dpp = [&](auto ctrl) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      x[i] += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x[i]), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  if (lanes > 1) dpp(std::integral_constant<int, 0xB1>{});           // lane ^ 1
  if (lanes > 2) dpp(std::integral_constant<int, 0x4E>{});           // lane ^ 2
  if (lanes > 4) dpp(std::integral_constant<int, 0x141>{});          // mirrored in eight: the other four
  if (lanes > 8) dpp(std::integral_constant<int, 0x140>{});          // mirrored in sixteen: the other eight
#pragma unroll
  for (int o = 16; o < 64; o <<= 1)
    if (lanes > o)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += __shfl_xor(x[i], o);
}
__device__ __forceinline__ double group_sum(double x, int lanes) {
  auto dpp = [&](auto ctrl) __attribute__((always_inline)) {
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), decltype(ctrl)::value, 0xF, 0xF, true);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), decltype(ctrl)::value, 0xF, 0xF, true);
    x += __hiloint2double(hi, lo);
  };
  if (lanes > 1) dpp(std::integral_constant<int, 0xB1>{});
  if (lanes > 2) dpp(std::integral_constant<int, 0x4E>{});
  if (lanes > 4) dpp(std::integral_constant<int, 0x141>{});
  if (lanes > 8) dpp(std::integral_constant<int, 0x140>{});
  for (int o = 16; o < lanes; o <<= 1) x += __shfl_xor(x, o);
  return x;
}

// STREAM: rows are read past the caches, where a group of lanes' pieces are whole lines of 128 bytes (a line read in halves would come twice).  For rows on their way into a
// cache, whose results are read next and they never again: 8 x 512 tokens, 32 / 8 heads, D = 128, into 4 bits 26.5 -> 24.7 us.  Forward pass and gradient gain where their results stay in the
// caches (68 -> 59 us and 119 -> 100, written to the same place again and again) and lose where they leave them, as in a training step of both (2 x 8192 tokens: 186 us
// without, 194 with, for the gradient finds part of what the forward pass has read), so they do not.
// What a lane has of every row: UPL units of VEC pairs, or of VEC channels that stay (x1 unused then).
template <class T, int VEC, int UPL, bool INTERLEAVED, bool STREAM = false>
struct NormLane {
  typedef RotaryPiece<T, VEC> Piece;
  typedef RotaryElem<T> E;
  typedef __attribute__((ext_vector_type(4))) uint32_t Quad;
  int at0[UPL], at1[UPL];
  bool has[UPL], turns[UPL];
  int lanes;

  __device__ __forceinline__ void init(const NormParams& p, int sub) {
    lanes = 1 << p.log_lanes;
#pragma unroll
    for (int n = 0; n < UPL; ++n) {
      const int unit = sub + n * lanes, turning = p.pairs / VEC;
      has[n] = unit < p.units;
      turns[n] = unit < turning;
      // (VEC neighbouring channels are whole pairs where neighbours pair, so that both kinds have the same pieces; VEC 1: a pair)
      at0[n] = turns[n] ? (INTERLEAVED && VEC == 1 ? 2 * unit : unit * VEC) : (has[n] ? 2 * p.pairs + (unit - turning) * VEC : 0);
      at1[n] = turns[n] ? (INTERLEAVED && VEC == 1 ? at0[n] + 1 : p.pairs + at0[n]) : at0[n];
    }
  }
  // the number of pair j of unit `unit`
  __device__ __forceinline__ static int pair_of(const NormParams& p, int unit, int j) {
    if (!INTERLEAVED || VEC == 1) return unit * VEC + j;
    return unit * (VEC / 2) + (j < VEC / 2 ? j : p.pairs / 2 + j - VEC / 2);
  }
  __device__ __forceinline__ void load(const T* row, Piece (&x0)[UPL], Piece (&x1)[UPL]) const {
#pragma unroll
    for (int n = 0; n < UPL; ++n) {                // (lanes without a unit read the row's first channels)
      if constexpr (STREAM) {
        x0[n] = __builtin_bit_cast(Piece, __builtin_nontemporal_load((const Quad*)(row + at0[n])));
        x1[n] = __builtin_bit_cast(Piece, __builtin_nontemporal_load((const Quad*)(row + at1[n])));
      } else {
        x0[n] = *(const Piece*)(row + at0[n]);
        x1[n] = *(const Piece*)(row + at1[n]);
      }
    }
  }
  __device__ __forceinline__ void store(T* row, const Piece (&x0)[UPL], const Piece (&x1)[UPL]) const {
#pragma unroll
    for (int n = 0; n < UPL; ++n) {
      if (has[n]) *(Piece*)(row + at0[n]) = x0[n];
      if (turns[n]) *(Piece*)(row + at1[n]) = x1[n];
    }
  }
  __device__ __forceinline__ void weights(const float* w, float (&w0)[UPL][VEC], float (&w1)[UPL][VEC]) const {
#pragma unroll
    for (int n = 0; n < UPL; ++n)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        w0[n][j] = w[at0[n] + j];
        w1[n][j] = w[at1[n] + j];
      }
  }
  // channels of pair j of a unit: (first piece, element) and (second piece, element)
  template <class P>
  __device__ __forceinline__ static auto& a_of(P& x0, P& x1, int j) { return INTERLEAVED ? (2 * j < VEC ? x0[(2 * j) % VEC] : x1[(2 * j) % VEC]) : x0[j]; }
  template <class P>
  __device__ __forceinline__ static auto& b_of(P& x0, P& x1, int j) {
    return INTERLEAVED ? (2 * j + 1 < VEC ? x0[(2 * j + 1) % VEC] : x1[(2 * j + 1) % VEC]) : x1[j];
  }
};

// What a wave's lanes have written to LDS before is there for what they read behind.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The angle of a token and channel pair in whole turns, reduced in 64 bits.
__device__ __forceinline__ double turn_of(const NormParams& p, int token, int pair) {
  int b, s;
  p.by_s.split(token, b, s);
  const int axis = pair < p.ends[0] ? 0 : (pair < p.ends[1] ? 1 : (pair < p.ends[2] ? 2 : 3));
  const double turn = (double)p.positions[b * p.pos_sb + s * p.pos_ss + axis * p.pos_sa] * ((double)p.inv_freq[pair] * 0.15915494309189533577);
  return turn - rint(turn);
}
// ... and sine and cosine of all pairs of n tokens from `token` on, [token][pair]
template <class T>
__device__ __forceinline__ void form_angles(const NormParams& p, int token, int n, float* cs, float* sn) {
  for (int i = threadIdx.x; i < n * p.pairs; i += 256) {
    int t, pair;
    p.by_pairs.split(i, t, pair);
    float c, x;
    RotaryElem<T>::sincos_turns((float)turn_of(p, token + t, pair), x, c);
    cs[i] = c;
    sn[i] = x;
  }
}
__device__ __forceinline__ int64_t row_at(const View& v, int b, int s) { return b * v.sb + s * v.ss; }

// Rows [row, row_end) of a workgroup's tokens, `heads` to a token: normalised, weighted and turned from `in` to `out`.  at_in(t), at_out(t): where token t's
// rows begin (at_out < 0: nowhere).
template <class T, int VEC, int UPL, bool INTERLEAVED, bool STREAM, class In, class Out>
__device__ __forceinline__ void norm_rows(const NormParams& p, const NormLane<T, VEC, UPL, INTERLEAVED, STREAM>& l, int sub, const T* in, int64_t in_sh, In at_in, T* out,
                                          int64_t out_sh, Out at_out, const float* weight, const Divisor& by_heads, int row, int row_end, const float* cs,
                                          const float* sn) {
#pragma clang fp contract(off)                     // one rounding order in training and in serving
  typedef NormLane<T, VEC, UPL, INTERLEAVED, STREAM> L;
  typedef RotaryElem<T> E;
  constexpr int HU = UPL * VEC <= 8 ? 2 : 1;       // rows whose loads are in flight together
  const int step = 256 >> p.log_lanes;
  float w0[UPL][VEC], w1[UPL][VEC];
  l.weights(weight, w0, w1);
  const float inv_d = 1.f / p.D;
  for (int r0 = row + (threadIdx.x >> p.log_lanes); r0 < row_end; r0 += HU * step) {
    typename L::Piece x0[HU][UPL], x1[HU][UPL];
    int t[HU], h[HU];
    float sum[HU] = {};
#pragma unroll
    for (int u = 0; u < HU; ++u) {
      by_heads.split(min(r0 + u * step, row_end - 1), t[u], h[u]);
      if (r0 + u * step < row_end) l.load(in + at_in(t[u]) + h[u] * in_sh, x0[u], x1[u]);
    }
    if (p.norm) {
#pragma unroll
      for (int u = 0; u < HU; ++u)
#pragma unroll
        for (int n = 0; n < UPL; ++n)
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float a = E::load(x0[u][n].x[j]), c = E::load(x1[u][n].x[j]);
            sum[u] = l.has[n] ? fmaf(a, a, sum[u]) : sum[u];
            sum[u] = l.turns[n] ? fmaf(c, c, sum[u]) : sum[u];
          }
      group_sum(sum, l.lanes);
    }
#pragma unroll
    for (int u = 0; u < HU; ++u) {
      if (r0 + u * step >= row_end) break;
      const float r = p.norm ? 1.f / sqrtf(fmaf(sum[u], inv_d, p.eps)) : 1.f;
#pragma unroll
      for (int n = 0; n < UPL; ++n) {
        float z0[VEC], z1[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          z0[j] = E::load(x0[u][n].x[j]) * r * w0[n][j];
          z1[j] = E::load(x1[u][n].x[j]) * r * w1[n][j];
        }
        if (l.turns[n]) {
          const int first = t[u] * p.pairs;
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            float &a = L::a_of(z0, z1, j), &c = L::b_of(z0, z1, j);
            const int pair = first + L::pair_of(p, sub + n * l.lanes, j);
            const float a_in = a, c_in = c, co = cs[pair], si = sn[pair];
            a = fmaf(a_in, co, -(c_in * si));
            c = fmaf(c_in, co, a_in * si);
          }
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          x0[u][n].x[j] = E::store(z0[j]);
          x1[u][n].x[j] = E::store(z1[j]);
        }
      }
      const int64_t to = at_out(t[u]);
      if (to >= 0) l.store(out + to + h[u] * out_sh, x0[u], x1[u]);
    }
  }
}

// A workgroup's LDS: cosines and sines [tokens][pairs], then `places` numbers a token, where its rows begin, the weights [2][D], then what a kernel has beside.
struct NormLds {
  float *cs, *sn;
  int64_t* at;
  float* w;
  void* rest;
};
__device__ __forceinline__ NormLds norm_lds(const NormParams& p, void* base, int places) {
  NormLds x;
  x.cs = (float*)base;
  x.sn = x.cs + p.tokens_per_block * p.pairs;
  x.at = (int64_t*)(x.sn + p.tokens_per_block * p.pairs);
  x.w = (float*)(x.at + places * p.tokens_per_block);
  x.rest = x.w + 2 * p.D;
  return x;
}
constexpr size_t norm_lds_bytes(int tokens, int pairs, int places, int D) { return (size_t)tokens * (pairs * 8 + places * 8) + (size_t)D * 8; }

// The weights of queries and keys into LDS.  (Read by every lane from memory when its rows begin, they cost a round trip behind the barrier: 8 x 512 tokens into
// a bf16 cache 29.6 us, without weights 24.6.)
__device__ __forceinline__ void hold_weights(const NormParams& p, float* w) {
  for (int i = threadIdx.x; i < 2 * p.D; i += 256) {
    const float* from = p.weight[i >= p.D];
    w[i] = from != nullptr ? from[i < p.D ? i : i - p.D] : 1.f;
  }
}

template <class T, int VEC, int UPL, bool INTERLEAVED>
__global__ void __launch_bounds__(256) norm_rotary_kernel(const NormParams p) {
  extern __shared__ int64_t norm_shared[];
  const NormLds x = norm_lds(p, norm_shared, 4);
  const int sub = threadIdx.x & ((1 << p.log_lanes) - 1);
  const int token = blockIdx.x * p.tokens_per_block, n = min(p.tokens_per_block, p.B * p.S - token);
  if ((int)threadIdx.x < n) {
    int b, s;
    p.by_s.split(token + threadIdx.x, b, s);
    int64_t* at = x.at + 4 * threadIdx.x;
    at[0] = row_at(p.q, b, s);
    at[1] = row_at(p.q_out, b, s);
    at[2] = row_at(p.k, b, s);
    at[3] = row_at(p.k_out, b, s);
  }
  hold_weights(p, x.w);
  form_angles<T>(p, token, n, x.cs, x.sn);
  __syncthreads();
  NormLane<T, VEC, UPL, INTERLEAVED> l;
  l.init(p, sub);
  auto rows = [&](const View& in, const View& out, int place, int heads, const Divisor& by, const float* weight) __attribute__((always_inline)) {
    norm_rows<T, VEC, UPL, INTERLEAVED, false>(p, l, sub, (const T*)in.ptr, in.sh, [&](int t) { return x.at[4 * t + place]; }, (T*)out.ptr, out.sh,
                                        [&](int t) { return x.at[4 * t + place + 1]; }, weight, by, 0, n * heads, x.cs, x.sn);
  };
  rows(p.q, p.q_out, 0, p.H, p.by_h, x.w);
  rows(p.k, p.k_out, 2, p.Hkv, p.by_hkv, x.w + p.D);
}

// The gradient: 115 - 118 us at those sizes, 4.3 - 4.4 TB/s of three tensors, and 5 for the weights' sums (fp32 225 and 7).  Its rows' angles stay in registers: a group of lanes keeps to a token and goes through the chunk of heads that the workgroup has of it, the next
// head's rows on their way while one is worked on.  (us with the rows shared out as in the forward pass / so: 2 x 8192 tokens, 32 / 8 heads, D = 128 121 / 118,
// D = 64 71 / 63, 512 tokens 18 / 15; here the exchange with LDS and the places of a row cost more than the runs give.)
// dw gathers in registers, then over the workgroup in LDS, and leaves as a row of partial sums for norm_weights_kernel: no atomics, so that the result does
// not depend on who comes first.
template <class T, int VEC, int UPL, bool INTERLEAVED>
__global__ void __launch_bounds__(256) norm_rotary_bwd_kernel(const NormParams p) {
  typedef NormLane<T, VEC, UPL, INTERLEAVED> L;
  typedef RotaryElem<T> E;
  extern __shared__ float dw_lds[];                // [waves][D]; before, the weights
  const int sub = threadIdx.x & ((1 << p.log_lanes) - 1), local = threadIdx.x >> p.log_lanes;
  L l;
  l.init(p, sub);
  const bool keys = (int)blockIdx.y >= p.q_chunks;
  const int heads = keys ? p.Hkv : p.H, h_begin = (blockIdx.y - (keys ? p.q_chunks : 0)) * p.heads_per_thread, h_end = min(h_begin + p.heads_per_thread, heads);
  const View &xv = keys ? p.k : p.q, &yv = p.dy[keys], &ov = p.dx[keys];
  float w0[UPL][VEC], w1[UPL][VEC], d0[UPL][VEC] = {}, d1[UPL][VEC] = {};
  for (int i = threadIdx.x; i < p.D; i += 256) dw_lds[i] = p.weight[keys] != nullptr ? p.weight[keys][i] : 1.f;
  __syncthreads();
  l.weights(dw_lds, w0, w1);
  __syncthreads();                                 // (before anyone's sums take their place)
  const float inv_d = 1.f / p.D;

  for (int group = blockIdx.x; group < p.groups; group += p.blocks) {
    const int64_t token = (int64_t)group * p.tokens_per_block + local;
    if (token >= (int64_t)p.B * p.S) continue;     // (whole groups of lanes)
    int b, s;
    p.by_s.split((int)token, b, s);
    const T* x_in = (const T*)xv.ptr + row_at(xv, b, s);
    const T* y_in = (const T*)yv.ptr + row_at(yv, b, s);
    T* out = (T*)ov.ptr + row_at(ov, b, s);
    typename L::Piece x0[UPL], x1[UPL], y0[UPL], y1[UPL];
    l.load(x_in + h_begin * xv.sh, x0, x1);
    l.load(y_in + h_begin * yv.sh, y0, y1);
    float cs[UPL][VEC], sn[UPL][VEC];
#pragma unroll
    for (int n = 0; n < UPL; ++n)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        cs[n][j] = 1.f;
        sn[n][j] = 0.f;
        if (l.turns[n]) E::sincos_turns((float)turn_of(p, (int)token, L::pair_of(p, sub + n * l.lanes, j)), sn[n][j], cs[n][j]);
      }
    for (int h = h_begin; h < h_end; ++h) {
      float sum[2] = {};                           // of x^2 and of x g
      float z0[UPL][VEC], z1[UPL][VEC], a0[UPL][VEC], a1[UPL][VEC];                  // dz, x
#pragma unroll
      for (int n = 0; n < UPL; ++n) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          a0[n][j] = l.has[n] ? E::load(x0[n].x[j]) : 0.f;
          a1[n][j] = l.turns[n] ? E::load(x1[n].x[j]) : 0.f;
          z0[n][j] = l.has[n] ? E::load(y0[n].x[j]) : 0.f;
          z1[n][j] = l.turns[n] ? E::load(y1[n].x[j]) : 0.f;
        }
      }
      const int next = min(h + 1, h_end - 1);
      l.load(x_in + next * xv.sh, x0, x1);
      l.load(y_in + next * yv.sh, y0, y1);
#pragma unroll
      for (int n = 0; n < UPL; ++n) {
        if (l.turns[n]) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            float &a = L::a_of(z0[n], z1[n], j), &c = L::b_of(z0[n], z1[n], j);
            const float a_in = a, c_in = c;
            a = a_in * cs[n][j] + c_in * sn[n][j];
            c = c_in * cs[n][j] - a_in * sn[n][j];
          }
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          sum[0] = fmaf(a0[n][j], a0[n][j], fmaf(a1[n][j], a1[n][j], sum[0]));
          sum[1] = fmaf(a0[n][j] * w0[n][j], z0[n][j], fmaf(a1[n][j] * w1[n][j], z1[n][j], sum[1]));
        }
      }
      group_sum(sum, l.lanes);
      // (r^3 is formed nowhere: it is subnormal from rows of 2^42 on and infinite for rows below 2^-43, where everything else here is an ordinary number)
      const float r = 1.f / sqrtf(fmaf(sum[0], inv_d, p.eps)), mean = r * (sum[1] * inv_d);     // of u g
      typename L::Piece o0[UPL], o1[UPL];
#pragma unroll
      for (int n = 0; n < UPL; ++n)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float a = a0[n][j] * r, c = a1[n][j] * r;
          d0[n][j] = fmaf(a, z0[n][j], d0[n][j]);
          d1[n][j] = fmaf(c, z1[n][j], d1[n][j]);
          o0[n].x[j] = E::store(r * fmaf(w0[n][j], z0[n][j], -a * mean));
          o1[n].x[j] = E::store(r * fmaf(w1[n][j], z1[n][j], -c * mean));
        }
      if (ov.ptr != nullptr) l.store(out + h * ov.sh, o0, o1);
    }
  }

  if (p.part == nullptr) return;
  // over the groups of lanes of a wave, then over the waves
#pragma unroll
  for (int n = 0; n < UPL; ++n)
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      for (int o = l.lanes; o < 64; o <<= 1) {
        d0[n][j] += __shfl_xor(d0[n][j], o);
        d1[n][j] += __shfl_xor(d1[n][j], o);
      }
  const int wave = threadIdx.x >> 6;
  if ((int)(threadIdx.x & 63) < l.lanes) {
#pragma unroll
    for (int n = 0; n < UPL; ++n)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if (l.has[n]) dw_lds[wave * p.D + l.at0[n] + j] = d0[n][j];
        if (l.turns[n]) dw_lds[wave * p.D + l.at1[n] + j] = d1[n][j];
      }
  }
  __syncthreads();
  float* to = p.part + ((int64_t)blockIdx.y * p.blocks + blockIdx.x) * p.D;
  for (int c = threadIdx.x; c < p.D; c += 256) to[c] = (dw_lds[c] + dw_lds[p.D + c]) + (dw_lds[2 * p.D + c] + dw_lds[3 * p.D + c]);
}

// dw: the sum of the workgroups' rows.  Workgroup (c, which) has channels 16 c .. + 15, a thread every 64th row of one of them.
__global__ void __launch_bounds__(1024) norm_weights_kernel(const NormParams p) {
  __shared__ float lds[1024];
  const int which = blockIdx.y, c = blockIdx.x * 16 + (threadIdx.x & 15);
  if (p.dweight[which] == nullptr) return;
  const int first = which ? p.q_chunks * p.blocks : 0, rows = (which ? p.k_chunks : p.q_chunks) * p.blocks;
  float sum = 0.f;
  if (c < p.D) {
#pragma unroll 8
    for (int r = threadIdx.x >> 4; r < rows; r += 64) sum += p.part[(int64_t)(first + r) * p.D + c];
  }
  lds[threadIdx.x] = sum;
  __syncthreads();
  for (int o = 512; o >= 16; o >>= 1) {
    if ((int)threadIdx.x < o) lds[threadIdx.x] += lds[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x < 16 && c < p.D) p.dweight[which][c] = lds[threadIdx.x];
}

// New tokens in serving: queries out, keys and values into the pages of a bf16 cache or of one in 4 bits (MX4).  A workgroup has some tokens, and of their
// keys', queries' and values' rows, in this order, a part.  A key that is held in 4 bits is computed in 64: its codes are those of the formula's
// result, and do not depend on the kernel that wrote them.  ALIGNED: a lane's pieces and its neighbours' make whole blocks of 32 channels (VEC = 8,
// pairs a multiple of 32), so that a key goes from registers to the page; else it is put together in LDS.
template <int VEC, int UPL, bool INTERLEAVED, bool STREAM, bool MX4, bool ALIGNED>
__global__ void __launch_bounds__(256) norm_append_kernel(const NormParams p) {
  typedef uint16_t T;
  typedef NormLane<T, VEC, UPL, INTERLEAVED, STREAM> L;
  typedef RotaryElem<T> E;
  static_assert(!ALIGNED || (MX4 && VEC == 8 && UPL == 1), "pieces of eight channels");
  extern __shared__ int64_t norm_shared[];
  constexpr int PLACES = 9;                        // q, q_out, k, v, the pages of k and v (< 0: none), the tokens' numbers there, k_held and v_held
  const NormLds x = norm_lds(p, norm_shared, PLACES);
  double* const cs64 = (double*)x.rest;            // MX4: [tokens][pairs] again
  double* const sn64 = cs64 + p.tokens_per_block * p.pairs;
  const int sub = threadIdx.x & ((1 << p.log_lanes) - 1), step = 256 >> p.log_lanes;
  const int token = blockIdx.x * p.tokens_per_block, n = min(p.tokens_per_block, p.B * p.S - token);
  const int D = p.D;
  // this workgroup's keys [lo, hi), queries and values
  const int part = blockIdx.y * p.rows_per_part, part_end = part + p.rows_per_part, n_k = n * p.Hkv, n_q = n * p.H;
  auto cut = [&](int first, int rows, int& lo, int& hi) __attribute__((always_inline)) {
    lo = min(max(part - first, 0), rows);
    hi = min(max(part_end - first, 0), rows);
  };
  int k_lo, k_hi, q_lo, q_hi, v_lo, v_hi;
  cut(0, n_k, k_lo, k_hi);
  cut(n_k, n_q, q_lo, q_hi);
  cut(n_k + n_q, n_k, v_lo, v_hi);

  if ((int)threadIdx.x < n) {
    int b, s;
    p.by_s.split(token + threadIdx.x, b, s);
    int64_t* at = x.at + PLACES * threadIdx.x;
    at[0] = row_at(p.q, b, s);
    at[1] = row_at(p.q_out, b, s);
    at[2] = row_at(p.k, b, s);
    at[3] = row_at(p.v, b, s);
    at[7] = row_at(p.k_held, b, s);
    at[8] = row_at(p.v_held, b, s);
    // the token's slot (from the true length: cut to the bound it would be an older token's)
    int64_t page = -1, within = 0;
    if (k_lo < k_hi || v_lo < v_hi) {
      const int slot = max(p.seq_lens[b], 0) - p.S + s;
      if (slot >= 0 && slot < p.max_len) {
        page = b, within = slot;
        if (p.block_table != nullptr) {
          page = p.block_table[(int64_t)b * p.table_stride + (slot >> p.page_shift)];
          within = slot & ((1 << p.page_shift) - 1);
        }
        if (page >= p.num_pages) page = -1;
      }
    }
    at[4] = page < 0 ? -1 : (MX4 ? page * p.mx4.k_sp : page * p.kc_sp + within * p.kc_st);
    at[5] = page < 0 ? -1 : (MX4 ? page * p.mx4.v_sp : page * p.vc_sp + within * p.vc_st);
    at[6] = within;
  }
  if (q_lo < q_hi || k_lo < k_hi) hold_weights(p, x.w);
  if (q_lo < q_hi || (!MX4 && k_lo < k_hi)) form_angles<T>(p, token, n, x.cs, x.sn);
  if (MX4 && k_lo < k_hi) {
    for (int i = threadIdx.x; i < n * p.pairs; i += 256) {
      int t, pair;
      p.by_pairs.split(i, t, pair);
      double c, y;
      sincospi(2. * turn_of(p, token + t, pair), &y, &c);
      cs64[i] = c;
      sn64[i] = y;
    }
  }
  __syncthreads();
  L l;
  l.init(p, sub);
  auto place = [&](int i) __attribute__((always_inline)) { return [=](int t) { return x.at[PLACES * t + i]; }; };

  // Eight channels of a row of token t from channel `at` on under the block's scale byte e: to the page (base: of the head) and to the caller
  auto put = [&](uint32_t codes, int e, int at, int t, uint8_t* base, int which, const View& held, int head) __attribute__((always_inline)) {
    const int64_t page = x.at[PLACES * t + 4 + which], within = x.at[PLACES * t + 6];
    if (page >= 0) {
      base += page;
      *(uint32_t*)(base + within * (D / 2) + at / 2) = codes;
      if ((at & 31) == 0) base[(int64_t)p.mx4.page_size * (D / 2) + (int64_t)(at >> 5) * p.mx4.page_size + within] = (uint8_t)e;
    }
    if (held.ptr != nullptr) *(uint4*)((T*)held.ptr + x.at[PLACES * t + 7 + which] + head * held.sh + at) = mx4_bf16x8(codes, mx4_scale_value(e));
  };
  // sixteen channels, 16 sub .. (lanes from D / 16 on have none), lane ^ 1 has the other half of the block
  auto put16 = [&](auto& y, int t, uint8_t* base, int which, const View& held, int head) __attribute__((always_inline)) {
    const int e = pair_max(mx4_own_scale(y));
    if (16 * sub >= D) return;
    put(mx4_pack8(y, e), e, 16 * sub, t, base, which, held, head);
    put(mx4_pack8(y + 8, e), e, 16 * sub + 8, t, base, which, held, head);
  };

  if constexpr (!MX4) {
    norm_rows<T, VEC, UPL, INTERLEAVED, STREAM>(p, l, sub, (const T*)p.k.ptr, p.k.sh, place(2), p.k_cache, p.kc_sh, place(4), x.w + D, p.by_hkv, k_lo, k_hi, x.cs, x.sn);
  } else if (k_lo < k_hi) {
    float w0[UPL][VEC], w1[UPL][VEC];
    l.weights(x.w + D, w0, w1);
    double* const mine = sn64 + p.tokens_per_block * p.pairs + (threadIdx.x >> p.log_lanes) * (D + 2);     // not ALIGNED: a row of this group of lanes
    typename L::Piece x0[UPL], x1[UPL];
    int t, h;
    auto load = [&](int r) __attribute__((always_inline)) {
      p.by_hkv.split(min(r, k_hi - 1), t, h);      // (groups behind the last row: that one again, for the exchanges between lanes; not stored)
      l.load((const T*)p.k.ptr + x.at[PLACES * t + 2] + h * p.k.sh, x0, x1);
    };
    load(k_lo + (threadIdx.x >> p.log_lanes));
    for (int r0 = k_lo; r0 < k_hi; r0 += step) {
      const int r = r0 + (threadIdx.x >> p.log_lanes), t_now = t, h_now = h;
      const bool real = r < k_hi;
      double z0[UPL][VEC], z1[UPL][VEC], sum = 0.;
#pragma unroll
      for (int n = 0; n < UPL; ++n)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          z0[n][j] = l.has[n] ? (double)E::load(x0[n].x[j]) : 0.;
          z1[n][j] = l.turns[n] ? (double)E::load(x1[n].x[j]) : 0.;
          sum = fma(z0[n][j], z0[n][j], fma(z1[n][j], z1[n][j], sum));
        }
      if (r0 + step < k_hi) load(r + step);
      const double rn = p.norm ? 1. / sqrt(group_sum(sum, l.lanes) / D + (double)p.eps) : 1.;
#pragma unroll
      for (int n = 0; n < UPL; ++n) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          z0[n][j] *= rn * w0[n][j];
          z1[n][j] *= rn * w1[n][j];
        }
        if (l.turns[n]) {
          const int first = t_now * p.pairs;
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            double &a = L::a_of(z0[n], z1[n], j), &c = L::b_of(z0[n], z1[n], j);
            const int pair = first + L::pair_of(p, sub + n * l.lanes, j);
            const double a_in = a, c_in = c, co = cs64[pair], si = sn64[pair];
            a = a_in * co - c_in * si;
            c = c_in * co + a_in * si;
          }
        }
      }
      uint8_t* base = p.mx4.k + h_now * p.mx4.k_sh;
      if constexpr (ALIGNED) {
        int e0 = mx4_own_scale(z0[0]), e1 = mx4_own_scale(z1[0]);
        e0 = four_max(e0);
        e1 = four_max(e1);
        if (real && l.has[0]) put(mx4_pack8(z0[0], e0), e0, l.at0[0], t_now, base, 0, p.k_held, h_now);
        if (real && l.turns[0]) put(mx4_pack8(z1[0], e1), e1, l.at1[0], t_now, base, 0, p.k_held, h_now);
      } else {
        wave_order();                              // (a row stays with its lanes, which lie in one wave: LDS keeps a wave's order)
#pragma unroll
        for (int n = 0; n < UPL; ++n)
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            if (l.has[n]) mine[l.at0[n] + j] = z0[n][j];
            if (l.turns[n]) mine[l.at1[n] + j] = z1[n][j];
          }
        wave_order();
        double y[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = 16 * sub < D ? mine[16 * sub + j] : 0.;
        if (real) put16(y, t_now, base, 0, p.k_held, h_now);
      }
    }
  }

  norm_rows<T, VEC, UPL, INTERLEAVED, STREAM>(p, l, sub, (const T*)p.q.ptr, p.q.sh, place(0), (T*)p.q_out.ptr, p.q_out.sh, place(1), x.w, p.by_h, q_lo, q_hi, x.cs,
                                      x.sn);

  if constexpr (MX4) {
    constexpr int HU = 2;
    for (int r0 = v_lo + (threadIdx.x >> p.log_lanes); r0 < v_hi; r0 += HU * step) {
      int t[HU], h[HU];
      RotaryPiece<T, 8> v0[HU], v1[HU];
#pragma unroll
      for (int u = 0; u < HU; ++u) {
        p.by_hkv.split(min(r0 + u * step, v_hi - 1), t[u], h[u]);
        const T* row = (const T*)p.v.ptr + x.at[PLACES * t[u] + 3] + h[u] * p.v.sh + (16 * sub < D ? 16 * sub : 0);
        v0[u] = *(const RotaryPiece<T, 8>*)row;
        v1[u] = *(const RotaryPiece<T, 8>*)(row + 8);
      }
#pragma unroll
      for (int u = 0; u < HU; ++u) {
        if (r0 + u * step >= v_hi) break;
        float y[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          y[j] = E::load(v0[u].x[j]);
          y[8 + j] = E::load(v1[u].x[j]);
        }
        put16(y, t[u], p.mx4.v + h[u] * p.mx4.v_sh, 1, p.v_held, h[u]);
      }
    }
  } else {
    for (int r = v_lo + (threadIdx.x >> p.log_lanes); r < v_hi; r += step) {
      int t, h;
      p.by_hkv.split(r, t, h);
      const int64_t to = x.at[PLACES * t + 5];
      if (to < 0) continue;
      const T* in = (const T*)p.v.ptr + x.at[PLACES * t + 3] + h * p.v.sh;
      T* out = p.v_cache + to + h * p.vc_sh;
      for (int c = sub * VEC; c < D; c += l.lanes * VEC) *(typename L::Piece*)(out + c) = *(const typename L::Piece*)(in + c);
    }
  }
}

}  // namespace fl
