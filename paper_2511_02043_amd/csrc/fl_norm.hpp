// Heads normalised and turned for gfx950: forward pass, gradient, and the write of new tokens into a paged cache.
//
// Every row x of a query or key head (D channels) becomes
//     y = R(t) z,   z = w r x,   r = (mean_c x_c^2 + eps)^(-1/2),
// with R the turn of channel pairs by the positions' angles (fl_rotary.hpp).  Its gradient, with dz = R(-t) dy and g = w dz:
//     dx = r g - r^3 mean_c(x_c g_c) x,     dw = sum over tokens and heads of r x dz.
// An element is read once (the gradient: x and dy) and written once, at some twenty operations: memory traffic, if the row's sum costs no second pass.  A
// row therefore lies in the registers of a few lanes: lane `sub` of a group of `lanes` has the row's pairs sub VEC .. (two pieces of VEC channels, 16 bytes
// each, at D = 128 eight lanes), the sum is three exchanges between neighbours, and the angles, formed once, serve several heads of the token.
#pragma once
#include "fl_mx4.hpp"
#include "fl_rotary.hpp"

namespace fl {

struct NormParams : RotaryParams {
  const float* weight[2];          // of queries and keys, [D], or null: ones
  float eps;
  int32_t norm;                    // 0: turns alone (appending only)
  int32_t log_lanes;               // lanes of a row: 2^log_lanes, times UPL at least the units
  int32_t q_chunks, k_chunks;      // workgroups along y that take queries, keys (appending: then values), heads_per_thread heads each
  // gradient
  View dy[2], dx[2];
  float* part;                     // [q_chunks + k_chunks][blocks][D]: sums of dw; null: not wanted
  float* dweight[2];               // [D] or null
  int32_t blocks, groups;          // workgroups along x; token groups that they share out
  // appending
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
  for (int o = 1; o < lanes; o <<= 1) x += __shfl_xor(x, o);
  return x;
}

// What a lane has of every row of its token: UPL units of VEC pairs, or of VEC channels that stay (x1 unused then).
template <class T, int VEC, int UPL, bool INTERLEAVED>
struct NormLane {
  typedef RotaryPiece<T, VEC> Piece;
  typedef RotaryElem<T> E;
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
      at0[n] = turns[n] ? (INTERLEAVED ? 2 * unit * VEC : unit * VEC) : (has[n] ? 2 * p.pairs + (unit - turning) * VEC : 0);
      at1[n] = turns[n] ? (INTERLEAVED ? at0[n] + VEC : p.pairs + at0[n]) : at0[n];
    }
  }
  __device__ __forceinline__ void load(const T* row, Piece (&x0)[UPL], Piece (&x1)[UPL]) const {
#pragma unroll
    for (int n = 0; n < UPL; ++n) {                // (lanes without a unit read the row's first channels)
      x0[n] = *(const Piece*)(row + at0[n]);
      x1[n] = *(const Piece*)(row + at1[n]);
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
        w0[n][j] = w != nullptr ? w[at0[n] + j] : 1.f;
        w1[n][j] = w != nullptr ? w[at1[n] + j] : 1.f;
      }
  }
  // in whole turns, reduced in 64 bits
  __device__ __forceinline__ static double turn_of(const NormParams& p, const int32_t (&pos)[4], int pair) {
    const int32_t at = pair < p.ends[0] ? pos[0] : (pair < p.ends[1] ? pos[1] : (pair < p.ends[2] ? pos[2] : pos[3]));
    const double turn = (double)at * ((double)p.inv_freq[pair] * 0.15915494309189533577);
    return turn - rint(turn);
  }
  __device__ __forceinline__ void angles(const NormParams& p, const int32_t (&pos)[4], int sub, float (&cs)[UPL][VEC], float (&sn)[UPL][VEC]) const {
#pragma unroll
    for (int n = 0; n < UPL; ++n)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        cs[n][j] = 1.f;
        sn[n][j] = 0.f;
        if (turns[n]) E::sincos_turns((float)turn_of(p, pos, (sub + n * lanes) * VEC + j), sn[n][j], cs[n][j]);
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

__device__ __forceinline__ void token_positions(const RotaryParams& p, int b, int s, int32_t (&pos)[4]) {
#pragma unroll
  for (int a = 0; a < 4; ++a) pos[a] = a < p.axes ? p.positions[b * p.pos_sb + s * p.pos_ss + a * p.pos_sa] : 0;
}

// Heads [h, h_end) of one token: normalised, weighted and turned from `in` to `out` (null: computed for nobody).
template <class T, int VEC, int UPL, bool INTERLEAVED>
__device__ __forceinline__ void norm_rows(const NormParams& p, const NormLane<T, VEC, UPL, INTERLEAVED>& l, const T* in, int64_t in_sh, T* out, int64_t out_sh,
                                          const float* weight, int h, int h_end, const float (&cs)[UPL][VEC], const float (&sn)[UPL][VEC]) {
#pragma clang fp contract(off)                     // one rounding order in training and in serving
  typedef NormLane<T, VEC, UPL, INTERLEAVED> L;
  typedef RotaryElem<T> E;
  constexpr int HU = UPL * VEC <= 8 ? 4 : 1;       // heads whose loads are in flight together
  float w0[UPL][VEC], w1[UPL][VEC];
  l.weights(weight, w0, w1);
  const float inv_d = 1.f / p.D;
  for (int h0 = h; h0 < h_end; h0 += HU) {
    typename L::Piece x0[HU][UPL], x1[HU][UPL];
    float sum[HU] = {};
#pragma unroll
    for (int u = 0; u < HU; ++u) l.load(in + min(h0 + u, h_end - 1) * in_sh, x0[u], x1[u]);
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
      if (h0 + u >= h_end) break;
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
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            float &a = L::a_of(z0, z1, j), &c = L::b_of(z0, z1, j);
            const float a_in = a, c_in = c;
            a = fmaf(a_in, cs[n][j], -(c_in * sn[n][j]));
            c = fmaf(c_in, cs[n][j], a_in * sn[n][j]);
          }
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          x0[u][n].x[j] = E::store(z0[j]);
          x1[u][n].x[j] = E::store(z1[j]);
        }
      }
      if (out != nullptr) l.store(out + (h0 + u) * out_sh, x0[u], x1[u]);
    }
  }
}

template <class T, int VEC, int UPL, bool INTERLEAVED>
__global__ void __launch_bounds__(256) norm_rotary_kernel(const NormParams p) {
  const int sub = threadIdx.x & ((1 << p.log_lanes) - 1), local = threadIdx.x >> p.log_lanes;
  const int64_t token = (int64_t)blockIdx.x * p.tokens_per_block + local;
  if (token >= (int64_t)p.B * p.S) return;         // (whole groups of lanes)
  int b, s;
  p.by_s.split((int)token, b, s);
  int32_t pos[4];
  token_positions(p, b, s, pos);
  NormLane<T, VEC, UPL, INTERLEAVED> l;
  l.init(p, sub);
  float cs[UPL][VEC], sn[UPL][VEC];
  l.angles(p, pos, sub, cs, sn);
  const bool keys = (int)blockIdx.y >= p.q_chunks;
  const int heads = keys ? p.Hkv : p.H, h = (blockIdx.y - (keys ? p.q_chunks : 0)) * p.heads_per_thread;
  const View &in = keys ? p.k : p.q, &out = keys ? p.k_out : p.q_out;
  norm_rows<T, VEC, UPL, INTERLEAVED>(p, l, (const T*)in.ptr + b * in.sb + s * in.ss, in.sh, (T*)out.ptr + b * out.sb + s * out.ss, out.sh, p.weight[keys],
                                      h, min(h + p.heads_per_thread, heads), cs, sn);
}

// The gradient.  A workgroup goes through groups of 256 / lanes tokens, one workgroup a chunk of heads; dw gathers in registers, then over the workgroup's tokens in
// LDS, and leaves as a row of partial sums for norm_weights_kernel: no atomics, so that the result does not depend on who comes first.
template <class T, int VEC, int UPL, bool INTERLEAVED>
__global__ void __launch_bounds__(256) norm_rotary_bwd_kernel(const NormParams p) {
  typedef NormLane<T, VEC, UPL, INTERLEAVED> L;
  typedef RotaryElem<T> E;
  extern __shared__ float dw_lds[];                // [waves][D]
  const int sub = threadIdx.x & ((1 << p.log_lanes) - 1), local = threadIdx.x >> p.log_lanes;
  L l;
  l.init(p, sub);
  const bool keys = (int)blockIdx.y >= p.q_chunks;
  const int heads = keys ? p.Hkv : p.H, h_begin = (blockIdx.y - (keys ? p.q_chunks : 0)) * p.heads_per_thread, h_end = min(h_begin + p.heads_per_thread, heads);
  const View &xv = keys ? p.k : p.q, &yv = p.dy[keys], &ov = p.dx[keys];
  float w0[UPL][VEC], w1[UPL][VEC], d0[UPL][VEC] = {}, d1[UPL][VEC] = {};
  l.weights(p.weight[keys], w0, w1);
  const float inv_d = 1.f / p.D;

  for (int group = blockIdx.x; group < p.groups; group += p.blocks) {
    const int64_t token = (int64_t)group * p.tokens_per_block + local;
    if (token >= (int64_t)p.B * p.S) continue;     // (whole groups of lanes)
    int b, s;
    p.by_s.split((int)token, b, s);
    int32_t pos[4];
    token_positions(p, b, s, pos);
    float cs[UPL][VEC], sn[UPL][VEC];
    l.angles(p, pos, sub, cs, sn);
    const T* x_in = (const T*)xv.ptr + b * xv.sb + s * xv.ss;
    const T* y_in = (const T*)yv.ptr + b * yv.sb + s * yv.ss;
    T* out = (T*)ov.ptr + b * ov.sb + s * ov.ss;
    constexpr int HU = UPL * VEC <= 8 ? 2 : 1;
    for (int h0 = h_begin; h0 < h_end; h0 += HU) {
      typename L::Piece x0[HU][UPL], x1[HU][UPL], y0[HU][UPL], y1[HU][UPL];
#pragma unroll
      for (int u = 0; u < HU; ++u) {
        const int h = min(h0 + u, h_end - 1);
        l.load(x_in + h * xv.sh, x0[u], x1[u]);
        l.load(y_in + h * yv.sh, y0[u], y1[u]);
      }
      float sum[2 * HU] = {};                      // of x^2 and of x g
      float z0[HU][UPL][VEC], z1[HU][UPL][VEC];    // dz
#pragma unroll
      for (int u = 0; u < HU; ++u)
#pragma unroll
        for (int n = 0; n < UPL; ++n) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            z0[u][n][j] = l.has[n] ? E::load(y0[u][n].x[j]) : 0.f;
            z1[u][n][j] = l.turns[n] ? E::load(y1[u][n].x[j]) : 0.f;
          }
          if (l.turns[n]) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              float &a = L::a_of(z0[u][n], z1[u][n], j), &c = L::b_of(z0[u][n], z1[u][n], j);
              const float a_in = a, c_in = c;
              a = a_in * cs[n][j] + c_in * sn[n][j];
              c = c_in * cs[n][j] - a_in * sn[n][j];
            }
          }
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float a = l.has[n] ? E::load(x0[u][n].x[j]) : 0.f, c = l.turns[n] ? E::load(x1[u][n].x[j]) : 0.f;
            sum[2 * u] = fmaf(a, a, fmaf(c, c, sum[2 * u]));
            sum[2 * u + 1] = fmaf(a * w0[n][j], z0[u][n][j], fmaf(c * w1[n][j], z1[u][n][j], sum[2 * u + 1]));
          }
        }
      group_sum(sum, l.lanes);
#pragma unroll
      for (int u = 0; u < HU; ++u) {
        if (h0 + u >= h_end) break;
        const float r = 1.f / sqrtf(fmaf(sum[2 * u], inv_d, p.eps)), back = r * r * r * (sum[2 * u + 1] * inv_d);
#pragma unroll
        for (int n = 0; n < UPL; ++n)
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float a = E::load(x0[u][n].x[j]), c = E::load(x1[u][n].x[j]);
            d0[n][j] = fmaf(a * r, z0[u][n][j], d0[n][j]);
            d1[n][j] = fmaf(c * r, z1[u][n][j], d1[n][j]);
            x0[u][n].x[j] = E::store(fmaf(r * w0[n][j], z0[u][n][j], -a * back));
            x1[u][n].x[j] = E::store(fmaf(r * w1[n][j], z1[u][n][j], -c * back));
          }
        if (ov.ptr != nullptr) l.store(out + (h0 + u) * ov.sh, x0[u], x1[u]);
      }
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

// New tokens in serving: queries out, keys and values into the pages of a bf16 cache or of one in 4 bits (MX4).  Chunks of heads along y: keys first,
// whose way is the longest, then queries, then values.  A key that is held in 4 bits is computed in 64: its codes are those of the formula's
// result, and do not depend on the kernel that wrote them.
template <int VEC, int UPL, bool INTERLEAVED, bool MX4>
__global__ void __launch_bounds__(256) norm_append_kernel(const NormParams p) {
  typedef uint16_t T;
  typedef NormLane<T, VEC, UPL, INTERLEAVED> L;
  typedef RotaryElem<T> E;
  extern __shared__ double key_lds[];              // MX4: a row of D for each group of lanes
  const int sub = threadIdx.x & ((1 << p.log_lanes) - 1), local = threadIdx.x >> p.log_lanes;
  const int64_t token = (int64_t)blockIdx.x * p.tokens_per_block + local;
  const bool real = token < (int64_t)p.B * p.S;
  int b = 0, s = 0;
  if (real) p.by_s.split((int)token, b, s);
  const int y = blockIdx.y;
  const bool keys = y < p.k_chunks, queries = !keys && y < p.k_chunks + p.q_chunks;
  const int h = (keys ? y : (queries ? y - p.k_chunks : y - p.k_chunks - p.q_chunks)) * p.heads_per_thread;
  const int h_end = min(h + p.heads_per_thread, queries ? p.H : p.Hkv);
  L l;
  l.init(p, sub);

  if (queries) {
    if (!real) return;
    int32_t pos[4];
    token_positions(p, b, s, pos);
    float cs[UPL][VEC], sn[UPL][VEC];
    l.angles(p, pos, sub, cs, sn);
    norm_rows<T, VEC, UPL, INTERLEAVED>(p, l, (const T*)p.q.ptr + b * p.q.sb + s * p.q.ss, p.q.sh, (T*)p.q_out.ptr + b * p.q_out.sb + s * p.q_out.ss, p.q_out.sh,
                                        p.weight[0], h, h_end, cs, sn);
    return;
  }

  // this token's slot (from the true length: cut to the bound it would be an older token's)
  int64_t page = -1, within = 0;
  if (real) {
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

  if constexpr (!MX4) {
    if (page < 0) return;
    if (keys) {
      int32_t pos[4];
      token_positions(p, b, s, pos);
      float cs[UPL][VEC], sn[UPL][VEC];
      l.angles(p, pos, sub, cs, sn);
      norm_rows<T, VEC, UPL, INTERLEAVED>(p, l, (const T*)p.k.ptr + b * p.k.sb + s * p.k.ss, p.k.sh, p.k_cache + page * p.kc_sp + within * p.kc_st, p.kc_sh,
                                          p.weight[1], h, h_end, cs, sn);
    } else {
      const T* in = (const T*)p.v.ptr + b * p.v.sb + s * p.v.ss;
      T* out = p.v_cache + page * p.vc_sp + within * p.vc_st;
      for (int h0 = h; h0 < h_end; ++h0) {
        typename L::Piece x0[UPL], x1[UPL];
        l.load(in + h0 * p.v.sh, x0, x1);
        l.store(out + h0 * p.vc_sh, x0, x1);
      }
    }
  } else {
    const int D = p.D;
    // sixteen channels of a row, 16 sub .., to the cache and to the caller (lanes from D / 16 on have none)
    auto put = [&](int head, auto& x, uint8_t* base, const View& held) __attribute__((always_inline)) {
      uint32_t codes[2];
      const int e = mx4_pack16(x, codes);
      if (!real || 16 * sub >= D) return;
      if (page >= 0) {
        *(uint2*)(base + within * (D / 2) + 8 * sub) = make_uint2(codes[0], codes[1]);
        if ((sub & 1) == 0) base[(int64_t)p.mx4.page_size * (D / 2) + (int64_t)(sub >> 1) * p.mx4.page_size + within] = (uint8_t)e;
      }
      if (held.ptr != nullptr) {
        uint4* to = (uint4*)((T*)held.ptr + b * held.sb + head * held.sh + s * held.ss + 16 * sub);
        to[0] = mx4_bf16x8(codes[0], mx4_scale_value(e));
        to[1] = mx4_bf16x8(codes[1], mx4_scale_value(e));
      }
    };
    if (!keys) {
      const T* in = (const T*)p.v.ptr + b * p.v.sb + s * p.v.ss + (16 * sub < D ? 16 * sub : 0);
      for (int h0 = h; h0 < h_end; ++h0) {
        const RotaryPiece<T, 8> v0 = *(const RotaryPiece<T, 8>*)(in + h0 * p.v.sh), v1 = *(const RotaryPiece<T, 8>*)(in + h0 * p.v.sh + 8);
        float x[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = E::load(v0.x[j]);
          x[8 + j] = E::load(v1.x[j]);
        }
        put(h0, x, p.mx4.v + page * p.mx4.v_sp + h0 * p.mx4.v_sh, p.v_held);
      }
      return;
    }
    int32_t pos[4];
    token_positions(p, b, s, pos);                 // (lanes behind the last token: the first one's)
    double cs[UPL][VEC], sn[UPL][VEC];
#pragma unroll
    for (int n = 0; n < UPL; ++n)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        cs[n][j] = 1.;
        sn[n][j] = 0.;
        if (l.turns[n]) sincospi(2. * L::turn_of(p, pos, (sub + n * l.lanes) * VEC + j), &sn[n][j], &cs[n][j]);
      }
    float w0[UPL][VEC], w1[UPL][VEC];
    l.weights(p.weight[1], w0, w1);
    const T* in = (const T*)p.k.ptr + b * p.k.sb + s * p.k.ss;
    double* const mine = key_lds + local * D;
    for (int h0 = h; h0 < h_end; ++h0) {
      typename L::Piece x0[UPL], x1[UPL];
      l.load(in + h0 * p.k.sh, x0, x1);
      double sum = 0.;
#pragma unroll
      for (int n = 0; n < UPL; ++n)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const double a = l.has[n] ? (double)E::load(x0[n].x[j]) : 0., c = l.turns[n] ? (double)E::load(x1[n].x[j]) : 0.;
          sum = fma(a, a, fma(c, c, sum));
        }
      const double r = p.norm ? 1. / sqrt(group_sum(sum, l.lanes) / D + (double)p.eps) : 1.;
      // (a row stays with its lanes, which lie in one wave: LDS keeps a wave's order)
      wave_order();
#pragma unroll
      for (int n = 0; n < UPL; ++n) {
        double z0[VEC], z1[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          z0[j] = E::load(x0[n].x[j]) * r * w0[n][j];
          z1[j] = E::load(x1[n].x[j]) * r * w1[n][j];
        }
        if (l.turns[n]) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            double &a = L::a_of(z0, z1, j), &c = L::b_of(z0, z1, j);
            const double a_in = a, c_in = c;
            a = a_in * cs[n][j] - c_in * sn[n][j];
            c = c_in * cs[n][j] + a_in * sn[n][j];
          }
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          if (l.has[n]) mine[l.at0[n] + j] = z0[j];
          if (l.turns[n]) mine[l.at1[n] + j] = z1[j];
        }
      }
      wave_order();
      double x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = 16 * sub < D ? mine[16 * sub + j] : 0.;
      put(h0, x, p.mx4.k + page * p.mx4.k_sp + h0 * p.mx4.k_sh, p.k_held);
    }
  }
}

}  // namespace fl
