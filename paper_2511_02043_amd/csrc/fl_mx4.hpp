// Keys and values in 4 bits (MX4) for gfx950: the format, and what moves rows into and out of it.
//
// 32 channels of a token and kv head share a scale 2^(E - 127), one byte; each channel is a code of 4 bits, a sign and one of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 (the OCP microscaling format e2m1 with e8m0 scales, which this machine converts from and to by itself).  E is
// the smallest with every magnitude below 7 of the scale, since 6 .. 7 round to 6, and between 1 and 252: a held value is finite and, but for
// scales near 2^-126, a bf16 number.  4.25 bits a value: of a unit normal row 11 % of its length are lost, as with 4-bit integers and a
// 16-bit scale and offset for 32 channels (5 bits).
//
// A page holds, for each kv head, the codes [page_size][D / 2] (the even channel in the low half of a byte), then the scales
// [D / 32][page_size]: one run of memory for a workgroup that reads one head.  A lane's codes are whole loads, and the scales of
// eight tokens in a row are one.
#pragma once
#include "fl_params.hpp"

namespace fl {

constexpr int mx4_token_bytes(int D) { return D / 2 + D / 32; }      // of one token and kv head

struct Mx4Cache {                  // page and kv head strides in bytes
  uint8_t* k;
  uint8_t* v;
  int64_t k_sp, k_sh, v_sp, v_sh;
  int32_t page_size;
};

// The scale byte of a block whose largest magnitude is `most` (infinite: the largest scale).
__device__ __forceinline__ int mx4_scale(float most) {
  const uint32_t u = __float_as_uint(most);
  return min(max((int)(u >> 23) - 2 + ((u & 0x7FFFFFu) >= 0x600000u ? 1 : 0), 1), 252);
}
__device__ __forceinline__ int mx4_scale(double most) {
  const uint32_t u = (uint32_t)__double2hiint(most);                 // (the mantissa's first bits decide: 1.75 is 0xC0000 of 20)
  return min(max((int)(u >> 20) - 1023 + 127 - 2 + ((u & 0xFFFFFu) >= 0xC0000u ? 1 : 0), 1), 252);
}
// 2^(127 - E): what a block's values are multiplied by
__device__ __forceinline__ float mx4_unit(int e, float) { return __uint_as_float((uint32_t)(254 - e) << 23); }
__device__ __forceinline__ double mx4_unit(int e, double) { return __hiloint2double((1023 + 127 - e) << 20, 0); }

// A value in units of its scale, cut to what a code can tell apart.
__device__ __forceinline__ float mx4_cut(float t) { return fminf(fmaxf(t, -8.f), 8.f); }
// ... in fp32 so that rounding it to a code is rounding the number in 64 bits: what is lost stays as a last bit that is set
__device__ __forceinline__ float mx4_cut(double x) {
  const double t = fmin(fmax(x, -8.), 8.);
  const float f = (float)t;
  const double back = (double)f;
  uint32_t u = __float_as_uint(f);
  if (back != t) u = (fabs(back) > fabs(t) ? u - 1 : u) | 1;
  return __uint_as_float(u);
}

// NaN is held as zero (before the maximum, which passes over quiet ones only); the scale byte that these channels ask for by themselves: a block's is the
// largest of its channels', since a scale grows with the magnitude.
template <class F, int N>
__device__ __forceinline__ int mx4_own_scale(F (&x)[N]) {
  F most = (F)0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = x[i] != x[i] ? (F)0 : x[i];
    most = fmax(most, fabs(x[i]));
  }
  return mx4_scale(most);
}
// the larger one of this lane's and lane ^ 1's (^ 2's)
template <int CTRL>
__device__ __forceinline__ int quad_max(int e) { return max(e, __builtin_amdgcn_update_dpp(0, e, CTRL, 0xF, 0xF, true)); }
__device__ __forceinline__ int pair_max(int e) { return quad_max<0xB1>(e); }
__device__ __forceinline__ int four_max(int e) { return quad_max<0x4E>(quad_max<0xB1>(e)); }

// Eight neighbouring channels under the scale byte e, channel 0 lowest.
template <class F>
__device__ __forceinline__ uint32_t mx4_pack8(const F* y, int e) {
  const F unit = mx4_unit(e, (F)0);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, mx4_cut(y[0] * unit), mx4_cut(y[1] * unit), 1.f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, mx4_cut(y[2] * unit), mx4_cut(y[3] * unit), 1.f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, mx4_cut(y[4] * unit), mx4_cut(y[5] * unit), 1.f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, mx4_cut(y[6] * unit), mx4_cut(y[7] * unit), 1.f, 3);
  return c;
}

__device__ __forceinline__ float mx4_scale_value(int e) { return __uint_as_float((uint32_t)e << 23); }

// Eight codes as bf16 numbers.
__device__ __forceinline__ uint4 mx4_bf16x8(uint32_t codes, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return r;
}

}  // namespace fl
