// Host side of the calls that turn heads by positions: checks of fl_rotary, and how a launch shares out tokens and heads.
#pragma once
#include <algorithm>

#include "fl_host.hpp"
#include "fl_rotary.hpp"

namespace fl {
namespace host {

// The common part of both calls: `any` is q or k, S its rows.
inline fl_status check_rotary(const fl_rotary* r, int64_t B, int64_t S, int64_t D, fl::RotaryParams* p) {
  if (r == nullptr) return fail(FL_ERR_NULL, "rotary is NULL");
  if (r->struct_size != sizeof(fl_rotary)) return fail(FL_ERR_DESC, "rotary->struct_size = %u, expected %zu", r->struct_size, sizeof(fl_rotary));
  if (r->axes < 1 || r->axes > 4) return fail(FL_ERR_DESC, "axes = %u, expected 1 .. 4", r->axes);
  if (r->interleaved > 1 || r->inverse > 1) return fail(FL_ERR_DESC, "interleaved and inverse are 0 or 1");
  int64_t pairs = 0;
  for (int a = 0; a < 4; ++a) {
    if (a < (int)r->axes) {
      if (r->sections[a] < 0) return fail(FL_ERR_DESC, "sections[%d] negative", a);
      pairs += r->sections[a];
    }
    p->ends[a] = (int32_t)std::min<int64_t>(pairs, 0x7fffffff);
  }
  if (pairs < 1 || 2 * pairs > D) return fail(FL_ERR_SHAPE, "%lld channel pairs in a head dim of %lld", (long long)pairs, (long long)D);
  if (B * S != 0 && (r->positions == nullptr || r->inv_freq == nullptr)) return fail(FL_ERR_NULL, "positions or inv_freq is NULL");
  if (B * S > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "too many tokens");
  p->axes = (int32_t)r->axes;
  p->pairs = (int32_t)pairs;
  p->D = (int32_t)D;
  p->inverse = (int32_t)r->inverse;
  p->positions = r->positions;
  p->pos_sb = r->stride[0];
  p->pos_ss = r->stride[1];
  p->pos_sa = r->stride[2];
  p->inv_freq = r->inv_freq;
  p->B = (int32_t)B;
  p->S = (int32_t)S;
  p->by_s = fl::Divisor::of(S);
  return FL_OK;
}

// Heads that a thread turns with the angles it has formed: as many as leave the chip a thousand workgroups.  (us with 512 / 1024 / 4096 of them:
// 8 chunks of 512 tokens into the cache, 32 / 8 heads, D = 128, 23.2 / 22.4 / 31.0; 2 x 8192 tokens forward 80.6 / 80.5 / 78.4)
inline int rotary_heads(int64_t blocks, int64_t heads) {
  int n = 16;
  while (n > 1 && blocks * ((heads + n - 1) / n) < 1024) n >>= 1;
  return n;
}

// 16-byte pieces where pairs and what stays are whole numbers of them (rows start 16-byte aligned), else one element at a time.
inline bool rotary_wide(const fl::RotaryParams& p, int dtype) {
  const int vec = dtype == FL_BF16 ? 8 : 4;
  return p.pairs % vec == 0 && (p.D - 2 * p.pairs) % vec == 0;
}

inline fl_status check_heads(int64_t H, int64_t Hkv) {
  return H > 16384 || Hkv > 16384 ? fail(FL_ERR_SHAPE, "more than 16384 heads") : FL_OK;
}

}  // namespace host
}  // namespace fl
