// Host-side helpers shared by the translation units that implement the C ABI: the thread-local
// error detail, and the checks / views of [B, G, H, S, D] tensors.
#pragma once
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/fl_attn.h"
#include "fl_params.hpp"

namespace fl {
namespace host {

inline thread_local char g_detail[384] = "";
inline void clear_detail() { g_detail[0] = 0; }

inline fl_status fail(fl_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_detail, sizeof(g_detail), fmt, ap);
  va_end(ap);
  return st;
}


// A window that reaches past both sequence ends changes nothing; cutting it there keeps the kernels'
// int32 arithmetic on i - window and j + window far from overflow (callers pass INT_MAX for "no limit").
inline int32_t clamp_window(int32_t window, int64_t Sq, int64_t Sk) {
  const int64_t lim = Sq > Sk ? Sq : Sk;
  return (int64_t)window > lim ? (int32_t)lim : window;
}

// Canonical mask bits: WINDOW implies CAUSAL.
inline uint32_t canonical_mask(uint32_t m) { return (m & FL_MASK_WINDOW) ? (m | FL_MASK_CAUSAL) : m; }

inline fl_status check_desc(const fl_variant_desc* d) {
  if (d == nullptr) return fail(FL_ERR_NULL, "desc is NULL");
  if (d->struct_size != sizeof(fl_variant_desc))
    return fail(FL_ERR_DESC, "desc->struct_size = %u, expected %zu", d->struct_size, sizeof(fl_variant_desc));
  if (!(d->scale > 0.f) || !std::isfinite(d->scale)) return fail(FL_ERR_DESC, "scale must be finite and > 0");
  if (d->score_mod > FL_MOD_SOFTCAP) return fail(FL_ERR_DESC, "unknown score_mod %u", d->score_mod);
  if (d->score_mod == FL_MOD_SOFTCAP && (!(d->softcap > 0.f) || !std::isfinite(d->softcap)))
    return fail(FL_ERR_DESC, "softcap must be finite and > 0");
  if (d->mask & ~(uint32_t)(FL_MASK_CAUSAL | FL_MASK_WINDOW | FL_MASK_DOC | FL_MASK_PREFIX))
    return fail(FL_ERR_DESC, "unknown mask bits 0x%x", d->mask);
  if ((d->mask & FL_MASK_PREFIX) && (d->mask & (FL_MASK_CAUSAL | FL_MASK_WINDOW)))
    return fail(FL_ERR_DESC, "FL_MASK_PREFIX excludes FL_MASK_CAUSAL and FL_MASK_WINDOW");
  if ((d->mask & FL_MASK_WINDOW) && d->window < 0) return fail(FL_ERR_DESC, "window must be >= 0");
  if ((d->mask & FL_MASK_PREFIX) && d->prefix_len < 0) return fail(FL_ERR_DESC, "prefix_len must be >= 0");
  if (d->n_bias > 2) return fail(FL_ERR_DESC, "n_bias must be 0..2");
  if (d->combine > FL_DIFFERENTIAL) return fail(FL_ERR_DESC, "unknown combine %u", d->combine);
  if (d->epilogue & ~(uint32_t)(FL_EPI_RMSNORM | FL_EPI_GATE_SIGMOID))
    return fail(FL_ERR_DESC, "unknown epilogue bits 0x%x", d->epilogue);
  if ((d->epilogue & FL_EPI_RMSNORM) && (!(d->rms_eps >= 0.f) || !std::isfinite(d->rms_eps)))
    return fail(FL_ERR_DESC, "rms_eps must be finite and >= 0");
  if (d->q_offset < 0 || d->q_offset > 0x3fffffff) return fail(FL_ERR_DESC, "q_offset must be in [0, 2^30)");
  return FL_OK;
}

inline int elem_size(int dtype) { return dtype == FL_BF16 ? 2 : 4; }

// Common checks of a [B, G, H, S, D] data tensor (q, k, v, out, gate, q2, k2).
inline fl_status check_data_tensor(const fl_tensor* t, const char* name, int want_dtype, const int64_t want[5]) {
  if (t == nullptr || t->ptr == nullptr) return fail(FL_ERR_NULL, "%s is NULL", name);
  if (t->dtype != want_dtype) return fail(FL_ERR_DTYPE, "%s has dtype %d, expected %d", name, t->dtype, want_dtype);
  for (int a = 0; a < 5; ++a)
    if (t->size[a] != want[a])
      return fail(FL_ERR_SHAPE, "%s size[%d] = %lld, expected %lld", name, a, (long long)t->size[a],
                  (long long)want[a]);
  if (t->stride[4] != 1) return fail(FL_ERR_STRIDE, "%s innermost stride must be 1", name);
  const int es = elem_size(t->dtype);
  if (((uintptr_t)t->ptr) % 16 != 0) return fail(FL_ERR_ALIGN, "%s base pointer not 16-byte aligned", name);
  for (int a = 0; a < 4; ++a) {
    if (t->stride[a] < 0) return fail(FL_ERR_STRIDE, "%s stride[%d] negative", name, a);
    if (t->size[a] > 1 && t->stride[a] == 0) return fail(FL_ERR_STRIDE, "%s stride[%d] is 0 (no broadcast here)", name, a);
    if (t->size[a] > 1 && (t->stride[a] * es) % 16 != 0)
      return fail(FL_ERR_ALIGN, "%s stride[%d] not a multiple of 16 bytes", name, a);
  }
  // the kernels address the rows of one key tile with 32-bit byte offsets from the tile's base
  if (t->size[3] > 1 && t->stride[3] >= (int64_t)1 << 23)
    return fail(FL_ERR_STRIDE, "%s row stride %lld is not below 2^23 elements", name, (long long)t->stride[3]);
  return FL_OK;
}

inline fl::View make_view(const fl_tensor* t) {
  fl::View v;
  v.ptr = t->ptr;
  v.sb = t->size[0] > 1 ? t->stride[0] : 0;
  v.sg = t->size[1] > 1 ? t->stride[1] : 0;
  v.sh = t->size[2] > 1 ? t->stride[2] : 0;
  v.ss = t->size[3] > 1 ? t->stride[3] : 0;
  return v;
}

// Rows of `bytes` each in memory: n0 x n1 of them, s0 and s1 bytes apart (>= bytes where there are several).
struct Rows {
  uintptr_t at;
  int64_t n0, s0, n1, s1, bytes;
};
inline Rows flat_rows(const void* p, int64_t bytes) { return {(uintptr_t)p, 1, 0, 1, 0, bytes}; }
// The first byte behind them; -1 where that is past every address.
inline int64_t rows_end(const Rows& r) {
  const __int128 e = (__int128)r.at + (__int128)(r.n0 - 1) * r.s0 + (__int128)(r.n1 - 1) * r.s1 + r.bytes;
  return e > (__int128)INT64_MAX ? -1 : (int64_t)e;
}
// True where `la` bytes from x on and rows of `lb` bytes at 0, s, 2 s, ... (n of them, s >= lb) have a byte in common.
inline bool row_meets(int64_t x, int64_t la, int64_t n, int64_t s, int64_t lb) {
  if (n == 1 || x < 0) return x < lb && x + la > 0;        // (from before the first row: that one or none)
  const int64_t i = x / s < n - 1 ? x / s : n - 1;         // the last row that starts at x or before
  return x < i * s + lb || (i + 1 < n && x + la > (i + 1) * s);
}
// True where a row of `a` and a row of `b` have a byte in common: exactly, since two views may take turns in one buffer.
inline bool rows_meet(const Rows& a, Rows b) {
  if (a.n0 <= 0 || a.n1 <= 0 || a.bytes <= 0 || b.n0 <= 0 || b.n1 <= 0 || b.bytes <= 0) return false;
  const int64_t end_a = rows_end(a), end_b = rows_end(b);
  if (end_a < 0 || end_b < 0) return true;                 // (no memory is like that)
  if (end_a <= (int64_t)b.at || end_b <= (int64_t)a.at) return false;
  if (b.n0 == 1 || (b.n1 > 1 && b.s1 > b.s0)) {            // axis 0 the one of the larger steps
    int64_t t = b.n0;
    b.n0 = b.n1, b.n1 = t;
    t = b.s0;
    b.s0 = b.s1, b.s1 = t;
  }
  const bool nested = b.n0 == 1 || (b.n1 - 1) * b.s1 + b.bytes <= b.s0;
  for (int64_t i0 = 0; i0 < a.n0; ++i0)
    for (int64_t i1 = 0; i1 < a.n1; ++i1) {
      const int64_t x = (int64_t)a.at + i0 * a.s0 + i1 * a.s1 - (int64_t)b.at;
      // of b's groups of rows, where they follow each other: the last one that starts at x or before, and the next (a row that reaches past
      // that one's start meets its first row)
      const int64_t j = !nested || b.n0 == 1 || x < 0 ? 0 : (x / b.s0 < b.n0 - 1 ? x / b.s0 : b.n0 - 1);
      const int64_t j_end = nested && j + 2 < b.n0 ? j + 2 : b.n0;
      for (int64_t j0 = j; j0 < j_end; ++j0)
        if (row_meets(x - j0 * b.s0, a.bytes, b.n1, b.s1, b.bytes)) return true;
    }
  return false;
}

// True where two rows of n0 x n1, s0 and s1 elements apart, `len` long (<= each step where there are several), lie over each other.
inline bool rows_overlap(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t len) {
  if (n0 <= 1 || n1 <= 1) return false;
  typedef __int128 wide;
  if ((wide)(n1 - 1) * s1 + len <= s0 || (wide)(n0 - 1) * s0 + len <= s1) return false;   // one axis within a step of the other
  for (int64_t i = 1; i < n0; ++i) {               // rows i apart along the first axis: the nearest ones along the second, on either side
    const wide k = (wide)i * s0 / s1, rest = (wide)i * s0 % s1;
    if ((k < n1 && rest < len) || (k + 1 < n1 && s1 - rest < len)) return true;
  }
  return false;
}

// The accumulated weights of cached keys, [B, 1, Hkv, 1, C] f32 with C >= least.  `written`: each row by a workgroup of its own.
inline fl_status check_weights(const fl_tensor* t, const char* name, int64_t B, int64_t Hkv, int64_t least, bool written = true) {
  if (t == nullptr || t->ptr == nullptr) return fail(FL_ERR_NULL, "%s is NULL", name);
  if (t->dtype != FL_F32) return fail(FL_ERR_DTYPE, "%s must be f32", name);
  const int64_t want[4] = {B, 1, Hkv, 1};
  for (int a = 0; a < 4; ++a)
    if (t->size[a] != want[a])
      return fail(FL_ERR_SHAPE, "%s size[%d] = %lld, expected %lld", name, a, (long long)t->size[a], (long long)want[a]);
  if (t->size[4] < least)
    return fail(FL_ERR_SHAPE, "%s has %lld slots per head, %lld needed", name, (long long)t->size[4], (long long)least);
  if (t->size[4] > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "%s has more slots than an int32 can count", name);
  if (t->stride[4] != 1) return fail(FL_ERR_STRIDE, "%s innermost stride must be 1", name);
  if (((uintptr_t)t->ptr) % 4 != 0) return fail(FL_ERR_ALIGN, "%s base pointer not 4-byte aligned", name);
  for (int a = 0; a < 4; a += 2)
    if (t->size[a] > 1 && t->stride[a] < t->size[4]) return fail(FL_ERR_STRIDE, "%s stride[%d]: rows overlap", name, a);
  if (written && rows_overlap(B, t->stride[0], Hkv, t->stride[2], t->size[4]))
    return fail(FL_ERR_STRIDE, "%s strides %lld and %lld: rows overlap", name, (long long)t->stride[0], (long long)t->stride[2]);
  return FL_OK;
}

// What fl_paged_kv says about a cache of `pages` pages, B sequences of which are used.  page_shift: log2 of the page size (0 where it is no power of
// two, which only a cache without a block table may have).
inline fl_status check_pages(const fl_paged_kv* kv, int64_t pages, int64_t page_size, int64_t B, int* page_shift) {
  if (kv->struct_size != sizeof(fl_paged_kv)) return fail(FL_ERR_DESC, "kv->struct_size = %u, expected %zu", kv->struct_size, sizeof(fl_paged_kv));
  if (pages < 0 || page_size <= 0) return fail(FL_ERR_SHAPE, "negative size");
  if (pages > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "more pages than an int32 table entry can name");
  if (kv->max_seq_len < 0) return fail(FL_ERR_SHAPE, "max_seq_len negative");
  if (pages == 0 && kv->max_seq_len > 0) return fail(FL_ERR_SHAPE, "max_seq_len = %d with an empty cache", kv->max_seq_len);
  if (kv->page_size != page_size) return fail(FL_ERR_SHAPE, "kv->page_size = %d, cache size[3] = %lld", kv->page_size, (long long)page_size);
  *page_shift = 0;
  const bool power = (page_size & (page_size - 1)) == 0;
  if (power)
    while ((1LL << *page_shift) < page_size) ++*page_shift;
  if (kv->block_table != nullptr) {
    if (page_size < 8 || !power) return fail(FL_ERR_SHAPE, "with a block table the page size (%lld) must be a power of two >= 8", (long long)page_size);
    if (kv->table_stride < (kv->max_seq_len + page_size - 1) / page_size)
      return fail(FL_ERR_SHAPE, "table_stride %d is less than the pages of max_seq_len", kv->table_stride);
  } else {
    if (pages < B) return fail(FL_ERR_SHAPE, "without a block table the cache needs a page per sequence");
    if (kv->max_seq_len > page_size) return fail(FL_ERR_SHAPE, "max_seq_len exceeds the page size");
  }
  return FL_OK;
}

// The caches [pages, 1, Hkv, page_size, D] bf16 that fl_paged_kv speaks of, B sequences of which are used.
inline fl_status check_cache(const fl_paged_kv* kv, const fl_tensor* k_cache, const fl_tensor* v_cache, int64_t B, int64_t Hkv, int64_t D,
                             int* page_shift) {
  if (kv == nullptr || k_cache == nullptr) return fail(FL_ERR_NULL, "kv or k_cache is NULL");
  const int64_t pages = k_cache->size[0], page_size = k_cache->size[3];
  fl_status st = check_pages(kv, pages, page_size, B, page_shift);
  if (st != FL_OK || B == 0 || Hkv == 0) return st;
  if (kv->seq_lens == nullptr) return fail(FL_ERR_NULL, "seq_lens is NULL");
  const int64_t size[5] = {pages, 1, Hkv, page_size, D};
  if (kv->max_seq_len > 0 && (st = check_data_tensor(k_cache, "k_cache", FL_BF16, size)) == FL_OK && v_cache != nullptr)
    st = check_data_tensor(v_cache, "v_cache", FL_BF16, size);
  return st;
}

// The same of caches in 4 bits: FL_MX4, of which only the strides of pages and kv heads, in bytes, say anything.
inline fl_status check_cache_mx4(const fl_paged_kv* kv, const fl_tensor* k_cache, const fl_tensor* v_cache, int64_t B, int64_t Hkv, int64_t D,
                                 int* page_shift) {
  if (kv == nullptr || k_cache == nullptr || v_cache == nullptr) return fail(FL_ERR_NULL, "kv, k_cache or v_cache is NULL");
  if (D != 64 && D != 128) return fail(FL_ERR_UNSUPPORTED, "D = %lld: caches in 4 bits take 64 or 128", (long long)D);
  const int64_t pages = k_cache->size[0], page_size = k_cache->size[3];
  fl_status st = check_pages(kv, pages, page_size, B, page_shift);
  if (st != FL_OK) return st;
  if (page_size % 8 != 0 || page_size > (1 << 24))
    return fail(FL_ERR_SHAPE, "pages of %lld tokens: caches in 4 bits take multiples of 8 up to 2^24", (long long)page_size);
  if (B == 0 || Hkv == 0) return FL_OK;
  if (kv->seq_lens == nullptr) return fail(FL_ERR_NULL, "seq_lens is NULL");
  if (kv->max_seq_len == 0) return FL_OK;
  const int64_t size[5] = {pages, 1, Hkv, page_size, D}, bytes = page_size * (D / 2 + D / 32);
  for (int w = 0; w < 2; ++w) {
    const fl_tensor* t = w ? v_cache : k_cache;
    const char* name = w ? "v_cache" : "k_cache";
    if (t->ptr == nullptr) return fail(FL_ERR_NULL, "%s is NULL", name);
    if (t->dtype != FL_MX4) return fail(FL_ERR_DTYPE, "%s has dtype %d, expected %d", name, t->dtype, FL_MX4);
    for (int a = 0; a < 5; ++a)
      if (t->size[a] != size[a])
        return fail(FL_ERR_SHAPE, "%s size[%d] = %lld, expected %lld", name, a, (long long)t->size[a], (long long)size[a]);
    if (((uintptr_t)t->ptr) % 16 != 0) return fail(FL_ERR_ALIGN, "%s base pointer not 16-byte aligned", name);
    for (int a = 0; a < 4; a += 2) {
      if (t->size[a] <= 1) continue;
      if (t->stride[a] < bytes) return fail(FL_ERR_STRIDE, "%s stride[%d] = %lld is less than a page and head's %lld bytes", name, a, (long long)t->stride[a], (long long)bytes);
      if (t->stride[a] % 16 != 0) return fail(FL_ERR_ALIGN, "%s stride[%d] not a multiple of 16 bytes", name, a);
    }
    if (pages > 1 && t->stride[0] >= (1LL << 32)) return fail(FL_ERR_STRIDE, "%s page stride is not below 2^32 bytes", name);
    if (rows_overlap(Hkv, t->stride[2], pages, t->stride[0], bytes)) return fail(FL_ERR_STRIDE, "%s strides: pages overlap", name);
  }
  return FL_OK;
}

// The forward pass behind fl_attn_fwd on keys and values [B, 1, Hkv, L, D] of which sequence b has kv_lens[b] (device): its query rows are the last of those.
fl_status forward_of_lengths(const fl_tensor* q, const fl_tensor* k, const fl_tensor* v, const fl_variant_desc* desc, const fl_aux* aux, fl_tensor* out,
                             fl_tensor* lse, void* stream, const int32_t* kv_lens);

// What fl_set_tuning("decode_splits") and fl_set_tuning("prefill_gather") ask for in this thread; 0: nothing.
int tuned_decode_splits();
int tuned_prefill_gather();

}  // namespace host
}  // namespace fl
