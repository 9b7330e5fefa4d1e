// C-ABI entry points of attention over a paged cache in 4 bits: the decode step and a chunk of query rows.  Argument validation and launch; the
// arithmetic is in fl_mx4_decode.hpp and, for chunks, in the forward kernels.
#include <algorithm>
#include <cstring>

#include "fl_bwd_registry.hpp"
#include "fl_host.hpp"
#include "fl_mx4_decode.hpp"

namespace {

using namespace fl::host;

constexpr int64_t kMostPairs = 64;                 // (query row, head) pairs of a kv head that a decode step takes
constexpr int64_t kMostRowPairs = 16384;           // ... that a chunk may bring through the decode kernels

int64_t pairs_of(int64_t H, int64_t Hkv, int64_t T) { return Hkv > 0 && T <= kMostRowPairs ? T * (H / Hkv) : kMostRowPairs + 1; }
// Blocks of pairs, each a workgroup's: 16 of them, where there are more 32 (16 rows of 8 sequences of 4k - 8k tokens, 32 / 8 heads, D = 128: 36 us in two blocks; 59 in one of
// 64, whose registers leave room for one wave per SIMD).
int64_t blocks_of(int64_t pairs) { return pairs <= 16 ? 1 : (pairs + 31) / 32; }

// Keys that the rows of one or all blocks see at most, `rows` of them under this mask.
int64_t keys_of(const fl_variant_desc* desc, int64_t max_seq_len, int64_t rows) {
  const bool window = canonical_mask(desc->mask) & FL_MASK_WINDOW;
  return window ? std::min<int64_t>(max_seq_len, clamp_window(desc->window, max_seq_len, max_seq_len) + rows) : max_seq_len;
}

// Splits of a sequence's keys, from the shapes, the host-side bound of the lengths and the most keys that a sequence's rows see: the power of two that
// brings the workgroups to 448 or more, or fewer where a shorter chain of tiles (0.65 us each, of 32 pairs 0.9) does not pay for the merge (3 us, and 1.6 ns and 0.3 a split
// for each row).  us, 32 / 8 heads, D = 128, splits: 64 sequences of 4k - 8k tokens 1: 87.7, 2: 89.9; 24 of them 1: 45.9, 2: 38.0, 4: 35.7, 8: 38; 8 of them 1: 43,
// 4: 17.8, 8: 16.9, 16: 18.0; 2 of 100k - 131k 16: 51.9, 32: 52.4, 64: 55.4; 48 of 512 - 1024 1: 12.5, 2: 15.2; eight rows of 24 of 1k - 2k 1: 20.0, 2: 23.8, 3: 28.3.
// Never more for fewer keys: a workspace that was sized without the window is large enough.  (A tile of D = 64 has half the bytes and conversions; its time was not taken apart,
// and D = 64 goes by the same rule.)
int splits_of(int64_t B, int64_t H, int64_t Hkv, int64_t T, int64_t keys) {
  const int64_t tiles = (keys + 31) / 32, pairs = pairs_of(H, Hkv, T), units = std::max<int64_t>(1, B * Hkv * blocks_of(pairs));
  if (tuned_decode_splits() > 0) return (int)std::max<int64_t>(1, std::min<int64_t>(tuned_decode_splits(), tiles));
  const double chain = (pairs <= 16 ? 0.65 : 0.9) * (double)tiles / 4, rows = (double)B * (double)T * (double)H;
  int best = 1;
  double least = chain;
  for (int ns = 2; ns <= 64 && ns * 4 <= tiles && units * (ns / 2) < 448; ns *= 2) {
    const double us = chain / ns + 3 + rows * (1.6e-3 + 3e-4 * ns);
    if (us < least) least = us, best = ns;
  }
  return best;
}

// Partial results; a sequence that is not split has none.
size_t decode_bytes(int64_t B, int64_t T, int64_t H, int64_t D, int ns) { return ns > 1 ? (size_t)(B * T * H * ns) * (size_t)(D + 2) * sizeof(float) : 0; }

size_t dense_bytes(int64_t B, int64_t Hkv, int64_t D, int64_t max_len) {
  return ((size_t)(B * Hkv * std::max<int64_t>(max_len, 1) * D) * 2 + 255) / 256 * 256;
}

// Whether a chunk's rows go through the decode kernels, 32 pairs of a kv head at a time, or its sequences are unpacked for the forward kernel.  The former read the keys
// again for each 32 pairs (52 000 keys of such a block a microsecond at D = 128, 72 000 at 64, and 256 keys' time to start); the latter have the unpacking, then a tile's chain over
// the keys or, if that is longer, their products.  us, rows / unpacked, T = 16, 64, 128, 256, 512 rows: 8 sequences of 4k - 8k tokens, 32 / 8 heads, D = 128 36 / 186, 91 / 235,
// 162 / 189, 311 / 250, 596 / 428; one of 8k 17 / 148, 25 / 199, 35 / 144, 56 / 144, 88 / 149; 16 of 500 - 1000 24 / 47, 31 / 48, 55 / 53, 99 / 78; 4 of 700 - 1500, 16 / 2 heads,
// D = 64, window 512 12 / 22, 14 / 24, 16 / 25, 12 / 25, 20 / 26.
bool through_decode(int64_t B, int64_t H, int64_t Hkv, int64_t T, int64_t D, int64_t max_len, const fl_variant_desc* desc) {
  const int64_t pairs = pairs_of(H, Hkv, T);
  if (pairs > kMostRowPairs || tuned_prefill_gather() == 1) return false;
  if (pairs <= kMostPairs) return true;
  const double wide = D == 128 ? 1. : 0., ahead = (double)std::max<int64_t>(0, max_len - T / 2);     // (rows of a prompt see half of it)
  const double rows_us = 10 + (double)(B * Hkv * blocks_of(pairs)) * (std::min(ahead, (double)keys_of(desc, max_len, 32)) + 256) / (wide ? 52e3 : 72e3);
  const double chain = (double)keys_of(desc, max_len, T) * (wide ? 0.0145 : 0.0112);
  const double products = 4. * (double)(B * H) * (double)T * std::min(ahead, (double)keys_of(desc, max_len, 0)) * (double)D / (wide ? 1.45e9 : 1.15e9);
  const double unpacked_us = 16 + (double)(B * Hkv) * (double)(max_len * D) * 7.2e-7 + std::max(chain, products);
  return rows_us <= unpacked_us;
}

template <int D, int MOD, int NB>
hipError_t launch_blocks(const fl::Mx4DecodeParams& p, int blocks, hipStream_t stream) {
  const hipError_t e = fl::raise_lds_limit(fl::mx4_decode_kernel<D, MOD, NB>);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((fl::mx4_decode_kernel<D, MOD, NB>), dim3(blocks), dim3(256), (fl::Mx4Ring<D, NB>::LDS), stream, p);
  return hipGetLastError();
}
template <int D, int MOD>
hipError_t launch_decode(const fl::Mx4DecodeParams& p, int blocks, int pairs, hipStream_t stream) {
  return pairs <= 16 ? launch_blocks<D, MOD, 1>(p, blocks, stream) : launch_blocks<D, MOD, 2>(p, blocks, stream);
}
template <int D>
hipError_t launch_decode(uint32_t mod, const fl::Mx4DecodeParams& p, int blocks, int pairs, hipStream_t stream) {
  const hipError_t e = mod == FL_MOD_NONE    ? launch_decode<D, fl::kModNone>(p, blocks, pairs, stream)
                       : mod == FL_MOD_ALIBI ? launch_decode<D, fl::kModAlibi>(p, blocks, pairs, stream)
                                             : launch_decode<D, fl::kModSoftcap>(p, blocks, pairs, stream);
  if (e != hipSuccess || p.nsplit == 1) return e;
  hipLaunchKernelGGL(fl::decode_combine_kernel<D>, dim3(p.B * p.T * p.H), dim3(64), 0, stream, p);
  return hipGetLastError();
}

fl::Mx4Cache cache_of(const fl_tensor* k_cache, const fl_tensor* v_cache, const fl_paged_kv* kv) {
  const fl::View k = make_view(k_cache), v = make_view(v_cache);
  return {(uint8_t*)k_cache->ptr, (uint8_t*)v_cache->ptr, k.sb, k.sh, v.sb, v.sh, kv->page_size};
}

// What both calls check; `name` in messages.
fl_status check_call(const char* name, const fl_tensor* q, const fl_tensor* k_cache, const fl_tensor* v_cache, const fl_paged_kv* kv, const fl_variant_desc* desc,
                     const fl_aux* aux, const fl_tensor* out, const fl_tensor* lse, int* page_shift, bool* empty) {
  fl_status st = check_desc(desc);
  if (st != FL_OK) return st;
  if (q == nullptr || k_cache == nullptr || v_cache == nullptr || kv == nullptr || out == nullptr) return fail(FL_ERR_NULL, "q, k_cache, v_cache, kv or out is NULL");
  if (aux != nullptr && aux->struct_size != sizeof(fl_aux)) return fail(FL_ERR_DESC, "aux->struct_size = %u, expected %zu", aux->struct_size, sizeof(fl_aux));
  const uint32_t mask = canonical_mask(desc->mask);
  if ((mask & (FL_MASK_DOC | FL_MASK_PREFIX)) || desc->n_bias != 0 || desc->combine != FL_SINGLE || desc->epilogue != 0 || desc->q_offset != 0)
    return fail(FL_ERR_UNSUPPORTED, "%s covers scale, score_mod and the sliding window only", name);
  if (q->dtype != FL_BF16) return fail(FL_ERR_DTYPE, "%s takes a bf16 q (dtype %d)", name, q->dtype);
  const int64_t B = q->size[0], H = q->size[2], T = q->size[3], D = q->size[4], Hkv = k_cache->size[2];
  if (B < 0 || H < 0 || T < 0 || D <= 0 || Hkv < 0) return fail(FL_ERR_SHAPE, "negative size");
  if (q->size[1] != 1) return fail(FL_ERR_SHAPE, "q must be [B, 1, H, rows, D]");
  if (T > 0x3fffffff) return fail(FL_ERR_SHAPE, "more than 2^30 rows");
  if (H != 0 && (Hkv <= 0 || H % Hkv != 0)) return fail(FL_ERR_SHAPE, "kv heads (%lld) must divide q heads (%lld)", (long long)Hkv, (long long)H);
  if ((st = check_cache_mx4(kv, k_cache, v_cache, B, Hkv, D, page_shift)) != FL_OK) return st;
  *empty = B == 0 || H == 0 || T == 0;
  if (*empty) return FL_OK;
  const int64_t qs[5] = {B, 1, H, T, D}, ls[5] = {B, 1, H, T, 1};
  if ((st = check_data_tensor(q, "q", FL_BF16, qs)) != FL_OK) return st;
  if (out->dtype != FL_BF16 && out->dtype != FL_F32) return fail(FL_ERR_DTYPE, "out dtype %d", out->dtype);
  if ((st = check_data_tensor(out, "out", out->dtype, qs)) != FL_OK) return st;
  if (lse != nullptr && lse->ptr != nullptr) {
    if (lse->dtype != FL_F32) return fail(FL_ERR_DTYPE, "lse must be f32");
    for (int a = 0; a < 5; ++a)
      if (lse->size[a] != ls[a]) return fail(FL_ERR_SHAPE, "lse size[%d] = %lld, expected %lld", a, (long long)lse->size[a], (long long)ls[a]);
  }
  if (aux == nullptr) return fail(FL_ERR_AUX_MISSING, "%s needs aux (workspace)", name);
  if (desc->score_mod == FL_MOD_ALIBI && aux->alibi_slopes == nullptr) return fail(FL_ERR_AUX_MISSING, "alibi_slopes");
  return FL_OK;
}

fl_status check_workspace(const fl_aux* aux, size_t need) {
  if (need == 0) return FL_OK;
  if (aux->workspace == nullptr || aux->workspace_bytes < need)
    return fail(FL_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", need, aux->workspace ? aux->workspace_bytes : (size_t)0);
  if (((uintptr_t)aux->workspace) % 16 != 0) return fail(FL_ERR_ALIGN, "workspace not 16-byte aligned");
  return FL_OK;
}

// The decode step, its arguments checked.
fl_status decode(const fl_tensor* q, const fl_tensor* k_cache, const fl_tensor* v_cache, const fl_paged_kv* kv, const fl_variant_desc* desc, const fl_aux* aux,
                 fl_tensor* out, fl_tensor* lse, int page_shift, hipStream_t stream) {
  const int64_t B = q->size[0], H = q->size[2], T = q->size[3], D = q->size[4], Hkv = k_cache->size[2];
  const int ns = splits_of(B, H, Hkv, T, keys_of(desc, kv->max_seq_len, T));
  const fl_status st = check_workspace(aux, decode_bytes(B, T, H, D, ns));
  if (st != FL_OK) return st;
  const int64_t row_blocks = blocks_of(pairs_of(H, Hkv, T));
  if (B * Hkv * ns * row_blocks > 0x7fffffffLL || B * T * H > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "too many workgroups");
  const uint32_t mask = canonical_mask(desc->mask);
  fl::Mx4DecodeParams p;
  memset(&p, 0, sizeof(p));
  const fl::View qv = make_view(q), ov = make_view(out);
  p.q = (const uint16_t*)q->ptr;
  p.q_sb = qv.sb; p.q_sh = qv.sh; p.q_st = qv.ss;
  p.cache = cache_of(k_cache, v_cache, kv);
  p.block_table = kv->block_table;
  p.table_stride = kv->table_stride;
  p.page_shift = page_shift;
  p.num_pages = (int)k_cache->size[0];
  p.seq_lens = kv->seq_lens;
  p.max_len = kv->max_seq_len;
  p.out = out->ptr;
  p.o_sb = ov.sb; p.o_sh = ov.sh; p.o_st = ov.ss;
  p.out_f32 = out->dtype == FL_F32;
  if (lse != nullptr && lse->ptr != nullptr) {
    const fl::View lv = make_view(lse);
    p.lse = (float*)lse->ptr;
    p.lse_sb = lv.sb; p.lse_sh = lv.sh; p.lse_st = lv.ss;
  }
  p.part_o = (float*)aux->workspace;
  p.part_ml = p.part_o + B * T * H * ns * D;
  p.alibi_slopes = aux->alibi_slopes;
  p.B = (int)B; p.H = (int)H; p.Hkv = (int)Hkv; p.T = (int)T;
  p.nsplit = ns;
  p.by_split = fl::Divisor::of(ns);
  p.by_block = fl::Divisor::of(row_blocks);
  p.by_hkv = fl::Divisor::of(Hkv);
  p.by_group = fl::Divisor::of(H / Hkv);
  p.by_h = fl::Divisor::of(H);
  p.by_t = fl::Divisor::of(T);
  p.window = (mask & FL_MASK_WINDOW) ? clamp_window(desc->window, kv->max_seq_len, kv->max_seq_len) : -1;
  p.scale = desc->scale;
  p.softcap = std::fmin(std::fmax(desc->softcap, 0x1p-120f), 0x1p120f);   // (both and twice them finite; beyond them every score is 0 in fp32, as at them)
  const int blocks = (int)(B * Hkv * ns * row_blocks), pairs = (int)(T * (H / Hkv));
  const hipError_t e = D == 128 ? launch_decode<128>(desc->score_mod, p, blocks, pairs, stream) : launch_decode<64>(desc->score_mod, p, blocks, pairs, stream);
  return e == hipSuccess ? FL_OK : fail(FL_ERR_LAUNCH, "decode launch: %s", hipGetErrorString(e));
}

}  // namespace

extern "C" {

size_t fl_attn_decode_mx4_workspace_size(const fl_tensor* q, const fl_tensor* k_cache, const fl_paged_kv* kv) {
  if (q == nullptr || k_cache == nullptr || kv == nullptr) return 0;
  const int64_t B = q->size[0], H = q->size[2], T = q->size[3];
  return decode_bytes(B, T, H, q->size[4], splits_of(B, H, k_cache->size[2], T, kv->max_seq_len));
}

fl_status fl_attn_decode_mx4(const fl_tensor* q, const fl_tensor* k_cache, const fl_tensor* v_cache, const fl_paged_kv* kv, const fl_variant_desc* desc,
                             const fl_aux* aux, fl_tensor* out, fl_tensor* lse, void* stream) {
  clear_detail();
  int page_shift = 0;
  bool empty = false;
  const fl_status st = check_call("the decode step over 4 bits", q, k_cache, v_cache, kv, desc, aux, out, lse, &page_shift, &empty);
  if (st != FL_OK) return st;
  if (q->size[2] != 0 && pairs_of(q->size[2], k_cache->size[2], q->size[3]) > kMostPairs)
    return fail(FL_ERR_SHAPE, "at most %lld (query row, q head) pairs per kv head (T = %lld)", (long long)kMostPairs, (long long)q->size[3]);
  if (empty) return FL_OK;
  return decode(q, k_cache, v_cache, kv, desc, aux, out, lse, page_shift, (hipStream_t)stream);
}

size_t fl_attn_prefill_mx4_workspace_size(const fl_tensor* q, const fl_tensor* k_cache, const fl_paged_kv* kv) {
  if (q == nullptr || k_cache == nullptr || kv == nullptr) return 0;
  const int64_t pairs = pairs_of(q->size[2], k_cache->size[2], q->size[3]);
  const size_t split = pairs <= kMostRowPairs ? fl_attn_decode_mx4_workspace_size(q, k_cache, kv) : 0;
  return pairs <= kMostPairs && tuned_prefill_gather() != 1 ? split : std::max(split, 2 * dense_bytes(q->size[0], k_cache->size[2], q->size[4], kv->max_seq_len));
}

size_t fl_attn_prefill_mx4_workspace_size_for(const fl_tensor* q, const fl_tensor* k_cache, const fl_paged_kv* kv, const fl_variant_desc* desc) {
  if (q == nullptr || k_cache == nullptr || kv == nullptr) return 0;
  const fl_status st = check_desc(desc);
  clear_detail();
  const int64_t B = q->size[0], H = q->size[2], T = q->size[3], D = q->size[4], Hkv = k_cache->size[2], L = kv->max_seq_len;
  if (st != FL_OK || B <= 0 || H <= 0 || T <= 0 || D <= 0 || Hkv <= 0 || L < 0) return 0;      // (refused, or nothing to do)
  return through_decode(B, H, Hkv, T, D, L, desc) ? decode_bytes(B, T, H, D, splits_of(B, H, Hkv, T, keys_of(desc, L, T))) : 2 * dense_bytes(B, Hkv, D, L);
}

fl_status fl_attn_prefill_mx4(const fl_tensor* q, const fl_tensor* k_cache, const fl_tensor* v_cache, const fl_paged_kv* kv, const fl_variant_desc* desc,
                              const fl_aux* aux, fl_tensor* out, fl_tensor* lse, void* stream_v) {
  clear_detail();
  int page_shift = 0;
  bool empty = false;
  fl_status st = check_call("prefill over 4 bits", q, k_cache, v_cache, kv, desc, aux, out, lse, &page_shift, &empty);
  if (st != FL_OK || empty) return st;
  hipStream_t stream = (hipStream_t)stream_v;
  const int64_t B = q->size[0], H = q->size[2], Sq = q->size[3], D = q->size[4], Hkv = k_cache->size[2], L = kv->max_seq_len;
  if (through_decode(B, H, Hkv, Sq, D, L, desc)) return decode(q, k_cache, v_cache, kv, desc, aux, out, lse, page_shift, stream);

  // the inner forward call: causal, every sequence's key count read on the device.  What it can refuse is checked before the first launch.
  fl_variant_desc inner = *desc;
  inner.mask = canonical_mask(desc->mask) | FL_MASK_CAUSAL;
  fl_aux ia;
  memset(&ia, 0, sizeof(ia));
  ia.struct_size = sizeof(fl_aux);
  ia.alibi_slopes = aux->alibi_slopes;
  if (!fl_variant_supported(&inner, FL_BF16, (int)D, (int)D)) return fail(FL_ERR_UNSUPPORTED, "no forward kernel for D=%lld score_mod=%u with this mask", (long long)D, desc->score_mod);
  const size_t half = dense_bytes(B, Hkv, D, L);
  if ((st = check_workspace(aux, 2 * half)) != FL_OK) return st;
  const int64_t per_head = (L + fl::kUnpackKeys - 1) / fl::kUnpackKeys, blocks = B * Hkv * 2 * per_head;
  if (blocks > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "too many rows to unpack");
  fl_tensor kd, vd;
  memset(&kd, 0, sizeof(kd));
  kd.dtype = FL_BF16;
  kd.size[0] = B; kd.size[1] = 1; kd.size[2] = Hkv; kd.size[3] = L; kd.size[4] = D;
  kd.stride[4] = 1; kd.stride[3] = D; kd.stride[2] = L * D; kd.stride[1] = Hkv * L * D; kd.stride[0] = Hkv * L * D;
  vd = kd;
  kd.ptr = aux->workspace;
  vd.ptr = (char*)aux->workspace + half;
  if (blocks > 0) {
    fl::Mx4UnpackParams u;
    memset(&u, 0, sizeof(u));
    u.cache = cache_of(k_cache, v_cache, kv);
    u.dst[0] = (uint16_t*)kd.ptr;
    u.dst[1] = (uint16_t*)vd.ptr;
    u.block_table = kv->block_table;
    u.seq_lens = kv->seq_lens;
    u.table_stride = kv->table_stride;
    u.page_shift = page_shift;
    u.num_pages = (int)k_cache->size[0];
    u.max_len = kv->max_seq_len;
    u.L = (int)L;
    u.by_blocks = fl::Divisor::of(per_head);
    u.by_heads = fl::Divisor::of(2);
    u.by_hkv = fl::Divisor::of(Hkv);
    if (D == 128) hipLaunchKernelGGL(fl::mx4_unpack_kernel<128>, dim3((unsigned)blocks), dim3(256), 0, stream, u);
    else hipLaunchKernelGGL(fl::mx4_unpack_kernel<64>, dim3((unsigned)blocks), dim3(256), 0, stream, u);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FL_ERR_LAUNCH, "unpack launch: %s", hipGetErrorString(e));
  }
  return forward_of_lengths(q, &kd, &vd, &inner, &ia, out, lse, stream_v, kv->seq_lens);
}

}  // extern "C"
