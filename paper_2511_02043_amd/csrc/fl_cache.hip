// C-ABI entry points around a bounded key/value cache: rotary positions, the write of new tokens into the pages, the weight that a prompt
// chunk gives to cached keys, eviction by it.  Argument validation and launch; the arithmetic is in the kernels.
#include <algorithm>
#include <cstring>

#include "fl_bwd_registry.hpp"
#include "fl_evict.hpp"
#include "fl_host.hpp"
#include "fl_key_weights.hpp"
#include "fl_rotary_host.hpp"

namespace {

using namespace fl::host;

// ---- rotary positions ----

template <class T, int VEC, bool APPEND>
hipError_t launch_rotary(fl::RotaryParams p, bool interleaved, hipStream_t stream) {
  const int heads = p.H + (APPEND ? 2 : 1) * p.Hkv;
  p.units = p.pairs / VEC + (p.D - 2 * p.pairs) / VEC;
  p.tokens_per_block = std::max(1, 256 / p.units);
  p.by_units = fl::Divisor::of(p.units);
  const int64_t blocks = ((int64_t)p.B * p.S + p.tokens_per_block - 1) / p.tokens_per_block;
  p.heads_per_thread = rotary_heads(blocks, heads);
  const dim3 grid((unsigned)blocks, (unsigned)((heads + p.heads_per_thread - 1) / p.heads_per_thread));
  if (interleaved) hipLaunchKernelGGL((fl::rotary_kernel<T, VEC, true, APPEND>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((fl::rotary_kernel<T, VEC, false, APPEND>), grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

extern "C" {

fl_status fl_rotary_embed(const fl_tensor* q, const fl_tensor* k, const fl_rotary* rotary, fl_tensor* q_out, fl_tensor* k_out, void* stream) {
  clear_detail();
  if (q == nullptr && k == nullptr) return fail(FL_ERR_NULL, "q and k are NULL");
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr)) return fail(FL_ERR_NULL, "q and q_out, k and k_out come together");
  const fl_tensor* any = q != nullptr ? q : k;
  const int64_t B = any->size[0], S = any->size[3], D = any->size[4];
  const int64_t H = q != nullptr ? q->size[2] : 0, Hkv = k != nullptr ? k->size[2] : 0;
  if (B < 0 || S < 0 || D <= 0 || H < 0 || Hkv < 0) return fail(FL_ERR_SHAPE, "negative size");
  if (any->size[1] != 1) return fail(FL_ERR_SHAPE, "q and k must be [B, 1, heads, S, D]");
  if (any->dtype != FL_BF16 && any->dtype != FL_F32) return fail(FL_ERR_DTYPE, "dtype %d, expected bf16 or f32", any->dtype);
  fl::RotaryParams p;
  memset(&p, 0, sizeof(p));
  fl_status st = check_rotary(rotary, B, S, D, &p);
  if (st != FL_OK || (st = check_heads(H, Hkv)) != FL_OK) return st;
  const int64_t qs[5] = {B, 1, H, S, D}, ks[5] = {B, 1, Hkv, S, D};
  if (k != nullptr)
    for (int a = 0; a < 5; ++a)
      if (k->size[a] != ks[a]) return fail(FL_ERR_SHAPE, "k size[%d] = %lld, expected %lld", a, (long long)k->size[a], (long long)ks[a]);
  if (B * S == 0) return FL_OK;
  if (H > 0) {
    if ((st = check_data_tensor(q, "q", any->dtype, qs)) != FL_OK || (st = check_data_tensor(q_out, "q_out", any->dtype, qs)) != FL_OK) return st;
    p.q = make_view(q);
    p.q_out = make_view(q_out);
  }
  if (Hkv > 0) {
    if ((st = check_data_tensor(k, "k", any->dtype, ks)) != FL_OK || (st = check_data_tensor(k_out, "k_out", any->dtype, ks)) != FL_OK) return st;
    p.k = make_view(k);
    p.k_out = make_view(k_out);
  }
  if (H + Hkv == 0) return FL_OK;
  p.H = (int)H;
  p.Hkv = (int)Hkv;
  const bool il = rotary->interleaved != 0, wide = rotary_wide(p, any->dtype);
  hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  if (any->dtype == FL_BF16) e = wide ? launch_rotary<uint16_t, 8, false>(p, il, s) : launch_rotary<uint16_t, 1, false>(p, il, s);
  else e = wide ? launch_rotary<float, 4, false>(p, il, s) : launch_rotary<float, 1, false>(p, il, s);
  return e == hipSuccess ? FL_OK : fail(FL_ERR_LAUNCH, "rotary launch: %s", hipGetErrorString(e));
}

fl_status fl_rotary_append(const fl_tensor* q, const fl_tensor* k, const fl_tensor* v, const fl_rotary* rotary, const fl_paged_kv* kv,
                           fl_tensor* q_out, fl_tensor* k_cache, fl_tensor* v_cache, void* stream) {
  clear_detail();
  if (q == nullptr || k == nullptr || v == nullptr || q_out == nullptr || kv == nullptr || k_cache == nullptr || v_cache == nullptr)
    return fail(FL_ERR_NULL, "q, k, v, q_out, kv, k_cache or v_cache is NULL");
  const int64_t B = q->size[0], H = q->size[2], T = q->size[3], D = q->size[4], Hkv = k_cache->size[2];
  if (B < 0 || T < 0 || D <= 0 || H < 0 || Hkv < 0) return fail(FL_ERR_SHAPE, "negative size");
  if (q->size[1] != 1) return fail(FL_ERR_SHAPE, "q must be [B, 1, H, T, D]");
  if (rotary != nullptr && rotary->inverse) return fail(FL_ERR_DESC, "keys enter a cache turned forwards: inverse is 0");
  fl::RotaryParams p;
  memset(&p, 0, sizeof(p));
  fl_status st = check_rotary(rotary, B, T, D, &p);
  if (st != FL_OK || (st = check_heads(H, Hkv)) != FL_OK) return st;
  int page_shift = 0;
  if ((st = check_cache(kv, k_cache, v_cache, B, Hkv, D, &page_shift)) != FL_OK) return st;
  if (B * T == 0) return FL_OK;
  if (kv->seq_lens == nullptr) return fail(FL_ERR_NULL, "seq_lens is NULL");   // (queries alone, which the check of the cache lets pass, read it too)
  const int64_t qs[5] = {B, 1, H, T, D}, ks[5] = {B, 1, Hkv, T, D};
  if (H > 0) {
    if ((st = check_data_tensor(q, "q", FL_BF16, qs)) != FL_OK || (st = check_data_tensor(q_out, "q_out", FL_BF16, qs)) != FL_OK) return st;
    p.q = make_view(q);
    p.q_out = make_view(q_out);
  }
  if (Hkv > 0) {
    if ((st = check_data_tensor(k, "k", FL_BF16, ks)) != FL_OK || (st = check_data_tensor(v, "v", FL_BF16, ks)) != FL_OK) return st;
    p.k = make_view(k);
    p.v = make_view(v);
  }
  if (H + Hkv == 0) return FL_OK;
  p.H = (int)H;
  p.Hkv = (int)Hkv;
  p.k_cache = (uint16_t*)k_cache->ptr;
  p.v_cache = (uint16_t*)v_cache->ptr;
  const fl::View kc = make_view(k_cache), vc = make_view(v_cache);
  p.kc_sp = kc.sb; p.kc_sh = kc.sh; p.kc_st = kc.ss;
  p.vc_sp = vc.sb; p.vc_sh = vc.sh; p.vc_st = vc.ss;
  p.block_table = kv->block_table;
  p.table_stride = kv->table_stride;
  p.page_shift = page_shift;
  p.num_pages = (int)k_cache->size[0];
  p.seq_lens = kv->seq_lens;
  p.max_len = kv->max_seq_len;
  const bool il = rotary->interleaved != 0;
  hipStream_t s = (hipStream_t)stream;
  const hipError_t e = rotary_wide(p, FL_BF16) ? launch_rotary<uint16_t, 8, true>(p, il, s) : launch_rotary<uint16_t, 1, true>(p, il, s);
  return e == hipSuccess ? FL_OK : fail(FL_ERR_LAUNCH, "rotary launch: %s", hipGetErrorString(e));
}

}  // extern "C"

// ---- weights that a prompt chunk gives ----

namespace {

constexpr int kKeysPerBlock = 256;

template <int D, int MOD>
hipError_t launch_key_weights(const fl::KeyWeightParams& p, int blocks, hipStream_t stream) {
  typedef fl::KeyWeightCfg<D, MOD> C;
  static_assert(C::KEYS == kKeysPerBlock, "keys per workgroup");
  hipError_t e = fl::raise_lds_limit(fl::key_weights_kernel<C>);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fl::key_weights_kernel<C>, dim3(blocks), dim3(C::NW * 64), C::LDS, stream, p);
  return hipGetLastError();
}
template <int D>
hipError_t launch_key_weights(uint32_t mod, const fl::KeyWeightParams& p, int blocks, hipStream_t stream) {
  return mod == FL_MOD_NONE ? launch_key_weights<D, fl::kModNone>(p, blocks, stream)
         : mod == FL_MOD_ALIBI ? launch_key_weights<D, fl::kModAlibi>(p, blocks, stream)
                               : launch_key_weights<D, fl::kModSoftcap>(p, blocks, stream);
}

// Workgroups that share a key block's (head, row tile) sequence: a thousand workgroups in all, each with four row tiles at least.
// (a prompt of 8192, 32 / 8 heads, D = 128: one workgroup a block 614 us, four 302 and 5 for the joining; 8 chunks of 512 rows on 4k - 8k
// keys, 2048 workgroups as they are, 250, cut in two 245 and 5)
int key_weight_splits(int64_t B, int64_t H, int64_t Hkv, int64_t Sq, int64_t max_len) {
  const int64_t blocks = B * Hkv * ((max_len + kKeysPerBlock - 1) / kKeysPerBlock);
  if (blocks <= 0 || Hkv <= 0) return 1;
  const int64_t items = H / Hkv * ((Sq + 63) / 64);
  return (int)std::max<int64_t>(1, std::min<int64_t>({(1024 + blocks - 1) / blocks, items / 4, 64}));
}

}  // namespace

extern "C" {

size_t fl_key_weights_workspace_size(const fl_tensor* q, const fl_tensor* k_cache, const fl_paged_kv* kv) {
  if (q == nullptr || k_cache == nullptr || kv == nullptr) return 0;
  const int64_t B = q->size[0], Hkv = k_cache->size[2];
  const int ns = key_weight_splits(B, q->size[2], Hkv, q->size[3], kv->max_seq_len);
  if (ns == 1) return 0;
  return (size_t)ns * (size_t)(B * Hkv) * (size_t)((kv->max_seq_len + (int64_t)kKeysPerBlock - 1) / kKeysPerBlock) * kKeysPerBlock * sizeof(float);
}

fl_status fl_key_weights(const fl_tensor* q, const fl_tensor* k_cache, const fl_tensor* lse, const fl_paged_kv* kv,
                         const fl_variant_desc* desc, const fl_aux* aux, fl_tensor* weights, void* stream_v) {
  clear_detail();
  fl_status st = check_desc(desc);
  if (st != FL_OK) return st;
  if (q == nullptr || k_cache == nullptr || lse == nullptr || kv == nullptr || weights == nullptr)
    return fail(FL_ERR_NULL, "q, k_cache, lse, kv or weights is NULL");
  if (aux != nullptr && aux->struct_size != sizeof(fl_aux)) return fail(FL_ERR_DESC, "aux->struct_size = %u, expected %zu", aux->struct_size, sizeof(fl_aux));
  const uint32_t mask = canonical_mask(desc->mask);
  if ((mask & (FL_MASK_DOC | FL_MASK_PREFIX)) || desc->n_bias != 0 || desc->combine != FL_SINGLE || desc->epilogue != 0 || desc->q_offset != 0)
    return fail(FL_ERR_UNSUPPORTED, "the weights of cached keys cover scale, score_mod and the sliding window only");
  const int64_t B = q->size[0], H = q->size[2], Sq = q->size[3], D = q->size[4], Hkv = k_cache->size[2];
  if (B < 0 || H < 0 || Sq < 0 || D <= 0 || Hkv < 0) return fail(FL_ERR_SHAPE, "negative size");
  if (q->size[1] != 1) return fail(FL_ERR_SHAPE, "q must be [B, 1, H, Sq, D]");
  if (Sq > 0x3fffffff) return fail(FL_ERR_SHAPE, "Sq must be below 2^30");
  if (D != 32 && D != 64 && D != 128) return fail(FL_ERR_UNSUPPORTED, "D = %lld, expected 32, 64 or 128", (long long)D);
  if (H != 0 && (Hkv <= 0 || H % Hkv != 0)) return fail(FL_ERR_SHAPE, "kv heads (%lld) must divide q heads (%lld)", (long long)Hkv, (long long)H);
  int page_shift = 0;
  if ((st = check_cache(kv, k_cache, nullptr, B, Hkv, D, &page_shift)) != FL_OK) return st;
  if (B == 0 || H == 0 || Sq == 0 || kv->max_seq_len == 0) return FL_OK;
  const int64_t qs[5] = {B, 1, H, Sq, D}, ls[5] = {B, 1, H, Sq, 1};
  if ((st = check_data_tensor(q, "q", FL_BF16, qs)) != FL_OK) return st;
  if (lse->ptr == nullptr) return fail(FL_ERR_NULL, "lse is NULL");
  if (lse->dtype != FL_F32) return fail(FL_ERR_DTYPE, "lse must be f32");
  for (int a = 0; a < 5; ++a)
    if (lse->size[a] != ls[a]) return fail(FL_ERR_SHAPE, "lse size[%d] = %lld, expected %lld", a, (long long)lse->size[a], (long long)ls[a]);
  if ((st = check_weights(weights, "weights", B, Hkv, kv->max_seq_len)) != FL_OK) return st;
  if (desc->score_mod == FL_MOD_ALIBI && (aux == nullptr || aux->alibi_slopes == nullptr)) return fail(FL_ERR_AUX_MISSING, "alibi_slopes");
  const int ns = key_weight_splits(B, H, Hkv, Sq, kv->max_seq_len);
  const size_t need = fl_key_weights_workspace_size(q, k_cache, kv);
  if (need != 0) {
    if (aux == nullptr || aux->workspace == nullptr || aux->workspace_bytes < need)
      return fail(FL_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", need, aux != nullptr && aux->workspace ? aux->workspace_bytes : (size_t)0);
    if (((uintptr_t)aux->workspace) % 16 != 0) return fail(FL_ERR_ALIGN, "workspace not 16-byte aligned");
  }
  const int64_t kblocks = (kv->max_seq_len + (int64_t)kKeysPerBlock - 1) / kKeysPerBlock;
  if (B * Hkv * kblocks * ns > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "too many workgroups");
  if ((Sq + 63) / 64 * (H / Hkv) > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "too many row tiles");

  fl::KeyWeightParams p;
  memset(&p, 0, sizeof(p));
  const fl::View qv = make_view(q), kc = make_view(k_cache);
  p.q = (const uint16_t*)q->ptr;
  p.q_sb = qv.sb; p.q_sh = qv.sh; p.q_ss = qv.ss;
  p.k = (const uint16_t*)k_cache->ptr;
  p.k_sp = kc.sb; p.k_sh = kc.sh; p.k_st = kc.ss;
  p.block_table = kv->block_table;
  p.table_stride = kv->table_stride;
  p.page_shift = page_shift;
  p.num_pages = (int)k_cache->size[0];
  p.seq_lens = kv->seq_lens;
  p.lse = (const float*)lse->ptr;
  p.lse_sb = lse->stride[0]; p.lse_sh = lse->stride[2]; p.lse_ss = lse->stride[3];
  p.weights = (float*)weights->ptr;
  p.w_sb = B > 1 ? weights->stride[0] : 0;
  p.w_sh = Hkv > 1 ? weights->stride[2] : 0;
  p.part = ns > 1 ? (float*)aux->workspace : nullptr;
  p.alibi_slopes = desc->score_mod == FL_MOD_ALIBI ? aux->alibi_slopes : nullptr;
  p.B = (int)B; p.H = (int)H; p.Hkv = (int)Hkv; p.Sq = (int)Sq;
  p.group = (int)(H / Hkv);
  p.max_len = kv->max_seq_len;
  p.n_kblocks = (int)kblocks;
  p.nsplit = ns;
  p.window = (mask & FL_MASK_WINDOW) ? clamp_window(desc->window, kv->max_seq_len, Sq) : -1;
  p.scale = desc->scale;
  p.softcap = desc->softcap;
  p.by_problems = fl::Divisor::of(B * Hkv);
  p.by_hkv = fl::Divisor::of(Hkv);
  p.by_kblocks = fl::Divisor::of(kblocks);
  p.by_split = fl::Divisor::of(ns);
  hipStream_t stream = (hipStream_t)stream_v;
  const int blocks = (int)(B * Hkv * kblocks * ns);
  hipError_t e = D == 128  ? launch_key_weights<128>(desc->score_mod, p, blocks, stream)
                 : D == 64 ? launch_key_weights<64>(desc->score_mod, p, blocks, stream)
                           : launch_key_weights<32>(desc->score_mod, p, blocks, stream);
  if (e != hipSuccess) return fail(FL_ERR_LAUNCH, "key weights launch: %s", hipGetErrorString(e));
  if (ns > 1) {
    hipLaunchKernelGGL(fl::key_weights_join_kernel, dim3((unsigned)(B * Hkv * kblocks)), dim3(256), 0, stream, p);
    if ((e = hipGetLastError()) != hipSuccess) return fail(FL_ERR_LAUNCH, "key weights join launch: %s", hipGetErrorString(e));
  }
  return FL_OK;
}

}  // extern "C"

// ---- eviction ----

namespace {

template <int THREADS, bool HELD>
hipError_t launch_select(const fl::EvictParams& p, unsigned blocks, hipStream_t stream) {
  const hipError_t e = fl::raise_lds_limit(fl::evict_select_kernel<THREADS, HELD>);
  if (e != hipSuccess) return e;
  const size_t lds = sizeof(fl::SelectShared) + (HELD ? (size_t)p.max_len * sizeof(float) : 0);
  hipLaunchKernelGGL((fl::evict_select_kernel<THREADS, HELD>), dim3(blocks), dim3(THREADS), lds, stream, p);
  return hipGetLastError();
}
// By the longest sequence that may come: short ones need no more than four waves, whose barriers are cheaper and of which several workgroups share
// a compute unit (us with 4 / 16 waves: 64 sequences x 8 heads of 2049 - 2304 slots 11.9 / 17.3, one of 500 - 700 6.7 / 7.7); the weights wait in LDS
// where they fit (8 x 8 of 16k - 32k slots 28.4, read again for every walk 48.9).
hipError_t launch_select(const fl::EvictParams& p, unsigned blocks, hipStream_t stream) {
  if (p.max_len <= 4096) return launch_select<256, true>(p, blocks, stream);
  return p.max_len <= fl::kSelectHeld ? launch_select<1024, true>(p, blocks, stream) : launch_select<1024, false>(p, blocks, stream);
}

}  // namespace

extern "C" {

fl_status fl_cache_evict(const fl_tensor* weights, fl_tensor* k_cache, fl_tensor* v_cache, const fl_paged_kv* kv, const fl_evict* evict,
                         fl_tensor* new_weights, void* stream_v) {
  clear_detail();
  if (weights == nullptr || k_cache == nullptr || v_cache == nullptr || kv == nullptr || evict == nullptr || new_weights == nullptr)
    return fail(FL_ERR_NULL, "weights, k_cache, v_cache, kv, evict or new_weights is NULL");
  if (evict->struct_size != sizeof(fl_evict)) return fail(FL_ERR_DESC, "evict->struct_size = %u, expected %zu", evict->struct_size, sizeof(fl_evict));
  const int64_t B = weights->size[0], Hkv = k_cache->size[2], D = k_cache->size[4], page_size = k_cache->size[3];
  if (B < 0 || Hkv < 0 || D <= 0) return fail(FL_ERR_SHAPE, "negative size");
  if (D % 8 != 0) return fail(FL_ERR_UNSUPPORTED, "D = %lld, expected a multiple of 8", (long long)D);
  if (evict->budget < 1 || evict->sinks < 0 || evict->recent < 0 || (int64_t)evict->sinks + evict->recent > evict->budget)
    return fail(FL_ERR_DESC, "budget = %d, sinks = %d, recent = %d: expected sinks + recent <= budget, budget >= 1", evict->budget, evict->sinks, evict->recent);
  int page_shift = 0;
  fl_status st = check_cache(kv, k_cache, v_cache, B, Hkv, D, &page_shift);
  if (st != FL_OK) return st;
  if (page_size < 8 || (page_size & (page_size - 1)) != 0)
    return fail(FL_ERR_SHAPE, "the page size (%lld) must be a power of two >= 8", (long long)page_size);
  if (B == 0 || Hkv == 0) return FL_OK;
  if (evict->new_lens == nullptr || evict->kept == nullptr || evict->dst_table == nullptr) return fail(FL_ERR_NULL, "new_lens, kept or dst_table is NULL");
  if (evict->dst_stride < ((int64_t)evict->budget + page_size - 1) / page_size)
    return fail(FL_ERR_SHAPE, "dst_stride %d is less than the pages of budget", evict->dst_stride);
  if ((st = check_weights(weights, "weights", B, Hkv, kv->max_seq_len, false)) != FL_OK) return st;
  if ((st = check_weights(new_weights, "new_weights", B, Hkv, evict->budget)) != FL_OK) return st;
  // workgroups read lengths, tables and weights while others write: no output may share memory with those or with another
  {
    using fl::host::Rows;
    const int64_t src_pages = (kv->max_seq_len + page_size - 1) / page_size, dst_pages = (evict->budget + page_size - 1) / page_size;
    auto of = [&](const fl_tensor* t, int64_t n) {
      return Rows{(uintptr_t)t->ptr, B, B > 1 ? t->stride[0] * 4 : 0, Hkv, Hkv > 1 ? t->stride[2] * 4 : 0, n * 4};
    };
    const struct { const char* name; Rows rows; } all[] = {
        {"new_lens", fl::host::flat_rows(evict->new_lens, B * 4)},
        {"kept", fl::host::flat_rows(evict->kept, B * Hkv * evict->budget * 4)},
        {"new_weights", of(new_weights, new_weights->size[4])},
        {"seq_lens", fl::host::flat_rows(kv->seq_lens, B * 4)},
        {"dst_table", Rows{(uintptr_t)evict->dst_table, B, evict->dst_stride * 4LL, 1, 0, dst_pages * 4}},
        {"block_table", Rows{(uintptr_t)kv->block_table, kv->block_table != nullptr ? B : 0, kv->table_stride * 4LL, 1, 0, src_pages * 4}},
        {"weights", of(weights, kv->max_seq_len)}};
    for (int o = 0; o < 3; ++o)
      for (int i = o + 1; i < 7; ++i)
        if (rows_meet(all[o].rows, all[i].rows)) return fail(FL_ERR_DESC, "%s and %s share memory", all[o].name, all[i].name);
  }
  if (B * Hkv > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "too many workgroups");

  fl::EvictParams p;
  memset(&p, 0, sizeof(p));
  const fl::View kc = make_view(k_cache), vc = make_view(v_cache);
  p.weights = (const float*)weights->ptr;
  p.w_sb = B > 1 ? weights->stride[0] : 0;
  p.w_sh = Hkv > 1 ? weights->stride[2] : 0;
  p.new_weights = (float*)new_weights->ptr;
  p.nw_sb = B > 1 ? new_weights->stride[0] : 0;
  p.nw_sh = Hkv > 1 ? new_weights->stride[2] : 0;
  p.kept = evict->kept;
  p.new_lens = evict->new_lens;
  p.k_cache = (uint16_t*)k_cache->ptr;
  p.v_cache = (uint16_t*)v_cache->ptr;
  p.k_sp = kc.sb; p.k_sh = kc.sh; p.k_st = kc.ss;
  p.v_sp = vc.sb; p.v_sh = vc.sh; p.v_st = vc.ss;
  p.block_table = kv->block_table;
  p.dst_table = evict->dst_table;
  p.table_stride = kv->table_stride;
  p.dst_stride = evict->dst_stride;
  p.page_shift = page_shift;
  p.num_pages = (int)k_cache->size[0];
  p.max_len = kv->max_seq_len;
  p.seq_lens = kv->seq_lens;
  p.B = (int)B; p.Hkv = (int)Hkv; p.D = (int)D;
  p.budget = evict->budget;
  p.sinks = evict->sinks;
  p.recent = evict->recent;
  p.capacity = (int)new_weights->size[4];
  p.pieces = (int)(D / 8);
  p.rows_per_block = 64;
  const int64_t groups = std::min<int64_t>(evict->budget, kv->max_seq_len) / p.rows_per_block + 1;
  if (B * Hkv * groups > 0x7fffffffLL) return fail(FL_ERR_SHAPE, "too many workgroups");
  p.by_hkv = fl::Divisor::of(Hkv);
  p.by_groups = fl::Divisor::of(groups);
  p.by_pieces = fl::Divisor::of(p.pieces);
  hipStream_t stream = (hipStream_t)stream_v;
  hipError_t e = launch_select(p, (unsigned)(B * Hkv), stream);
  if (e != hipSuccess) return fail(FL_ERR_LAUNCH, "eviction launch: %s", hipGetErrorString(e));
  hipLaunchKernelGGL(fl::evict_move_kernel, dim3((unsigned)(B * Hkv * groups)), dim3(256), 0, stream, p);
  if ((e = hipGetLastError()) != hipSuccess) return fail(FL_ERR_LAUNCH, "eviction copy launch: %s", hipGetErrorString(e));
  return FL_OK;
}

}  // extern "C"
