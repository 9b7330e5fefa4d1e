// C-ABI entry points of heads that are normalised and turned in one pass: forward pass, gradient, and new tokens into a bf16 or 4-bit cache.
// Argument validation and launch; the arithmetic is in fl_norm.hpp.
#include <cstring>

#include "fl_norm.hpp"
#include "fl_rotary_host.hpp"

namespace {

using namespace fl::host;

constexpr int64_t kMostChannels = 1024;

fl_status check_norm(const fl_head_norm* n, fl::NormParams* p) {
  if (n->struct_size != sizeof(fl_head_norm)) return fail(FL_ERR_DESC, "norm->struct_size = %u, expected %zu", n->struct_size, sizeof(fl_head_norm));
  if (!(n->eps >= 0.f) || !std::isfinite(n->eps)) return fail(FL_ERR_DESC, "eps must be finite and >= 0");
  p->norm = 1;
  p->eps = n->eps;
  p->weight[0] = n->q_weight;
  p->weight[1] = n->k_weight;
  return FL_OK;
}

// How the kernels share out a row: VEC channels a piece, UPL units a lane.
struct RowShape {
  bool wide;
  int upl;
};
RowShape shape_row(fl::NormParams* p, int dtype) {
  RowShape r;
  r.wide = rotary_wide(*p, dtype);
  const int vec = r.wide ? (dtype == FL_BF16 ? 8 : 4) : 1;
  p->units = p->pairs / vec + (p->D - 2 * p->pairs) / vec;
  // a lane of a wave has one unit of wide rows where those fit (D = 128: 8 to 16 units of bf16, 16 to 32 of f32)
  r.upl = r.wide ? (p->units <= 64 ? 1 : 4) : (p->units <= 128 ? 2 : 16);
  p->log_lanes = 0;
  while ((r.upl << p->log_lanes) < p->units) ++p->log_lanes;
  p->by_pairs = fl::Divisor::of(p->pairs);
  p->by_h = fl::Divisor::of(p->H);
  p->by_hkv = fl::Divisor::of(p->Hkv);
  return r;
}

// Tokens of a workgroup: enough workgroups for the chip, then enough rows for long runs; their angles take LDS.  (Forward pass of 2 x 8192 tokens, 32 / 8 heads, us with at
// least 1024 / 2048 / 4096 / 8192 workgroups: D = 128 70.6 / 68.5 / 67.6 / 72.0, D = 64 33.3 / 32.1 / 32.7 / 39.3, D = 80 44.2 / 44.2 / 46.6 / 54.8.  Appending: below.)
constexpr int64_t kMostTokens = 16;
int tokens_of(const fl::NormParams& p, int64_t workgroups) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)p.B * p.S / workgroups, kMostTokens, 16 * 1024 / p.pairs / 8}));
}

template <class T, int VEC, int UPL>
hipError_t launch_forward(const fl::NormParams& p, bool il, dim3 grid, hipStream_t stream) {
  const size_t lds = fl::norm_lds_bytes(p.tokens_per_block, p.pairs, 4, p.D);
  if (il) hipLaunchKernelGGL((fl::norm_rotary_kernel<T, VEC, UPL, true>), grid, dim3(256), lds, stream, p);
  else hipLaunchKernelGGL((fl::norm_rotary_kernel<T, VEC, UPL, false>), grid, dim3(256), lds, stream, p);
  return hipGetLastError();
}
template <class T, int VEC, int UPL>
hipError_t launch_gradient(const fl::NormParams& p, bool il, dim3 grid, hipStream_t stream) {
  const size_t lds = 4 * p.D * sizeof(float);
  if (il) hipLaunchKernelGGL((fl::norm_rotary_bwd_kernel<T, VEC, UPL, true>), grid, dim3(256), lds, stream, p);
  else hipLaunchKernelGGL((fl::norm_rotary_bwd_kernel<T, VEC, UPL, false>), grid, dim3(256), lds, stream, p);
  return hipGetLastError();
}
template <int VEC, int UPL, bool MX4, bool ALIGNED = false, bool STREAM = false>
hipError_t launch_append(const fl::NormParams& p, bool il, dim3 grid, hipStream_t stream) {
  size_t lds = fl::norm_lds_bytes(p.tokens_per_block, p.pairs, 9, p.D);
  if (MX4) lds += (size_t)p.tokens_per_block * p.pairs * 16;
  if (MX4 && !ALIGNED) lds += (size_t)(256 >> p.log_lanes) * (p.D + 2) * sizeof(double);
  if (il) hipLaunchKernelGGL((fl::norm_append_kernel<VEC, UPL, true, STREAM, MX4, ALIGNED>), grid, dim3(256), lds, stream, p);
  else hipLaunchKernelGGL((fl::norm_append_kernel<VEC, UPL, false, STREAM, MX4, ALIGNED>), grid, dim3(256), lds, stream, p);
  return hipGetLastError();
}

// The checks that forward pass and gradient share, up to the tensors; `empty`: nothing to launch.
fl_status check_call(const fl_tensor* q, const fl_tensor* k, const fl_rotary* rotary, const fl_head_norm* norm, fl::NormParams* p, bool* empty) {
  if (q == nullptr && k == nullptr) return fail(FL_ERR_NULL, "q and k are NULL");
  if (norm == nullptr) return fail(FL_ERR_NULL, "norm is NULL");
  const fl_tensor* any = q != nullptr ? q : k;
  const int64_t B = any->size[0], S = any->size[3], D = any->size[4];
  const int64_t H = q != nullptr ? q->size[2] : 0, Hkv = k != nullptr ? k->size[2] : 0;
  if (B < 0 || S < 0 || D <= 0 || H < 0 || Hkv < 0) return fail(FL_ERR_SHAPE, "negative size");
  if (any->size[1] != 1) return fail(FL_ERR_SHAPE, "q and k must be [B, 1, heads, S, D]");
  if (any->dtype != FL_BF16 && any->dtype != FL_F32) return fail(FL_ERR_DTYPE, "dtype %d, expected bf16 or f32", any->dtype);
  if (D > kMostChannels) return fail(FL_ERR_UNSUPPORTED, "D = %lld, expected 1 .. %lld", (long long)D, (long long)kMostChannels);
  fl_status st = check_rotary(rotary, B, S, D, p);
  if (st != FL_OK || (st = check_heads(H, Hkv)) != FL_OK || (st = check_norm(norm, p)) != FL_OK) return st;
  if (rotary->inverse) return fail(FL_ERR_DESC, "inverse is 0");
  if (k != nullptr) {
    const int64_t ks[5] = {B, 1, Hkv, S, D};
    for (int a = 0; a < 5; ++a)
      if (k->size[a] != ks[a]) return fail(FL_ERR_SHAPE, "k size[%d] = %lld, expected %lld", a, (long long)k->size[a], (long long)ks[a]);
  }
  p->H = (int)H;
  p->Hkv = (int)Hkv;
  *empty = B * S == 0 || H + Hkv == 0;
  return FL_OK;
}

// A tensor of q's sizes (k's: `keys`) as a view.
fl_status view_of(const fl_tensor* t, const char* name, const fl::NormParams& p, bool keys, int dtype, fl::View* v) {
  const int64_t size[5] = {p.B, 1, keys ? p.Hkv : p.H, p.S, p.D};
  if (size[2] == 0) return FL_OK;
  const fl_status st = check_data_tensor(t, name, dtype, size);
  if (st == FL_OK) *v = make_view(t);
  return st;
}

// The gradient's launch: enough workgroups for the chip, few enough that their rows of partial sums are soon added up.  (2 x 8192 tokens, 32 / 8 heads, us with up to 1024 / 2048 /
// 4096 workgroups, the last with eight heads of a token at most: D = 128 120.5 / 119.0 / 116.8, 32 pairs of it turning 139 / 128 / 140, D = 64 67.5 / 62.9 / 62.9.)
constexpr int64_t kGradientBlocks = 2048;
void share_gradient(fl::NormParams* p) {
  p->tokens_per_block = 256 >> p->log_lanes;
  p->groups = (int)(((int64_t)p->B * p->S + p->tokens_per_block - 1) / p->tokens_per_block);
  p->heads_per_thread = rotary_heads(p->groups, p->H + p->Hkv);
  p->q_chunks = (p->H + p->heads_per_thread - 1) / p->heads_per_thread;
  p->k_chunks = (p->Hkv + p->heads_per_thread - 1) / p->heads_per_thread;
  p->blocks = (int)std::max<int64_t>(1, std::min<int64_t>(p->groups, kGradientBlocks / std::max(1, p->q_chunks + p->k_chunks)));
}

}  // namespace

extern "C" {

fl_status fl_norm_rotary(const fl_tensor* q, const fl_tensor* k, const fl_rotary* rotary, const fl_head_norm* norm, fl_tensor* q_out, fl_tensor* k_out,
                         void* stream) {
  clear_detail();
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr)) return fail(FL_ERR_NULL, "q and q_out, k and k_out come together");
  fl::NormParams p;
  memset(&p, 0, sizeof(p));
  bool empty = false;
  fl_status st = check_call(q, k, rotary, norm, &p, &empty);
  if (st != FL_OK || empty) return st;
  const int dtype = (q != nullptr ? q : k)->dtype;
  if ((st = view_of(q, "q", p, false, dtype, &p.q)) != FL_OK || (st = view_of(q_out, "q_out", p, false, dtype, &p.q_out)) != FL_OK ||
      (st = view_of(k, "k", p, true, dtype, &p.k)) != FL_OK || (st = view_of(k_out, "k_out", p, true, dtype, &p.k_out)) != FL_OK)
    return st;
  const RowShape r = shape_row(&p, dtype);
  p.tokens_per_block = tokens_of(p, 2048);
  const dim3 grid((unsigned)(((int64_t)p.B * p.S + p.tokens_per_block - 1) / p.tokens_per_block));
  const bool il = rotary->interleaved != 0;
  hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  if (dtype == FL_BF16)
    e = r.wide ? (r.upl == 1 ? launch_forward<uint16_t, 8, 1>(p, il, grid, s) : launch_forward<uint16_t, 8, 4>(p, il, grid, s))
               : (r.upl == 2 ? launch_forward<uint16_t, 1, 2>(p, il, grid, s) : launch_forward<uint16_t, 1, 16>(p, il, grid, s));
  else
    e = r.wide ? (r.upl == 1 ? launch_forward<float, 4, 1>(p, il, grid, s) : launch_forward<float, 4, 4>(p, il, grid, s))
               : (r.upl == 2 ? launch_forward<float, 1, 2>(p, il, grid, s) : launch_forward<float, 1, 16>(p, il, grid, s));
  return e == hipSuccess ? FL_OK : fail(FL_ERR_LAUNCH, "norm launch: %s", hipGetErrorString(e));
}

size_t fl_norm_rotary_bwd_workspace_size(const fl_tensor* q, const fl_tensor* k, const fl_rotary* rotary) {
  if ((q == nullptr && k == nullptr) || rotary == nullptr) return 0;
  fl::NormParams p;
  memset(&p, 0, sizeof(p));
  bool empty = false;
  fl_head_norm norm = {sizeof(fl_head_norm), 0.f, nullptr, nullptr};
  fl_rotary r = *rotary;
  r.positions = (const int32_t*)1, r.inv_freq = (const float*)1;      // (not looked at)
  const fl_status st = check_call(q, k, &r, &norm, &p, &empty);
  clear_detail();
  if (st != FL_OK || empty) return 0;
  shape_row(&p, (q != nullptr ? q : k)->dtype);
  share_gradient(&p);
  return (size_t)(p.q_chunks + p.k_chunks) * p.blocks * p.D * sizeof(float);
}

fl_status fl_norm_rotary_bwd(const fl_tensor* q, const fl_tensor* k, const fl_tensor* dq_out, const fl_tensor* dk_out, const fl_rotary* rotary,
                             const fl_head_norm* norm, fl_tensor* dq, fl_tensor* dk, float* dq_weight, float* dk_weight, void* workspace,
                             size_t workspace_bytes, void* stream_v) {
  clear_detail();
  if ((q == nullptr) != (dq_out == nullptr) || (k == nullptr) != (dk_out == nullptr)) return fail(FL_ERR_NULL, "q and dq_out, k and dk_out come together");
  if ((q == nullptr && (dq != nullptr || dq_weight != nullptr)) || (k == nullptr && (dk != nullptr || dk_weight != nullptr)))
    return fail(FL_ERR_NULL, "a gradient is wanted of what is NULL");
  fl::NormParams p;
  memset(&p, 0, sizeof(p));
  bool empty = false;
  fl_status st = check_call(q, k, rotary, norm, &p, &empty);
  if (st != FL_OK) return st;
  hipStream_t stream = (hipStream_t)stream_v;
  p.dweight[0] = dq_weight;
  p.dweight[1] = dk_weight;
  const bool weights = dq_weight != nullptr || dk_weight != nullptr;
  const dim3 weight_grid((unsigned)((p.D + 15) / 16), 2);
  hipError_t e = hipSuccess;
  if (!empty) {
    const int dtype = (q != nullptr ? q : k)->dtype;
    if ((st = view_of(q, "q", p, false, dtype, &p.q)) != FL_OK || (st = view_of(dq_out, "dq_out", p, false, dtype, &p.dy[0])) != FL_OK ||
        (st = view_of(k, "k", p, true, dtype, &p.k)) != FL_OK || (st = view_of(dk_out, "dk_out", p, true, dtype, &p.dy[1])) != FL_OK)
      return st;
    if (dq != nullptr && (st = view_of(dq, "dq", p, false, dtype, &p.dx[0])) != FL_OK) return st;
    if (dk != nullptr && (st = view_of(dk, "dk", p, true, dtype, &p.dx[1])) != FL_OK) return st;
    const RowShape r = shape_row(&p, dtype);
    share_gradient(&p);
    if (weights) {
      const size_t need = (size_t)(p.q_chunks + p.k_chunks) * p.blocks * p.D * sizeof(float);
      if (workspace == nullptr || workspace_bytes < need)
        return fail(FL_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", need, workspace ? workspace_bytes : (size_t)0);
      if (((uintptr_t)workspace) % 16 != 0) return fail(FL_ERR_ALIGN, "workspace not 16-byte aligned");
      p.part = (float*)workspace;
    }
    if (!weights && dq == nullptr && dk == nullptr) return FL_OK;
    const dim3 grid((unsigned)p.blocks, (unsigned)(p.q_chunks + p.k_chunks));
    const bool il = rotary->interleaved != 0;
    if (dtype == FL_BF16)
      e = r.wide ? (r.upl == 1 ? launch_gradient<uint16_t, 8, 1>(p, il, grid, stream) : launch_gradient<uint16_t, 8, 4>(p, il, grid, stream))
                 : (r.upl == 2 ? launch_gradient<uint16_t, 1, 2>(p, il, grid, stream) : launch_gradient<uint16_t, 1, 16>(p, il, grid, stream));
    else
      e = r.wide ? (r.upl == 1 ? launch_gradient<float, 4, 1>(p, il, grid, stream) : launch_gradient<float, 4, 4>(p, il, grid, stream))
                 : (r.upl == 2 ? launch_gradient<float, 1, 2>(p, il, grid, stream) : launch_gradient<float, 1, 16>(p, il, grid, stream));
    if (e != hipSuccess) return fail(FL_ERR_LAUNCH, "norm gradient launch: %s", hipGetErrorString(e));
  }
  if (weights) {                                   // (no tokens: sums over nothing)
    hipLaunchKernelGGL(fl::norm_weights_kernel, weight_grid, dim3(1024), 0, stream, p);
    if ((e = hipGetLastError()) != hipSuccess) return fail(FL_ERR_LAUNCH, "norm weights launch: %s", hipGetErrorString(e));
  }
  return FL_OK;
}

fl_status fl_norm_rotary_append(const fl_tensor* q, const fl_tensor* k, const fl_tensor* v, const fl_rotary* rotary, const fl_head_norm* norm,
                                const fl_paged_kv* kv, fl_tensor* q_out, fl_tensor* k_cache, fl_tensor* v_cache, fl_tensor* k_held, fl_tensor* v_held,
                                void* stream) {
  clear_detail();
  if (q == nullptr || k == nullptr || v == nullptr || q_out == nullptr || kv == nullptr || k_cache == nullptr || v_cache == nullptr)
    return fail(FL_ERR_NULL, "q, k, v, q_out, kv, k_cache or v_cache is NULL");
  const int64_t B = q->size[0], H = q->size[2], T = q->size[3], D = q->size[4], Hkv = k_cache->size[2];
  if (B < 0 || T < 0 || D <= 0 || H < 0 || Hkv < 0) return fail(FL_ERR_SHAPE, "negative size");
  if (q->size[1] != 1) return fail(FL_ERR_SHAPE, "q must be [B, 1, H, T, D]");
  if (D > kMostChannels) return fail(FL_ERR_UNSUPPORTED, "D = %lld, expected 1 .. %lld", (long long)D, (long long)kMostChannels);
  if (rotary != nullptr && rotary->inverse) return fail(FL_ERR_DESC, "keys enter a cache turned forwards: inverse is 0");
  if (k_cache->dtype != v_cache->dtype) return fail(FL_ERR_DTYPE, "k_cache has dtype %d, v_cache %d", k_cache->dtype, v_cache->dtype);
  const bool mx4 = k_cache->dtype == FL_MX4;
  if (!mx4 && (k_held != nullptr || v_held != nullptr)) return fail(FL_ERR_DESC, "k_held and v_held go with caches in 4 bits");
  fl::NormParams p;
  memset(&p, 0, sizeof(p));
  fl_status st = check_rotary(rotary, B, T, D, &p);
  if (st != FL_OK || (st = check_heads(H, Hkv)) != FL_OK || (norm != nullptr && (st = check_norm(norm, &p)) != FL_OK)) return st;
  int page_shift = 0;
  if ((st = mx4 ? check_cache_mx4(kv, k_cache, v_cache, B, Hkv, D, &page_shift) : check_cache(kv, k_cache, v_cache, B, Hkv, D, &page_shift)) != FL_OK) return st;
  if (B * T == 0) return FL_OK;
  p.H = (int)H;
  p.Hkv = (int)Hkv;
  if ((st = view_of(q, "q", p, false, FL_BF16, &p.q)) != FL_OK || (st = view_of(q_out, "q_out", p, false, FL_BF16, &p.q_out)) != FL_OK ||
      (st = view_of(k, "k", p, true, FL_BF16, &p.k)) != FL_OK || (st = view_of(v, "v", p, true, FL_BF16, &p.v)) != FL_OK)
    return st;
  if (k_held != nullptr && (st = view_of(k_held, "k_held", p, true, FL_BF16, &p.k_held)) != FL_OK) return st;
  if (v_held != nullptr && (st = view_of(v_held, "v_held", p, true, FL_BF16, &p.v_held)) != FL_OK) return st;
  if (H + Hkv == 0) return FL_OK;
  const fl::View kc = make_view(k_cache), vc = make_view(v_cache);
  if (mx4) {
    p.mx4.k = (uint8_t*)k_cache->ptr;
    p.mx4.v = (uint8_t*)v_cache->ptr;
    p.mx4.k_sp = kc.sb; p.mx4.k_sh = kc.sh;
    p.mx4.v_sp = vc.sb; p.mx4.v_sh = vc.sh;
    p.mx4.page_size = kv->page_size;
  } else {
    p.k_cache = (uint16_t*)k_cache->ptr;
    p.v_cache = (uint16_t*)v_cache->ptr;
    p.kc_sp = kc.sb; p.kc_sh = kc.sh; p.kc_st = kc.ss;
    p.vc_sp = vc.sb; p.vc_sh = vc.sh; p.vc_st = vc.ss;
  }
  p.block_table = kv->block_table;
  p.table_stride = kv->table_stride;
  p.page_shift = page_shift;
  p.num_pages = (int)k_cache->size[0];
  p.seq_lens = kv->seq_lens;
  p.max_len = kv->max_seq_len;
  const RowShape r = shape_row(&p, FL_BF16);
  p.tokens_per_block = tokens_of(p, 256);
  const int64_t blocks = (B * T + p.tokens_per_block - 1) / p.tokens_per_block, rows = p.tokens_per_block * (H + 2 * Hkv), at_once = 256 >> p.log_lanes;
  // a column of workgroups shares its tokens' rows, down to one for each group of lanes, while that leaves a compute unit three workgroups at most (8 x 512 tokens,
  // 32 / 8 heads, D = 128, 16 tokens a column, inputs from memory, with 512 / 768 / 1024 workgroups: into 4 bits 28.7 / 26.2 / 28.8 us, into bf16 pages 23.6 / 22.9 / 23.0)
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((rows + at_once - 1) / at_once, (768 + blocks - 1) / blocks));
  p.rows_per_part = (int)((rows + parts - 1) / parts);
  const dim3 grid((unsigned)blocks, (unsigned)parts);
  const bool il = rotary->interleaved != 0, streams = r.wide && r.upl == 1 && p.pairs % 64 == 0 && (p.D - 2 * p.pairs) % 64 == 0;
  hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  if (mx4)                                         // (D is 64 or 128)
    e = !r.wide ? launch_append<1, 2, true>(p, il, grid, s) : (streams ? launch_append<8, 1, true, true, true>(p, il, grid, s) : p.pairs % 32 == 0 ? launch_append<8, 1, true, true>(p, il, grid, s) : launch_append<8, 1, true>(p, il, grid, s));
  else
    e = r.wide ? (streams ? launch_append<8, 1, false, false, true>(p, il, grid, s) : r.upl == 1 ? launch_append<8, 1, false>(p, il, grid, s) : launch_append<8, 4, false>(p, il, grid, s))
               : (r.upl == 2 ? launch_append<1, 2, false>(p, il, grid, s) : launch_append<1, 16, false>(p, il, grid, s));
  return e == hipSuccess ? FL_OK : fail(FL_ERR_LAUNCH, "append launch: %s", hipGetErrorString(e));
}

}  // extern "C"
