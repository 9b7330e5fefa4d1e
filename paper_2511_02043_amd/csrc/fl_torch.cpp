// Marshalling of the PyTorch entry points (attention and its backward pass, with and without the variants' extra tensors, a decode
// step, a chunk of a paged prefill, rotary positions, weights of cached keys, eviction): torch tensors in, C-ABI descriptors filled, outputs and workspace taken from torch's
// allocator, one call of libflattn.so, the fl_status and the outputs back.  No attention arithmetic and no kernel is here.
//
// The same in Python (ctypes structures filled field by field) cost 20 us of a 31 us causal call on [1, 8, 128, 64] and of
// a 31 us decode step of one sequence, whose kernels take 8 and 10 us; a training step with a bias and a gate on
// [1, 16, 4, 64, 32] took 252 us that way and 117 this way with autograd nodes in Python, most of it in the autograd engine.
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/extension.h>

#include <optional>
#include <tuple>

#include "../../include/fl_attn.h"

namespace py = pybind11;
using at::Tensor;
typedef std::optional<Tensor> OptTensor;

namespace {

int dtype_code(const Tensor& t) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return FL_BF16;
    case at::kFloat: return FL_F32;
    case at::kInt: return FL_I32;
    default: throw py::key_error(c10::toString(t.scalar_type()));
  }
}

// The 5-D descriptor of a tensor whose axes are `axes` (-1: an axis of size 1).
fl_tensor desc5(const Tensor& t, const int (&axes)[5]) {
  fl_tensor d = {};
  d.ptr = t.data_ptr();
  d.dtype = dtype_code(t);
  for (int a = 0; a < 5; ++a) {
    d.size[a] = axes[a] < 0 ? 1 : t.size(axes[a]);
    d.stride[a] = axes[a] < 0 ? 0 : t.stride(axes[a]);
  }
  return d;
}
// [B, H, S, D] or [B, G, H, S, D]
fl_tensor desc(const Tensor& t) {
  if (t.dim() == 5) return desc5(t, {0, 1, 2, 3, 4});
  if (t.dim() != 4) throw py::value_error("expected [B, H, S, D] or [B, G, H, S, D], got " + std::to_string(t.dim()) + " axes");
  return desc5(t, {0, -1, 1, 2, 3});
}

template <class T>
T* ptr(const OptTensor& t) {
  return t.has_value() ? (T*)t->data_ptr() : nullptr;
}

fl_variant_desc variant(double scale, int mod, double softcap, int mask, int window, int prefix, int q_offset) {
  fl_variant_desc d = {};
  d.struct_size = sizeof(d);
  d.scale = (float)scale;
  d.score_mod = (uint32_t)mod;
  d.softcap = (float)softcap;
  d.mask = (uint32_t)mask;
  d.window = window;
  d.prefix_len = prefix;
  d.q_offset = q_offset;
  return d;
}

fl_aux aux_of(const OptTensor& slopes, const OptTensor& q_ids, const OptTensor& kv_ids, const Tensor& workspace) {
  fl_aux a = {};
  a.struct_size = sizeof(a);
  a.alibi_slopes = ptr<const float>(slopes);
  a.q_doc_ids = ptr<const int32_t>(q_ids);
  a.kv_doc_ids = ptr<const int32_t>(kv_ids);
  if (workspace.defined()) {
    a.workspace = workspace.data_ptr();
    a.workspace_bytes = workspace.nbytes();
  }
  return a;
}

// An output gradient in a layout that the kernels read: unit inner stride, 16-byte aligned rows and base, no broadcast axis
// (autograd hands over a sum over an outer axis as one).
Tensor readable(const Tensor& t) {
  bool ok = t.stride(-1) == 1 && (uintptr_t)t.data_ptr() % 16 == 0;
  for (int64_t a = 0; a + 1 < t.dim(); ++a) ok = ok && (t.size(a) == 1 || (t.stride(a) != 0 && t.stride(a) % 8 == 0));
  return ok ? t : t.clone(at::MemoryFormat::Contiguous);
}

Tensor bytes(size_t n, const Tensor& like) { return at::empty({(int64_t)n}, like.options().dtype(at::kByte)); }

// out [B, (G,) H, Sq, Dv] in q's dtype and rank, lse [B, G, H, Sq, 1]
std::tuple<int, Tensor, Tensor> attention_fwd(const Tensor& q, const Tensor& k, const Tensor& v, double scale, int mod, double softcap,
                                              int mask, int window, int prefix, int q_offset, const OptTensor& slopes,
                                              const OptTensor& q_ids, const OptTensor& kv_ids, int64_t stream) {
  const fl_tensor tq = desc(q), tk = desc(k), tv = desc(v);
  const fl_variant_desc d = variant(scale, mod, softcap, mask, window, prefix, q_offset);
  std::vector<int64_t> size(q.sizes().begin(), q.sizes().end());
  size.back() = tv.size[4];
  Tensor out = at::empty(size, q.options());
  Tensor lse = at::empty({tq.size[0], tq.size[1], tq.size[2], tq.size[3], 1}, q.options().dtype(at::kFloat));
  fl_tensor tout = desc(out), tlse = desc(lse);
  Tensor ws;
  const size_t need = fl_attn_fwd_workspace_size(&tq, &tk, &d);
  if (need != 0) ws = bytes(need, q);
  const fl_aux a = aux_of(slopes, q_ids, kv_ids, ws);
  const int status = fl_attn_fwd(&tq, &tk, &tv, &d, &a, &tout, &tlse, (void*)stream);
  return {status, out, lse};
}

// dq, dk, dv in the layouts of q, k, v
std::tuple<int, Tensor, Tensor, Tensor> attention_bwd(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& out,
                                                      const Tensor& lse, const Tensor& dout_in, double scale, int mod, double softcap,
                                                      int mask, int window, int prefix, int q_offset, const OptTensor& slopes,
                                                      const OptTensor& q_ids, const OptTensor& kv_ids, int64_t stream) {
  const Tensor dout = readable(dout_in);
  const fl_tensor tq = desc(q), tk = desc(k), tv = desc(v), tout = desc(out), tlse = desc(lse), tdo = desc(dout);
  const fl_variant_desc d = variant(scale, mod, softcap, mask, window, prefix, q_offset);
  Tensor dq = at::empty_like(q), dk = at::empty_like(k), dv = at::empty_like(v);
  fl_tensor tdq = desc(dq), tdk = desc(dk), tdv = desc(dv);
  const Tensor ws = bytes(std::max<size_t>(fl_attn_bwd_workspace_size(&tq, &tk, &d), 16), q);
  const fl_aux a = aux_of(slopes, q_ids, kv_ids, ws);
  const int status = fl_attn_bwd(&tq, &tk, &tv, &tout, &tdo, &tlse, &d, &a, &tdq, &tdk, &tdv, (void*)stream);
  return {status, dq, dk, dv};
}

// The tensors of a variant beyond q, k and v (absent ones are None), as variant_fwd and variant_bwd take them.
struct Extras {
  const OptTensor &q2, &k2, &lam, &gate, &bias0, &bias1, &rms_weight;
  int n_bias() const { return (int)bias0.has_value() + (int)bias1.has_value(); }
  fl_variant_desc describe(fl_variant_desc d, bool rmsnorm, double rms_eps) const {
    d.n_bias = (uint32_t)n_bias();
    d.combine = q2.has_value() ? FL_DIFFERENTIAL : FL_SINGLE;
    d.epilogue = (rmsnorm ? FL_EPI_RMSNORM : 0) | (gate.has_value() ? FL_EPI_GATE_SIGMOID : 0);
    d.rms_eps = rmsnorm ? (float)rms_eps : 0.f;
    return d;
  }
  fl_aux fill(fl_aux a) const {
    int n = 0;
    for (const OptTensor* b : {&bias0, &bias1})
      if (b->has_value()) a.bias[n++] = desc(**b);
    if (gate.has_value()) a.gate = desc(*gate);
    if (q2.has_value()) a.q2 = desc(*q2);
    if (k2.has_value()) a.k2 = desc(*k2);
    a.lambda = ptr<const float>(lam);
    a.rms_weight = ptr<const float>(rms_weight);
    return a;
  }
};

// out in q's dtype and rank, lse [B, G or 2 G (two streams), H, Sq, 1]
std::tuple<int, Tensor, Tensor> variant_fwd(const Tensor& q, const Tensor& k, const Tensor& v, const OptTensor& q2, const OptTensor& k2,
                                            const OptTensor& lam, const OptTensor& gate, const OptTensor& bias0, const OptTensor& bias1,
                                            const OptTensor& rms_weight, double scale, int mod, double softcap, int mask, int window,
                                            int prefix, int q_offset, bool rmsnorm, double rms_eps, const OptTensor& slopes,
                                            const OptTensor& q_ids, const OptTensor& kv_ids, int64_t stream) {
  const Extras x{q2, k2, lam, gate, bias0, bias1, rms_weight};
  const fl_tensor tq = desc(q), tk = desc(k), tv = desc(v);
  const fl_variant_desc d = x.describe(variant(scale, mod, softcap, mask, window, prefix, q_offset), rmsnorm, rms_eps);
  std::vector<int64_t> size(q.sizes().begin(), q.sizes().end());
  size.back() = tv.size[4];
  Tensor out = at::empty(size, q.options());
  Tensor lse = at::empty({tq.size[0], (q2.has_value() ? 2 : 1) * tq.size[1], tq.size[2], tq.size[3], 1}, q.options().dtype(at::kFloat));
  fl_tensor tout = desc(out), tlse = desc(lse);
  Tensor ws;
  const size_t need = fl_attn_fwd_workspace_size(&tq, &tk, &d);
  if (need != 0) ws = bytes(need, q);
  const fl_aux a = x.fill(aux_of(slopes, q_ids, kv_ids, ws));
  const int status = fl_attn_fwd(&tq, &tk, &tv, &d, &a, &tout, &tlse, (void*)stream);
  return {status, out, lse};
}

// The status and the gradients of q, k, v, q2, k2, lam, gate, bias0, bias1, rms_weight in their layouts (None where absent).  The
// kernels sum bias gradients in fp32; they are rounded to the biases' dtype here.
std::tuple<int, std::vector<OptTensor>> variant_bwd(const Tensor& q, const Tensor& k, const Tensor& v, const OptTensor& q2,
                                                    const OptTensor& k2, const OptTensor& lam, const OptTensor& gate,
                                                    const OptTensor& bias0, const OptTensor& bias1, const OptTensor& rms_weight,
                                                    const Tensor& out, const Tensor& lse, const Tensor& dout_in, double scale, int mod,
                                                    double softcap, int mask, int window, int prefix, int q_offset, bool rmsnorm,
                                                    double rms_eps, const OptTensor& slopes, const OptTensor& q_ids,
                                                    const OptTensor& kv_ids, int64_t stream) {
  const Extras x{q2, k2, lam, gate, bias0, bias1, rms_weight};
  const Tensor dout = readable(dout_in);
  const fl_tensor tq = desc(q), tk = desc(k), tv = desc(v), tout = desc(out), tlse = desc(lse), tdo = desc(dout);
  const fl_variant_desc d = x.describe(variant(scale, mod, softcap, mask, window, prefix, q_offset), rmsnorm, rms_eps);
  auto like = [](const OptTensor& t) { return t.has_value() ? OptTensor(at::empty_like(*t)) : OptTensor(); };
  auto fp32 = [](const OptTensor& t) { return t.has_value() ? OptTensor(at::empty(t->sizes(), t->options().dtype(at::kFloat))) : OptTensor(); };
  Tensor dq = at::empty_like(q), dk = at::empty_like(k), dv = at::empty_like(v);
  const OptTensor dq2 = like(q2), dk2 = like(k2), dlam = like(lam), dgate = like(gate), drms = fp32(rms_weight);
  OptTensor dbias0 = fp32(bias0), dbias1 = fp32(bias1);
  fl_bwd_extra e = {};
  e.struct_size = sizeof(e);
  if (dq2.has_value()) e.dq2 = desc(*dq2);
  if (dk2.has_value()) e.dk2 = desc(*dk2);
  if (dgate.has_value()) e.dgate = desc(*dgate);
  int n = 0;
  for (const OptTensor* b : {&dbias0, &dbias1})
    if (b->has_value()) e.dbias[n++] = desc(**b);
  e.dlambda = ptr<float>(dlam);
  e.drms_weight = ptr<float>(drms);
  fl_tensor tdq = desc(dq), tdk = desc(dk), tdv = desc(dv);
  const Tensor ws = bytes(std::max<size_t>(fl_attn_bwd_ex_workspace_size(&tq, &tk, &tv, &d), 16), q);
  const fl_aux a = x.fill(aux_of(slopes, q_ids, kv_ids, ws));
  const int status = fl_attn_bwd_ex(&tq, &tk, &tv, &tout, &tdo, &tlse, &d, &a, &tdq, &tdk, &tdv, &e, (void*)stream);
  if (status == 0) {
    if (dbias0.has_value()) dbias0 = dbias0->to(bias0->scalar_type());
    if (dbias1.has_value()) dbias1 = dbias1->to(bias1->scalar_type());
  }
  return {status, {dq, dk, dv, dq2, dk2, dlam, dgate, dbias0, dbias1, drms}};
}

template <class... Parts>
void need(bool ok, const Parts&... parts) {
  if (!ok) throw py::value_error(c10::str(parts...));
}
// A caller's workspace is written through its address alone, nbytes() of it from there on: memory of the call's device without gaps or repeats.
void check_workspace(const OptTensor& workspace, const Tensor& q) {
  need(!workspace.has_value() || workspace->device() == q.device(), "workspace must be on ", q.device());
  need(!workspace.has_value() || workspace->is_non_overlapping_and_dense(), "workspace must be contiguous memory, got strides ",
       workspace.has_value() ? workspace->strides() : at::IntArrayRef());
}

// From row to row of a table; a single row's stride says nothing.
int32_t row_step(const Tensor& table) { return (int32_t)(table.size(0) > 1 ? table.stride(0) : table.size(1)); }

// A decode step (q [B, H, D]) or a chunk of a paged prefill (q [B, H, Sq, D]) over caches [pages, page_size, Hkv, D].  Returns
// the status, the workspace bytes the call needs, out (q's shape) and lse ([B, H] or [B, H, Sq]; undefined unless wanted).  A
// workspace that is too small is reported by the second value alone: nothing has been launched then.
std::tuple<int, int64_t, Tensor, OptTensor> paged(bool decode, const Tensor& q, const Tensor& k_cache, const Tensor& v_cache,
                                                  const Tensor& seq_lens, const OptTensor& table, int max_seq_len, double scale,
                                                  int mod, double softcap, int mask, int window, const OptTensor& slopes,
                                                  const OptTensor& workspace, bool want_lse, int64_t stream) {
  TORCH_CHECK(k_cache.dim() == 4 && v_cache.dim() == 4, "the caches must be [pages, page_size, Hkv, D]");
  check_workspace(workspace, q);
  const fl_tensor tq = decode ? desc5(q, {0, -1, 1, -1, 2}) : desc5(q, {0, -1, 1, 2, 3});
  const fl_tensor tk = desc5(k_cache, {0, -1, 2, 1, 3}), tv = desc5(v_cache, {0, -1, 2, 1, 3});
  Tensor out = at::empty(q.sizes(), q.options());
  fl_tensor tout = decode ? desc5(out, {0, -1, 1, -1, 2}) : desc5(out, {0, -1, 1, 2, 3});
  OptTensor lse;
  fl_tensor tlse = {};
  if (want_lse) {
    lse = at::empty(q.sizes().slice(0, q.dim() - 1), q.options().dtype(at::kFloat));
    tlse = decode ? desc5(*lse, {0, -1, 1, -1, -1}) : desc5(*lse, {0, -1, 1, 2, -1});
  }
  fl_paged_kv kv = {};
  kv.struct_size = sizeof(kv);
  kv.block_table = ptr<const int32_t>(table);
  kv.table_stride = table.has_value() ? row_step(*table) : 0;
  kv.page_size = (int32_t)k_cache.size(1);
  kv.seq_lens = (const int32_t*)seq_lens.data_ptr();
  kv.max_seq_len = max_seq_len;
  const size_t need = std::max<size_t>(
      decode ? fl_attn_decode_workspace_size(&tq, &tk, &kv) : fl_attn_prefill_paged_workspace_size(&tq, &tk, &kv), 16);
  if (workspace.has_value() && workspace->nbytes() < need) return {0, (int64_t)need, out, lse};
  const Tensor ws = workspace.has_value() ? *workspace : bytes(need, q);
  const fl_variant_desc d = variant(scale, mod, softcap, mask, window, 0, 0);
  const fl_aux a = aux_of(slopes, std::nullopt, std::nullopt, ws);
  const int status = (decode ? fl_attn_decode : fl_attn_prefill_paged)(&tq, &tk, &tv, &kv, &d, &a, &tout, want_lse ? &tlse : nullptr,
                                                                      (void*)stream);
  return {status, (int64_t)need, out, lse};
}

// ---- a bounded key/value cache: positions, weights of cached keys, eviction ----

// The checks of these calls' tensors are here too (one token of 64 sequences into the cache: 10.2 us a call with them in Python, 5.8 here).
// an array that the C ABI reads as raw memory of a fixed type and shape
void check_array(const char* name, const OptTensor& t, at::ScalarType dtype, at::IntArrayRef shape, at::Device device, bool contiguous, bool inner_unit) {
  need(t.has_value(), name, " must be a torch.Tensor");
  need(t->scalar_type() == dtype, name, " must be ", dtype, ", got ", t->scalar_type());
  need(t->device() == device, name, " is on ", t->device(), ", expected ", device);
  need(t->sizes() == shape, name, " must have shape ", shape, ", got ", t->sizes());
  need(!contiguous || t->is_contiguous(), name, " must be contiguous");
  need(!inner_unit || t->size(-1) <= 1 || t->stride(-1) == 1, name, " must have unit stride along its last axis");
}
typedef std::optional<std::vector<int64_t>> Sections;

// The positions as [B, S, axes] and the sections, for q [B, heads, (S,) D] and k, which may be missing
std::tuple<Tensor, std::vector<int64_t>> check_rotary(const Tensor& q, const OptTensor& k, const OptTensor& positions, const OptTensor& inv_freq,
                                                      const Sections& given, int64_t B, int64_t S) {
  need(positions.has_value() && positions->dim() == 3, "positions must be a tensor [B, S, axes]");
  const int64_t axes = positions->size(2);
  const Tensor p = positions->size(0) == 1 && B != 1 ? positions->expand({B, -1, -1}) : *positions;
  check_array("positions", p, at::kInt, {B, S, axes}, q.device(), false, false);
  need(inv_freq.has_value() && inv_freq->dim() == 1, "inv_freq must be a tensor [pairs]");
  const int64_t pairs = inv_freq->size(0);
  check_array("inv_freq", inv_freq, at::kFloat, {pairs}, q.device(), true, false);
  std::vector<int64_t> sections = given.has_value() ? *given : std::vector<int64_t>{pairs};
  need((int64_t)sections.size() == axes && axes >= 1 && axes <= 4, sections.size(), " sections for positions with ", axes, " axes (1 to 4 of both)");
  int64_t sum = 0;
  for (int64_t n : sections) {
    need(n >= 0 && n <= pairs, "sections must be >= 0 and add up to the ", pairs, " pairs of inv_freq");
    sum += n;
  }
  need(sum == pairs, "sections must be >= 0 and add up to the ", pairs, " pairs of inv_freq");
  if (k.has_value())
    need(k->device() == q.device() && k->scalar_type() == q.scalar_type() && k->dim() == q.dim() && k->size(0) == q.size(0) &&
             k->sizes().slice(2) == q.sizes().slice(2),
         "k ", k->sizes(), " ", k->scalar_type(), " does not go with q ", q.sizes(), " ", q.scalar_type());
  return {p, std::move(sections)};
}

// The host-side bound of the lengths, after the checks that every call over the paged cache makes; q: a tensor of B sequences
int64_t check_cache(const Tensor& q, const Tensor& k_cache, const OptTensor& v_cache, const OptTensor& seq_lens, const OptTensor& table,
                    std::optional<int64_t> max_seq_len) {
  for (const Tensor* c : {&k_cache, v_cache.has_value() ? &*v_cache : &k_cache})
    need(c->dim() == 4 && c->scalar_type() == at::kBFloat16 && c->device() == q.device(), "the caches must be bf16 tensors [pages, page_size, Hkv, D] on ",
         q.device());
  need(!v_cache.has_value() || v_cache->sizes() == k_cache.sizes(), "k_cache and v_cache must have one shape");
  const int64_t B = q.size(0);
  check_array("seq_lens", seq_lens, at::kInt, {B}, q.device(), true, false);
  if (table.has_value()) {
    need(table->dim() == 2, "block_table must be [B, max_pages]");
    check_array("block_table", table, at::kInt, {B, table->size(1)}, q.device(), false, true);
  }
  const int64_t held = (table.has_value() ? table->size(1) : 1) * k_cache.size(1), n = max_seq_len.value_or(held);
  need(n >= 0 && n <= INT32_MAX, "max_seq_len = ", n);
  need(!table.has_value() || n <= held, "max_seq_len = ", n, " is more than the ", table.has_value() ? table->size(1) : 1, " pages of block_table hold");
  return n;
}

void check_weights(const OptTensor& weights, const Tensor& q, const Tensor& k_cache) {
  need(weights.has_value() && weights->dim() == 3, "weights must be a tensor [B, Hkv, capacity]");
  check_array("weights", weights, at::kFloat, {q.size(0), k_cache.size(2), weights->size(2)}, q.device(), false, true);
}
void check_slopes(const OptTensor& slopes, const Tensor& q) {
  if (slopes.has_value()) check_array("alibi_slopes", slopes, at::kFloat, {q.size(1)}, q.device(), true, false);
}

fl_paged_kv paged_kv(const Tensor& cache, const Tensor& seq_lens, const OptTensor& table, int max_seq_len) {
  fl_paged_kv kv = {};
  kv.struct_size = sizeof(kv);
  kv.block_table = ptr<const int32_t>(table);
  kv.table_stride = table.has_value() ? row_step(*table) : 0;
  kv.page_size = (int32_t)cache.size(1);
  kv.seq_lens = (const int32_t*)seq_lens.data_ptr();
  kv.max_seq_len = max_seq_len;
  return kv;
}
// [B, heads, D] or [B, heads, T, D]
fl_tensor rows_desc(const Tensor& t) { return t.dim() == 3 ? desc5(t, {0, -1, 1, -1, 2}) : desc5(t, {0, -1, 1, 2, 3}); }
fl_tensor cache_desc(const Tensor& t) { return desc5(t, {0, -1, 2, 1, 3}); }

fl_rotary rotary_desc(const Tensor& positions, const Tensor& inv_freq, const std::vector<int64_t>& sections, bool interleaved, bool inverse) {
  fl_rotary r = {};
  r.struct_size = sizeof(r);
  r.axes = (uint32_t)sections.size();              // (more than four are refused by the call)
  for (size_t a = 0; a < sections.size() && a < 4; ++a) r.sections[a] = (int32_t)sections[a];
  r.interleaved = interleaved;
  r.inverse = inverse;
  r.positions = (const int32_t*)positions.data_ptr();
  for (int a = 0; a < 3; ++a) r.stride[a] = positions.size(a) > 1 ? positions.stride(a) : 0;
  r.inv_freq = (const float*)inv_freq.data_ptr();
  return r;
}

// q and k [B, heads, S, D], either may be missing; the outputs have their layouts
std::tuple<int, OptTensor, OptTensor> rotary(const OptTensor& q, const OptTensor& k, const Tensor& positions, const Tensor& inv_freq,
                                             const std::vector<int64_t>& sections, bool interleaved, bool inverse, int64_t stream) {
  const c10::DeviceGuard guard(positions.device());
  const fl_rotary r = rotary_desc(positions, inv_freq, sections, interleaved, inverse);
  OptTensor qo, ko;
  fl_tensor tq = {}, tk = {}, tqo = {}, tko = {};
  if (q.has_value()) {
    qo = at::empty_like(*q);
    tq = rows_desc(*q);
    tqo = rows_desc(*qo);
  }
  if (k.has_value()) {
    ko = at::empty_like(*k);
    tk = rows_desc(*k);
    tko = rows_desc(*ko);
  }
  const int status = fl_rotary_embed(q.has_value() ? &tq : nullptr, k.has_value() ? &tk : nullptr, &r, q.has_value() ? &tqo : nullptr,
                                     k.has_value() ? &tko : nullptr, (void*)stream);
  return {status, qo, ko};
}

// ... of a call, with its checks
std::tuple<int, OptTensor, OptTensor> rotary_checked(const Tensor& q, const OptTensor& k, const OptTensor& positions, const OptTensor& inv_freq,
                                                     const Sections& given, bool interleaved, int64_t stream) {
  const auto [p, sections] = check_rotary(q, k, positions, inv_freq, given, q.size(0), q.size(2));
  return rotary(q, k, p, *inv_freq, sections, interleaved, false, stream);
}

// q [B, H, (T,) D], k and v [B, Hkv, (T,) D]: the turned q, in a layout of its own; keys and values into the caches
std::tuple<int, Tensor> rotary_append(const Tensor& q, const Tensor& k, const Tensor& v, const OptTensor& positions, const OptTensor& inv_freq,
                                      const Sections& given, bool interleaved, const Tensor& k_cache, const Tensor& v_cache,
                                      const OptTensor& seq_lens, const OptTensor& table, std::optional<int64_t> bound, int64_t stream) {
  const c10::DeviceGuard guard(q.device());
  const auto [p, sections] = check_rotary(q, k, positions, inv_freq, given, q.size(0), q.dim() == 4 ? q.size(2) : 1);
  const int max_seq_len = (int)check_cache(q, k_cache, v_cache, seq_lens, table, bound);
  need(k.sizes() == v.sizes() && v.scalar_type() == q.scalar_type() && v.device() == q.device() && k.size(1) == k_cache.size(2), "k ", k.sizes(),
       " and v ", v.sizes(), " do not go with the cache ", k_cache.sizes());
  const fl_rotary r = rotary_desc(p, *inv_freq, sections, interleaved, false);
  Tensor qo = at::empty_like(q);
  const fl_tensor tq = rows_desc(q), tk = rows_desc(k), tv = rows_desc(v);
  fl_tensor tqo = rows_desc(qo), tkc = cache_desc(k_cache), tvc = cache_desc(v_cache);
  const fl_paged_kv kv = paged_kv(k_cache, *seq_lens, table, max_seq_len);
  const int status = fl_rotary_append(&tq, &tk, &tv, &r, &kv, &tqo, &tkc, &tvc, (void*)stream);
  return {status, qo};
}

// paged() for a decode step (q [B, H, D] or [B, H, T, D]) that adds up the keys' weights [B, Hkv, C]
std::tuple<int, int64_t, Tensor, OptTensor> decode_weights(const Tensor& q, const Tensor& k_cache, const Tensor& v_cache, const OptTensor& w,
                                                           const OptTensor& lens, const OptTensor& table, std::optional<int64_t> bound, double scale,
                                                           int mod, double softcap, int mask, int window, const OptTensor& slopes,
                                                           const OptTensor& workspace, bool want_lse, int64_t stream) {
  const c10::DeviceGuard guard(q.device());
  const int max_seq_len = (int)check_cache(q, k_cache, v_cache, lens, table, bound);
  check_weights(w, q, k_cache);
  check_slopes(slopes, q);
  check_workspace(workspace, q);
  const Tensor &weights = *w, &seq_lens = *lens;
  const fl_tensor tq = rows_desc(q), tk = cache_desc(k_cache), tv = cache_desc(v_cache);
  Tensor out = at::empty(q.sizes(), q.options());
  fl_tensor tout = rows_desc(out), tw = desc5(weights, {0, -1, 1, -1, 2}), tlse = {};
  OptTensor lse;
  if (want_lse) {
    lse = at::empty(q.sizes().slice(0, q.dim() - 1), q.options().dtype(at::kFloat));
    tlse = q.dim() == 3 ? desc5(*lse, {0, -1, 1, -1, -1}) : desc5(*lse, {0, -1, 1, 2, -1});
  }
  const fl_paged_kv kv = paged_kv(k_cache, seq_lens, table, max_seq_len);
  const size_t room = std::max<size_t>(fl_attn_decode_weights_workspace_size(&tq, &tk, &kv), 16);
  if (workspace.has_value() && workspace->nbytes() < room) return {0, (int64_t)room, out, lse};
  const Tensor ws = workspace.has_value() ? *workspace : bytes(room, q);
  const fl_variant_desc d = variant(scale, mod, softcap, mask, window, 0, 0);
  const fl_aux a = aux_of(slopes, std::nullopt, std::nullopt, ws);
  const int status = fl_attn_decode_weights(&tq, &tk, &tv, &kv, &d, &a, &tout, want_lse ? &tlse : nullptr, &tw, (void*)stream);
  return {status, (int64_t)room, out, lse};
}

// The weights that a chunk's rows (q [B, H, Sq, D], lse [B, H, Sq]) give to cached keys; status and the workspace bytes needed
std::tuple<int, int64_t> key_weights(const Tensor& q, const Tensor& k_cache, const OptTensor& lse, const OptTensor& w, const OptTensor& lens,
                                     const OptTensor& table, std::optional<int64_t> bound, double scale, int mod, double softcap, int mask,
                                     int window, const OptTensor& slopes, const OptTensor& workspace, int64_t stream) {
  const c10::DeviceGuard guard(q.device());
  const int max_seq_len = (int)check_cache(q, k_cache, std::nullopt, lens, table, bound);
  check_weights(w, q, k_cache);
  check_array("lse", lse, at::kFloat, {q.size(0), q.size(1), q.size(2)}, q.device(), false, false);
  check_slopes(slopes, q);
  check_workspace(workspace, q);
  const Tensor &weights = *w, &seq_lens = *lens;
  const fl_tensor tq = rows_desc(q), tk = cache_desc(k_cache), tlse = desc5(*lse, {0, -1, 1, 2, -1});
  fl_tensor tw = desc5(weights, {0, -1, 1, -1, 2});
  const fl_paged_kv kv = paged_kv(k_cache, seq_lens, table, max_seq_len);
  const size_t room = fl_key_weights_workspace_size(&tq, &tk, &kv);
  if (workspace.has_value() && workspace->nbytes() < room) return {0, (int64_t)room};
  Tensor ws;
  if (room != 0) ws = workspace.has_value() ? *workspace : bytes(room, q);
  const fl_variant_desc d = variant(scale, mod, softcap, mask, window, 0, 0);
  const fl_aux a = aux_of(slopes, std::nullopt, std::nullopt, ws);
  return {fl_key_weights(&tq, &tk, &tlse, &kv, &d, &a, &tw, (void*)stream), (int64_t)room};
}

// status, new lengths [B], weights [B, Hkv, capacity] and kept slots [B, Hkv, budget]
std::tuple<int, Tensor, Tensor, Tensor> evict(const Tensor& weights, const Tensor& k_cache, const Tensor& v_cache, const OptTensor& seq,
                                              const OptTensor& table, const OptTensor& dst, std::optional<int64_t> bound, int64_t budget, int sinks,
                                              int recent, std::optional<int64_t> room, int64_t stream) {
  const c10::DeviceGuard guard(weights.device());
  const int max_seq_len = (int)check_cache(weights, k_cache, v_cache, seq, table, bound);
  check_weights(weights, weights, k_cache);
  need(dst.has_value() && dst->dim() == 2, "dst_table must be [B, pages]");
  check_array("dst_table", dst, at::kInt, {weights.size(0), dst->size(1)}, weights.device(), false, true);
  need(budget >= 1 && budget <= INT32_MAX && dst->size(1) * k_cache.size(1) >= budget, "budget = ", budget, " with ", dst->size(1), " pages of ",
       k_cache.size(1), " tokens in dst_table");
  const int64_t capacity = room.value_or(budget);
  need(capacity >= budget, "capacity = ", capacity, " is less than budget = ", budget);
  const Tensor &seq_lens = *seq, &dst_table = *dst;
  const int64_t B = weights.size(0), Hkv = weights.size(1);
  Tensor lens = at::empty({B}, seq_lens.options()), new_weights = at::empty({B, Hkv, capacity}, weights.options()),
         kept = at::empty({B, Hkv, budget}, seq_lens.options());
  const fl_tensor tw = desc5(weights, {0, -1, 1, -1, 2});
  fl_tensor tk = cache_desc(k_cache), tv = cache_desc(v_cache), tn = desc5(new_weights, {0, -1, 1, -1, 2});
  const fl_paged_kv kv = paged_kv(k_cache, seq_lens, table, max_seq_len);
  fl_evict e = {};
  e.struct_size = sizeof(e);
  e.budget = (int32_t)budget;
  e.sinks = sinks;
  e.recent = recent;
  e.dst_table = (const int32_t*)dst_table.data_ptr();
  e.dst_stride = row_step(dst_table);
  e.new_lens = (int32_t*)lens.data_ptr();
  e.kept = (int32_t*)kept.data_ptr();
  return {fl_cache_evict(&tw, &tk, &tv, &kv, &e, &tn, (void*)stream), lens, new_weights, kept};
}

// ---- the autograd nodes of training calls.  A node written in Python is entered by the engine's thread under the interpreter's lock, which
// the calling thread has just given up.  A causal forward and backward call on [1, 8, 110, 128] took 45 or 89 us with one, by where the
// process runs, and takes 38 or 72 with these; documents and windows 3 x 32/8 x 182 61 or 97, and 49 or 84.  Calls under a transform, a
// trace, forward-mode derivatives or torch.compile keep the Python node (functional.py).

PyObject* g_check = nullptr;                       // binding.check: raises for a status

// The exception that binding.check raises for `status`, thrown on a thread without the interpreter's lock; the engine carries it to the caller.
[[noreturn]] void throw_status(int status) {
  py::gil_scoped_acquire gil;
  PyObject* r = PyObject_CallFunction(g_check, "i", status);
  if (r != nullptr) {                              // (not reached: it raises for every status but 0)
    Py_DECREF(r);
    PyErr_SetString(PyExc_RuntimeError, "backward pass failed");
  }
  python_error e;
  e.persist();
  throw e;
}

int64_t current_stream(const Tensor& t) { return (int64_t)c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

// The outputs of a forward pass, taken through Function::apply unseen, and what its backward pass needs beside tensors that autograd saves.
struct Done {
  const Tensor &out, &lse;
  const std::vector<double>& scalars;
  const OptTensor &slopes, &q_ids, &kv_ids;

  void keep(torch::autograd::AutogradContext* ctx) const {
    ctx->saved_data["scalars"] = scalars;
    if (slopes.has_value()) ctx->saved_data["slopes"] = *slopes;
    if (q_ids.has_value()) ctx->saved_data["q_ids"] = *q_ids;
    if (kv_ids.has_value()) ctx->saved_data["kv_ids"] = *kv_ids;
  }
};
OptTensor kept(torch::autograd::AutogradContext* ctx, const char* name) {
  const auto it = ctx->saved_data.find(name);
  return it == ctx->saved_data.end() ? OptTensor() : OptTensor(it->second.toTensor());
}
// (slopes are an input without a gradient: a call that only they would need a derivative of has a node all the same)
struct AttentionNode : torch::autograd::Function<AttentionNode> {
  static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v, const OptTensor&, const Done& done) {
    ctx->save_for_backward({q, k, v, done.out, done.lse});
    done.keep(ctx);
    return done.out;
  }
  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, const torch::autograd::variable_list& grads) {
    const auto t = ctx->get_saved_variables();
    const auto s = ctx->saved_data["scalars"].toDoubleVector();
    auto [status, dq, dk, dv] = attention_bwd(t[0], t[1], t[2], t[3], t[4], grads[0], s[0], (int)s[1], s[2], (int)s[3], (int)s[4], (int)s[5],
                                              (int)s[6], kept(ctx, "slopes"), kept(ctx, "q_ids"), kept(ctx, "kv_ids"), current_stream(t[0]));
    if (status != 0) throw_status(status);
    return {dq, dk, dv, Tensor(), Tensor()};
  }
};

// attention_fwd with a node: the status and out
std::tuple<int, Tensor> attention_node(const Tensor& q, const Tensor& k, const Tensor& v, double scale, int mod, double softcap, int mask,
                                       int window, int prefix, int q_offset, const OptTensor& slopes, const OptTensor& q_ids,
                                       const OptTensor& kv_ids, int64_t stream) {
  auto [status, out, lse] = attention_fwd(q, k, v, scale, mod, softcap, mask, window, prefix, q_offset, slopes, q_ids, kv_ids, stream);
  if (status != 0) return {status, out};
  const std::vector<double> scalars = {scale, (double)mod, softcap, (double)mask, (double)window, (double)prefix, (double)q_offset};
  return {0, AttentionNode::apply(q, k, v, slopes, Done{out, lse, scalars, slopes, q_ids, kv_ids})};
}

struct VariantNode : torch::autograd::Function<VariantNode> {
  static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v, const OptTensor& q2,
                        const OptTensor& k2, const OptTensor& lam, const OptTensor& gate, const OptTensor& bias0, const OptTensor& bias1,
                        const OptTensor& rms_weight, const Done& done) {
    torch::autograd::variable_list saved = {q, k, v};
    for (const OptTensor* x : {&q2, &k2, &lam, &gate, &bias0, &bias1, &rms_weight}) saved.push_back(x->has_value() ? **x : Tensor());
    saved.push_back(done.out);
    saved.push_back(done.lse);
    ctx->save_for_backward(std::move(saved));
    done.keep(ctx);
    return done.out;
  }
  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, const torch::autograd::variable_list& grads) {
    const auto t = ctx->get_saved_variables();
    const auto s = ctx->saved_data["scalars"].toDoubleVector();
    auto opt = [](const Tensor& x) { return x.defined() ? OptTensor(x) : OptTensor(); };
    auto [status, g] = variant_bwd(t[0], t[1], t[2], opt(t[3]), opt(t[4]), opt(t[5]), opt(t[6]), opt(t[7]), opt(t[8]), opt(t[9]), t[10], t[11],
                                   grads[0], s[0], (int)s[1], s[2], (int)s[3], (int)s[4], (int)s[5], (int)s[6], s[7] != 0, s[8], kept(ctx, "slopes"),
                                   kept(ctx, "q_ids"), kept(ctx, "kv_ids"), current_stream(t[0]));
    if (status != 0) throw_status(status);
    torch::autograd::variable_list out;
    for (const OptTensor& x : g) out.push_back(x.has_value() ? *x : Tensor());
    out.emplace_back();                            // the forward pass's results
    return out;
  }
};

// variant_fwd with a node: the status and out
std::tuple<int, Tensor> variant_node(const Tensor& q, const Tensor& k, const Tensor& v, const OptTensor& q2, const OptTensor& k2, const OptTensor& lam,
                                     const OptTensor& gate, const OptTensor& bias0, const OptTensor& bias1, const OptTensor& rms_weight,
                                     double scale, int mod, double softcap, int mask, int window, int prefix, int q_offset, bool rmsnorm,
                                     double rms_eps, const OptTensor& slopes, const OptTensor& q_ids, const OptTensor& kv_ids, int64_t stream) {
  auto [status, out, lse] = variant_fwd(q, k, v, q2, k2, lam, gate, bias0, bias1, rms_weight, scale, mod, softcap, mask, window, prefix, q_offset,
                                        rmsnorm, rms_eps, slopes, q_ids, kv_ids, stream);
  if (status != 0) return {status, out};
  const std::vector<double> scalars = {scale,          (double)mod,      softcap, (double)mask, (double)window,
                                       (double)prefix, (double)q_offset, rmsnorm ? 1.0 : 0.0, rms_eps};
  return {0, VariantNode::apply(q, k, v, q2, k2, lam, gate, bias0, bias1, rms_weight, Done{out, lse, scalars, slopes, q_ids, kv_ids})};
}

// The outputs of rotary(), taken through Function::apply unseen.
struct Turned {
  const OptTensor &q, &k;
};
// Autograd keeps no tensors made in inference mode, which have no version to compare: a copy of one.
Tensor savable(const Tensor& t) { return t.is_inference() ? t.clone() : t; }
// The turn by -t of what arrives; itself differentiable, the map being linear.
struct RotaryNode : torch::autograd::Function<RotaryNode> {
  static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const OptTensor& q, const OptTensor&, const Tensor& positions,
                                                const Tensor& inv_freq, const std::vector<int64_t>& sections, bool interleaved, bool inverse,
                                                const Turned& turned) {
    ctx->set_materialize_grads(false);
    ctx->save_for_backward({savable(positions), savable(inv_freq)});           // (changed in place before the backward pass: torch raises there)
    ctx->saved_data["sections"] = sections;
    ctx->saved_data["how"] = std::vector<int64_t>{q.has_value(), interleaved, inverse};
    torch::autograd::variable_list out;
    if (turned.q.has_value()) out.push_back(*turned.q);
    if (turned.k.has_value()) out.push_back(*turned.k);
    return out;
  }
  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, const torch::autograd::variable_list& grads) {
    const auto how = ctx->saved_data["how"].toIntVector();
    const auto sections = ctx->saved_data["sections"].toIntVector();
    const auto saved = ctx->get_saved_variables();
    const Tensor &positions = saved[0], &inv_freq = saved[1];
    const int first = how[0] != 0 ? 0 : 1;
    OptTensor g[2];                                // of q and k, where one has arrived and is wanted
    for (size_t n = 0; n < grads.size(); ++n)
      if (grads[n].defined() && ctx->needs_input_grad(n)) g[first + n] = readable(grads[n]);
    torch::autograd::variable_list out(8);
    if (!g[0].has_value() && !g[1].has_value()) return out;
    const bool inverse = how[2] == 0;
    auto [status, q, k] = rotary(g[0], g[1], positions, inv_freq, sections, how[1] != 0, inverse, current_stream(positions));
    if (status != 0) throw_status(status);
    if (at::GradMode::is_enabled()) {
      const auto t = apply(g[0], g[1], positions, inv_freq, sections, how[1] != 0, inverse, Turned{q, k});
      if (q.has_value()) q = t[0];
      if (k.has_value()) k = t.back();
    }
    if (q.has_value()) out[0] = *q;
    if (k.has_value()) out[1] = *k;
    return out;
  }
};

// rotary_checked with a node
std::tuple<int, OptTensor, OptTensor> rotary_node(const Tensor& q, const OptTensor& k, const OptTensor& positions, const OptTensor& inv_freq,
                                                  const Sections& given, bool interleaved, int64_t stream) {
  const auto [p, sections] = check_rotary(q, k, positions, inv_freq, given, q.size(0), q.size(2));
  auto [status, qo, ko] = rotary(q, k, p, *inv_freq, sections, interleaved, false, stream);
  if (status != 0) return {status, qo, ko};
  const auto t = RotaryNode::apply(OptTensor(q), k, p, *inv_freq, sections, interleaved, false, Turned{qo, ko});
  if (qo.has_value()) qo = t[0];
  if (ko.has_value()) ko = t.back();
  return {0, qo, ko};
}

}  // namespace

PYBIND11_MODULE(_fltorch, m) {
  typedef py::call_guard<py::gil_scoped_release> nogil;
  m.def("attention_fwd", &attention_fwd, nogil());
  m.def("attention_bwd", &attention_bwd, nogil());
  m.def("attention_node", &attention_node, nogil());
  m.def("variant_fwd", &variant_fwd, nogil());
  m.def("variant_bwd", &variant_bwd, nogil());
  m.def("variant_node", &variant_node, nogil());
  m.def("paged", &paged, nogil());
  m.def("check_rotary", &check_rotary);
  m.def("check_cache", &check_cache);
  m.def("rotary", &rotary, nogil());
  m.def("rotary_checked", &rotary_checked, nogil());
  m.def("rotary_node", &rotary_node, nogil());
  m.def("rotary_append", &rotary_append, nogil());
  m.def("decode_weights", &decode_weights, nogil());
  m.def("key_weights", &key_weights, nogil());
  m.def("evict", &evict, nogil());
  m.def("set_check", [](py::object check) {
    Py_XDECREF(g_check);
    g_check = check.release().ptr();
  });
}
