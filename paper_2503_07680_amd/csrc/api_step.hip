// C ABI of the operators around a pack's attention and loss: argument validation on the host, then kernel launches on the
// caller's stream.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "common.hpp"
#include "cross_rules.hpp"
#include "rows.hpp"

namespace {

constexpr int32_t kMaxDim = 1 << 24, kMaxTokens = 1 << 24;

int type_bytes(int32_t type) { return type == HBP_BF16 ? 2 : type == HBP_F32 ? 4 : 0; }
bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

hbp_status check_embed(const hbp_embed_desc* d, hbp::EmbedParams* p) {
  if (!d) return HBP_ERR_INVALID_ARG;
  if (d->total_tokens < 0 || d->vocab < 1 || d->dim < 1 || !std::isfinite(d->scale)) return HBP_ERR_INVALID_ARG;
  if (!type_bytes(d->table_type) || !type_bytes(d->row_type)) return HBP_ERR_INVALID_ARG;
  if (d->dim > kMaxDim || d->total_tokens > kMaxTokens || d->vocab == INT32_MAX) return HBP_ERR_UNSUPPORTED;
  p->T = d->total_tokens;
  p->V = d->vocab;
  p->dim = d->dim;
  p->table_st = d->table_stride ? d->table_stride : d->dim;
  p->row_st = d->row_stride ? d->row_stride : d->dim;
  p->scale = d->scale;
  if (p->table_st < d->dim || p->row_st < d->dim) return HBP_ERR_SHAPE;
  return HBP_OK;
}

// The tensors that have elements, in the batches of the launches; false: bad arguments.
hbp_status grad_batches(const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, int32_t n,
                        std::vector<hbp::GradBatch>& batches) {
  if (n < 0 || (n > 0 && (!in || !sizes || !types))) return HBP_ERR_INVALID_ARG;
  int64_t all = 0;
  for (int32_t i = 0; i < n; ++i) all += sizes[i] > 0 && sizes[i] <= ((int64_t)1 << 40) ? sizes[i] : 0;
  // few elements: smaller chunks, or most of the chip is idle (0.8 million elements in 24 tensors: 60 workgroups, or 200)
  const int chunk_log2 = all <= ((int64_t)1 << 23) ? hbp::kGradSmallChunkLog2 : hbp::kGradChunkLog2;
  for (int32_t i = 0; i < n; ++i) {
    if (sizes[i] < 0 || !type_bytes(types[i])) return HBP_ERR_INVALID_ARG;
    if (sizes[i] == 0) continue;
    if (sizes[i] > ((int64_t)1 << 40)) return HBP_ERR_UNSUPPORTED;
    const int es = type_bytes(types[i]);
    if (!in[i] || !aligned_to(in[i], es) || (out && (!out[i] || !aligned_to(out[i], es)))) return HBP_ERR_INVALID_ARG;
    const uint64_t chunks = ((uint64_t)(sizes[i] - 1) >> chunk_log2) + 1;
    if (batches.empty() || batches.back().n == hbp::kGradBatch || batches.back().first_chunk[batches.back().n] + chunks > INT32_MAX) {
      batches.emplace_back();
      batches.back().n = 0;
      batches.back().first_chunk[0] = 0;
      batches.back().chunk_log2 = chunk_log2;
    }
    hbp::GradBatch& b = batches.back();
    b.in[b.n] = in[i];
    b.out[b.n] = out ? out[i] : const_cast<void*>(in[i]);
    b.size[b.n] = sizes[i];
    b.type[b.n] = (uint8_t)types[i];
    b.first_chunk[b.n + 1] = b.first_chunk[b.n] + (uint32_t)chunks;
    ++b.n;
  }
  return HBP_OK;
}
int groups_of(const hbp::GradBatch& b) { return (int)std::min<uint32_t>(b.first_chunk[b.n], hbp::kGradMaxGroups); }

// Whether what is written overlaps anything else that is written, or anything read but the same tensor at the same place.
bool overlaps(const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, int32_t n) {
  struct Range {
    uintptr_t from, to;
    int32_t i;
    bool written;
  };
  std::vector<Range> r;
  r.reserve(2 * (size_t)n);
  for (int32_t i = 0; i < n; ++i) {
    if (sizes[i] == 0) continue;
    const uintptr_t bytes = (uintptr_t)sizes[i] * type_bytes(types[i]), a = (uintptr_t)in[i], b = out ? (uintptr_t)out[i] : a;
    r.push_back({b, b + bytes, i, true});
    if (a != b) r.push_back({a, a + bytes, i, false});
  }
  std::sort(r.begin(), r.end(), [](const Range& x, const Range& y) { return x.from < y.from; });
  // two ranges that overlap, one of them written
  uintptr_t end_written = 0, end_any = 0;
  for (const Range& x : r) {
    if (x.from < end_written || (x.written && x.from < end_any)) return true;
    end_any = std::max(end_any, x.to);
    if (x.written) end_written = std::max(end_written, x.to);
  }
  return false;
}

constexpr int64_t kMaxRows = INT32_MAX - 4096;  // rounding up to whole tiles and parts stays in 32 bits
constexpr int64_t kMaxTokenStride = int64_t{1} << 22;  // elements: rows of a tile are addressed in 32 bits, as in hbp_varlen_attn_*

hbp_status check_cross(const hbp_cross_desc* d) {
  if (!d) return HBP_ERR_INVALID_ARG;
  if (d->total_queries < 0 || d->total_keys < 0 || d->n_samples < 0 || d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->d_qk <= 0 || d->d_v <= 0)
    return HBP_ERR_INVALID_ARG;
  if (!std::isfinite(d->softmax_scale) || d->longest_keys < 0 || d->longest_queries < 0 || d->pairs < 0) return HBP_ERR_INVALID_ARG;
  if (d->n_q_heads % d->n_kv_heads) return HBP_ERR_SHAPE;
  if (!((d->d_qk == 64 && d->d_v == 64) || (d->d_qk == 128 && d->d_v == 128) || (d->d_qk == 192 && d->d_v == 128))) return HBP_ERR_UNSUPPORTED;
  const hbp::CrossStrides s = hbp::cross_strides(*d);
  const int64_t t[4] = {s.q_t, s.k_t, s.v_t, s.o_t}, h[4] = {s.q_h, s.k_h, s.v_h, s.o_h}, dim[4] = {d->d_qk, d->d_qk, d->d_v, d->d_v};
  for (int i = 0; i < 4; ++i)
    if (t[i] % 8 || h[i] % 8 || t[i] < dim[i] || h[i] < dim[i] || t[i] > kMaxTokenStride) return HBP_ERR_SHAPE;
  // the kernels count folded rows, and steps over them, in 32 bits
  if (((int64_t)d->total_queries << hbp::cross_fold_log2(*d)) > kMaxRows || d->total_keys > kMaxRows ||
      (int64_t)d->total_queries * d->n_q_heads > ((int64_t)1 << 36))
    return HBP_ERR_UNSUPPORTED;
  return HBP_OK;
}
float scale_of(const hbp_cross_desc* d) { return d->softmax_scale > 0.f ? d->softmax_scale : 1.0f / std::sqrt((float)d->d_qk); }
bool aligned16(const void* p) { return aligned_to(p, 16); }
constexpr float kLog2e = 1.4426950408889634f;

}  // namespace

extern "C" hbp_status hbp_cross_tile_rows(const hbp_cross_desc* desc, int32_t which, int32_t* rows_out) {
  if (!rows_out || (which != HBP_FWD && which != HBP_BWD)) return HBP_ERR_INVALID_ARG;
  const hbp_status st = check_cross(desc);
  if (st != HBP_OK) return st;
  *rows_out = which == HBP_BWD ? hbp::kCrossKeys : hbp::kCrossRows >> hbp::cross_fold_log2(*desc);
  return HBP_OK;
}

extern "C" hbp_status hbp_cross_workspace_bytes(const hbp_cross_desc* desc, int32_t which, size_t* bytes_out) {
  if (!bytes_out || (which != HBP_FWD && which != HBP_BWD)) return HBP_ERR_INVALID_ARG;
  const hbp_status st = check_cross(desc);
  if (st != HBP_OK) return st;
  *bytes_out = which == HBP_FWD ? hbp::cross_fwd_layout(*desc).total : hbp::cross_bwd_layout(*desc).total;
  return HBP_OK;
}

extern "C" hbp_status hbp_cross_attn_fwd(const hbp_cross_desc* desc, const void* q, const void* k, const void* v, const int32_t* cu_q,
                                         const int32_t* cu_kv, const hbp_tile* q_tiles, int32_t n_q_tiles, void* o, float* lse,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  const hbp_status st = check_cross(desc);
  if (st != HBP_OK) return st;
  if (n_q_tiles < 0) return HBP_ERR_INVALID_ARG;
  const hbp::CrossFwdLayout lay = hbp::cross_fwd_layout(*desc);
  if (lay.total > 0 && (!workspace || !aligned_to(workspace, 256) || workspace_bytes < lay.total)) return HBP_ERR_WORKSPACE;
  if (desc->total_queries == 0 || n_q_tiles == 0) return HBP_OK;
  if (!q || !o || !lse || !cu_q || !cu_kv || !q_tiles || (desc->total_keys > 0 && (!k || !v))) return HBP_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return HBP_ERR_INVALID_ARG;
  const hbp::CrossStrides s = hbp::cross_strides(*desc);
  hbp::FwdParams p;
  std::memset(&p, 0, sizeof(p));
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.cu = cu_q;
  p.cu_kv = cu_kv;
  p.tiles = q_tiles;
  p.n_tiles = n_q_tiles;
  p.n_samples = desc->n_samples;
  p.T = desc->total_queries;
  p.Tk = desc->total_keys;
  p.Hq = desc->n_q_heads;
  p.Hkv = desc->n_kv_heads;
  p.fold_log2 = hbp::cross_fold_log2(*desc);
  p.g = (desc->n_q_heads / desc->n_kv_heads) >> p.fold_log2;
  p.q_st = s.q_t; p.q_sh = s.q_h; p.k_st = s.k_t; p.k_sh = s.k_h;
  p.v_st = s.v_t; p.v_sh = s.v_h; p.o_st = s.o_t; p.o_sh = s.o_h;
  p.scale_log2 = scale_of(desc) * kLog2e;
  p.parts = lay.parts;
  p.part_keys = lay.part_keys;
  p.o_part = reinterpret_cast<float*>(static_cast<char*>(workspace) + lay.o_off);
  p.ml_part = reinterpret_cast<float*>(static_cast<char*>(workspace) + lay.ml_off);
  return hbp::launch_cross_fwd(desc->d_qk, desc->d_v, p, static_cast<hipStream_t>(stream)) ? HBP_ERR_DEVICE : HBP_OK;
}

extern "C" hbp_status hbp_cross_attn_bwd(const hbp_cross_desc* desc, const void* q, const void* k, const void* v, const void* o,
                                         const float* lse, const void* d_o, const int32_t* cu_q, const int32_t* cu_kv,
                                         const hbp_tile* q_tiles, int32_t n_q_tiles, const hbp_tile* kv_tiles, int32_t n_kv_tiles,
                                         void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes, void* stream) {
  const hbp_status st = check_cross(desc);
  if (st != HBP_OK) return st;
  if (n_q_tiles < 0 || n_kv_tiles < 0) return HBP_ERR_INVALID_ARG;
  const hbp::CrossBwdLayout lay = hbp::cross_bwd_layout(*desc);
  if (lay.total > 0 && (!workspace || !aligned_to(workspace, 256) || workspace_bytes < lay.total)) return HBP_ERR_WORKSPACE;
  const bool queries = desc->total_queries > 0, keys = desc->total_keys > 0;
  if (!queries) n_q_tiles = 0;
  if (!keys) n_kv_tiles = 0;
  if (n_q_tiles == 0 && n_kv_tiles == 0) return HBP_OK;
  if (!cu_q || !cu_kv || (n_q_tiles > 0 && !q_tiles) || (n_kv_tiles > 0 && !kv_tiles)) return HBP_ERR_INVALID_ARG;
  if ((queries && (!q || !o || !lse || !d_o || !dq)) || (keys && (!k || !v || !dk || !dv))) return HBP_ERR_INVALID_ARG;
  for (const void* x : {q, k, v, o, d_o, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!aligned16(x)) return HBP_ERR_INVALID_ARG;
  const hbp::CrossStrides s = hbp::cross_strides(*desc);
  char* const ws = static_cast<char*>(workspace);
  hbp::BwdParams p;
  std::memset(&p, 0, sizeof(p));
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.o = static_cast<const uint16_t*>(o);
  p.d_o = static_cast<const uint16_t*>(d_o);
  p.lse = lse;
  p.dq = static_cast<uint16_t*>(dq);
  p.dk = static_cast<uint16_t*>(dk);
  p.dv = static_cast<uint16_t*>(dv);
  p.D = reinterpret_cast<float*>(ws + lay.d_off);
  p.lse2 = reinterpret_cast<float*>(ws + lay.lse2_off);
  p.cu = cu_q;
  p.cu_kv = cu_kv;
  p.tiles = kv_tiles;
  p.n_tiles = n_kv_tiles;
  p.q_tiles = q_tiles;
  p.n_q_tiles = n_q_tiles;
  p.n_samples = desc->n_samples;
  p.T = desc->total_queries;
  p.Tk = desc->total_keys;
  p.Hq = desc->n_q_heads;
  p.Hkv = desc->n_kv_heads;
  p.fold_log2 = hbp::cross_fold_log2(*desc);
  p.g = (desc->n_q_heads / desc->n_kv_heads) >> p.fold_log2;
  p.q_st = s.q_t; p.q_sh = s.q_h; p.k_st = s.k_t; p.k_sh = s.k_h;
  p.v_st = s.v_t; p.v_sh = s.v_h; p.o_st = s.o_t; p.o_sh = s.o_h;
  p.scale = scale_of(desc);
  p.scale_log2 = p.scale * kLog2e;
  p.n_split = lay.parts;
  p.n_split_dq = 1;
  p.dk_part = reinterpret_cast<float*>(ws + lay.dk_part_off);
  p.dv_part = reinterpret_cast<float*>(ws + lay.dv_part_off);
  p.part_steps = lay.part_steps;
  p.dq_part_keys = lay.dq_part_keys;
  p.dq_parts = lay.dq_parts;
  p.dq_first = lay.dq_first;
  p.dq_part = reinterpret_cast<float*>(ws + lay.dq_part_off);
  return hbp::launch_cross_bwd(desc->d_qk, desc->d_v, p, static_cast<hipStream_t>(stream)) ? HBP_ERR_DEVICE : HBP_OK;
}

extern "C" hbp_status hbp_embed_fwd(const hbp_embed_desc* desc, const void* table, const int32_t* tokens, void* rows, void* stream) {
  hbp::EmbedParams p;
  const hbp_status st = check_embed(desc, &p);
  if (st != HBP_OK) return st;
  if (p.T == 0) return HBP_OK;
  if (!table || !tokens || !rows) return HBP_ERR_INVALID_ARG;
  if (!aligned_to(table, type_bytes(desc->table_type)) || !aligned_to(rows, type_bytes(desc->row_type)) || !aligned_to(tokens, 4))
    return HBP_ERR_INVALID_ARG;
  p.tokens = tokens;
  return hbp::launch_embed_fwd(p, desc->table_type, desc->row_type, table, rows, static_cast<hipStream_t>(stream)) ? HBP_ERR_DEVICE : HBP_OK;
}

extern "C" hbp_status hbp_embed_bwd_workspace_bytes(const hbp_embed_desc* desc, size_t* bytes_out) {
  if (!bytes_out) return HBP_ERR_INVALID_ARG;
  hbp::EmbedParams p;
  const hbp_status st = check_embed(desc, &p);
  if (st != HBP_OK) return st;
  *bytes_out = hbp::embed_bwd_layout(p.T, p.V, p.dim).total;
  return HBP_OK;
}

extern "C" hbp_status hbp_embed_bwd(const hbp_embed_desc* desc, const void* d_rows, const int32_t* tokens, int32_t accumulate,
                                    void* d_table, void* workspace, size_t workspace_bytes, void* stream) {
  hbp::EmbedParams p;
  const hbp_status st = check_embed(desc, &p);
  if (st != HBP_OK) return st;
  if (accumulate != 0 && accumulate != 1) return HBP_ERR_INVALID_ARG;
  if (p.T > 0 && (!workspace || !aligned_to(workspace, 256) || workspace_bytes < hbp::embed_bwd_layout(p.T, p.V, p.dim).total))
    return HBP_ERR_WORKSPACE;
  if (p.T == 0 && accumulate) return HBP_OK;
  if (!d_table || (p.T > 0 && (!d_rows || !tokens))) return HBP_ERR_INVALID_ARG;
  if (!aligned_to(d_table, type_bytes(desc->table_type)) || !aligned_to(d_rows, type_bytes(desc->row_type)) || !aligned_to(tokens, 4))
    return HBP_ERR_INVALID_ARG;
  p.tokens = tokens;
  return hbp::launch_embed_bwd(p, desc->table_type, desc->row_type, d_rows, d_table, accumulate != 0, static_cast<char*>(workspace),
                               static_cast<hipStream_t>(stream))
             ? HBP_ERR_DEVICE
             : HBP_OK;
}

extern "C" hbp_status hbp_grad_workspace_bytes(int32_t n_tensors, size_t* bytes_out) {
  if (!bytes_out || n_tensors < 0) return HBP_ERR_INVALID_ARG;
  // a batch ends at kGradBatch tensors, or where its chunks fill 31 bits: at most one more a tensor of 2^40 elements
  *bytes_out = ((size_t)n_tensors / hbp::kGradBatch + 1) * hbp::kGradMaxGroups * sizeof(double);
  return HBP_OK;
}

extern "C" hbp_status hbp_grad_sumsq(const void* const* tensors, const int64_t* sizes, const int32_t* types, int32_t n_tensors,
                                     int32_t accumulate, double* sumsq, void* workspace, size_t workspace_bytes, void* stream) {
  try {
    if (n_tensors < 0 || !sumsq || !aligned_to(sumsq, 8) || (accumulate != 0 && accumulate != 1)) return HBP_ERR_INVALID_ARG;
    std::vector<hbp::GradBatch> batches;
    const hbp_status st = grad_batches(tensors, nullptr, sizes, types, n_tensors, batches);
    if (st != HBP_OK) return st;
    size_t partials = 0;
    for (const auto& b : batches) partials += groups_of(b);
    if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < partials * sizeof(double)) return HBP_ERR_WORKSPACE;
    double* partial = static_cast<double*>(workspace);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    int at = 0;
    for (const auto& b : batches) {
      if (hbp::launch_grad_sumsq(b, groups_of(b), partial + at, s) != 0) return HBP_ERR_DEVICE;
      at += groups_of(b);
    }
    return hbp::launch_grad_total(partial, at, sumsq, accumulate != 0, s) ? HBP_ERR_DEVICE : HBP_OK;
  } catch (const std::bad_alloc&) {
    return HBP_ERR_NO_MEMORY;
  } catch (...) {
    return HBP_ERR_INVALID_ARG;
  }
}

namespace {
// The clipping, the sum of squares given as in GradNorm.  Later batches first: their elements have been read last.
hbp_status clip(const void* const* tensors, void* const* outs, const int64_t* sizes, const int32_t* types, int32_t n_tensors,
                std::vector<hbp::GradBatch>& batches, hbp::GradNorm norm, hipStream_t s) {
  if (overlaps(tensors, outs, sizes, types, n_tensors)) return HBP_ERR_INVALID_ARG;
  if (batches.empty()) {  // the norm is wanted all the same
    batches.emplace_back();
    batches.back().n = 0;
    batches.back().first_chunk[0] = 0;
    batches.back().chunk_log2 = hbp::kGradSmallChunkLog2;
  }
  bool in_place = true;
  for (const auto& b : batches)
    for (int i = 0; i < b.n; ++i) in_place = in_place && b.in[i] == b.out[i];
  for (size_t i = batches.size(); i-- > 0;) {
    if (hbp::launch_grad_clip(batches[i], std::max(1, groups_of(batches[i])), norm, in_place, s) != 0) return HBP_ERR_DEVICE;
    norm.norm_out = nullptr;
    norm.sumsq_out = nullptr;
  }
  return HBP_OK;
}
}  // namespace

extern "C" hbp_status hbp_grad_clip(const void* const* tensors, void* const* outs_or_null, const int64_t* sizes, const int32_t* types,
                                    int32_t n_tensors, const double* sumsq, float max_norm, float* norm_out_or_null, void* stream) {
  try {
    if (n_tensors < 0 || !sumsq || !aligned_to(sumsq, 8) || !(max_norm >= 0.f)) return HBP_ERR_INVALID_ARG;
    std::vector<hbp::GradBatch> batches;
    const hbp_status st = grad_batches(tensors, outs_or_null, sizes, types, n_tensors, batches);
    if (st != HBP_OK) return st;
    return clip(tensors, outs_or_null, sizes, types, n_tensors, batches, {sumsq, 1, nullptr, max_norm, norm_out_or_null}, static_cast<hipStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return HBP_ERR_NO_MEMORY;
  } catch (...) {
    return HBP_ERR_INVALID_ARG;
  }
}

extern "C" hbp_status hbp_grad_clip_norm(const void* const* tensors, void* const* outs_or_null, const int64_t* sizes, const int32_t* types,
                                         int32_t n_tensors, float max_norm, double* sumsq_out, float* norm_out_or_null, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  try {
    if (n_tensors < 0 || !sumsq_out || !aligned_to(sumsq_out, 8) || !(max_norm >= 0.f)) return HBP_ERR_INVALID_ARG;
    std::vector<hbp::GradBatch> batches;
    const hbp_status st = grad_batches(tensors, outs_or_null, sizes, types, n_tensors, batches);
    if (st != HBP_OK) return st;
    int n = 0;
    for (const auto& b : batches) n += groups_of(b);
    if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < (size_t)n * sizeof(double)) return HBP_ERR_WORKSPACE;
    if (overlaps(tensors, outs_or_null, sizes, types, n_tensors)) return HBP_ERR_INVALID_ARG;  // before the first launch
    double* partial = static_cast<double*>(workspace);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    int at = 0;
    for (const auto& b : batches) {
      if (hbp::launch_grad_sumsq(b, groups_of(b), partial + at, s) != 0) return HBP_ERR_DEVICE;
      at += groups_of(b);
    }
    // Few partial sums: every workgroup of the clipping adds them up for itself, in the same order, and a launch falls away (24
    // tensors of 0.8 million elements: 18.1 -> 10.2 us a call, with shorter arguments and smaller chunks).  Many of them would cost each workgroup longer than that.
    if (n < 2 || n > 512) {
      if (hbp::launch_grad_total(partial, n, sumsq_out, false, s) != 0) return HBP_ERR_DEVICE;
      return clip(tensors, outs_or_null, sizes, types, n_tensors, batches, {sumsq_out, 1, nullptr, max_norm, norm_out_or_null}, s);
    }
    return clip(tensors, outs_or_null, sizes, types, n_tensors, batches, {partial, n, sumsq_out, max_norm, norm_out_or_null}, s);
  } catch (const std::bad_alloc&) {
    return HBP_ERR_NO_MEMORY;
  } catch (...) {
    return HBP_ERR_INVALID_ARG;
  }
}
