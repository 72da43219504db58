// How a cross attention call is laid out and launched: plain host functions of sizes, without HIP.
#pragma once
#include <stdint.h>

#include "hbp.h"

namespace hbp {

// Strides with the dense ones in the place of zeros.
struct CrossStrides {
  int64_t q_t, q_h, k_t, k_h, v_t, v_h, o_t, o_h;
};
inline CrossStrides cross_strides(const hbp_cross_desc& d) {
  auto fix = [](int64_t s, int64_t dense) { return s == 0 ? dense : s; };
  return {fix(d.q_stride_t, (int64_t)d.n_q_heads * d.d_qk), fix(d.q_stride_h, d.d_qk),
          fix(d.k_stride_t, (int64_t)d.n_kv_heads * d.d_qk), fix(d.k_stride_h, d.d_qk),
          fix(d.v_stride_t, (int64_t)d.n_kv_heads * d.d_v), fix(d.v_stride_h, d.d_v),
          fix(d.o_stride_t, (int64_t)d.n_q_heads * d.d_v), fix(d.o_stride_h, d.d_v)};
}

// log2 of F, the query heads of a kv head that are rows beside each other (struct Fold): the largest power of two up to 32 in
// the group size, where a token's F heads lie inside its stride, else 1.
inline int cross_fold_log2(const hbp_cross_desc& d) {
  const CrossStrides s = cross_strides(d);
  const int g = d.n_q_heads / d.n_kv_heads;
  int l = 0;
  while (l < 5 && g % (2 << l) == 0 && (((int64_t)2 << l) - 1) * s.q_h + d.d_qk <= s.q_t && (((int64_t)2 << l) - 1) * s.o_h + d.d_v <= s.o_t) ++l;
  return l;
}
constexpr int kCrossRows = 256, kCrossKeys = 128;  // folded rows of a query tile, keys of a key tile

// In how many parts the steps over a key tile's query rows are dealt out, each an item of its own (their sums of dK and dV are
// added up by the reduce kernel): as many as give every compute unit two, of at least 8 steps in the mean.
inline int cross_parts(const hbp_cross_desc& d) {
  if (d.total_keys == 0 || d.total_queries == 0) return 1;
  const int64_t items = ((int64_t)d.total_keys + kCrossKeys - 1) / kCrossKeys * d.n_kv_heads;
  const int64_t steps = (int64_t)d.total_queries * (d.n_q_heads / d.n_kv_heads) / (d.n_samples > 0 ? d.n_samples : 1) / 64;
  int64_t parts = (512 + items - 1) / items;
  if (parts > steps / 8) parts = steps / 8;
  return (int)(parts < 1 ? 1 : parts > 16 ? 16 : parts);
}

// In how many parts the forward deals out the keys of a query tile: where there are few tiles (tokens of generation, a few
// learned queries) a workgroup for each and every key in turn leaves the chip idle.
inline int cross_fwd_parts(const hbp_cross_desc& d) {
  if (d.total_keys == 0 || d.total_queries == 0 || d.n_samples == 0) return 1;
  const int l = cross_fold_log2(d);
  const int64_t full = (((int64_t)d.total_queries << l) + kCrossRows - 1) / kCrossRows, some = d.n_samples < d.total_queries ? d.n_samples : d.total_queries;
  const int64_t items = (full > some ? full : some) * (d.n_q_heads >> l), keys = d.total_keys / d.n_samples;
  int64_t parts = 2048 / items;
  if (parts > keys / 128) parts = keys / 128;
  return (int)(parts < 1 ? 1 : parts > 32 ? 32 : parts);
}
struct CrossFwdLayout {
  size_t o_off, ml_off, total;
  int parts;
};
inline CrossFwdLayout cross_fwd_layout(const hbp_cross_desc& d) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  CrossFwdLayout l;
  l.parts = cross_fwd_parts(d);
  const size_t rows = l.parts > 1 ? (size_t)l.parts * d.n_q_heads * d.total_queries : 0;
  l.o_off = 0;
  l.ml_off = up(rows * d.d_v * 4);
  l.total = l.ml_off + up(rows * 8);
  return l;
}

struct CrossBwdLayout {
  size_t d_off, lse2_off, dk_part_off, dv_part_off, total;
  int parts;
};
inline CrossBwdLayout cross_bwd_layout(const hbp_cross_desc& d) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  CrossBwdLayout l;
  l.parts = cross_parts(d);
  const size_t rows = up((size_t)d.n_q_heads * d.total_queries * 4), sums = l.parts > 1 ? (size_t)l.parts * d.total_keys * d.n_kv_heads * 4 : 0;
  l.d_off = 0;
  l.lse2_off = rows;
  l.dk_part_off = 2 * rows;
  l.dv_part_off = l.dk_part_off + up(sums * d.d_qk);
  l.total = l.dv_part_off + up(sums * d.d_v);
  return l;
}

}  // namespace hbp
