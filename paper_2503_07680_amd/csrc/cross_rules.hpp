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

// In how many parts the steps over a key tile's query rows (64 of them a step) are dealt out, each an item of its own, whose sums
// of dK and dV are added up by the reduce kernel: where there are fewer than some 192 key tiles (a tile and a kv head each), of
// six steps at least.  Backward, us, in one part -> as here (best of 1 to 32): 4407 queries, 113 keys, 32/8 heads of 128: 375 -> 82
// (75); 3458, 60, 8/1: 370 -> 32.7 (32.7); 9588, 1356, 8/1: 1524 -> 196 (192); 9682, 963, 32/8: 857 -> 508 (508); 4 samples of
// 1240, 150, 32/8: 156 -> 85 (82); 16 of 530, 860, 8/1: 202 -> 137 (137); 4 of 1080, 105, 24/24: 55.8 -> 63.8 (55.8); 280 tiles of 29
// steps: 79.5 in one part, 95.4 in two.
inline int cross_parts(const hbp_cross_desc& d) {
  if (d.total_keys == 0 || d.total_queries == 0) return 1;
  const int64_t items = ((int64_t)d.total_keys + kCrossKeys - 1) / kCrossKeys * d.n_kv_heads;
  const int64_t steps = (int64_t)d.total_queries * (d.n_q_heads / d.n_kv_heads) / (d.n_samples > 0 ? d.n_samples : 1) / 64;
  int64_t parts = (192 + items / 2) / items;
  if (parts > steps / 6) parts = steps / 6;
  return (int)(parts < 1 ? 1 : parts > 32 ? 32 : parts);
}

// Query tiles of the mean sample, as far as the descriptor tells, for all folded groups of heads; rows of one; key tiles (of 64).
struct CrossTiles {
  int64_t items, rows, key_tiles;
};
inline CrossTiles cross_tiles(const hbp_cross_desc& d) {
  const int l = cross_fold_log2(d);
  const int64_t rows = (int64_t)d.total_queries << l, full = (rows + kCrossRows - 1) / kCrossRows;
  const int64_t some = d.n_samples < d.total_queries ? d.n_samples : d.total_queries, tiles = full > some ? full : some;
  return {tiles * (d.n_q_heads >> l), rows / tiles, d.total_keys / d.n_samples / 64};
}

// In how many parts the forward deals out the keys of a query tile: where there are few tiles (tokens of generation, a few
// learned queries) a workgroup for each, and every key in turn, leaves the chip idle.  A tile of few rows is bound by the latency
// of its key tiles: some 768 workgroups, of three tiles at least.  One of many rows computes, and its parts cost their O in fp32
// twice: some 384 workgroups of four wavefronts, of six tiles at least, and nothing below 16.
// Forward, us, in one part -> as here (best of 1 to 32), lengths log-normal with a spread of .4:
//   rows to 32: 32 samples of one token, some 1700 keys, 32/8 heads of 128: 72.8 -> 44.9 (44.9); 4 of 64: 43.0 -> 20.7 (20.6)
//               1 token, 19278 keys, 32/8 heads: 269 -> 26.8 (26.8); 8 tokens, 24 heads: 41.6 -> 33.2 (31.8); 16 of 192: 59.5 -> 40.0 (34.4)
//   more:       64 queries, 4000 keys: 59.0 -> 21.6 (21.6), 64/8: 50.6 -> 26 (24.5); 4 samples: 50.4 -> 29.8 (29.7)
//               256 queries, 8000 keys, 32/8 heads: 131 -> 48.4 (45.3); 1308, 16859 keys, 8/1: 269 -> 113 (98.7)
//               517, 12494 keys, 64/8: 260 in one part (231 in three); 16 samples of 100 queries, 300 keys: 12 to 41 in one part,
//               14 to 85 in two
//
// The mean sample's parts are long for one that is much longer.  Where that one's would be more than 32 tiles, and 1.5 times a workgroup's
// fair share of all tiles (three times, if there was one part for all), the share is the length of a part: the longest sample has as
// many as it takes, the others fewer, and workgroups without keys end at once.  By the mean -> here, one token each:
//   50000 keys and 31 of 200, 32/8 heads of 128: 238 -> 76; 24 heads: 907 -> 193; 127 of 200, 32/8: 888 -> 222, 8/1: 237 -> 85
//   lengths log-normal, a spread of .8: 32 samples of 1500, 16 heads of 192: 204 -> 170, 32/8: 61 -> 57; 300 of 700, 8/1: 64 -> 54
//   100 queries each, 20000 keys and 15 of 300, 32/8: 316 -> 112.  Below these lines it loses: parts of 12 to 22 tiles, 5 to 39 %
struct CrossFwdParts {
  int parts, keys;  // at most, for one sample; keys of a part at least
};
inline CrossFwdParts cross_fwd_parts(const hbp_cross_desc& d) {
  if (d.total_keys == 0 || d.total_queries == 0 || d.n_samples == 0) return {1, 0};
  const CrossTiles t = cross_tiles(d);
  const bool few = t.rows <= 32;
  const int64_t groups = few ? 768 : 384, items = few ? t.items : t.items * ((t.rows + 127) / 128);
  const int64_t least = few ? 3 : 6, most = few ? 32 : 16, begin = few ? 6 : 16;  // tiles of a part; parts; tiles below which there is one
  int64_t parts = groups / items;
  if (parts > t.key_tiles / least) parts = t.key_tiles / least;
  if (parts > most) parts = most;
  if (parts < 1 || t.key_tiles < begin) parts = 1;
  const int64_t longest = ((int64_t)(d.longest_keys < d.total_keys ? d.longest_keys : d.total_keys) + 63) / 64;
  int64_t share = (items * t.key_tiles + groups - 1) / groups;
  if (share < least) share = least;
  const int64_t part = longest / parts;
  if (part <= 32 || 2 * part <= (parts > 1 ? 3 : 6) * share) return {(int)parts, 0};
  parts = (longest + share - 1) / share;
  return {(int)(parts > most ? most : parts), (int)(share * 64)};
}
struct CrossFwdLayout {
  size_t o_off, ml_off, total;
  int parts, part_keys;
};
inline CrossFwdLayout cross_fwd_layout(const hbp_cross_desc& d) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  CrossFwdLayout l;
  const CrossFwdParts parts = cross_fwd_parts(d);
  l.parts = parts.parts;
  l.part_keys = parts.keys;
  const size_t rows = l.parts > 1 ? (size_t)l.parts * d.n_q_heads * d.total_queries : 0;
  l.o_off = 0;
  l.ml_off = up(rows * d.d_v * 4);
  l.total = l.ml_off + up(rows * 8);
  return l;
}

// A workgroup's fair share of the backward, in dK/dV's steps (64 rows of a head, 128 keys): one of dQ, 256 rows and 64 keys, is 1.5 of
// them.  By the mean lengths with their tiles' empty rows, or by the pairs of rows and keys, where long samples are long on both sides.
inline int64_t cross_bwd_share(const hbp_cross_desc& d) {
  const CrossTiles t = cross_tiles(d);
  const int64_t items = ((int64_t)d.total_keys + kCrossKeys - 1) / kCrossKeys * d.n_kv_heads;
  const int64_t steps = (int64_t)d.total_queries * (d.n_q_heads / d.n_kv_heads) / d.n_samples / 64;
  const int64_t by_mean = (2 * items * steps + 3 * t.items * t.key_tiles) / 2 / 256;
  const int64_t by_pairs = d.pairs / (64 * kCrossKeys) * d.n_q_heads / 256 * 7 / 4;
  return by_mean > by_pairs ? by_mean : by_pairs;
}
// Whether an item of so many of dK/dV's steps (some 1.1 us each) holds up the launch by more than its parts cost, of which most have
// nothing to do (a workgroup 2 us) where few samples are long: then the share is the length of a part.  Backward, us, by the mean -> here:
// one sample of 8000 queries and 200 keys, 30 of 100 and 100, 32/8 heads of 128: 673 -> 212, 8/1: 210 -> 108; 20000 and 1500, 24 of 500 and
// 1500, 8/1: 3277 -> 1217, 12/3 of 64: 1142 -> 566; 10 and 30000, 30 of 100 and 100, 32/8: 484 -> 157, 24 heads: 565 -> 364; 300 and 4000,
// 11 of 300 and 300, 8/1: 121 -> 64; 16 samples log-normal with a spread of 1, 8/1: 735 -> 432.  Without the parts' cost in the rule 8000
// and 200 with 24 heads went from 196 to 265, 300 and 4000 from 146 to 161.
inline bool cross_holds_up(int64_t steps, int64_t share, int64_t workgroups) { return steps > 64 + workgroups / 32 && steps > 2 * share; }
// At head size 192 dQ's items are halves of a tile, and an item of dK/dV that is one part goes through the workspace too.
inline int64_t cross_items_cost(const hbp_cross_desc& d) { return d.d_qk > 128 ? 2 : 1; }
constexpr int64_t kCrossMostParts = 16;  // of a long sample: the workspace has room for as many of every one
struct CrossBwdParts {
  int parts, least;  // at most, for one item; steps or keys of a part at least
};
inline CrossBwdParts cross_dkdv_parts(const hbp_cross_desc& d) {
  const int parts = cross_parts(d);
  if (d.total_keys == 0 || d.total_queries == 0 || d.n_samples == 0) return {parts, 0};
  const int64_t longest = (int64_t)(d.longest_queries < d.total_queries ? d.longest_queries : d.total_queries) * (d.n_q_heads / d.n_kv_heads) / 64;
  const int64_t share = cross_bwd_share(d), least = share < 32 ? 32 : share;
  int64_t more = (longest + least - 1) / least;
  if (more > kCrossMostParts) more = kCrossMostParts;
  if (!cross_holds_up(longest / parts, share, ((int64_t)d.total_keys + kCrossKeys - 1) / kCrossKeys * d.n_kv_heads * more * cross_items_cost(d))) return {parts, 0};
  return {(int)more, (int)least};
}

// The same for dQ, beside dK/dV in one launch.  In products of 64-column blocks: an item of dQ takes 3 x 256 rows x its keys, all
// of dQ that times its items, all of dK/dV 4 x rows x keys.  An item that is longer than a compute unit's share of the two is cut.
// Backward, us, in one part -> as here: 118 queries, 7467 keys, 32/8 heads of 128: 172 -> 69; 74, 5994, 6/2 of 64: 73 -> 22.5; 34,
// 5300, 8/1: 109 -> 24; 112, 5400, 12/3: 117 -> 31; 52, 4222, 24: 103 -> 50.  (By the forward's rule 16 samples of 450 queries and
// 800 keys, 8/1 heads, went from 132 to 167.)
inline CrossBwdParts cross_dq_parts(const hbp_cross_desc& d) {
  if (d.total_keys == 0 || d.total_queries == 0 || d.n_samples == 0) return {1, 0};
  const CrossTiles t = cross_tiles(d);
  int64_t parts = 256 * 3 * kCrossRows / (t.items * 3 * kCrossRows + (int64_t)d.total_queries * d.n_q_heads * 4);
  if (parts > t.key_tiles / 2) parts = t.key_tiles / 2;
  parts = parts < 1 ? 1 : parts > 32 ? 32 : parts;
  const int64_t longest = ((int64_t)(d.longest_keys < d.total_keys ? d.longest_keys : d.total_keys) + 63) / 64;
  const int64_t share = cross_bwd_share(d), least = share < 32 ? 21 : share * 2 / 3;
  int64_t more = (longest + least - 1) / least;
  if (more > kCrossMostParts) more = kCrossMostParts;
  if (!cross_holds_up(longest * 3 / 2 / parts, share, t.items * more * cross_items_cost(d))) return {(int)parts, 0};
  return {(int)more, (int)(least * 64)};
}

// Workgroups that share the rows of a tile where parts are added up: some 1024 in all, and no more than a tile has work for.
inline int cross_join_shares(int groups, int tiles) {
  const int64_t n = 1024 / ((int64_t)groups * tiles);
  return n < 4 ? 4 : n > 32 ? 32 : (int)n;
}

// dK/dV and dQ in one launch, a workgroup an item, as long as the items' numbers stay exact in the kernel's quotients.  Against two
// launches, 77 packs of 40 to 19600 tokens a side, 4/4 to 128/128 heads: 1.1 to 1.6 where the launches have few rounds, 1.0 to 1.1 in
// large packs, .99 at worst.
inline bool cross_one_launch(int64_t n_dkdv, int64_t n_dq) { return n_dkdv > 0 && n_dq > 0 && n_dkdv + n_dq < (1 << 22); }

// Whether dQ's items come before those of dK/dV: those that are longer, in the mean, or, where long samples have parts of their own, at most.
inline bool cross_dq_first(const hbp_cross_desc& d, const CrossBwdParts& dkdv, const CrossBwdParts& dq) {
  const int64_t group = d.n_q_heads / d.n_kv_heads;
  if (dkdv.least == 0 && dq.least == 0) return (int64_t)d.total_keys * 3 * 256 / dq.parts > d.total_queries * group * 4 * 128 / dkdv.parts;
  const int64_t steps = dkdv.least ? dkdv.least : d.longest_queries * group / 64 / dkdv.parts;
  const int64_t tiles = dq.least ? dq.least / 64 : d.longest_keys / 64 / dq.parts;
  return 3 * tiles > 2 * steps;
}

struct CrossBwdLayout {
  size_t d_off, lse2_off, dk_part_off, dv_part_off, dq_part_off, total;
  int parts, part_steps, dq_parts, dq_part_keys;
  bool dq_first;
};
inline CrossBwdLayout cross_bwd_layout(const hbp_cross_desc& d) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  CrossBwdLayout l;
  const CrossBwdParts dkdv = cross_dkdv_parts(d), dq = cross_dq_parts(d);
  l.parts = dkdv.parts;
  l.part_steps = dkdv.least;
  const size_t rows = up((size_t)d.n_q_heads * d.total_queries * 4), sums = l.parts > 1 ? (size_t)l.parts * d.total_keys * d.n_kv_heads * 4 : 0;
  l.d_off = 0;
  l.lse2_off = rows;
  l.dk_part_off = 2 * rows;
  l.dv_part_off = l.dk_part_off + up(sums * d.d_qk);
  l.dq_parts = dq.parts;
  l.dq_part_keys = dq.least;
  l.dq_first = cross_dq_first(d, dkdv, dq);
  l.dq_part_off = l.dv_part_off + up(sums * d.d_v);
  l.total = l.dq_part_off + (l.dq_parts > 1 ? up((size_t)l.dq_parts * d.n_q_heads * d.total_queries * d.d_qk * 4) : 0);
  return l;
}

}  // namespace hbp
