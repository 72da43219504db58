// Driver for cross attention's host code (the plan, and the rules of csrc/cross_rules.hpp) under AddressSanitizer and
// UndefinedBehaviorSanitizer: seeded random and extreme lengths and descriptors, exact-size output buffers, size queries, error
// paths.  Prints "ok" and returns 0 when every call returned the expected status and every rule kept its bounds.
#include <climits>
#include <cstdio>
#include <vector>

#include "cross_rules.hpp"
#include "hbp.h"

static uint64_t rng_state = 0x7654321;
static uint32_t rnd() {
  rng_state = rng_state * 6364136223846793005ull + 1442695040888963407ull;
  return (uint32_t)(rng_state >> 33);
}
#define CHECK(cond)                                           \
  do {                                                        \
    if (!(cond)) {                                            \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #cond); \
      return 1;                                               \
    }                                                         \
  } while (0)

static int32_t size_up_to(int bits) { return (int32_t)(rnd() & ((1u << (1 + rnd() % bits)) - 1)); }

int main() {
  for (int round = 0; round < 400; ++round) {
    const int n = (int)(rnd() % 50);
    std::vector<int32_t> q(n), k(n);
    for (auto& v : q) v = rnd() % 4 ? (int32_t)(rnd() % 900) : 0;
    for (auto& v : k) v = rnd() % 4 ? (int32_t)(rnd() % 2000) : 0;
    const int32_t rows = 1 + (int32_t)(rnd() % 300), kind = rnd() & 1;
    int32_t nt = -1;
    int64_t pairs = -1;
    CHECK(hbp_cross_plan(q.data(), k.data(), n, rows, kind, nullptr, nullptr, 0, nullptr, 0, &nt, &pairs) == HBP_OK);
    std::vector<int32_t> cu_q(n + 1), cu_kv(n + 1);
    std::vector<hbp_tile> tiles(nt);
    CHECK(hbp_cross_plan(q.data(), k.data(), n, rows, kind, cu_q.data(), cu_kv.data(), n + 1, tiles.data(), nt, &nt, &pairs) == HBP_OK);
    int64_t want = 0, covered = 0;
    for (int i = 0; i < n; ++i) want += (int64_t)q[i] * k[i];
    CHECK(pairs == want);
    const auto& cu = kind == HBP_TILES_QUERY ? cu_q : cu_kv;
    for (const auto& t : tiles) {
      CHECK(t.sample >= 0 && t.sample < n && cu[t.sample] <= t.row_begin && t.row_begin < t.row_end && t.row_end <= cu[t.sample + 1]);
      CHECK(t.row_end - t.row_begin <= rows && t.row_begin == cu[t.sample] + t.tile * rows);
      covered += t.row_end - t.row_begin;
    }
    CHECK(covered == cu[n]);
    if (nt > 0) CHECK(hbp_cross_plan(q.data(), k.data(), n, rows, kind, nullptr, nullptr, 0, tiles.data(), nt - 1, &nt, &pairs) == HBP_ERR_CAPACITY);
  }
  {
    const int32_t most[3] = {INT_MAX, INT_MAX, INT_MAX}, one[3] = {1, 1, 1}, fits[1] = {INT_MAX};
    int32_t nt;
    int64_t pairs;
    CHECK(hbp_cross_plan(most, most, 3, 1 << 20, 0, nullptr, nullptr, 0, nullptr, 0, &nt, &pairs) == HBP_ERR_INVALID_ARG);
    CHECK(hbp_cross_plan(one, most, 2, 1 << 20, 1, nullptr, nullptr, 0, nullptr, 0, &nt, &pairs) == HBP_ERR_INVALID_ARG);
    CHECK(hbp_cross_plan(fits, fits, 1, 1 << 20, 1, nullptr, nullptr, 0, nullptr, 0, &nt, &pairs) == HBP_OK);
    CHECK(pairs == (int64_t)INT_MAX * INT_MAX && nt == 2048);
  }
  const int dims[3][2] = {{64, 64}, {128, 128}, {192, 128}};
  for (int round = 0; round < 200000; ++round) {
    hbp_cross_desc d = {};
    d.total_queries = size_up_to(31) >> 5;
    d.total_keys = size_up_to(31);
    d.n_samples = size_up_to(20);
    d.n_kv_heads = 1 + (int32_t)(rnd() % 64);
    d.n_q_heads = d.n_kv_heads * (1 + (int32_t)(rnd() % 64));
    d.longest_keys = rnd() % 2 ? 0 : size_up_to(31);
    d.longest_queries = rnd() % 2 ? 0 : size_up_to(31);
    d.pairs = rnd() % 2 ? 0 : (int64_t)size_up_to(31) * size_up_to(31);
    d.d_qk = dims[round % 3][0];
    d.d_v = dims[round % 3][1];
    const int fold = hbp::cross_fold_log2(d), parts = hbp::cross_parts(d), dq = hbp::cross_dq_parts(d).parts;
    const hbp::CrossFwdParts f_parts = hbp::cross_fwd_parts(d);
    const int fwd = f_parts.parts;
    CHECK(f_parts.keys >= 0 && f_parts.keys % 64 == 0 && (f_parts.keys == 0 || (d.longest_keys > 0 && fwd > 1 && f_parts.keys < INT_MAX - 4096)));
    CHECK(fold >= 0 && fold <= 5 && (d.n_q_heads / d.n_kv_heads) % (1 << fold) == 0);
    CHECK(parts >= 1 && parts <= 32 && fwd >= 1 && fwd <= 32 && dq >= 1 && dq <= 32);
    const hbp::CrossBwdParts dkdv = hbp::cross_dkdv_parts(d);
    CHECK(dkdv.parts >= 1 && dkdv.parts <= 32 && dkdv.least >= 0);
    const hbp::CrossFwdLayout f = hbp::cross_fwd_layout(d);
    const hbp::CrossBwdLayout b = hbp::cross_bwd_layout(d);
    CHECK(f.total % 256 == 0 && b.total % 256 == 0 && f.o_off <= f.ml_off && f.ml_off <= f.total);
    CHECK((f.total == 0) == (f.parts == 1));
    CHECK(b.d_off <= b.lse2_off && b.lse2_off <= b.dk_part_off && b.dk_part_off <= b.dv_part_off && b.dv_part_off <= b.dq_part_off && b.dq_part_off <= b.total);
    const int shares = hbp::cross_join_shares(d.n_q_heads >> fold, 1 + (int)(rnd() % 30000));
    CHECK(shares >= 4 && shares <= 32);
  }
  std::printf("ok\n");
  return 0;
}
