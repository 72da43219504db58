// Token embedding of a packed buffer and its gradient, gfx950.
//
//   lookup     Y[t] = s W[x_t], zeros where x_t is no token (negative, or the vocabulary's size and beyond)
//   gradient   dW[v] (+)= s sum over t with x_t = v, in ascending t, of dY[t]
//
// Both move bytes and compute next to nothing.  The gradient works on the tokens sorted by id, equal ids in the order of
// their positions, so that every row of dW is summed in one fixed order, in 32 bits, and written once, without atomics:
// (1) the stable sort of (id, position); (2) the sorted positions are cut into chunks of a fixed number, whatever the ids, so
// that a frequent id costs no workgroup more than the others: a run of equal ids inside a chunk is summed and written, of one
// that goes beyond it the chunk's part is kept; (3) the parts of such runs are added up in the chunks' order.
//
// The sort is one launch (embed_group_kernel): a workgroup owns a range of up to 1024 ids, reads all tokens (4 KB to 1 MB, from
// its die's L2; twice again where a few of its ids have very many), counts those below its range, which is where its part of the order
// begins, and places its own.  It also zeroes those rows of a fresh dW that have no token.  Very many tokens or ids take a radix
// sort of nine bits a pass instead.
//
// 8192 tokens, width 4096, added to a bf16 table of 128256 rows: 40 us (sort 7.4, sums 23 at 4.2 TB/s, joined runs 6);
// 32767 tokens of width 2056, fresh fp32 table of 32000 rows: 106 (sort and zeros 44, sums 51, joined runs 8).
#include "lds_limit.hpp"
#include "rows.hpp"

namespace hbp {

namespace {

constexpr int kRowThreads = 256;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kGroupList = 12288, kGroupBins = 1024;  // tokens that a workgroup lists, ids of it (embed_group_kernel)
constexpr int kWaveList = kGroupList / 16;           // of each of its wavefronts
constexpr int kTileRounds = 4, kTile = kTileRounds * kSortThreads;  // of each workgroup where there are more
constexpr int kSmallChunks = 16384;          // up to so many tokens: chunks of 16, else of 32
constexpr uint32_t kNoKey = 0xffffffffu;

int log2_threads_per_row(int n_vec) {  // 64 to 256: a wavefront is always on one row
  return n_vec > 128 ? 8 : n_vec > 64 ? 7 : 6;
}
int waves_per_row(int n_vec) { return (n_vec + 63) / 64; }
// Ids of a workgroup of the one-launch sort; 0: the radix sort is taken, where every workgroup would read very many tokens, or there
// would be very many of them (a compute unit holds one).  Whole calls on narrow rows, us, one launch / radix sort, ids of frequencies
// 1/n, or (equal / half of the tokens one id): 1000 tokens 17 / 28; 32768: 33 / 46; 65536: 44 / 50 (30 / 47; 73 / 54);
// 131072: 69 / 59 (43 / 56; 125 / 67); 196608: 166 / 68; a million ids: 1000 29 / 37, 32768 49 / 63, 131072 80 / 67; two million: 42 /
// 37, 51 / 52 with 8192, 71 / 62 with 32768; four million: 65 / 38, 82 / 52 with 8192.
int group_bins(int32_t T, int32_t V) {
  const int bins = V <= 256 * kGroupBins ? (V + 255) / 256 : kGroupBins;
  const int64_t groups = (V + (int64_t)bins - 1) / bins;
  return T <= 65536 && groups <= 2048 && T * groups <= ((int64_t)1 << 25) ? bins : 0;
}
int n_vectors(int dim) { return dim >= 8 ? (dim + 7) / 8 : dim; }
int key_bits(int32_t V) { return 32 - __builtin_clz((uint32_t)V); }  // ids 0 .. V - 1, and V for "no token"

// A thread's share of a row: VEC values from column col on, of which the first `skip` belong to the thread before (the last
// eight of a row whose width is no multiple of eight).
struct Span {
  int col, skip;
};
template <int VEC>
__device__ __forceinline__ Span span_of(int v, int dim) {
  const int col = VEC == 8 ? min(8 * v, dim - 8) : v;
  return {col, VEC * v - col};
}
template <int TYPE, int VEC>
__device__ __forceinline__ f32x8_row load_span(const typename RowType<TYPE>::T* p) {
  if constexpr (VEC == 8) return RowType<TYPE>::widen(RowType<TYPE>::load_raw(p));
  f32x8_row x = {};
  x[0] = RowType<TYPE>::load1(p);
  return x;
}

// ------------------------------------------------------------------------------------- lookup
// A workgroup takes U rows a pass with its rows' loads under way together.  Many rows (U > 1, from 16 million elements on) are stored
// past the caches: 65536 rows of 1025 bf16, which start anywhere: 57 -> 35 us; 32768 of 2056 from fp32: 59 -> 47; 131072 of 4096:
// 297 -> 285 (4.7 TB/s; a copy reaches 4.8).  Fewer rows are left in the caches for what reads them next.
template <int TABLE, int ROW, int VEC, int U>
__global__ __launch_bounds__(kRowThreads) void embed_lookup_kernel(EmbedParams p, const typename RowType<TABLE>::T* table,
                                                                   typename RowType<ROW>::T* out, int log2_tpr) {
  const int tpr = 1 << log2_tpr, per_pass = kRowThreads >> log2_tpr;
  const int sub = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> log2_tpr);
  const int64_t row0 = (int64_t)blockIdx.x * (per_pass * U) + sub;
  int id[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t r = row0 + (int64_t)u * per_pass;
    id[u] = r < p.T ? p.tokens[r] : -1;
  }
  const int n_vec = VEC == 8 ? (p.dim + 7) / 8 : p.dim;
  for (int v = threadIdx.x & (tpr - 1); v < n_vec; v += tpr) {
    const int col = span_of<VEC>(v, p.dim).col;
    f32x8_row x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = f32x8_row{};
      if (id[u] >= 0 && id[u] < p.V) x[u] = load_span<TABLE, VEC>(table + (int64_t)id[u] * p.table_st + col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = row0 + (int64_t)u * per_pass;
      if (r >= p.T) break;
      auto* to = out + r * p.row_st + col;
      const f32x8_row y = x[u] * p.scale;
      if constexpr (VEC == 8 && U > 1) RowType<ROW>::store_past(to, y);
      else if constexpr (VEC == 8) RowType<ROW>::store(to, y);
      else RowType<ROW>::store1(to, y[0]);
    }
  }
}

// --------------------------------------------------------------------------------------- sort
typedef volatile __attribute__((address_space(3))) uint32_t* LdsCounts;

// One tile of up to E * 1024 elements, element (wave * rounds + e) * 64 + lane in key[e] of a thread (kNoKey: none).  Counts
// the digit `shift` of its elements into counts[digit][wave] and returns in rank[e] how many of the same digit the wavefront
// has in front of each.  counts start as zeros.
template <int E>
__device__ __forceinline__ void wave_ranks(const uint32_t (&key)[E], uint32_t (&rank)[E], int rounds, int shift, LdsCounts counts) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (e >= rounds) continue;
    const bool is = key[e] != kNoKey;
    const uint32_t d = (key[e] >> shift) & (kDigits - 1);
    uint64_t same = __builtin_amdgcn_ballot_w64(is);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
      const bool one = (d >> b) & 1;
      const uint64_t ones = __builtin_amdgcn_ballot_w64(one);
      same &= one ? ones : ~ones;
    }
    rank[e] = 0;
    if (is) {  // LDS operations of a wavefront are in order: all read the count before the first of each digit raises it
      const uint32_t before = counts[d * kSortWaves + wave];
      const uint32_t in_front = (uint32_t)__popcll(same & below);
      __builtin_amdgcn_wave_barrier();
      if (in_front == 0) counts[d * kSortWaves + wave] = before + (uint32_t)__popcll(same);
      __builtin_amdgcn_wave_barrier();
      rank[e] = before + in_front;
    }
  }
}
// exclusive sum over the workgroup of one value a thread; sums: one word a wavefront
__device__ __forceinline__ uint32_t before_me(uint32_t x, uint32_t* sums) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  uint32_t s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(s, d, 64);
    if (lane >= d) s += y;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = s;
  __syncthreads();
  uint32_t base = 0;
  for (int w = 0; w < wave; ++w) base += sums[w];
  return base + s - x;
}
// counts[digit][wave] -> the tile's elements of smaller digits, and of the same one in the wavefronts before
__device__ __forceinline__ void scan_counts(uint32_t* counts, uint32_t* sums) {
  constexpr int N = kDigits * kSortWaves / kSortThreads;
  uint32_t c[N], total = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    c[i] = counts[threadIdx.x * N + i];
    total += c[i];
  }
  uint32_t at = before_me(total, sums);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    counts[threadIdx.x * N + i] = at;
    at += c[i];
  }
  __syncthreads();
}
__device__ __forceinline__ void clear_counts(uint32_t* counts) {
  for (int i = threadIdx.x; i < kDigits * kSortWaves; i += kSortThreads) counts[i] = 0;
  __syncthreads();
}
__device__ __forceinline__ uint32_t key_of(int32_t token, int32_t V) { return token >= 0 && token < V ? (uint32_t)token : (uint32_t)V; }

// Zeros into rows [V part / parts, V (part + 1) / parts) of dW, by the workgroups from `first` on; 2^lanes_log2 lanes a row.
struct Fill {
  char* table;
  int64_t stride_bytes, row_bytes;
  int32_t V, part, parts, blocks;  // blocks: 0 for none
  int32_t lanes_log2;
};
typedef uint32_t u32x4_line __attribute__((ext_vector_type(4)));
// A row by the lanes sub = 0 .. of it.  A wavefront on a row stores whole lines past the caches, and leaves in them what the row's
// ends share with its neighbours, until those are written (23000 rows of 8224 bytes: 39 us
// past the caches altogether, 30).  Lanes for several short rows: half a million of 16 bytes, 51 -> 23 us a call.
__device__ __forceinline__ void zero_row(const Fill& f, int64_t r, int sub) {
  char* row = f.table + r * f.stride_bytes;
  int64_t from = 0;  // rows are whole elements of 2 or 4 bytes
  if (f.lanes_log2 == 6) {
    const int head = (int)(-(uintptr_t)row & 127);
    if (2 * sub < head) *(uint16_t*)(row + 2 * sub) = 0;
    from = head + ((f.row_bytes - head) & ~(int64_t)127);
    for (int64_t b = head + sub * 16; b < from; b += 1024) __builtin_nontemporal_store(u32x4_line{0, 0, 0, 0}, (u32x4_line*)(row + b));
  }
  for (from += sub * 16; from + 16 <= f.row_bytes; from += 16 << f.lanes_log2) *(u32x4_any*)(row + from) = u32x4_any{0, 0, 0, 0};
  // at most one piece of the row's end is left, to one lane
  if (from < f.row_bytes)
    for (; from < f.row_bytes; from += 2) *(uint16_t*)(row + from) = 0;
}
// lanes for a row of so many bytes: a wavefront where it has a whole line at least, wherever it starts
int fill_lanes_log2(int64_t row_bytes) {
  int l = 0;
  while (l < 6 && (16 << l) < row_bytes) ++l;
  return l;
}
__device__ __forceinline__ void fill_rows(const Fill& f, int block) {
  const int lane = threadIdx.x & 63, sub = lane & ((1 << f.lanes_log2) - 1);
  const int64_t waves = (int64_t)f.blocks * kSortWaves, wave = (int64_t)block * kSortWaves + (threadIdx.x >> 6);
  const int64_t from = (int64_t)f.V * f.part / f.parts, to = (int64_t)f.V * (f.part + 1) / f.parts;
  for (int64_t r = from + (wave << (6 - f.lanes_log2)) + (lane >> f.lanes_log2); r < to; r += waves << (6 - f.lanes_log2)) zero_row(f, r, sub);
}

// The one-launch sort: workgroup w owns the ids [w bins, (w + 1) bins), and each of its wavefronts reads a stretch of the tokens,
// counts those of each of its ids and of all smaller ones and lists the former in LDS, in order.  A wavefront then ranks 64 listed
// ones at a time among those of the same id by ballots over the bits; the counts of the wavefronts in front and of the smaller ids
// make up the rest of a place.  Bound by the instructions of the scan, some 13 a token of a lane.  Where a few ids have so many of
// the tokens that a wavefront's part of the list is too short, all are read twice again, to count each wavefront's tokens of each id
// and to place them (16384 tokens of width 2048, half of them one id: a call of 90 us, half of that the joins below, is 48).
// 65536 tokens, 32000 ids, us: tiles of 16384 tokens listed one after the other in a second reading 28, the whole stretch in a second
// reading 24, in the first 21; 8192 tokens, 128256 ids: 26.8 with one workgroup that sorts nine bits at a time in LDS, 7.5.
struct GroupLds {
  uint16_t counts[kGroupBins * kSortWaves];  // of the listed tokens, [id][wavefront]
  union {
    struct {
      uint16_t id[kGroupList], rank[kGroupList];
      uint32_t pos[kGroupList];
    };
    uint32_t next[kGroupBins * kSortWaves];  // without a list: a wavefront's next place of each id, [id][wavefront]
  };
  uint32_t place[kGroupBins];                // counts, then the next place, of each id
  uint32_t sums[kSortWaves], below[kSortWaves], mine[kSortWaves];
  uint64_t has[kSortWaves];                  // ids with a token, a bit each
};
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ i32x4_any load_tokens(const int32_t* tokens, int end, int i) {  // -1 from end on
  if (i + 4 <= end) return *(const i32x4_any*)(tokens + i);
  i32x4_any t;
#pragma unroll
  for (int j = 0; j < 4; ++j) t[j] = i + j < end ? tokens[i + j] : -1;
  return t;
}
__global__ __launch_bounds__(kSortThreads) void embed_group_kernel(const int32_t* tokens, int T, int V, int bins, uint32_t* keys,
                                                                   uint32_t* order, Fill fill) {
  extern __shared__ __attribute__((aligned(16))) char group_lds[];
  GroupLds& l = *(GroupLds*)group_lds;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int lo = (int)((int64_t)blockIdx.x * bins), own_ids = min(bins, V - lo);
  const uint64_t in_front = ((uint64_t)1 << lane) - 1;
  auto of_mine = [&](int t) { return (uint32_t)(t - lo) < (uint32_t)own_ids; };  // tokens that are none are below 0 or from V on
  // Counts of this range's ids.  The first lane's id is counted once for all that have it: frequent ones do not queue up in LDS.
  // Whole numbers, the order does not matter.
  auto count = [&](const i32x4_any& t, const uint64_t (&b)[4], uint32_t* counts, int step) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (b[j] == 0) continue;
      const int lead = __builtin_ctzll(b[j]), id = __builtin_amdgcn_readlane(t[j], lead);
      const uint32_t same = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(t[j] == id));
      if (of_mine(t[j]) && (t[j] != id || lane == lead)) atomicAdd(&counts[(t[j] - lo) * step], t[j] == id ? same : 1u);
    }
  };
  // A lane's four tokens from position pos on into the wavefront's part of the list behind its first `at`.  Returns how many of the
  // wavefront's tokens there are.
  auto list = [&](const i32x4_any& t, int pos, uint32_t at) {
    uint64_t b[4];
    uint32_t n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      b[j] = __builtin_amdgcn_ballot_w64(of_mine(t[j]));
      n += (uint32_t)__popcll(b[j]);
    }
    if (n == 0) return 0u;
    count(t, b, l.place, 1);
    uint32_t to = at;  // of this lane's first: the lanes in front, four tokens each
#pragma unroll
    for (int j = 0; j < 4; ++j) to += (uint32_t)__popcll(b[j] & in_front);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (of_mine(t[j])) {
        if (to < kWaveList) {
          l.id[wave * kWaveList + to] = (uint16_t)(t[j] - lo);
          l.pos[wave * kWaveList + to] = (uint32_t)(pos + j);
        }
        ++to;
      }
    return n;
  };
  const int stretch = (T + kSortWaves * 256 - 1) / (kSortWaves * 256) * 256, begin = wave * stretch, end = min(begin + stretch, T);
  l.place[tid] = 0;
  __syncthreads();
  uint32_t below = 0, mine = 0;  // of this wavefront
  for (int i0 = begin; i0 < end; i0 += 1024) {
    i32x4_any t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = load_tokens(tokens, end, i0 + k * 256 + lane * 4);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        below += (uint32_t)__popcll(__builtin_amdgcn_ballot_w64((uint32_t)t[k][j] < (uint32_t)lo));
      }
#pragma unroll
    for (int k = 0; k < 4; ++k) mine += list(t[k], i0 + k * 256 + lane * 4, mine);
  }
  if (lane == 0) {
    l.below[wave] = below;
    l.mine[wave] = mine;
  }
  __syncthreads();
  const uint32_t of_id = l.place[tid];
  const uint64_t has = __builtin_amdgcn_ballot_w64(of_id != 0);
  if (lane == 0) l.has[wave] = has;
  // places in front of this range; its tokens; the longest part of the list
  uint32_t base = 0, all = 0, longest = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    base += l.below[w];
    all += l.mine[w];
    longest = max(longest, l.mine[w]);
  }
  const uint32_t place = base + before_me(of_id, l.sums);
  __syncthreads();
  l.place[tid] = place;
  // which of the tokens (id d; a lane each) have the same id, and how many of them are in front
  auto of_same_id = [&](bool is, uint32_t d) {
    uint64_t same = __builtin_amdgcn_ballot_w64(is);
#pragma unroll
    for (int b = 0; b < 10; ++b) {
      const bool one = (d >> b) & 1;
      const uint64_t ones = __builtin_amdgcn_ballot_w64(one);
      same &= one ? ones : ~ones;
    }
    return same;
  };
  // LDS operations of a wavefront are in order: all read a count before the first token of each id raises it
  if (__builtin_amdgcn_readfirstlane(longest) <= kWaveList) {
    for (int i = tid; i < kGroupBins * kSortWaves / 8; i += kSortThreads) ((u32x4_any*)l.counts)[i] = u32x4_any{0, 0, 0, 0};
    __syncthreads();
    const uint32_t first = wave * kWaveList + lane, end_of_list = wave * kWaveList + mine;
    volatile uint16_t* const counts = l.counts;
    for (uint32_t i = first; i - lane < end_of_list; i += 64) {
      const bool is = i < end_of_list;
      const uint32_t d = is ? l.id[i] : 0;
      const uint64_t same = of_same_id(is, d);
      if (is) {
        const uint32_t before = counts[d * kSortWaves + wave], r = (uint32_t)__popcll(same & in_front);
        __builtin_amdgcn_wave_barrier();
        if (r == 0) counts[d * kSortWaves + wave] = (uint16_t)(before + (uint32_t)__popcll(same));
        __builtin_amdgcn_wave_barrier();
        l.rank[i] = (uint16_t)(before + r);
      }
    }
    __syncthreads();
    for (uint32_t i = first; i < end_of_list; i += 64) {
      const uint32_t d = l.id[i];
      uint32_t to = l.place[d] + l.rank[i];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) to += w < wave ? l.counts[d * kSortWaves + w] : 0;
      keys[to] = (uint32_t)lo + d;
      order[to] = l.pos[i];
    }
  } else {
    __syncthreads();  // the places are there, and nothing reads the list any more
    for (int i = tid; i < kGroupBins * kSortWaves / 4; i += kSortThreads) ((u32x4_any*)l.next)[i] = u32x4_any{0, 0, 0, 0};
    __syncthreads();
    for (int i0 = begin; i0 < end; i0 += 1024) {
      i32x4_any t[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) t[k] = load_tokens(tokens, end, i0 + k * 256 + lane * 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint64_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = __builtin_amdgcn_ballot_w64(of_mine(t[k][j]));
        count(t[k], b, l.next + wave, kSortWaves);
      }
    }
    __syncthreads();
    uint32_t at = place;  // of this thread's id
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = l.next[tid * kSortWaves + w];
      l.next[tid * kSortWaves + w] = at;
      at += c;
    }
    __syncthreads();
    volatile uint32_t* const next = l.next;
    for (int i0 = begin; i0 < end; i0 += 512) {
      int t[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] = i0 + k * 64 + lane < end ? tokens[i0 + k * 64 + lane] : -1;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const bool is = of_mine(t[k]);
        const uint64_t any = __builtin_amdgcn_ballot_w64(is);
        if (any == 0) continue;
        const int lead = __builtin_amdgcn_readlane(t[k], __builtin_ctzll(any));
        uint64_t same = __builtin_amdgcn_ballot_w64(t[k] == lead);
        const uint32_t d = is ? (uint32_t)(t[k] - lo) : 0;
        if (same != any) same = of_same_id(is, d);
        if (is) {
          const uint32_t before = next[d * kSortWaves + wave], r = (uint32_t)__popcll(same & in_front);
          __builtin_amdgcn_wave_barrier();
          if (r == 0) next[d * kSortWaves + wave] = before + (uint32_t)__popcll(same);
          __builtin_amdgcn_wave_barrier();
          keys[before + r] = (uint32_t)lo + d;
          order[before + r] = (uint32_t)(i0 + k * 64 + lane);
        }
      }
    }
  }
  if ((int)blockIdx.x == (int)gridDim.x - 1)  // behind the last token: none
    for (int64_t i = (int64_t)base + all + tid; i < T; i += kSortThreads) keys[i] = (uint32_t)V;
  if (fill.blocks) {
    const int shift = 6 - fill.lanes_log2, sub = lane & ((1 << fill.lanes_log2) - 1);
    for (int r = (wave << shift) + (lane >> fill.lanes_log2); r < own_ids; r += kSortWaves << shift)
      if (!(l.has[r >> 6] >> (r & 63) & 1)) zero_row(fill, (int64_t)lo + r, sub);
  }
}

// The radix sort: a workgroup a tile.  counts[tile][digit] of one pass; first pass: the keys are the tokens.
__global__ __launch_bounds__(kSortThreads) void embed_count_kernel(const int32_t* tokens, const uint32_t* keys, int T, int V, int shift,
                                                                   int tiles, uint32_t* counts, Fill fill) {
  __shared__ uint32_t c[kDigits];
  if ((int)blockIdx.x >= tiles) {
    fill_rows(fill, blockIdx.x - tiles);
    return;
  }
  if (threadIdx.x < kDigits) c[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kTileRounds; ++e) {
    const int64_t i = (int64_t)blockIdx.x * kTile + e * kSortThreads + threadIdx.x;
    if (i < T) {
      const uint32_t k = keys ? keys[i] : key_of(tokens[i], V);
      atomicAdd(&c[(k >> shift) & (kDigits - 1)], 1u);  // whole numbers: the order does not matter
    }
  }
  __syncthreads();
  if (threadIdx.x < kDigits) counts[(int64_t)blockIdx.x * kDigits + threadIdx.x] = c[threadIdx.x];
}
__global__ __launch_bounds__(kSortThreads) void embed_scatter_kernel(const int32_t* tokens, const uint32_t* keys, const uint32_t* order,
                                                                     int T, int V, int shift, int tiles, const uint32_t* tile_counts,
                                                                     uint32_t* keys_out, uint32_t* order_out, Fill fill) {
  __shared__ uint32_t counts[kDigits * kSortWaves];
  __shared__ uint32_t sums[kSortWaves], start[kDigits], total[2][kDigits], earlier[2][kDigits];
  if ((int)blockIdx.x >= tiles) {
    fill_rows(fill, blockIdx.x - tiles);
    return;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  uint32_t key[kTileRounds], pos[kTileRounds], rank[kTileRounds];
#pragma unroll
  for (int e = 0; e < kTileRounds; ++e) {
    const int64_t i = (int64_t)blockIdx.x * kTile + (wave * kTileRounds + e) * 64 + lane;
    key[e] = kNoKey;
    pos[e] = (uint32_t)i;
    if (i < T) {
      key[e] = keys ? keys[i] : key_of(tokens[i], V);
      if (order) pos[e] = order[i];
    }
  }
  clear_counts(counts);
  // a digit's elements in the tiles before this one, and in all (half of the threads take every second tile)
  {
    const int d = threadIdx.x & (kDigits - 1), half = threadIdx.x >> kDigitBits;
    uint32_t all = 0, before = 0;
    for (int t = half; t < tiles; t += 2) {
      const uint32_t x = tile_counts[(int64_t)t * kDigits + d];
      all += x;
      if (t < (int)blockIdx.x) before += x;
    }
    total[half][d] = all;
    earlier[half][d] = before;
  }
  wave_ranks<kTileRounds>(key, rank, kTileRounds, shift, (LdsCounts)counts);
  __syncthreads();
  scan_counts(counts, sums);
  {
    const int d = threadIdx.x & (kDigits - 1);
    const uint32_t all = threadIdx.x < kDigits ? total[0][d] + total[1][d] : 0;
    const uint32_t smaller = before_me(all, sums);
    // a digit's first place, less what scan_counts has in front of it in this tile
    if (threadIdx.x < kDigits) start[d] = smaller + earlier[0][d] + earlier[1][d] - counts[d * kSortWaves];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kTileRounds; ++e) {
    if (key[e] == kNoKey) continue;
    const uint32_t d = (key[e] >> shift) & (kDigits - 1), to = start[d] + counts[d * kSortWaves + wave] + rank[e];
    keys_out[to] = key[e];
    order_out[to] = pos[e];
  }
}

// --------------------------------------------------------------------------------------- sums
// A thread's values of a row as they lie in memory.
template <int TYPE, int VEC>
struct RawSpan {
  typename RowType<TYPE>::Raw raw;
  typename RowType<TYPE>::T one;
  RawSpan() = default;
  __device__ __forceinline__ explicit RawSpan(const typename RowType<TYPE>::T* p) {
    if constexpr (VEC == 8) raw = RowType<TYPE>::load_raw(p);
    else one = *p;
  }
  __device__ __forceinline__ f32x8_row widen() const {
    if constexpr (VEC == 8) return RowType<TYPE>::widen(raw);
    f32x8_row x = {};
    x[0] = RowType<TYPE>::load1(&one);
    return x;
  }
};
// The thread's own values of them to the row.
template <int TYPE, int VEC>
__device__ __forceinline__ void store_span(typename RowType<TYPE>::T* row, const Span& at, const f32x8_row& y) {
  auto* p = row + at.col;
  if constexpr (VEC == 1) {
    RowType<TYPE>::store1(p, y[0]);
  } else if (at.skip == 0) {
    RowType<TYPE>::store(p, y);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= at.skip) RowType<TYPE>::store1(p + i, y[i]);
  }
}
template <int VEC>
__device__ __forceinline__ void put_part(float* p, const f32x8_row& acc) {
  if constexpr (VEC == 8) RowType<HBP_F32>::store(p, acc);
  else *p = acc[0];
}

struct Sorted {
  const uint32_t *keys, *order;
  float* part;  // [chunk][2][dim]: the end of a run that began earlier; the beginning of one that goes on
  int chunk, n_chunks;
};

// A wavefront takes 64 vectors of a chunk's rows.  The chunk's ids and places are read once, a lane each (with the neighbours on
// both sides), and handed out from there, so that a batch of rows, and what dW holds where runs begin (ADD), is under way at a time:
// with a scalar read in front of every row 32767 tokens of width 2048 took 75 us of the kernel.
template <int ROW, int TABLE, int VEC, bool ADD, int U>
__global__ __launch_bounds__(kRowThreads) void embed_sum_kernel(EmbedParams p, Sorted s, const typename RowType<ROW>::T* d_out,
                                                                typename RowType<TABLE>::T* d_table, int wpr) {
  const int64_t w = (int64_t)blockIdx.x * (kRowThreads / 64) + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int c = (int)(w / wpr), lane = threadIdx.x & 63, n_vec = VEC == 8 ? (p.dim + 7) / 8 : p.dim;
  const int v = (int)(w - (int64_t)c * wpr) * 64 + lane;
  if (c >= s.n_chunks) return;
  const bool mine = v < n_vec;  // the other lanes stay: their registers hold ids and places too
  const int first = c * s.chunk, m = min(s.chunk, p.T - first);
  // lane l: entry l - 1 of the chunk
  const int i = first - 1 + lane;
  const uint32_t none = (uint32_t)p.V;
  uint32_t key = none, place = 0;
  if (i >= 0 && i < p.T && lane <= m + 1) {
    key = s.keys[i];
    if (lane >= 1 && lane <= m && key != none) place = s.order[i];
  }
  const int n = __popcll(__builtin_amdgcn_ballot_w64(lane >= 1 && lane <= m && key != none));  // those that are none come last
  if (n == 0) return;
  const uint32_t before = __shfl_up(key, 1, 64);
  const uint64_t begins = __builtin_amdgcn_ballot_w64(lane >= 1 && lane <= n && key != before) >> 1;  // bit e: entry e begins a run
  const bool goes_on = n == m && __builtin_amdgcn_readlane(key, m + 1) == __builtin_amdgcn_readlane(key, m);
  const Span at = span_of<VEC>(min(v, n_vec - 1), p.dim);
  bool from_before = !(begins & 1);
  f32x8_row acc = {}, old = {};
  uint32_t cur = __builtin_amdgcn_readlane(key, 1);
  auto end_run = [&](bool goes_on) {
    if (!mine) return;
    if (from_before || goes_on) put_part<VEC>(s.part + ((int64_t)c * 2 + (from_before ? 0 : 1)) * p.dim + at.col, acc);
    else store_span<TABLE, VEC>(d_table + (int64_t)cur * p.table_st, at, ADD ? old + acc * p.scale : acc * p.scale);
  };
  for (int e0 = 0; e0 < n; e0 += U) {
    RawSpan<ROW, VEC> x[U];
    RawSpan<TABLE, VEC> had[ADD ? U : 1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = min(e0 + u, n - 1);
      x[u] = RawSpan<ROW, VEC>(d_out + (int64_t)(uint32_t)__builtin_amdgcn_readlane(place, e + 1) * p.row_st + at.col);
      if (ADD && (begins >> e & 1))
        had[u] = RawSpan<TABLE, VEC>(d_table + (int64_t)(uint32_t)__builtin_amdgcn_readlane(key, e + 1) * p.table_st + at.col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = e0 + u;
      if (e >= n) break;
      if (begins >> e & 1) {
        if (e > 0) {
          end_run(false);
          from_before = false;
        }
        cur = __builtin_amdgcn_readlane(key, e + 1);
        acc = f32x8_row{};
        if (ADD) old = had[ADD ? u : 0].widen();
      }
      acc += x[u].widen();
    }
  }
  end_run(goes_on);
}

// The runs that go beyond their chunk: the parts in the chunks' order.
//
// A run over fewer than kLongRun chunks behind its first: a wavefront has 64 vectors of it, and looks from every chunk whether one
// begins there.  A longer one (a filler's id may have half of the tokens) covers some chunk whose number is a multiple of kLongRun, and
// is found from the first of these: a workgroup has 16 vectors of it and sums 16 stretches of the parts side by side, in order in
// the end.  131072 tokens of width 4096, half of them one id: 296 us with a wavefront for it, 35.
constexpr int kLongRun = 64, kLongStretches = 16, kLongVectors = 16;
template <int TABLE, int VEC, bool ADD>
__device__ __forceinline__ void add_run(const EmbedParams& p, typename RowType<TABLE>::T* d_table, uint32_t k, const Span& at, const f32x8_row& acc,
                                        const RawSpan<TABLE, VEC>& had) {
  store_span<TABLE, VEC>(d_table + (int64_t)k * p.table_st, at, ADD ? had.widen() + acc * p.scale : acc * p.scale);
}
// parts [from, to) of the run that begins in chunk c; part 0 is that chunk's end, the others are their chunks' beginnings
template <int VEC>
__device__ __forceinline__ f32x8_row sum_parts(const Sorted& s, int dim, int c, int col, int from, int to) {
  constexpr int U = 16;
  const float* part = s.part + (int64_t)c * 2 * dim + col;
  f32x8_row acc = {};
  for (int i = from; i < to; i += U) {
    f32x8_row x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      x[u] = i + u < to ? load_span<HBP_F32, VEC>(part + (i + u == 0 ? (int64_t)dim : (int64_t)(i + u) * 2 * dim)) : f32x8_row{};
#pragma unroll
    for (int u = 0; u < U; ++u) acc += x[u];
  }
  return acc;
}
template <int TABLE, int VEC, bool ADD>
__global__ __launch_bounds__(kRowThreads) void embed_join_kernel(EmbedParams p, Sorted s, typename RowType<TABLE>::T* d_table, int wpr, int long_groups) {
  __shared__ f32x8_row sums[kLongStretches][kLongVectors];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n_vec = VEC == 8 ? (p.dim + 7) / 8 : p.dim;
  if ((int)blockIdx.x < long_groups) {
    const int per_run = (n_vec + kLongVectors - 1) / kLongVectors, here = (blockIdx.x / (unsigned)per_run + 1) * kLongRun;
    const uint32_t k = s.keys[here * s.chunk];
    if (k >= (uint32_t)p.V || s.keys[here * s.chunk - 1] != k) return;
    // the chunk that it begins in: the nearest before this one whose first entry does not go on with it
    const int b = here - 1 - lane;
    const uint64_t begins = __builtin_amdgcn_ballot_w64(b == 0 || s.keys[b * s.chunk - 1] != k);
    if (begins == 0) return;  // further away: another multiple's
    const int c = here - 1 - __builtin_ctzll(begins);
    int last = here, end = s.n_chunks;  // the last chunk that begins with it is in [last, end)
    while (end - last > 1) {
      const int step = (end - last + 63) / 64, at = last + (lane + 1) * step;
      const int n = __popcll(__builtin_amdgcn_ballot_w64(at < end && s.keys[(at < end ? at : 0) * s.chunk] == k));
      end = min(end, last + (n + 1) * step);
      last += n * step;
    }
    const int n = last - c;
    if (n < kLongRun) return;
    const int v = (int)(blockIdx.x % (unsigned)per_run) * kLongVectors + (lane & (kLongVectors - 1)), stretch = wave * 4 + (lane >> 4);
    const Span at = span_of<VEC>(min(v, n_vec - 1), p.dim);
    const int per = (n + kLongStretches) / kLongStretches, from = stretch * per;  // of n + 1 parts
    sums[stretch][lane & (kLongVectors - 1)] = sum_parts<VEC>(s, p.dim, c, at.col, from, min(from + per, n + 1));
    __syncthreads();
    if ((int)threadIdx.x >= kLongVectors || v >= n_vec) return;
    RawSpan<TABLE, VEC> had;
    if (ADD) had = RawSpan<TABLE, VEC>(d_table + (int64_t)k * p.table_st + at.col);
    f32x8_row acc = sums[0][lane];
#pragma unroll
    for (int i = 1; i < kLongStretches; ++i) acc += sums[i][lane];
    add_run<TABLE, VEC, ADD>(p, d_table, k, at, acc, had);
    return;
  }
  const int64_t w = (int64_t)(blockIdx.x - long_groups) * (kRowThreads / 64) + wave;
  const int c = (int)(w / wpr);
  if (c + 1 >= s.n_chunks) return;  // nothing goes beyond the last one
  const int first = c * s.chunk, next = first + s.chunk;
  const uint32_t k = s.keys[next - 1];
  if (k >= (uint32_t)p.V || s.keys[next] != k) return;
  if (s.keys[first] == k && first > 0 && s.keys[first - 1] == k) return;  // it began earlier
  const int b = c + 1 + lane;
  const uint64_t in = __builtin_amdgcn_ballot_w64(b < s.n_chunks && s.keys[(b < s.n_chunks ? b : 0) * s.chunk] == k);
  const int n = __popcll(in);  // chunks behind this one that begin with the run
  if (n == kLongRun) return;
  const int v = (int)(w - (int64_t)c * wpr) * 64 + lane;
  if (v >= n_vec) return;
  const Span at = span_of<VEC>(v, p.dim);
  RawSpan<TABLE, VEC> had;
  if (ADD) had = RawSpan<TABLE, VEC>(d_table + (int64_t)k * p.table_st + at.col);
  add_run<TABLE, VEC, ADD>(p, d_table, k, at, sum_parts<VEC>(s, p.dim, c, at.col, 0, n + 1), had);
}

template <int TABLE, int ROW, int VEC>
void lookup(const EmbedParams& p, const void* table, void* out, hipStream_t s) {
  const int log2_tpr = log2_threads_per_row(n_vectors(p.dim)), per_pass = kRowThreads >> log2_tpr;
  const int64_t passes = ((int64_t)p.T + per_pass - 1) / per_pass;
  const auto* w = (const typename RowType<TABLE>::T*)table;
  auto* y = (typename RowType<ROW>::T*)out;
  if (passes >= 8 * 1024)
    hipLaunchKernelGGL((embed_lookup_kernel<TABLE, ROW, VEC, 8>), dim3((unsigned)((passes + 7) / 8)), dim3(kRowThreads), 0, s, p, w, y, log2_tpr);
  else
    hipLaunchKernelGGL((embed_lookup_kernel<TABLE, ROW, VEC, 1>), dim3((unsigned)passes), dim3(kRowThreads), 0, s, p, w, y, log2_tpr);
}

template <int ROW, int TABLE, int VEC, bool ADD>
int sums(const EmbedParams& p, const Sorted& srt, const void* d_out, void* d_table, hipStream_t s) {
  const int wpr = waves_per_row(n_vectors(p.dim)), per_group = kRowThreads / 64;
  const int64_t groups = ((int64_t)srt.n_chunks * wpr + per_group - 1) / per_group;
  if (groups > 0x7fffffff) return (int)hipErrorInvalidValue;
  const dim3 grid((unsigned)groups);
  auto* w = (typename RowType<TABLE>::T*)d_table;
  hipLaunchKernelGGL((embed_sum_kernel<ROW, TABLE, VEC, ADD, 8>), grid, dim3(kRowThreads), 0, s, p, srt, (const typename RowType<ROW>::T*)d_out, w, wpr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || srt.n_chunks < 2) return (int)e;
  const int64_t long_groups = (int64_t)((srt.n_chunks - 1) / kLongRun) * ((n_vectors(p.dim) + kLongVectors - 1) / kLongVectors);
  if (long_groups + groups > 0x7fffffff) return (int)hipErrorInvalidValue;
  hipLaunchKernelGGL((embed_join_kernel<TABLE, VEC, ADD>), dim3((unsigned)(long_groups + groups)), dim3(kRowThreads), 0, s, p, srt, w, wpr, (int)long_groups);
  return (int)hipGetLastError();
}
template <int ROW, int TABLE>
int sums(const EmbedParams& p, const Sorted& srt, const void* d_out, void* d_table, bool accumulate, hipStream_t s) {
  if (p.dim >= 8) return accumulate ? sums<ROW, TABLE, 8, true>(p, srt, d_out, d_table, s) : sums<ROW, TABLE, 8, false>(p, srt, d_out, d_table, s);
  return accumulate ? sums<ROW, TABLE, 1, true>(p, srt, d_out, d_table, s) : sums<ROW, TABLE, 1, false>(p, srt, d_out, d_table, s);
}

int group(const EmbedParams& p, int bins, uint32_t* keys, uint32_t* order, const Fill& fill, hipStream_t s) {
  static LdsLimitDone done;
  if (const int e = raise_lds_limit((const void*)embed_group_kernel, (int)sizeof(GroupLds), done)) return e;
  hipLaunchKernelGGL(embed_group_kernel, dim3((unsigned)((p.V + (int64_t)bins - 1) / bins)), dim3(kSortThreads), sizeof(GroupLds), s, p.tokens, p.T, p.V, bins,
                     keys, order, fill);
  return (int)hipGetLastError();
}

size_t up(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int launch_embed_fwd(const EmbedParams& p, int table_type, int row_type, const void* table, void* out, hipStream_t s) {
  const bool wide = p.dim >= 8;
  if (table_type == HBP_BF16 && row_type == HBP_BF16) wide ? lookup<HBP_BF16, HBP_BF16, 8>(p, table, out, s) : lookup<HBP_BF16, HBP_BF16, 1>(p, table, out, s);
  else if (table_type == HBP_BF16) wide ? lookup<HBP_BF16, HBP_F32, 8>(p, table, out, s) : lookup<HBP_BF16, HBP_F32, 1>(p, table, out, s);
  else if (row_type == HBP_BF16) wide ? lookup<HBP_F32, HBP_BF16, 8>(p, table, out, s) : lookup<HBP_F32, HBP_BF16, 1>(p, table, out, s);
  else wide ? lookup<HBP_F32, HBP_F32, 8>(p, table, out, s) : lookup<HBP_F32, HBP_F32, 1>(p, table, out, s);
  return (int)hipGetLastError();
}

EmbedBwdLayout embed_bwd_layout(int32_t T, int32_t V, int32_t dim) {
  EmbedBwdLayout l;
  l.chunk = T <= kSmallChunks ? 16 : 32;
  l.n_chunks = (T + l.chunk - 1) / l.chunk;
  const size_t ints = up((size_t)T * 4), tiles = (size_t)(T / kTile + 1);
  l.keys_off[0] = 0;
  l.order_off[0] = ints;
  const bool one = group_bins(T, V) != 0;  // sorted where it ends
  l.keys_off[1] = one ? 0 : 2 * ints;
  l.order_off[1] = one ? ints : 3 * ints;
  l.hist_off = one ? 2 * ints : 4 * ints;
  l.part_off = l.hist_off + (one ? 0 : up(tiles * kDigits * 4));
  // fewer tokens never need more: a workspace for the longest pack serves all
  const size_t parts = (size_t)(T <= kSmallChunks ? l.n_chunks : l.n_chunks > kSmallChunks / 16 ? l.n_chunks : kSmallChunks / 16);
  l.total = l.part_off + up(parts * 2 * (size_t)dim * 4);
  return l;
}

int launch_embed_bwd(const EmbedParams& p, int table_type, int row_type, const void* d_out, void* d_table, bool accumulate,
                     char* ws, hipStream_t s) {
  const EmbedBwdLayout l = embed_bwd_layout(p.T, p.V, p.dim);
  const int es = table_type == HBP_BF16 ? 2 : 4, bits = key_bits(p.V);
  uint32_t* keys[2] = {(uint32_t*)(ws + l.keys_off[0]), (uint32_t*)(ws + l.keys_off[1])};
  uint32_t* order[2] = {(uint32_t*)(ws + l.order_off[0]), (uint32_t*)(ws + l.order_off[1])};
  Fill fill{(char*)d_table, p.table_st * es, (int64_t)p.dim * es, p.V, 0, 1, 0, fill_lanes_log2((int64_t)p.dim * es)};
  // workgroups of 16 wavefronts, a row a wavefront at a time
  const int fill_blocks = accumulate ? 0 : (int)((p.V + kSortWaves - 1) / kSortWaves < 2048 ? (p.V + kSortWaves - 1) / kSortWaves : 2048);
  int at = 0;
  if (p.T == 0 && accumulate) return 0;
  if (const int bins = group_bins(p.T, p.V)) {
    fill.blocks = accumulate ? 0 : 1;
    const int e = group(p, bins, keys[0], order[0], fill, s);
    if (e || p.T == 0) return e;
  } else {
    const int tiles = (p.T + kTile - 1) / kTile, passes = (bits + kDigitBits - 1) / kDigitBits;
    uint32_t* hist = (uint32_t*)(ws + l.hist_off);
    fill.parts = 2 * passes;
    fill.blocks = (fill_blocks + fill.parts - 1) / fill.parts;
    for (int pass = 0; pass < passes; ++pass) {
      const uint32_t* from = pass ? keys[at] : nullptr;
      const int shift = pass * kDigitBits, to = at ^ 1;
      fill.part = 2 * pass;
      hipLaunchKernelGGL(embed_count_kernel, dim3(tiles + fill.blocks), dim3(kSortThreads), 0, s, p.tokens, from, p.T, p.V, shift, tiles, hist, fill);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return (int)e;
      fill.part = 2 * pass + 1;
      hipLaunchKernelGGL(embed_scatter_kernel, dim3(tiles + fill.blocks), dim3(kSortThreads), 0, s, p.tokens, from, pass ? order[at] : nullptr,
                         p.T, p.V, shift, tiles, hist, keys[to], order[to], fill);
      e = hipGetLastError();
      if (e != hipSuccess) return (int)e;
      at = to;
    }
  }
  const Sorted srt{keys[at], order[at], (float*)(ws + l.part_off), l.chunk, l.n_chunks};
  if (row_type == HBP_BF16)
    return table_type == HBP_BF16 ? sums<HBP_BF16, HBP_BF16>(p, srt, d_out, d_table, accumulate, s) : sums<HBP_BF16, HBP_F32>(p, srt, d_out, d_table, accumulate, s);
  return table_type == HBP_BF16 ? sums<HBP_F32, HBP_BF16>(p, srt, d_out, d_table, accumulate, s) : sums<HBP_F32, HBP_F32>(p, srt, d_out, d_table, accumulate, s);
}

}  // namespace hbp
