// What the embedding's and the gradients' kernels share: eight values of either type at any element's address, and the
// parameters that the C ABI hands to their launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hbp.h"

namespace hbp {

// 16-byte accesses at the alignment of an element: rows of an odd width and views into a bucket start anywhere, and the
// hardware takes such an address as it is.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8_row __attribute__((ext_vector_type(8)));
typedef float f32x8_row __attribute__((ext_vector_type(8)));

template <int TYPE>
struct RowType;
template <>
struct RowType<HBP_BF16> {
  typedef uint16_t T;
  typedef u32x4_any Raw;  // of eight values
  static __device__ __forceinline__ Raw load_raw(const T* p) { return *(const u32x4_any*)p; }
  static __device__ __forceinline__ f32x8_row widen(const Raw& r) {
    f32x8_row x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(r[i] << 16);
      x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
    return x;
  }
  static __device__ __forceinline__ float load1(const T* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ __forceinline__ Raw narrow(const f32x8_row& x) {  // to nearest, ties to even
    return __builtin_bit_cast(u32x4_any, __builtin_convertvector(x, bf16x8_row));
  }
  static __device__ __forceinline__ void store(T* p, const f32x8_row& x) { *(u32x4_any*)p = narrow(x); }
  static __device__ __forceinline__ void store_past(T* p, const f32x8_row& x) { __builtin_nontemporal_store(narrow(x), (u32x4_any*)p); }
  static __device__ __forceinline__ void store1(T* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }
};
template <>
struct RowType<HBP_F32> {
  typedef float T;
  struct Raw {
    f32x4_any lo, hi;
  };
  static __device__ __forceinline__ Raw load_raw(const T* p) { return Raw{*(const f32x4_any*)p, *(const f32x4_any*)(p + 4)}; }
  static __device__ __forceinline__ f32x8_row widen(const Raw& r) {
    return f32x8_row{r.lo[0], r.lo[1], r.lo[2], r.lo[3], r.hi[0], r.hi[1], r.hi[2], r.hi[3]};
  }
  static __device__ __forceinline__ float load1(const T* p) { return *p; }
  static __device__ __forceinline__ void store(T* p, const f32x8_row& x) {
    *(f32x4_any*)p = f32x4_any{x[0], x[1], x[2], x[3]};
    *(f32x4_any*)(p + 4) = f32x4_any{x[4], x[5], x[6], x[7]};
  }
  static __device__ __forceinline__ void store_past(T* p, const f32x8_row& x) {
    __builtin_nontemporal_store(f32x4_any{x[0], x[1], x[2], x[3]}, (f32x4_any*)p);
    __builtin_nontemporal_store(f32x4_any{x[4], x[5], x[6], x[7]}, (f32x4_any*)(p + 4));
  }
  static __device__ __forceinline__ void store1(T* p, float x) { *p = x; }
};

struct EmbedParams {
  const int32_t* tokens;
  int32_t T, V, dim;
  int64_t table_st, row_st;  // elements
  float scale;
};
int launch_embed_fwd(const EmbedParams& p, int table_type, int row_type, const void* table, void* out, hipStream_t s);

// Workspace of the embedding's gradient (offsets from its base).
struct EmbedBwdLayout {
  size_t keys_off[2], order_off[2], hist_off, part_off, total;
  int chunk, n_chunks;
};
EmbedBwdLayout embed_bwd_layout(int32_t T, int32_t V, int32_t dim);
int launch_embed_bwd(const EmbedParams& p, int table_type, int row_type, const void* d_out, void* d_table, bool accumulate,
                     char* ws, hipStream_t s);

// A list of gradients as a launch's arguments: up to N tensors (a short list has short arguments: 3.5 KB of them cost a launch
// 1.6 us on the host).  Chunks of 1 << chunk_log2 elements are dealt to the workgroups in turn.
constexpr int kGradBatch = 120, kGradFew = 24, kGradMaxGroups = 2048;
constexpr int kGradChunkLog2 = 14, kGradSmallChunkLog2 = 12;
template <int N>
struct GradBatchOf {
  const void* in[N];
  void* out[N];
  int64_t size[N];
  uint32_t first_chunk[N + 1];
  uint8_t type[N];
  int32_t n, chunk_log2;
};
typedef GradBatchOf<kGradBatch> GradBatch;
int launch_grad_sumsq(const GradBatch& b, int groups, double* partial, hipStream_t s);
int launch_grad_total(const double* partial, int n, double* sumsq, bool accumulate, hipStream_t s);
// The sum of squares: sums[0] (n = 1), or the sum of n partial ones, which goes to sumsq_out then.
struct GradNorm {
  const double* sums;
  int32_t n;
  double* sumsq_out;
  float max_norm;
  float* norm_out;  // both outputs may be null
};
int launch_grad_clip(const GradBatch& b, int groups, const GradNorm& norm, bool in_place, hipStream_t s);

}  // namespace hbp
