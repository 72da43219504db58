// The norm of a training step's gradients over all their tensors, and clipping to it, gfx950.
//
//   q = sum g^2 over every element of every tensor;  n = sqrt(q);  out = g (m / n) where n > m and n is finite, else g
//
// Bound by memory: the factor is known only when everything has been read, so the elements are read twice and written once.
// The list of tensors goes to the kernels as their arguments, kGradBatch of them a launch: nothing is copied to the device
// in front of a step, and a captured call holds its list.  The tensors' elements are cut into chunks, dealt to the
// workgroups in turn.  Squares are added in 64 bits: no sum overflows or loses the small tensors beside the large ones, and
// the additions hide behind the loads (three vector instructions more an element).  The order of all additions is fixed by
// the list of sizes.
#include <type_traits>

#include "rows.hpp"

namespace hbp {

namespace {

constexpr int kThreads = 256;

// the tensor that chunk c of the batch lies in
template <class Batch>
__device__ __forceinline__ int tensor_of(const Batch& b, uint32_t c) {
  int lo = 0, hi = b.n;  // first_chunk[lo] <= c < first_chunk[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.first_chunk[mid] <= c) lo = mid;
    else hi = mid;
  }
  return lo;
}

// A workgroup's chunks, c0, c0 + step, ...: f(tensor, first element, elements)
template <class Batch, class F>
__device__ __forceinline__ void for_chunks(const Batch& b, bool backwards, F f) {
  const uint32_t n = b.first_chunk[b.n];
  for (uint32_t i = blockIdx.x; i < n; i += gridDim.x) {
    const uint32_t c = backwards ? n - 1 - i : i;
    const int t = tensor_of(b, c);
    const int64_t first = (int64_t)(c - b.first_chunk[t]) << b.chunk_log2, left = b.size[t] - first, chunk = (int64_t)1 << b.chunk_log2;
    f(t, first, (int)(left < chunk ? left : chunk));
  }
}

// Elements of a whole chunk in accesses of 16 bytes, a wavefront's beside each other: four or eight of them each.
template <int TYPE>
struct Quad {
  static constexpr int N = 16 / sizeof(typename RowType<TYPE>::T);
  typedef float Values __attribute__((ext_vector_type(N)));
  static __device__ __forceinline__ Values widen(const u32x4_any& r) {
    if constexpr (N == 8) return RowType<HBP_BF16>::widen(r);
    else return __builtin_bit_cast(Values, r);
  }
  static __device__ __forceinline__ u32x4_any narrow(const Values& x) {
    if constexpr (N == 8) return RowType<HBP_BF16>::narrow(x);
    else return __builtin_bit_cast(u32x4_any, x);
  }
};

template <int TYPE, int CHUNK>
__device__ __forceinline__ double chunk_sumsq(const void* tensor, int64_t first, int n) {
  typedef RowType<TYPE> R;
  const auto* p = (const typename R::T*)tensor + first;
  double q0 = 0, q1 = 0;
  auto add = [&](const typename R::Raw& raw) {
    const f32x8_row x = R::widen(raw);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      q0 = fma((double)x[j], (double)x[j], q0);
      q1 = fma((double)x[j + 1], (double)x[j + 1], q1);
    }
  };
  typedef Quad<TYPE> Q;
  constexpr int PASSES = CHUNK / (kThreads * Q::N);
  if (n == CHUNK) {
    u32x4_any raw[PASSES];
#pragma unroll
    for (int u = 0; u < PASSES; ++u) raw[u] = *(const u32x4_any*)(p + Q::N * (u * kThreads + (int)threadIdx.x));
#pragma unroll
    for (int u = 0; u < PASSES; ++u) {
      const auto x = Q::widen(raw[u]);
#pragma unroll
      for (int j = 0; j < Q::N; j += 2) {
        q0 = fma((double)x[j], (double)x[j], q0);
        q1 = fma((double)x[j + 1], (double)x[j + 1], q1);
      }
    }
  } else {
    const int whole = n / 8;
    for (int i = threadIdx.x; i < whole; i += kThreads) add(R::load_raw(p + 8 * i));
    const int i = whole * 8 + (int)threadIdx.x;
    if (i < n) {
      const double x = R::load1(p + i);
      q0 = fma(x, x, q0);
    }
  }
  return q0 + q1;
}

// sum over the workgroup, the same in every thread; lds: a double a wavefront
__device__ __forceinline__ double group_sum(double q, double* lds) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) q += __shfl_xor(q, d, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = q;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}
// sum of n partial ones, in an order that goes by n alone; eight loads under way
__device__ __forceinline__ double sum_of_partials(const double* partial, int n, double* lds) {
  double q = 0;
  for (int i = threadIdx.x; i < n; i += 8 * kThreads) {
    double x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = i + u * kThreads < n ? partial[i + u * kThreads] : 0.0;
#pragma unroll
    for (int u = 0; u < 8; ++u) q += x[u];
  }
  return group_sum(q, lds);
}

template <int N, int CHUNK>
__global__ __launch_bounds__(kThreads) void grad_sumsq_kernel(GradBatchOf<N> b, double* partial) {
  __shared__ double lds[kThreads / 64];
  double q = 0;
  for_chunks(b, false, [&](int t, int64_t first, int n) {
    q += b.type[t] == HBP_BF16 ? chunk_sumsq<HBP_BF16, CHUNK>(b.in[t], first, n) : chunk_sumsq<HBP_F32, CHUNK>(b.in[t], first, n);
  });
  q = group_sum(q, lds);
  if (threadIdx.x == 0) partial[blockIdx.x] = q;
}

__global__ __launch_bounds__(kThreads) void grad_total_kernel(const double* partial, int n, double* sumsq, bool accumulate) {
  __shared__ double lds[kThreads / 64];
  const double q = sum_of_partials(partial, n, lds);
  if (threadIdx.x == 0) *sumsq = accumulate ? *sumsq + q : q;
}

template <int TYPE, int CHUNK>
__device__ __forceinline__ void chunk_clip(const void* in, void* out, int64_t first, int n, float factor) {
  typedef RowType<TYPE> R;
  const auto* p = (const typename R::T*)in + first;
  auto* o = (typename R::T*)out + first;
  typedef Quad<TYPE> Q;
  constexpr int PASSES = CHUNK / (kThreads * Q::N);
  if (n == CHUNK) {
    u32x4_any raw[PASSES];
#pragma unroll
    for (int u = 0; u < PASSES; ++u) raw[u] = *(const u32x4_any*)(p + Q::N * (u * kThreads + (int)threadIdx.x));
    // Long lists go past the caches: 1.4 billion bf16 elements 1577 -> 1538 us, 150 million fp32 365 -> 341 (383 with the 32 bytes of
    // eight elements a thread in two stores).  Short ones are left in them for what reads them next.
#pragma unroll
    for (int u = 0; u < PASSES; ++u) {
      const u32x4_any y = Q::narrow(Q::widen(raw[u]) * factor);
      auto* const to = (u32x4_any*)(o + Q::N * (u * kThreads + (int)threadIdx.x));
      if constexpr (CHUNK == 1 << kGradChunkLog2) __builtin_nontemporal_store(y, to);
      else *to = y;
    }
  } else {
    const int whole = n / 8;
    for (int i = threadIdx.x; i < whole; i += kThreads) R::store(o + 8 * i, R::widen(R::load_raw(p + 8 * i)) * factor);
    const int i = whole * 8 + (int)threadIdx.x;
    if (i < n) R::store1(o + i, R::load1(p + i) * factor);
  }
}

// The chunks are taken from the last one on: what the sum of squares has read last is still in the cache of 256 MB.
template <int N, int CHUNK>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradBatchOf<N> b, GradNorm g, bool in_place) {
  __shared__ double lds[kThreads / 64];
  const double q = g.n == 1 ? *g.sums : sum_of_partials(g.sums, g.n, lds), norm = sqrt(q);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (g.n != 1 && g.sumsq_out) *g.sumsq_out = q;
    if (g.norm_out) *g.norm_out = (float)norm;
  }
  const bool clips = norm > (double)g.max_norm && norm <= 1.7976931348623157e308;  // not where it is infinite, or no number
  if (!clips && in_place) return;
  const float factor = clips ? (float)((double)g.max_norm / norm) : 1.f;
  for_chunks(b, true, [&](int t, int64_t first, int n) {
    if (b.type[t] == HBP_BF16) chunk_clip<HBP_BF16, CHUNK>(b.in[t], b.out[t], first, n, factor);
    else chunk_clip<HBP_F32, CHUNK>(b.in[t], b.out[t], first, n, factor);
  });
}

template <int N>
GradBatchOf<N> shortened(const GradBatch& b) {
  GradBatchOf<N> f;
  for (int i = 0; i < b.n; ++i) {
    f.in[i] = b.in[i];
    f.out[i] = b.out[i];
    f.size[i] = b.size[i];
    f.type[i] = b.type[i];
    f.first_chunk[i] = b.first_chunk[i];
  }
  f.first_chunk[b.n] = b.first_chunk[b.n];
  f.n = b.n;
  f.chunk_log2 = b.chunk_log2;
  return f;
}
// f(batch of the shortest kind that holds it, its chunks' size as a constant)
template <class F>
int with_batch(const GradBatch& b, F f) {
  typedef std::integral_constant<int, 1 << kGradChunkLog2> Large;
  typedef std::integral_constant<int, 1 << kGradSmallChunkLog2> Small;
  const bool small = b.chunk_log2 == kGradSmallChunkLog2;
  if (b.n <= kGradFew) {
    const auto few = shortened<kGradFew>(b);
    if (small) f(few, Small{});
    else f(few, Large{});
  } else {
    if (small) f(b, Small{});
    else f(b, Large{});
  }
  return (int)hipGetLastError();
}

}  // namespace

int launch_grad_sumsq(const GradBatch& b, int groups, double* partial, hipStream_t s) {
  return with_batch(b, [&](const auto& batch, auto chunk) {
    constexpr int N = sizeof(batch.in) / sizeof(batch.in[0]);
    hipLaunchKernelGGL((grad_sumsq_kernel<N, decltype(chunk)::value>), dim3(groups), dim3(kThreads), 0, s, batch, partial);
  });
}
int launch_grad_total(const double* partial, int n, double* sumsq, bool accumulate, hipStream_t s) {
  hipLaunchKernelGGL(grad_total_kernel, dim3(1), dim3(kThreads), 0, s, partial, n, sumsq, accumulate);
  return (int)hipGetLastError();
}
int launch_grad_clip(const GradBatch& b, int groups, const GradNorm& norm, bool in_place, hipStream_t s) {
  return with_batch(b, [&](const auto& batch, auto chunk) {
    constexpr int N = sizeof(batch.in) / sizeof(batch.in[0]);
    hipLaunchKernelGGL((grad_clip_kernel<N, decltype(chunk)::value>), dim3(groups), dim3(kThreads), 0, s, batch, norm, in_place);
  });
}

}  // namespace hbp
