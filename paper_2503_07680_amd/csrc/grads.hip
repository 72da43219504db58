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
#include "rows.hpp"

namespace hbp {

namespace {

constexpr int kThreads = 256;

// the tensor that chunk c of the batch lies in
__device__ __forceinline__ int tensor_of(const GradBatch& b, uint32_t c) {
  int lo = 0, hi = b.n;  // first_chunk[lo] <= c < first_chunk[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.first_chunk[mid] <= c) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int TYPE>
__device__ __forceinline__ double chunk_sumsq(const void* tensor, int64_t first, int64_t n) {
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
  constexpr int PASSES = (int)(kGradChunk / (kThreads * 8));
  if (n == kGradChunk) {
    typename R::Raw x[PASSES];
#pragma unroll
    for (int u = 0; u < PASSES; ++u) x[u] = R::load_raw(p + 8 * (u * kThreads + (int)threadIdx.x));
#pragma unroll
    for (int u = 0; u < PASSES; ++u) add(x[u]);
  } else {
    const int whole = (int)(n / 8);
    for (int i = threadIdx.x; i < whole; i += kThreads) add(R::load_raw(p + 8 * i));
    const int i = whole * 8 + (int)threadIdx.x;
    if (i < (int)n) {
      const double x = R::load1(p + i);
      q0 = fma(x, x, q0);
    }
  }
  return q0 + q1;
}

__device__ __forceinline__ double group_sum(double q, double* lds) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) q += __shfl_xor(q, d, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = q;
  __syncthreads();
  double s = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += lds[w];
  return s;
}

__global__ __launch_bounds__(kThreads) void grad_sumsq_kernel(GradBatch b, double* partial) {
  __shared__ double lds[kThreads / 64];
  const uint32_t n_chunks = b.first_chunk[b.n];
  double q = 0;
  for (uint32_t c = blockIdx.x; c < n_chunks; c += gridDim.x) {
    const int t = tensor_of(b, c);
    const int64_t first = (int64_t)(c - b.first_chunk[t]) * kGradChunk, left = b.size[t] - first, n = left < kGradChunk ? left : kGradChunk;
    q += b.type[t] == HBP_BF16 ? chunk_sumsq<HBP_BF16>(b.in[t], first, n) : chunk_sumsq<HBP_F32>(b.in[t], first, n);
  }
  q = group_sum(q, lds);
  if (threadIdx.x == 0) partial[blockIdx.x] = q;
}

__global__ __launch_bounds__(1024) void grad_total_kernel(const double* partial, int n, double* sumsq, bool accumulate) {
  __shared__ double lds[16];
  double q = 0;
  for (int i = threadIdx.x; i < n; i += 1024) q += partial[i];
  q = group_sum(q, lds);
  if (threadIdx.x == 0) *sumsq = accumulate ? *sumsq + q : q;
}

template <int TYPE>
__device__ __forceinline__ void chunk_clip(const void* in, void* out, int64_t first, int64_t n, float factor) {
  typedef RowType<TYPE> R;
  const auto* p = (const typename R::T*)in + first;
  auto* o = (typename R::T*)out + first;
  constexpr int PASSES = (int)(kGradChunk / (kThreads * 8));
  if (n == kGradChunk) {
    typename R::Raw x[PASSES];
#pragma unroll
    for (int u = 0; u < PASSES; ++u) x[u] = R::load_raw(p + 8 * (u * kThreads + (int)threadIdx.x));
#pragma unroll
    for (int u = 0; u < PASSES; ++u) R::store(o + 8 * (u * kThreads + (int)threadIdx.x), R::widen(x[u]) * factor);
  } else {
    const int whole = (int)(n / 8);
    for (int i = threadIdx.x; i < whole; i += kThreads) R::store(o + 8 * i, R::widen(R::load_raw(p + 8 * i)) * factor);
    const int i = whole * 8 + (int)threadIdx.x;
    if (i < (int)n) R::store1(o + i, R::load1(p + i) * factor);
  }
}

__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradBatch b, const double* sumsq, float max_norm, bool in_place, float* norm_out) {
  const double norm = sqrt(*sumsq);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const bool clips = norm > (double)max_norm && norm <= 1.7976931348623157e308;  // not where it is infinite, or no number
  if (!clips && in_place) return;
  const float factor = clips ? (float)((double)max_norm / norm) : 1.f;
  const uint32_t n_chunks = b.first_chunk[b.n];
  for (uint32_t c = blockIdx.x; c < n_chunks; c += gridDim.x) {
    const int t = tensor_of(b, c);
    const int64_t first = (int64_t)(c - b.first_chunk[t]) * kGradChunk, left = b.size[t] - first, n = left < kGradChunk ? left : kGradChunk;
    if (b.type[t] == HBP_BF16) chunk_clip<HBP_BF16>(b.in[t], b.out[t], first, n, factor);
    else chunk_clip<HBP_F32>(b.in[t], b.out[t], first, n, factor);
  }
}

}  // namespace

int launch_grad_sumsq(const GradBatch& b, int groups, double* partial, hipStream_t s) {
  hipLaunchKernelGGL(grad_sumsq_kernel, dim3(groups), dim3(kThreads), 0, s, b, partial);
  return (int)hipGetLastError();
}
int launch_grad_total(const double* partial, int n, double* sumsq, bool accumulate, hipStream_t s) {
  hipLaunchKernelGGL(grad_total_kernel, dim3(1), dim3(1024), 0, s, partial, n, sumsq, accumulate);
  return (int)hipGetLastError();
}
int launch_grad_clip(const GradBatch& b, int groups, const double* sumsq, float max_norm, bool in_place, float* norm_out, hipStream_t s) {
  hipLaunchKernelGGL(grad_clip_kernel, dim3(groups), dim3(kThreads), 0, s, b, sumsq, max_norm, in_place, norm_out);
  return (int)hipGetLastError();
}

}  // namespace hbp
