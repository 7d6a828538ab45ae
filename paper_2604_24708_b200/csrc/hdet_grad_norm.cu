// Global gradient norms over a handle's tensors: n_r = sqrt(sum of g_r^2), for every replica, or for the replicas' mean gradient.
//
// Bound by reading the gradients once.  A CTA sums one span (consecutive elements of one tensor of one replica) and leaves an fp64
// partial sum; the CTA that finishes a replica's last span adds the partial sums in a fixed order, so that there is one launch, and the
// same bits on every run whichever CTA it is.
#include <cuda_bf16.h>

#include "hdet_kernels.cuh"

namespace hdet {
namespace {

constexpr int kNormThreads = 256;
constexpr int kAhead = 8;              // 16-byte loads of a thread under way

template <typename GradT> struct Packed;      // 16 bytes of gradients, and what a mean of them is summed in
template <> struct Packed<float> { static constexpr int n = 4; using Sum = double; };
template <> struct Packed<__nv_bfloat16> { static constexpr int n = 8; using Sum = float; };

__device__ __forceinline__ void unpack16(const uint4& u, float (&g)[4]) {
  g[0] = __uint_as_float(u.x); g[1] = __uint_as_float(u.y); g[2] = __uint_as_float(u.z); g[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack16(const uint4& u, float (&g)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    g[2 * i] = __uint_as_float(w[i] << 16);
    g[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ float one(const float* p) { return __ldcs(p); }
__device__ __forceinline__ float one(const __nv_bfloat16* p) {
  return __uint_as_float((unsigned)__ldcs(reinterpret_cast<const unsigned short*>(p)) << 16);
}

// Squares are added in fp32 over 16 bytes and in fp64 from there on.  Where an fp32 square could leave its range (gradients above 1e15
// or, all of them, below 1e-15) those 16 bytes are taken in fp64, but for zeros: a table's rows without tokens are full of them.
template <int kN>
__device__ __forceinline__ double squares(const float (&g)[kN]) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < kN; ++i) s = fmaf(g[i], g[i], s);
  if (s >= 1e-30f && s <= 1e30f) return (double)s;
  unsigned bits = 0;
#pragma unroll
  for (int i = 0; i < kN; ++i) bits |= __float_as_uint(g[i]);
  if (bits << 1 == 0) return 0.0;                  // (-0, too)
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < kN; ++i) d += (double)g[i] * (double)g[i];
  return d;
}

__device__ __forceinline__ double block_sum(double x) {      // valid in thread 0
  __shared__ double s_warp[kNormThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = x;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < kNormThreads / 32; ++w) x += s_warp[w];
  return x;
}

template <typename GradT>
__device__ __forceinline__ double span_squares(const GradT* p, int len) {
  constexpr int kN = Packed<GradT>::n;
  const int head = min(len, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(GradT));
  const int vecs = (len - head) / kN;
  const uint4* v = reinterpret_cast<const uint4*>(p + head);
  double acc = 0.0;
  int j = threadIdx.x;
  for (; j + (kAhead - 1) * kNormThreads < vecs; j += kAhead * kNormThreads) {
    uint4 u[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) u[k] = __ldcs(v + j + k * kNormThreads);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float g[kN];
      unpack16(u[k], g);
      acc += squares(g);
    }
  }
  for (; j < vecs; j += kNormThreads) {
    float g[kN];
    unpack16(__ldcs(v + j), g);
    acc += squares(g);
  }
  // what lies before the first and behind the last 16-byte boundary: fewer than 2 kN elements
  const int tail = head + vecs * kN;
  if (threadIdx.x < head) { const double g = one(p + threadIdx.x); acc += g * g; }
  if (tail + (int)threadIdx.x < len) { const double g = one(p + tail + threadIdx.x); acc += g * g; }
  return acc;
}

// What a sum over replicas takes of one: in fp32 a 32nd, which changes no digit and lets no sum leave the range that the mean is in.
// to_mean makes the mean of it.
constexpr float kPart = 32.0f;
static_assert(HDET_MAX_REPLICAS <= kPart, "a sum of 32nds is at most the largest gradient");
__device__ __forceinline__ void add_part(double& sum, float g) { sum += (double)g; }
__device__ __forceinline__ void add_part(float& sum, float g) { sum = fmaf(g, 1.0f / kPart, sum); }

// The same of the mean over n replicas, summed in their order: fp32 gradients in fp64, as the update does, bf16 ones in fp32, whose rounding is
// 2^15 times finer than theirs (in fp64 the conversions took 976 us for four of the 350 M list, whose bytes take 440).
template <typename GradT>
__device__ __forceinline__ double span_mean_squares(const GradT* p, long long stride, int n, double to_mean, int len) {
  using Sum = typename Packed<GradT>::Sum;
  constexpr int kN = Packed<GradT>::n;
  const bool wide = (stride * (long long)sizeof(GradT)) % 16 == 0;
  const int head = wide ? min(len, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(GradT)) : len;
  const int vecs = (len - head) / kN;
  double acc = 0.0;
  // 16 bytes of kReplicas replicas under way (of four bf16 gradients of the 350 M list 441 us, of four fp32 ones of the 125 M list 346; with two times 16
  // bytes and fewer threads at once 493 and 353; with three replicas 483 and 371).
  constexpr int kReplicas = 4;
  for (int j = threadIdx.x; j < vecs; j += kNormThreads) {
    Sum sum[kN] = {};
    for (int r0 = 0; r0 < n; r0 += kReplicas) {
      uint4 u[kReplicas];
#pragma unroll
      for (int r = 0; r < kReplicas; ++r) {
        u[r] = make_uint4(0, 0, 0, 0);
        if (r0 + r < n) u[r] = __ldcs(reinterpret_cast<const uint4*>(p + (r0 + r) * stride + head) + j);
      }
#pragma unroll
      for (int r = 0; r < kReplicas; ++r) {
        float g[kN];
        unpack16(u[r], g);
#pragma unroll
        for (int i = 0; i < kN; ++i) add_part(sum[i], g[i]);
      }
    }
    float g[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) g[i] = (float)(sum[i] * (Sum)to_mean);
    acc += squares(g);
  }
  const auto single = [&](int e) {
    Sum sum = 0;
    for (int r = 0; r < n; ++r) add_part(sum, one(p + r * stride + e));
    const double g = (float)(sum * (Sum)to_mean);
    acc += g * g;
  };
  for (int e = threadIdx.x; e < head; e += kNormThreads) single(e);
  const int tail = head + vecs * kN;
  if (tail + (int)threadIdx.x < len) single(tail + threadIdx.x);
  return acc;
}

template <typename GradT, bool kMean>
__global__ void __launch_bounds__(kNormThreads) grad_norm_kernel(const __grid_constant__ NormPlan plan, int first, double max_norm, void* norms,
                                                                 bool norms_f64) {
  __shared__ bool s_last;
  const int row = blockIdx.y, at = first + blockIdx.x;
  const GradSpan span = plan.spans[at];
  const TensorDesc* td = plan.tensors + span.tensor;
  const long long stride = td->grad_stride;
  const GradT* p = static_cast<const GradT*>(td->grad) + span.off;
  double sum = kMean ? span_mean_squares(p, stride, plan.n_replicas, (sizeof(GradT) == 2 ? (double)kPart : 1.0) / (double)plan.n_replicas, span.len)
                     : span_squares(p + row * stride, span.len);
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    plan.partial[(long long)row * plan.n_spans + at] = sum;
    __threadfence();
    s_last = atomicAdd(plan.done + row, 1u) == (unsigned)plan.n_spans - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  const double* partial = plan.partial + (long long)row * plan.n_spans;
  sum = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < plan.n_spans; i += kNormThreads) sum += __ldcg(partial + i);
  sum = block_sum(sum);
  if (threadIdx.x != 0) return;
  plan.done[row] = 0;
  const double norm = sqrt(sum);
  // a norm that is not finite clips nothing: what is not finite in the gradient reaches the parameters, where it is reported
  const float clip = norm > max_norm && norm <= 1.7976931348623157e308 ? (float)(max_norm / norm) : 1.0f;
  for (int r = row; r < plan.n_replicas; r += plan.rows) {      // rows 1: all replicas' norm
    if (max_norm > 0.0) plan.clip[r] = clip;
    if (norms) {
      if (norms_f64) static_cast<double*>(norms)[r] = norm; else static_cast<float*>(norms)[r] = (float)norm;
    }
  }
}

}  // namespace

cudaError_t launch_grad_norm(const NormPlan& plan, int first, int count, double max_norm, void* norms, bool norms_f64, cudaStream_t stream) {
  if (count == 0) return cudaSuccess;
  const dim3 grid((unsigned)count, (unsigned)plan.rows);
  const bool bf16 = plan.grad_dtype == HDET_DTYPE_BF16;
  if (plan.mean) {
    if (bf16) grad_norm_kernel<__nv_bfloat16, true><<<grid, kNormThreads, 0, stream>>>(plan, first, max_norm, norms, norms_f64);
    else grad_norm_kernel<float, true><<<grid, kNormThreads, 0, stream>>>(plan, first, max_norm, norms, norms_f64);
  } else {
    if (bf16) grad_norm_kernel<__nv_bfloat16, false><<<grid, kNormThreads, 0, stream>>>(plan, first, max_norm, norms, norms_f64);
    else grad_norm_kernel<float, false><<<grid, kNormThreads, 0, stream>>>(plan, first, max_norm, norms, norms_f64);
  }
  return cudaGetLastError();
}

}  // namespace hdet
