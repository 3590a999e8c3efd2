// The global gradient norm over many tensors, and clipping by it:
//   S = sum of g^2 over the finite entries (64 bits), B = number of the others
//   c = min(1, max_norm / (sqrt(S) + eps)), dst = c * src
// The tensors' addresses and sizes travel as kernel arguments, kClipTensors to a launch, so a call keeps nothing and can be
// captured.  Tensors are cut into chunks of kClipChunk entries; a launch's workgroups take its chunks in turn.
#pragma once
#include "common.h"
#include "pipeline_ends.h"

namespace varuna {

constexpr int kClipTensors = 96;
constexpr int kClipChunk = 8192;
constexpr int kClipBlocks = 1024;

struct ClipJobs {
  const void* src[kClipTensors];
  void* dst[kClipTensors];
  int64_t count[kClipTensors];
  uint32_t first[kClipTensors + 1];  // chunk at which the tensor begins
  uint8_t bf16[kClipTensors];        // 1: src is bf16, 2: dst is
  int32_t n;
};

__device__ __forceinline__ int job_of(const ClipJobs& j, uint32_t chunk) {
  int lo = 0, hi = j.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (j.first[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float load_any(const void* p, int64_t i, bool b) {
  return b ? to_f32(static_cast<const bf16*>(p)[i]) : static_cast<const float*>(p)[i];
}

__global__ __launch_bounds__(256) void grad_norm_partial_kernel(ClipJobs j, double* __restrict__ partial) {
  __shared__ double ss[256], sb[256];
  double s = 0.0, bad = 0.0;
  for (uint32_t c = blockIdx.x; c < j.first[j.n]; c += gridDim.x) {
    const int k = job_of(j, c);
    const int64_t begin = (int64_t)(c - j.first[k]) * kClipChunk;
    const int64_t end = begin + kClipChunk < j.count[k] ? begin + kClipChunk : j.count[k];
    for (int64_t i = begin + threadIdx.x; i < end; i += 256) {
      const float v = load_any(j.src[k], i, j.bf16[k] & 1);
      if (isfinite(v)) s += (double)v * (double)v; else bad += 1.0;
    }
  }
  ss[threadIdx.x] = s; sb[threadIdx.x] = bad;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) { ss[threadIdx.x] += ss[threadIdx.x + w]; sb[threadIdx.x] += sb[threadIdx.x + w]; }
    __syncthreads();
  }
  if (threadIdx.x == 0) { partial[2 * blockIdx.x] = ss[0]; partial[2 * blockIdx.x + 1] = sb[0]; }
}

__global__ __launch_bounds__(256) void grad_norm_final_kernel(const double* __restrict__ partial, int n, double* __restrict__ sum_sq,
                                                              float* __restrict__ nonfinite) {
  __shared__ double ss[256], sb[256];
  double s = 0.0, bad = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) { s += partial[2 * i]; bad += partial[2 * i + 1]; }
  ss[threadIdx.x] = s; sb[threadIdx.x] = bad;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) { ss[threadIdx.x] += ss[threadIdx.x + w]; sb[threadIdx.x] += sb[threadIdx.x + w]; }
    __syncthreads();
  }
  if (threadIdx.x == 0) { *sum_sq = ss[0]; *nonfinite = (float)sb[0]; }
}

__global__ __launch_bounds__(256) void grad_clip_kernel(ClipJobs j, const double* __restrict__ sum_sq, double max_norm, double eps) {
  const float by = (float)fmin(1.0, max_norm / (sqrt(*sum_sq) + eps));
  for (uint32_t c = blockIdx.x; c < j.first[j.n]; c += gridDim.x) {
    const int k = job_of(j, c);
    const int64_t begin = (int64_t)(c - j.first[k]) * kClipChunk;
    const int64_t end = begin + kClipChunk < j.count[k] ? begin + kClipChunk : j.count[k];
    for (int64_t i = begin + threadIdx.x; i < end; i += 256) {
      const float v = by * load_any(j.src[k], i, j.bf16[k] & 1);
      if (j.bf16[k] & 2) static_cast<bf16*>(j.dst[k])[i] = from_f32<bf16>(v);
      else static_cast<float*>(j.dst[k])[i] = v;
    }
  }
}

// Runs f(jobs, workgroups) for every kClipTensors tensors that are not empty.
template <typename F>
inline void clip_launches(const TensorSpan& src, const TensorSpan* dst, F f) {
  ClipJobs j;
  j.n = 0;
  uint32_t chunks = 0;
  auto flush = [&] {
    if (j.n == 0) return;
    j.first[j.n] = chunks;
    f(j, chunks < (uint32_t)kClipBlocks ? chunks : (uint32_t)kClipBlocks);
    j.n = 0;
    chunks = 0;
  };
  for (int32_t i = 0; i < src.n; ++i) {
    if (src.count[i] == 0) continue;
    j.src[j.n] = src.p[i];
    j.dst[j.n] = dst ? const_cast<void*>(dst->p[i]) : nullptr;
    j.bf16[j.n] = (uint8_t)((src.dtype[i] != 0 ? 1 : 0) | (dst && dst->dtype[i] != 0 ? 2 : 0));
    j.count[j.n] = src.count[i];
    j.first[j.n] = chunks;
    chunks += (uint32_t)((src.count[i] + kClipChunk - 1) / kClipChunk);
    if (++j.n == kClipTensors) flush();
  }
  flush();
}

size_t grad_norm_scratch_bytes(const int64_t*, int32_t n) {
  return (size_t)(n / kClipTensors + 1) * kClipBlocks * 2 * sizeof(double);
}

hipError_t launch_grad_norm(const TensorSpan& t, double* sum_sq, float* nonfinite, void* scratch, hipStream_t st) {
  double* partial = static_cast<double*>(scratch);
  int n = 0;
  clip_launches(t, nullptr, [&](const ClipJobs& j, uint32_t blocks) {
    hipLaunchKernelGGL(grad_norm_partial_kernel, dim3(blocks), dim3(256), 0, st, j, partial + 2 * (size_t)n);
    n += (int)blocks;
  });
  hipLaunchKernelGGL(grad_norm_final_kernel, dim3(1), dim3(256), 0, st, partial, n, sum_sq, nonfinite);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const TensorSpan& dst, const TensorSpan& src, const double* sum_sq, double max_norm, double eps, hipStream_t st) {
  clip_launches(src, &dst, [&](const ClipJobs& j, uint32_t blocks) {
    hipLaunchKernelGGL(grad_clip_kernel, dim3(blocks), dim3(256), 0, st, j, sum_sq, max_norm, eps);
  });
  return hipGetLastError();
}

}  // namespace varuna
