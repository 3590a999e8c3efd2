// The last stage's loss: cross entropy over the vocabulary with label smoothing e, and the gradient of the logits,
//   m = max_j x_j, s = sum_j exp(x_j - m), loss = (1 - e) (log s + m - x_y) + e (log s + m - mean_j x_j)
//   dx_j = g (exp(x_j - m) / s - (1 - e) [j = y] - e / V)
// A row whose target is none of [0, V) has loss 0 and gradient 0 and is not counted.
#pragma once
#include "common.h"
#include "pipeline_ends.h"

namespace varuna {

template <int THREADS> __device__ __forceinline__ float block_sum(float v, float* lds) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) v += lds[i];
  return v;
}
template <int THREADS> __device__ __forceinline__ float block_max(float v, float* lds) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) v = fmaxf(v, lds[i]);
  return v;
}

__device__ __forceinline__ int64_t target_of(const LossArgs& a, int64_t r) {
  const int64_t y = a.wide ? static_cast<const int64_t*>(a.targets)[r] : (int64_t)static_cast<const int32_t*>(a.targets)[r];
  return y >= 0 && y < a.vocab ? y : -1;
}

// One workgroup per row, which it reads three times.
template <typename T>
__global__ __launch_bounds__(256) void cross_entropy_kernel(LossArgs a) {
  __shared__ float lds[4];
  const int64_t r = blockIdx.x;
  const int64_t y = target_of(a, r);
  const T* x = static_cast<const T*>(a.logits) + r * a.ld;
  T* dx = a.dlogits ? static_cast<T*>(a.dlogits) + r * a.ldd : nullptr;
  if (y < 0) {
    if (threadIdx.x == 0) a.loss[r] = 0.f;
    if (dx)
      for (int j = threadIdx.x; j < a.vocab; j += 256) dx[j] = from_f32<T>(0.f);
    return;
  }
  float m = -INFINITY;
  for (int j = threadIdx.x; j < a.vocab; j += 256) m = fmaxf(m, to_f32(x[j]));
  m = block_max<256>(m, lds);
  float s = 0.f, total = 0.f;   // total: the mean; the values are scaled before they are summed, so that the type's lowest value as a mask does not overflow it
  const float inv_v = 1.f / (float)a.vocab;
  for (int j = threadIdx.x; j < a.vocab; j += 256) {
    const float v = to_f32(x[j]);
    s += expf(v - m);
    total += v * inv_v;
  }
  s = block_sum<256>(s, lds);
  const float eps = a.smoothing, xy = to_f32(x[y]);
  float loss = logf(s) + (m - xy);
  if (eps != 0.f) {
    total = block_sum<256>(total, lds);
    loss = (1.f - eps) * loss + eps * (logf(s) + (m - total));
  }
  __syncthreads();   // x[y] has been read
  if (threadIdx.x == 0) a.loss[r] = loss;
  if (!dx) return;
  const float g = a.scale ? a.grad_scale * *a.scale : a.grad_scale;
  for (int j = threadIdx.x; j < a.vocab; j += 256)
    dx[j] = from_f32<T>(g * (expf(to_f32(x[j]) - m) / s - eps / (float)a.vocab - (j == y ? 1.f - eps : 0.f)));
}

// out2 = sum of the losses (in 64 bits, rounded once), number of counted rows.
__global__ __launch_bounds__(1024) void loss_sum_kernel(LossArgs a) {
  __shared__ double ss[1024];
  __shared__ int sn[1024];
  double s = 0.0;
  int n = 0;
  for (int64_t r = threadIdx.x; r < a.rows; r += 1024)
    if (target_of(a, r) >= 0) { s += (double)a.loss[r]; ++n; }
  ss[threadIdx.x] = s; sn[threadIdx.x] = n;
  __syncthreads();
  for (int w = 512; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) { ss[threadIdx.x] += ss[threadIdx.x + w]; sn[threadIdx.x] += sn[threadIdx.x + w]; }
    __syncthreads();
  }
  if (threadIdx.x == 0) { a.out2[0] = (float)ss[0]; a.out2[1] = (float)sn[0]; }
}

template <typename T>
hipError_t launch_cross_entropy(const LossArgs& a, hipStream_t st) {
  if (a.rows > 0) hipLaunchKernelGGL(cross_entropy_kernel<T>, dim3((unsigned)a.rows), dim3(256), 0, st, a);
  if (a.out2) hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace varuna
