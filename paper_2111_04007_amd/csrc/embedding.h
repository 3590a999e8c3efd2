// The first stage's embedding: out[t] = scale * table[id_t] + places[position_t], and the table's fp32 gradient.
#pragma once
#include "common.h"
#include "pipeline_ends.h"

namespace varuna {

// The id of row t, or -1 where it is none of [0, n).
__device__ __forceinline__ int64_t row_id(const IdArgs& a, int64_t t, int64_t n) {
  const int64_t v = a.p == nullptr ? t % a.period : (a.wide ? static_cast<const int64_t*>(a.p)[t] : (int64_t)static_cast<const int32_t*>(a.p)[t]);
  return v >= 0 && v < n ? v : -1;
}

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(EmbedArgs a) {
  const int64_t t = blockIdx.x;
  const int64_t id = row_id(a.ids, t, a.vocab);
  const int64_t at = a.places ? row_id(a.positions, t, a.n_positions) : -1;
  const T* e = static_cast<const T*>(a.table) + (id < 0 ? 0 : id * a.h);
  const T* p = static_cast<const T*>(a.places) + (at < 0 ? 0 : at * a.h);
  T* out = static_cast<T*>(a.out) + t * a.h;
  for (int j = threadIdx.x; j < a.h; j += 256) {
    float v = id < 0 ? 0.f : a.scale * to_f32(e[j]);
    if (at >= 0) v += to_f32(p[j]);
    out[j] = from_f32<T>(v);
  }
}

template <typename T>
hipError_t launch_embedding_fwd(const EmbedArgs& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  hipLaunchKernelGGL(embedding_fwd_kernel<T>, dim3((unsigned)a.rows), dim3(256), 0, st, a);
  return hipGetLastError();
}

// One wave per row of the table: it looks at the ids of all rows, 64 at a time, and sums those that are its own in order.
template <typename T>
__global__ __launch_bounds__(64) void embedding_bwd_kernel(EmbedGradArgs a) {
  const int64_t v = blockIdx.x;
  const int lane = threadIdx.x;
  float* out = a.dtable + v * a.h;
  for (int j0 = 0; j0 < a.h; j0 += 64) {
    const int j = j0 + lane;
    float s = 0.f;
    bool any = false;
    for (int64_t t0 = 0; t0 < a.rows; t0 += 64) {
      const int64_t t = t0 + lane;
      uint64_t own = __ballot(t < a.rows && row_id(a.ids, t, a.vocab) == v);
      for (; own != 0; own &= own - 1) {
        any = true;
        if (j < a.h) s += to_f32(static_cast<const T*>(a.dy)[(t0 + __builtin_ctzll(own)) * a.h + j]);
      }
    }
    if (j >= a.h) continue;
    if (!a.accumulate) out[j] = a.scale * s;
    else if (any) out[j] += a.scale * s;
  }
}

size_t embedding_bwd_scratch_bytes(int64_t, int64_t, int64_t) { return 256; }

template <typename T>
hipError_t launch_embedding_bwd(const EmbedGradArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(embedding_bwd_kernel<T>, dim3((unsigned)a.vocab), dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace varuna
