// The global gradient norm over many tensors, and clipping by it:
//   S = sum of g^2 over the finite entries (64 bits), B = number of the others
//   c = min(1, max_norm / (sqrt(S) + eps)), dst = c * src
// The tensors' addresses and sizes travel as kernel arguments, kClipTensors to a launch, so a call keeps nothing and can be
// captured.  Tensors are cut into chunks of kClipChunk entries; a workgroup takes consecutive ones.
#pragma once
#include "common.h"
#include "pipeline_ends.h"

namespace varuna {

constexpr int kClipTensors = 96;             // of a launch: 3 KB of kernel arguments
constexpr int kClipChunk = 8192;             // entries; 4096 is equal
constexpr int kNormBlocks = 2048;            // workgroups of a launch, each with a partial sum; 4096 are equal
// The clipping gives every chunk a workgroup of its own (274 M fp32 entries into bf16 498 us; 541 on 8192 workgroups, 576 on 2048).
constexpr int kClipBlocks = 1 << 16;
// The destination is written past the caches where sources and destinations together, in place once, exceed the last-level cache.  us of the norm,
// the clip and a pass that reads the result, through / past, by the result's size: fp32 in place 64 MB 55.0 / 55.7, 128 MB 92 / 94, 192 MB 127.5 /
// 129.2, 256 MB 174 / 172, 512 MB 399 / 392; fp32 into another buffer 64 MB 55 / 60, 96 MB 72 / 76, 128 MB 97 / 99, 192 MB 153 / 136, 512 MB
// 410 / 393; fp32 into bf16 64 MB 79 / 85, 96 MB 115 / 110, 192 MB 239 / 218; bf16 into another buffer 64 MB 65.5 / 71, 128 MB 112.5 / 113.5,
// 192 MB 169 / 155.  (An optimizer step behind it, which reads three more buffers, leaves no difference over 3 %: fp32 in place 64 MB 188 / 185,
// into another buffer 64 MB 196 / 191, 128 MB 385 / 377.)
constexpr int64_t kClipPast = 256ll << 20;

struct ClipJobs {
  const void* src[kClipTensors];
  void* dst[kClipTensors];
  int64_t count[kClipTensors];
  uint32_t first[kClipTensors + 1];  // chunk at which the tensor begins
  uint32_t bf16[kClipTensors];       // 1: src is bf16, 2: dst is
  int32_t n;
};

// U entries from any element on, loaded in one piece of up to 16 bytes, which needs no more than an element's alignment.
template <int U> struct Some { float v[U]; };
template <int U, typename T>
__device__ __forceinline__ Some<U> load_some(const T* p) {
  typedef T Any __attribute__((ext_vector_type(U), aligned(sizeof(T))));
  const Any a = *reinterpret_cast<const Any*>(p);
  Some<U> e;
#pragma unroll
  for (int i = 0; i < U; ++i) e.v[i] = to_f32(a[i]);
  return e;
}
template <bool PAST, int U, typename T>
__device__ __forceinline__ void store_some(T* p, const Some<U>& e) {   // on U entries; PAST: past the caches
  typedef T Vec __attribute__((ext_vector_type(U)));
  Vec a;
#pragma unroll
  for (int i = 0; i < U; ++i) a[i] = from_f32<T>(e.v[i]);
  if (PAST) __builtin_nontemporal_store(a, reinterpret_cast<Vec*>(p));
  else *reinterpret_cast<Vec*>(p) = a;
}

// The chunks of one workgroup: `per` consecutive ones.
struct ClipRange { uint32_t begin, end; };
__device__ __forceinline__ ClipRange chunks_of(const ClipJobs& j, uint32_t per, uint32_t group) {
  const uint32_t b = group * per, all = j.first[j.n];
  return {b, all - b < per ? all : b + per};
}
// The tensor that a chunk belongs to: how many begin at it or before, counted by a wave's ballots.
__device__ __forceinline__ int job_of(const ClipJobs& j, uint32_t chunk) {
  int k = -1;
#pragma unroll
  for (int b = 0; b < kClipTensors; b += 64) {
    const int i = b + (threadIdx.x & 63);
    k += __popcll(__ballot(i < j.n && j.first[i < kClipTensors ? i : 0] <= chunk));
  }
  return __builtin_amdgcn_readfirstlane(k);
}

__device__ __forceinline__ void add_square(float v, double& s, uint32_t& bad) {
  const bool fine = __builtin_isfinite(v);
  const double d = fine ? (double)v : 0.0;
  s += d * d;
  bad += !fine;
}
// Squares of p[0 .. n), n <= kClipChunk.
template <typename T>
__device__ __forceinline__ void add_squares(const T* p, int n, double& s, uint32_t& bad) {
  constexpr int U = 16 / (int)sizeof(T), AHEAD = kClipChunk / (U * 256);
  Some<U> e[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int at = (i * 256 + (int)threadIdx.x) * U;
    if (at + U <= n) e[i] = load_some<U>(p + at);
  }
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int at = (i * 256 + (int)threadIdx.x) * U;
    if (at + U <= n) {
#pragma unroll
      for (int k = 0; k < U; ++k) add_square(e[i].v[k], s, bad);
    } else {
      for (int k = at; k < n; ++k) add_square(to_f32(p[k]), s, bad);
    }
  }
}

__global__ __launch_bounds__(256) void grad_norm_partial_kernel(ClipJobs j, uint32_t per, double* __restrict__ partial) {
  __shared__ double ss[4], sb[4];
  double s = 0.0;
  uint32_t bad = 0;
  const ClipRange r = chunks_of(j, per, blockIdx.x);
  int k = job_of(j, r.begin);
  for (uint32_t c = r.begin; c < r.end; ++c) {
    if (c >= j.first[k + 1]) ++k;
    const int64_t begin = (int64_t)(c - j.first[k]) * kClipChunk, left = j.count[k] - begin;
    const int n = left < kClipChunk ? (int)left : kClipChunk;
    if (j.bf16[k] & 1) add_squares(static_cast<const bf16*>(j.src[k]) + begin, n, s, bad);
    else add_squares(static_cast<const float*>(j.src[k]) + begin, n, s, bad);
  }
  double b = (double)bad;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { s += __shfl_xor(s, o, kWave); b += __shfl_xor(b, o, kWave); }
  if ((threadIdx.x & 63) == 0) { ss[threadIdx.x >> 6] = s; sb[threadIdx.x >> 6] = b; }
  __syncthreads();
  if (threadIdx.x == 0) { partial[2 * blockIdx.x] = (ss[0] + ss[1]) + (ss[2] + ss[3]); partial[2 * blockIdx.x + 1] = (sb[0] + sb[1]) + (sb[2] + sb[3]); }
}

__global__ __launch_bounds__(1024) void grad_norm_final_kernel(const double* __restrict__ partial, int n, double* __restrict__ sum_sq,
                                                               float* __restrict__ nonfinite) {
  __shared__ double ss[16], sb[16];
  double s = 0.0, bad = 0.0;
#pragma unroll 2
  for (int i = threadIdx.x; i < n; i += 1024) { s += partial[2 * i]; bad += partial[2 * i + 1]; }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { s += __shfl_xor(s, o, kWave); bad += __shfl_xor(bad, o, kWave); }
  if ((threadIdx.x & 63) == 0) { ss[threadIdx.x >> 6] = s; sb[threadIdx.x >> 6] = bad; }
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0; bad = 0.0;
#pragma unroll
    for (int w = 0; w < 16; ++w) { s += ss[w]; bad += sb[w]; }
    *sum_sq = s; *nonfinite = (float)bad;
  }
}

// dst[0 .. n) = by * src[0 .. n), n <= kClipChunk: groups of U entries that begin where dst lies on U of them, and what is left
// before and behind.
template <bool PAST, typename D, typename S>
__device__ __forceinline__ void clip_chunk(D* dst, const S* src, int n, float by) {
  constexpr int U = sizeof(D) == 2 && sizeof(S) == 2 ? 8 : 4, AHEAD = kClipChunk / (U * 256);
  int head = (U - (int)(reinterpret_cast<uintptr_t>(dst) / sizeof(D)) % U) % U;
  if (head > n) head = n;
  const int groups = (n - head) / U, tail = head + groups * U;
  Some<U> e[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int k = i * 256 + (int)threadIdx.x;
    if (k < groups) e[i] = load_some<U>(src + head + U * k);
  }
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int k = i * 256 + (int)threadIdx.x;
    if (k < groups) {
#pragma unroll
      for (int w = 0; w < U; ++w) e[i].v[w] *= by;
      store_some<PAST>(dst + head + U * k, e[i]);
    }
  }
  const int t = (int)threadIdx.x;
  const int edge = t < head ? t : (t >= 8 && t - 8 < n - tail ? tail + t - 8 : -1);
  if (edge >= 0) dst[edge] = from_f32<D>(by * to_f32(src[edge]));
}

// A launch's chunks are taken last to first: what the norm has read last is still in the last-level cache (launches themselves follow each other
// in the tensors' order, so beyond kClipTensors of them that holds for the last launch's).
template <bool PAST>
__global__ __launch_bounds__(256) void grad_clip_kernel(ClipJobs j, uint32_t per, const double* __restrict__ sum_sq, double max_norm, double eps) {
  const float by = (float)fmin(1.0, max_norm / (sqrt(*sum_sq) + eps));
  const ClipRange r = chunks_of(j, per, gridDim.x - 1 - blockIdx.x);
  int k = job_of(j, r.end - 1);
  for (uint32_t c = r.end; c-- > r.begin;) {
    if (c < j.first[k]) --k;
    if (by == 1.f && j.dst[k] == j.src[k]) continue;
    const int64_t begin = (int64_t)(c - j.first[k]) * kClipChunk, left = j.count[k] - begin;
    const int n = left < kClipChunk ? (int)left : kClipChunk;
    const int types = j.bf16[k];
    if (types == 0) clip_chunk<PAST>(static_cast<float*>(j.dst[k]) + begin, static_cast<const float*>(j.src[k]) + begin, n, by);
    else if (types == 1) clip_chunk<PAST>(static_cast<float*>(j.dst[k]) + begin, static_cast<const bf16*>(j.src[k]) + begin, n, by);
    else if (types == 2) clip_chunk<PAST>(static_cast<bf16*>(j.dst[k]) + begin, static_cast<const float*>(j.src[k]) + begin, n, by);
    else clip_chunk<PAST>(static_cast<bf16*>(j.dst[k]) + begin, static_cast<const bf16*>(j.src[k]) + begin, n, by);
  }
}

// Runs f(jobs, workgroups, chunks of each) for every kClipTensors tensors that are not empty.
template <typename F>
inline void clip_launches(const TensorSpan& src, const TensorSpan* dst, uint32_t blocks, F f) {
  ClipJobs j;
  j.n = 0;
  uint32_t chunks = 0;
  auto flush = [&] {
    if (j.n == 0) return;
    j.first[j.n] = chunks;
    const uint32_t per = (chunks + blocks - 1) / blocks;
    f(j, (chunks + per - 1) / per, per);
    j.n = 0;
    chunks = 0;
  };
  for (int32_t i = 0; i < src.n; ++i) {
    if (src.count[i] == 0) continue;
    j.src[j.n] = src.p[i];
    j.dst[j.n] = dst ? const_cast<void*>(dst->p[i]) : nullptr;
    j.bf16[j.n] = (uint32_t)((src.dtype[i] != 0 ? 1 : 0) | (dst && dst->dtype[i] != 0 ? 2 : 0));
    j.count[j.n] = src.count[i];
    j.first[j.n] = chunks;
    chunks += (uint32_t)((src.count[i] + kClipChunk - 1) / kClipChunk);
    if (++j.n == kClipTensors) flush();
  }
  flush();
}

size_t grad_norm_scratch_bytes(const int64_t*, int32_t n) {
  return (size_t)(n / kClipTensors + 1) * kNormBlocks * 2 * sizeof(double);
}

hipError_t launch_grad_norm(const TensorSpan& t, double* sum_sq, float* nonfinite, void* scratch, hipStream_t st) {
  double* partial = static_cast<double*>(scratch);
  int n = 0;
  clip_launches(t, nullptr, kNormBlocks, [&](const ClipJobs& j, uint32_t blocks, uint32_t per) {
    hipLaunchKernelGGL(grad_norm_partial_kernel, dim3(blocks), dim3(256), 0, st, j, per, partial + 2 * (size_t)n);
    n += (int)blocks;
  });
  hipLaunchKernelGGL(grad_norm_final_kernel, dim3(1), dim3(1024), 0, st, partial, n, sum_sq, nonfinite);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const TensorSpan& dst, const TensorSpan& src, const double* sum_sq, double max_norm, double eps, hipStream_t st) {
  int64_t bytes = 0;
  for (int32_t i = 0; i < dst.n; ++i) bytes += dst.count[i] * ((dst.dtype[i] != 0 ? 2 : 4) + (dst.p[i] == src.p[i] ? 0 : src.dtype[i] != 0 ? 2 : 4));
  const bool past = bytes >= kClipPast;
  clip_launches(src, &dst, kClipBlocks, [&](const ClipJobs& j, uint32_t blocks, uint32_t per) {
    if (past) hipLaunchKernelGGL(grad_clip_kernel<true>, dim3(blocks), dim3(256), 0, st, j, per, sum_sq, max_norm, eps);
    else hipLaunchKernelGGL(grad_clip_kernel<false>, dim3(blocks), dim3(256), 0, st, j, per, sum_sq, max_norm, eps);
  });
  return hipGetLastError();
}

}  // namespace varuna
