// One AdamW step (Kingma & Ba, Algorithm 1, decoupled weight decay) over many tensors, their gradients multiplied by a scale and a clip factor on the way:
//   g = c * gradient;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  w -= lr (m / (1 - b1^step) / (sqrt(v / (1 - b2^step)) + eps) + decay w)
// w: the fp32 master of a bf16 parameter, which is w rounded, or the fp32 parameter itself.  Moments are fp32, or e4m3 codes of m / s and sqrt(v) / s'
// with powers of two s, s' for every 256 consecutive entries: s = 2^(e - 7), e the exponent of the block's largest finite value, so that the
// largest code is below 256 and rounding up never leaves the type.  A value between two codes goes up in proportion to its distance from the lower, v's by v
// itself: an average that moves by a hundredth of a code's distance a step would stand still if it were rounded to the nearest, and one rounded
// by its root would grow on its own.  What decides is u = frac(i a + step b), an evenly spread sequence over steps and entries both; nothing is
// drawn, so a step repeats bit for bit.  v > 0 keeps at least the smallest code, or the next division would be by eps alone.
//
// Bound by memory: 30 bytes an entry of a bf16 parameter with fp32 gradient and moments, 18 with moments in 8 bits.
#pragma once
#include "common.h"
#include "layer_ops.h"

namespace varuna {

constexpr int kAdamTensors = 80;          // of a launch: 3.2 KB of kernel arguments
constexpr int kAdamChunk = 4096;          // entries, 16 blocks: a workgroup's
constexpr uint32_t kWeylA = 0xC13FA9A9u, kWeylB = 0x91E10DA5u;   // 2^32 over the plastic number and over its square

struct AdamWJobs {
  void* p[kAdamTensors];
  const void* g[kAdamTensors];
  int64_t count[kAdamTensors];
  uint32_t first[kAdamTensors + 1];   // chunk at which the tensor begins
  uint32_t block[kAdamTensors];       // first block of its state
  float decay[kAdamTensors];
  uint32_t types[kAdamTensors];       // 1: the parameter is bf16, 2: the gradient is
  int32_t n;
};

// What is the same for all entries of a step.
struct AdamWStep { float by, lr, inv1, inv2, decay; uint32_t shift_m, shift_v; };

__device__ __forceinline__ AdamWStep adamw_step(const AdamWArgs& a) {
  double lr = a.lr, step = (double)a.step;
  if (a.lr_step) { lr = a.lr_step[0]; step = a.lr_step[1]; }
  AdamWStep s;
  s.lr = (float)lr;
  s.decay = (float)(lr * a.weight_decay);
  s.inv1 = (float)(1.0 / (1.0 - exp2(step * a.log2_beta1)));
  s.inv2 = (float)(1.0 / (1.0 - exp2(step * a.log2_beta2)));
  s.by = a.grad_scale;
  if (a.sum_sq) s.by = (float)((double)a.grad_scale * fmin(1.0, a.max_norm / (fabs((double)a.grad_scale) * sqrt(*a.sum_sq) + a.clip_eps)));
  const uint32_t n = (uint32_t)(int64_t)step;
  s.shift_m = n * kWeylB;
  s.shift_v = n * kWeylA;
  return s;
}

// u in [0, 1) on 24 binary digits.
__device__ __forceinline__ float adamw_u(uint32_t i, uint32_t a, uint32_t shift) { return (float)((i * a + shift) >> 8) * 0x1p-24f; }

// The step between the codes around x in [0, 256): a power of two.
__device__ __forceinline__ float code_gap(float x) {
  const uint32_t e = __float_as_uint(x) >> 23;
  return __uint_as_float(((e < 121u ? 121u : e) - 3u) << 23);   // below 2^-6: as there
}
__device__ __forceinline__ float code_below(float x, float gap) {   // both powers of two times small whole numbers: exact
  return __builtin_truncf(x * __uint_as_float((254u << 23) - __float_as_uint(gap))) * gap;
}
__device__ __forceinline__ float code_m(float x, float u) {
#pragma clang fp contract(off)
  const float a = fabsf(x), gap = code_gap(a), lo = code_below(a, gap);
  return copysignf(a - lo > u * gap ? lo + gap : lo, x);
}
__device__ __forceinline__ float code_v(float r, float u) {
#pragma clang fp contract(off)
  const float gap = code_gap(r), lo = code_below(r, gap);
  const float c = (r - lo) * (r + lo) > u * gap * (lo + lo + gap) ? lo + gap : lo;
  return r > 0.f ? fmaxf(c, 0x1p-9f) : c;
}
// The power of two by which a block whose largest value is `most` is divided, and its inverse.
__device__ __forceinline__ float block_scale(float most) {
  const uint32_t e = __float_as_uint(most) >> 23;
  return __uint_as_float(((e < 8u ? 8u : e) - 7u) << 23);
}
__device__ __forceinline__ float inverse_power(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// Each product and sum is rounded by itself: codes and bf16 gradients are so coarse that their means meet a power of two exactly now and then, and which
// side of it the largest value of a block comes out on, its scale's exponent, should not depend on what the compiler contracts.
__device__ __forceinline__ void adamw_one(float g, float& w, float& m, float& v, const AdamWArgs& a, const AdamWStep& s, float decay) {
#pragma clang fp contract(off)
  g *= s.by;
  m = a.beta1 * m + a.one_minus_beta1 * g;
  v = a.beta2 * v + a.one_minus_beta2 * (g * g);
  w -= s.lr * (m * s.inv1 / (sqrtf(v * s.inv2) + a.eps)) + decay * w;
}

// Four entries of a block on a lane.  P, G: types of the parameter and the gradient; BITS8: moments are codes.
template <typename P, typename G, bool BITS8>
__device__ __forceinline__ void adamw_block(const AdamWArgs& a, const AdamWStep& s, float decay, P* p, const G* g, uint32_t block, int n) {
  const int lane = threadIdx.x & 63, at = lane * 4, have = n - at;
  const int64_t i = (int64_t)block * kStateBlock + at;
  const Piece<G, 4> ge = load_piece<4>(g + at, have);
  float w[4], m[4], v[4];
  if constexpr (sizeof(P) == 2) {
    const Piece<float, 4> e = load_piece<4>(a.master + i, 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = e.v[k];
  } else {
    const Piece<float, 4> e = load_piece<4>(p + at, have);
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = e.v[k];
  }
  if constexpr (BITS8) {
    const int cm = static_cast<const int*>(a.m)[i / 4], cv = static_cast<const int*>(a.v)[i / 4];
    const float sm = a.scales[2 * (int64_t)block], sv = a.scales[2 * (int64_t)block + 1];
    m[0] = __builtin_amdgcn_cvt_f32_fp8(cm, 0) * sm; m[1] = __builtin_amdgcn_cvt_f32_fp8(cm, 1) * sm;
    m[2] = __builtin_amdgcn_cvt_f32_fp8(cm, 2) * sm; m[3] = __builtin_amdgcn_cvt_f32_fp8(cm, 3) * sm;
    v[0] = __builtin_amdgcn_cvt_f32_fp8(cv, 0) * sv; v[1] = __builtin_amdgcn_cvt_f32_fp8(cv, 1) * sv;
    v[2] = __builtin_amdgcn_cvt_f32_fp8(cv, 2) * sv; v[3] = __builtin_amdgcn_cvt_f32_fp8(cv, 3) * sv;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] *= v[k];
  } else {
    const floatx4 em = reinterpret_cast<const floatx4*>(a.m)[i / 4], ev = reinterpret_cast<const floatx4*>(a.v)[i / 4];
#pragma unroll
    for (int k = 0; k < 4; ++k) { m[k] = em[k]; v[k] = ev[k]; }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) adamw_one(to_f32(ge.v[k]), w[k], m[k], v[k], a, s, decay);
  if constexpr (BITS8) {
    float r[4], mm = 0.f, mr = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r[k] = sqrtf(v[k]);
      if (k < have) {
        mm = fmaxf(mm, __builtin_isfinite(m[k]) ? fabsf(m[k]) : 0.f);
        mr = fmaxf(mr, __builtin_isfinite(r[k]) ? r[k] : 0.f);
      }
    }
    const float sm = block_scale(wave_max(mm)), sv = block_scale(wave_max(mr)), im = inverse_power(sm), iv = inverse_power(sv);
    float cm[4], cv[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t e = (uint32_t)i + (uint32_t)k;
      cm[k] = __builtin_isfinite(m[k]) ? code_m(m[k] * im, adamw_u(e, kWeylA, s.shift_m)) : __builtin_nanf("");
      cv[k] = __builtin_isfinite(r[k]) ? code_v(r[k] * iv, adamw_u(e, kWeylB, s.shift_v)) : __builtin_nanf("");
    }
    const int um = __builtin_amdgcn_cvt_pk_fp8_f32(cm[2], cm[3], __builtin_amdgcn_cvt_pk_fp8_f32(cm[0], cm[1], 0, false), true);
    const int uv = __builtin_amdgcn_cvt_pk_fp8_f32(cv[2], cv[3], __builtin_amdgcn_cvt_pk_fp8_f32(cv[0], cv[1], 0, false), true);
    if (have >= 4) {
      static_cast<int*>(a.m)[i / 4] = um;
      static_cast<int*>(a.v)[i / 4] = uv;
    } else {
      for (int k = 0; k < have; ++k) {
        static_cast<uint8_t*>(a.m)[i + k] = (uint8_t)(um >> (8 * k));
        static_cast<uint8_t*>(a.v)[i + k] = (uint8_t)(uv >> (8 * k));
      }
    }
    if (lane == 0) { a.scales[2 * (int64_t)block] = sm; a.scales[2 * (int64_t)block + 1] = sv; }
  } else {
    store_piece<4>(static_cast<float*>(a.m) + i, have, Piece<float, 4>{{m[0], m[1], m[2], m[3]}});
    store_piece<4>(static_cast<float*>(a.v) + i, have, Piece<float, 4>{{v[0], v[1], v[2], v[3]}});
  }
  if constexpr (sizeof(P) == 2) store_piece<4>(a.master + i, have, Piece<float, 4>{{w[0], w[1], w[2], w[3]}});
  store_piece<4>(p + at, have, Piece<P, 4>{{from_f32<P>(w[0]), from_f32<P>(w[1]), from_f32<P>(w[2]), from_f32<P>(w[3])}});
}

template <typename P, typename G, bool BITS8>
__device__ __forceinline__ void adamw_chunk(const AdamWArgs& a, const AdamWStep& s, const AdamWJobs& j, int k, int64_t begin) {
  P* p = static_cast<P*>(j.p[k]) + begin;
  const G* g = static_cast<const G*>(j.g[k]) + begin;
  const int64_t left = j.count[k] - begin;
  const int n = left < kAdamChunk ? (int)left : kAdamChunk;
  const float decay = s.decay * j.decay[k];
  const uint32_t block = j.block[k] + (uint32_t)(begin / kStateBlock);
  for (int b = (int)(threadIdx.x >> 6); b * kStateBlock < n; b += 4)
    adamw_block<P, G, BITS8>(a, s, decay, p + b * kStateBlock, g + b * kStateBlock, block + (uint32_t)b, n - b * kStateBlock);
}

template <bool BITS8>
__global__ __launch_bounds__(256) void adamw_kernel(AdamWJobs j, AdamWArgs a) {
  if (a.skip && *a.skip != 0.f) return;
  const uint32_t c = blockIdx.x;
  int k = -1;   // the tensor that the chunk belongs to: how many begin at it or before
#pragma unroll
  for (int b = 0; b < kAdamTensors; b += 64) {
    const int i = b + (int)(threadIdx.x & 63);
    k += __popcll(__ballot(i < j.n && j.first[i < kAdamTensors ? i : 0] <= c));
  }
  k = __builtin_amdgcn_readfirstlane(k);
  const AdamWStep s = adamw_step(a);
  const int64_t begin = (int64_t)(c - j.first[k]) * kAdamChunk;
  switch (j.types[k]) {
    case 0: return adamw_chunk<float, float, BITS8>(a, s, j, k, begin);
    case 1: return adamw_chunk<bf16, float, BITS8>(a, s, j, k, begin);
    case 2: return adamw_chunk<float, bf16, BITS8>(a, s, j, k, begin);
    default: return adamw_chunk<bf16, bf16, BITS8>(a, s, j, k, begin);
  }
}

hipError_t launch_adamw(const TensorSpan& params, const TensorSpan& grads, const float* decays, const AdamWArgs& a, hipStream_t st) {
  AdamWJobs j;
  j.n = 0;
  uint32_t chunks = 0, blocks = 0;
  auto flush = [&] {
    if (j.n == 0) return;
    j.first[j.n] = chunks;
    if (a.scales) hipLaunchKernelGGL(adamw_kernel<true>, dim3(chunks), dim3(256), 0, st, j, a);
    else hipLaunchKernelGGL(adamw_kernel<false>, dim3(chunks), dim3(256), 0, st, j, a);
    j.n = 0;
    chunks = 0;
  };
  for (int32_t i = 0; i < params.n; ++i) {
    const int64_t n = params.count[i];
    if (n == 0) continue;
    j.p[j.n] = const_cast<void*>(params.p[i]);
    j.g[j.n] = grads.p[i];
    j.count[j.n] = n;
    j.first[j.n] = chunks;
    j.block[j.n] = blocks;
    j.decay[j.n] = decays ? decays[i] : 1.f;
    j.types[j.n] = (uint32_t)((params.dtype[i] != 0 ? 1 : 0) | (grads.dtype[i] != 0 ? 2 : 0));
    chunks += (uint32_t)((n + kAdamChunk - 1) / kAdamChunk);
    blocks += (uint32_t)((n + kStateBlock - 1) / kStateBlock);
    if (++j.n == kAdamTensors) flush();
  }
  flush();
  return hipGetLastError();
}

}  // namespace varuna
