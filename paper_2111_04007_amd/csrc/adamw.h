// One AdamW step (Kingma & Ba, Algorithm 1, decoupled weight decay) over many tensors, their gradients multiplied by a scale and a clip factor on the way:
//   g = c * gradient;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  w -= lr (m / (1 - b1^step) / (sqrt(v / (1 - b2^step)) + eps) + decay w)
// w: the fp32 master of a bf16 parameter, which is w rounded, or the fp32 parameter itself.  Moments are fp32, or e4m3 codes of m / s and sqrt(v) / s'
// with powers of two s, s' for every 256 consecutive entries: s = 2^(e - 7), e the exponent of the block's largest finite value, so that the
// largest code is below 256 and rounding up never leaves the type.  A value between two codes goes up in proportion to its distance from the lower, v's by v
// itself: an average that moves by a hundredth of a code's distance a step would stand still if it were rounded to the nearest, and one rounded
// by its root would grow on its own.  What decides is u = frac(i a + step b), an evenly spread sequence over steps and entries both; nothing is
// drawn, so a step repeats bit for bit.  v > 0 keeps at least the smallest code, or the next division would be by eps alone.
//
// Bound by memory: 30 bytes an entry of a bf16 parameter with fp32 gradient and moments, 18 with moments in 8 bits, where the vector unit is as busy (some 90 operations an entry).
// 274 M entries in 50 tensors: 1528 us (5.4 TB/s) and 822 us (6.0 TB/s).
#pragma once
#include "common.h"
#include "layer_ops.h"

#include <cmath>
#include <type_traits>

namespace varuna {

constexpr int kAdamTensors = 80;          // of a launch: 3.2 KB of kernel arguments
// Entries of a workgroup, a block for each wave.  274 M bf16 parameters, moments of 8 bits / 32, us: 847 / 1515; 2048 entries 890 / 1555, 4096 932 / 1555, 8192 966 / 1583, 32768
// 1032 / 1661, each wave's next block fetched ahead; its blocks side by side 4096 938 / 1523.
constexpr int kAdamChunk = 1024;
// From this many bytes of all tensors on a step goes past the caches, which then hold nothing of it when the next one comes.  us through / past: 8 bits (12 bytes an entry) 60 MB 19.8 /
// 19.9, 120 MB 33.6 / 34.8, 216 MB 66.7 / 58.3, 360 MB 109 / 95, 3.3 GB 1026 / 843; 32 bits (18 bytes) 90 MB 25.5 / 28.6, 180 MB 55.3 / 53.4, 324 MB 108 / 97, 4.9 GB 1752 / 1520.
constexpr int64_t kAdamPast = 160ll << 20;
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

// What is the same for all entries of a step: the update is rate * m / (root * sqrt(v) + eps) + decay * w.
struct AdamWStep { float by, rate, root, decay; uint32_t shift_m, shift_v; };

__host__ __device__ inline AdamWStep adamw_step(double lr, double step, double weight_decay, double log2_beta1, double log2_beta2) {
  AdamWStep s;
  s.by = 1.f;
  s.rate = (float)(lr / (1.0 - exp2(step * log2_beta1)));
  s.root = (float)sqrt(1.0 / (1.0 - exp2(step * log2_beta2)));
  s.decay = (float)(lr * weight_decay);
  const uint32_t n = (uint32_t)(int64_t)step;
  s.shift_m = n * kWeylB;
  s.shift_v = n * kWeylA;
  return s;
}

// The largest of a wave's values, each at least 0 as a whole number, in every lane.
__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
  auto dpp = [](uint32_t x, auto ctrl) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(ctrl)::value, 0xf, 0xf, true); };
  auto most = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  v = most(v, dpp(v, std::integral_constant<int, 0xb1>{}));    // quad_perm 1 0 3 2
  v = most(v, dpp(v, std::integral_constant<int, 0x4e>{}));    // quad_perm 2 3 0 1
  v = most(v, dpp(v, std::integral_constant<int, 0x141>{}));   // row_half_mirror
  v = most(v, dpp(v, std::integral_constant<int, 0x140>{}));   // row_mirror
  auto lane = [&](int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
  return most(most(lane(0), lane(16)), most(lane(32), lane(48)));
}

// sqrt(v) of v >= 0, rounded to nearest but for values within 2^-45 or so of a tie: one step of Newton's method from the hardware's reciprocal root; of 0, infinity and NaN these themselves.
// exact: below 2^-126 too, where the root counts as 2^-63 otherwise (in an update, not in a code).
__device__ __forceinline__ float adamw_root(float v, bool exact) {
  const bool low = exact && v < 0x1p-96f;
  const float x = fmaxf(low ? v * 0x1p64f : v, 0x1p-126f), y = __builtin_amdgcn_rsqf(x), r = x * y;
  const float root = __builtin_fmaf(__builtin_fmaf(-r, r, x), 0.5f * y, r);
  return __builtin_amdgcn_classf(v, 0x180) ? (low ? root * 0x1p-32f : root) : v;   // of the numbers above 0
}
// An eps of at least 2^-30 leaves no 2^-23 of an update to roots of at most 2^-63, times 2^10 for the steps' correction.
constexpr float kEpsOfTinyRoots = 0x1p-30f;
// Codes of r = sqrt(v) over its block's scale: the upper neighbour where (r^2 - lo^2) / (hi^2 - lo^2) > u, u of 24 binary digits.  Below 2^-6 codes lie 2^-9 apart: r + 2^-6 has that spacing.
// Both neighbours are sums of few digits: exact.  A root above 0 counts as the smallest code at least.
__device__ __forceinline__ float code_v(float root, uint32_t u) {
#pragma clang fp contract(off)
  const float r = fmaxf(root, 0x1p-9f), low = r < 0x1p-6f ? 0x1p-6f : 0.f;
  const uint32_t t = __float_as_uint(r + low) & 0xfff00000u;
  const float lo = __uint_as_float(t) - low, hi = __uint_as_float(t + 0x100000u) - low;
  const float c = (r - lo) * (r + lo) > (float)(u >> 8) * ((hi - lo) * 0x1p-24f) * (lo + hi) ? hi : lo;
  return root > 0.f ? c : 0.f;
}
// The power of two by which a block whose largest value has these exponent bits is divided, and its inverse.
__device__ __forceinline__ float block_scale(uint32_t e) { return __uint_as_float(((e < 8u ? 8u : e) - 7u) << 23); }
__device__ __forceinline__ float inverse_power(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }
// The exponent bits of the root of a value.
__device__ __forceinline__ uint32_t root_exponent(float v) { return __float_as_uint(adamw_root(v, true)) >> 23; }
constexpr uint32_t kTinyRootsShow = (127 - 94) << 23;   // bits of 2^-94

// Each product and sum is rounded by itself: codes and bf16 gradients are so coarse that their means meet a power of two exactly now and then, and which
// side of it the largest value of a block comes out on, its scale's exponent, should not depend on what the compiler contracts.
__device__ __forceinline__ void adamw_moments(float g, float& m, float& v, const AdamWArgs& a) {
#pragma clang fp contract(off)
  m = a.beta1 * m + a.one_minus_beta1 * g;
  v = a.beta2 * v + a.one_minus_beta2 * (g * g);
}

// Four entries of a block on a lane, as they are read.
template <typename P, typename G, bool BITS8> struct AdamWEntries {
  Piece<G, 4> g;
  Piece<float, 4> w, m, v;
  int cm, cv;
  float sm, sv;
};
// P, G: types of the parameter and the gradient; BITS8: moments are codes; PAST: past the caches.
template <typename P, typename G, bool BITS8, bool PAST>
__device__ __forceinline__ AdamWEntries<P, G, BITS8> adamw_fetch(const AdamWArgs& a, const P* p, const G* g, uint32_t block, int n) {
  const int at = (int)(threadIdx.x & 63) * 4, have = n - at;
  const int64_t i = (int64_t)block * kStateBlock + at;
  AdamWEntries<P, G, BITS8> e;
  if (n >= kStateBlock) {
    e.g = load_piece<4, PAST>(g + at, 4);
    if constexpr (sizeof(P) == 4) e.w = load_piece<4, PAST>(p + at, 4);
  } else {
    e.g = load_piece<4, PAST>(g + at, have);
    if constexpr (sizeof(P) == 4) e.w = load_piece<4, PAST>(p + at, have);
  }
  if constexpr (sizeof(P) == 2) e.w = load_piece<4, PAST>(static_cast<const float*>(a.master) + i, 4);
  if constexpr (BITS8) {
    const int *m = static_cast<const int*>(a.m) + i / 4, *v = static_cast<const int*>(a.v) + i / 4;
    e.cm = PAST ? __builtin_nontemporal_load(m) : *m;
    e.cv = PAST ? __builtin_nontemporal_load(v) : *v;
    e.sm = a.scales[2 * (int64_t)block];
    e.sv = a.scales[2 * (int64_t)block + 1];
  } else {
    e.m = load_piece<4, PAST>(static_cast<const float*>(a.m) + i, 4);
    e.v = load_piece<4, PAST>(static_cast<const float*>(a.v) + i, 4);
  }
  return e;
}
template <typename P, typename G, bool BITS8, bool PAST>
__device__ __forceinline__ void adamw_block(const AdamWArgs& a, const AdamWStep& s, float decay, const AdamWEntries<P, G, BITS8>& in, P* p, uint32_t block, int n) {
  const int lane = threadIdx.x & 63, at = lane * 4, have = n - at;
  const int64_t i = (int64_t)block * kStateBlock + at;
  float w[4], m[4], v[4], r[4];
  if constexpr (BITS8) {
    const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8(in.cm, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(in.cm, true);
    const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8(in.cv, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8(in.cv, true);
    const float cm[4] = {m01[0], m01[1], m23[0], m23[1]}, cv[4] = {v01[0], v01[1], v23[0], v23[1]};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = cm[k] * in.sm;
      v[k] = cv[k] * in.sv;
      v[k] *= v[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) { m[k] = in.m.v[k]; v[k] = in.v.v[k]; }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) adamw_moments(to_f32(in.g.v[k]) * s.by, m[k], v[k], a);
  const bool exact = a.eps < kEpsOfTinyRoots;
  if (exact) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = adamw_root(v[k], true);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = adamw_root(v[k], false);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    w[k] = in.w.v[k];
    w[k] -= s.rate * m[k] * __builtin_amdgcn_rcpf(s.root * r[k] + a.eps) + decay * w[k];
  }
  const Piece<P, 4> pe{{from_f32<P>(w[0]), from_f32<P>(w[1]), from_f32<P>(w[2]), from_f32<P>(w[3])}};
  const Piece<float, 4> we{{w[0], w[1], w[2], w[3]}}, me{{m[0], m[1], m[2], m[3]}}, ve{{v[0], v[1], v[2], v[3]}};
  const bool whole = n >= kStateBlock;   // all lanes of the wave alike
  if (whole) {
    if constexpr (sizeof(P) == 2) store_piece<4, PAST>(a.master + i, 4, we);
    store_piece<4, PAST>(p + at, 4, pe);
    if constexpr (!BITS8) {
      store_piece<4, PAST>(static_cast<float*>(a.m) + i, 4, me);
      store_piece<4, PAST>(static_cast<float*>(a.v) + i, 4, ve);
    }
  } else {
    if constexpr (sizeof(P) == 2) store_piece<4>(a.master + i, have, we);
    store_piece<4>(p + at, have, pe);
    if constexpr (!BITS8) {
      store_piece<4>(static_cast<float*>(a.m) + i, have, me);
      store_piece<4>(static_cast<float*>(a.v) + i, have, ve);
    }
  }
  if constexpr (BITS8) {
    // Bits of values that are at least 0 are ordered as the values are, infinities and NaNs above them all.
    constexpr uint32_t kInf = 0x7f800000u;
    uint32_t bm[4], bv[4], mm = 0, mv = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      bm[k] = __float_as_uint(m[k]) & 0x7fffffffu;
      bv[k] = __float_as_uint(v[k]);   // never below 0, but for a NaN, which is above infinity with its sign too
      if (!whole && k >= have) bm[k] = bv[k] = 0;   // what lies between the tensors' states
      mm = bm[k] > mm ? bm[k] : mm;
      mv = bv[k] > mv ? bv[k] : mv;
    }
    mm = wave_most(mm);
    mv = wave_most(mv);
    const bool broken = mm >= kInf || mv >= kInf;   // of all lanes
    if (broken) {   // the largest of what is finite
      mm = mv = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (bm[k] < kInf) mm = bm[k] > mm ? bm[k] : mm;
        if (bv[k] < kInf) mv = bv[k] > mv ? bv[k] : mv;
      }
      mm = wave_most(mm);
      mv = wave_most(mv);
    }
    // Roots that counted as 2^-63 in the update are what they are in a code.  In blocks with a v of 2^-94 and more 2^-63 is at most 2^-9 of the scale, which is the smallest code and what
    // every lesser root becomes too.
    if (!exact && mv < kTinyRootsShow) {
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = adamw_root(v[k], true);
    }
    const float sm = block_scale(mm >> 23), sv = block_scale(root_exponent(__uint_as_float(mv))), im = inverse_power(sm), iv = inverse_power(sv);
    // The conversion rounds up where the 20 digits behind a code and the upper 20 of its second operand carry: the operand is 1 - u.
    const uint32_t seed = ~((uint32_t)i * kWeylA + s.shift_m), u = (uint32_t)i * kWeylB + s.shift_v;
    int um = 0;
    um = __builtin_amdgcn_cvt_sr_fp8_f32(m[0] * im, (int)seed, um, 0);
    um = __builtin_amdgcn_cvt_sr_fp8_f32(m[1] * im, (int)(seed - kWeylA), um, 1);
    um = __builtin_amdgcn_cvt_sr_fp8_f32(m[2] * im, (int)(seed - 2 * kWeylA), um, 2);
    um = __builtin_amdgcn_cvt_sr_fp8_f32(m[3] * im, (int)(seed - 3 * kWeylA), um, 3);
    int uv = __builtin_amdgcn_cvt_pk_fp8_f32(code_v(r[0] * iv, u), code_v(r[1] * iv, u + kWeylB), 0, false);
    uv = __builtin_amdgcn_cvt_pk_fp8_f32(code_v(r[2] * iv, u + 2 * kWeylB), code_v(r[3] * iv, u + 3 * kWeylB), uv, true);
    if (broken) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (bm[k] >= kInf) um |= 0x7f << (8 * k);
        if (bv[k] >= kInf) uv |= 0x7f << (8 * k);
      }
    }
    if (whole) {
      int *qm = static_cast<int*>(a.m) + i / 4, *qv = static_cast<int*>(a.v) + i / 4;
      if (PAST) { __builtin_nontemporal_store(um, qm); __builtin_nontemporal_store(uv, qv); }
      else { *qm = um; *qv = uv; }
    } else {
      for (int k = 0; k < 4 && k < have; ++k) {
        static_cast<uint8_t*>(a.m)[i + k] = (uint8_t)(um >> (8 * k));
        static_cast<uint8_t*>(a.v)[i + k] = (uint8_t)(uv >> (8 * k));
      }
    }
    if (lane == 0) { a.scales[2 * (int64_t)block] = sm; a.scales[2 * (int64_t)block + 1] = sv; }
  }
}

template <typename P, typename G, bool BITS8, bool PAST>
__device__ __forceinline__ void adamw_chunk(const AdamWArgs& a, const AdamWStep& s, const AdamWJobs& j, int k, int64_t begin) {
  begin += __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * kStateBlock;
  const int64_t left = j.count[k] - begin;
  if (left <= 0) return;
  P* p = static_cast<P*>(j.p[k]) + begin;
  const int n = left < kStateBlock ? (int)left : kStateBlock;
  const uint32_t block = j.block[k] + (uint32_t)(begin / kStateBlock);
  const AdamWEntries<P, G, BITS8> e = adamw_fetch<P, G, BITS8, PAST>(a, p, static_cast<const G*>(j.g[k]) + begin, block, n);
  adamw_block<P, G, BITS8, PAST>(a, s, s.decay * j.decay[k], e, p, block, n);
}

template <bool BITS8, bool PAST>
__global__ __launch_bounds__(256) void adamw_kernel(AdamWJobs j, AdamWArgs a, AdamWStep s) {
  if (a.skip && *a.skip != 0.f) return;
  const uint32_t c = blockIdx.x;
  int k = -1;   // the tensor that the chunk belongs to: how many begin at it or before
#pragma unroll
  for (int b = 0; b < kAdamTensors; b += 64) {
    const int i = b + (int)(threadIdx.x & 63);
    k += __popcll(__ballot(i < j.n && j.first[i < kAdamTensors ? i : 0] <= c));
  }
  k = __builtin_amdgcn_readfirstlane(k);
  if (a.lr_step) s = adamw_step(a.lr_step[0], a.lr_step[1], a.weight_decay, a.log2_beta1, a.log2_beta2);
  s.by = a.grad_scale;
  if (a.sum_sq) s.by = (float)((double)a.grad_scale * fmin(1.0, a.max_norm / (fabs((double)a.grad_scale) * sqrt(*a.sum_sq) + a.clip_eps)));
  const int64_t begin = (int64_t)(c - j.first[k]) * kAdamChunk;
  switch (j.types[k]) {
    case 0: return adamw_chunk<float, float, BITS8, PAST>(a, s, j, k, begin);
    case 1: return adamw_chunk<bf16, float, BITS8, PAST>(a, s, j, k, begin);
    case 2: return adamw_chunk<float, bf16, BITS8, PAST>(a, s, j, k, begin);
    default: return adamw_chunk<bf16, bf16, BITS8, PAST>(a, s, j, k, begin);
  }
}

hipError_t launch_adamw(const TensorSpan& params, const TensorSpan& grads, const float* decays, const AdamWArgs& a, hipStream_t st) {
  AdamWJobs j;
  j.n = 0;
  uint32_t chunks = 0, blocks = 0;
  int64_t bytes = 0;
  for (int32_t i = 0; i < params.n; ++i)
    bytes += params.count[i] * ((a.scales ? 2 : 8) + (grads.dtype[i] != 0 ? 2 : 4) + (params.dtype[i] != 0 ? 6 : 4));
  const bool past = bytes >= kAdamPast;
  const AdamWStep step = adamw_step(a.lr, (double)a.step, a.weight_decay, a.log2_beta1, a.log2_beta2);
  auto flush = [&] {
    if (j.n == 0) return;
    j.first[j.n] = chunks;
    auto kernel = a.scales ? (past ? adamw_kernel<true, true> : adamw_kernel<true, false>) : (past ? adamw_kernel<false, true> : adamw_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3(chunks), dim3(256), 0, st, j, a, step);
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
