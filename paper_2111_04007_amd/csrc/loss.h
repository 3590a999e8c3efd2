// The last stage's loss: cross entropy over the vocabulary with label smoothing e, and the gradient of the logits,
//   m = max_j x_j, s = sum_j exp(x_j - m), loss = (1 - e) (log s + m - x_y) + e (log s + m - mean_j x_j)
//   dx_j = g (exp(x_j - m) / s - (1 - e) [j = y] - e / V)
// A row whose target is none of [0, V) has loss 0 and gradient 0 and is not counted.
#pragma once
#include "common.h"
#include "pipeline_ends.h"

namespace varuna {

__device__ __forceinline__ int64_t target_of(const LossArgs& a, int64_t r) {
  const int64_t y = a.wide ? static_cast<const int64_t*>(a.targets)[r] : (int64_t)static_cast<const int32_t*>(a.targets)[r];
  return y >= 0 && y < a.vocab ? y : -1;
}

// How a row lies on 16-byte pieces: `head` entries, `n` pieces of W, `tail` entries.
template <typename T>
struct RowPieces {
  static constexpr int W = 16 / (int)sizeof(T);
  int head, n, tail;
  __device__ __forceinline__ RowPieces(const T* x, int vocab) {
    head = (W - (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T)) % W) % W;
    if (head > vocab) head = vocab;
    n = (vocab - head) / W;
    tail = vocab - head - n * W;
  }
  // The entry outside of the pieces that thread i holds, or -1.
  __device__ __forceinline__ int edge(int i) const {
    return i < head ? i : (i >= W && i - W < tail ? head + n * W + i - W : -1);
  }
};

// exp(x - m); m is the largest value, or 0 where that is -inf.  One rounding of the product and the hardware's base-2 exponential: off by up to
// about 3 (m - x) 2^-24 of itself (1e-5 where it is e^-88; an exact product would cost a second fma for every entry, and the sum, whose large terms
// have a small m - x, gains nothing), and 0 below 2^-126.
__device__ __forceinline__ float exp_less(float x, float m) { return __builtin_amdgcn_exp2f((x - m) * 1.4426950408889634f); }
__device__ __forceinline__ float exp_base(float m) { return m == -INFINITY ? 0.f : m; }
// (m - x) / 2, rounded once: no overflow between finite values.
__device__ __forceinline__ float half_gap(float m, float x) { return fmaf(-0.5f, x, 0.5f * m); }

// bf16 values are unpacked where they are used, one piece after the other: a row that is kept unpacked takes three times the
// registers.  The compiler can neither take an unpacked value from before this point nor put off what `after` depends on.
template <typename T, typename R> __device__ __forceinline__ void unpack_anew(R& raw, float& after) {
  if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(raw), "+v"(after)::"memory");
}

// Entry w of a piece.
template <typename T, typename R> __device__ __forceinline__ float entry(const R& raw, int w) {
  const uint32_t u = sizeof(T) == 2 ? ((w & 1) ? raw[w / 2] & 0xffff0000u : raw[w / 2] << 16) : raw[w];
  return __builtin_bit_cast(float, u);
}

// What goes past the caches: the gradient where it is larger than the last-level cache, so that what reads it next finds none of it
// there anyway; the logits where nothing but the loss is asked for and no one reads them again.  us, through / past:
// gradient of 4096 x 50257 153 / 144, of 8192 x 128000 773 / 772; loss of 2048 x 50257 fp32 alone 75.7 / 71.6.  A smaller gradient
// is written faster past them as well (1023 x 30523 33.7 / 26.8), but the products that read it lose more: together with the two
// products of a head 1024 wide, 512 x 30528 219 / 233, 1024 x 30528 267 / 267, 2048 x 30528 524 / 531, 4096 x 50304 2131 / 2125.
enum : int { kPastNone = 0, kPastStores = 1, kPastLoads = 2 };
constexpr int64_t kLastLevelCache = 256ll << 20;

// One workgroup of 64 WAVES threads per row.  RES: the row stays in registers, NV pieces of it per thread, from its one reading to its
// gradient; otherwise it is read in chunks of that size, with a running maximum and sum, and once more for the gradient.
// Every thread keeps its own maximum and sum; one exchange through LDS joins them.  The smoothing's term is lse - mean = log s + (m - mean):
// threads sum (m - x_j) / V below their own maximum and add (m' - m) / V for each of their entries when they join a larger one m'.  All of these are
// positive, so the error follows the row's spread and not its size (values summed by themselves lose log2 |x| bits: 3e-3 at 3e4, all of them in a row
// of the type's lowest value).  Differences are halved, since m - x_j alone may overflow.  With RES all blocks of 64 WAVES pieces but
// the last are whole (the launch sees to it): no branch stands between the loads.  same: a gradient's row lies on 16 bytes as its logits do.
template <typename T, int WAVES, int NV, bool RES, int PAST>
__global__ __launch_bounds__(64 * WAVES) void cross_entropy_kernel(LossArgs a, bool same) {
  typedef RowPieces<T> P;
  constexpr int W = P::W, THREADS = 64 * WAVES;
  typedef T Vec __attribute__((ext_vector_type(W)));
  typedef uint32_t Raw __attribute__((ext_vector_type(4)));
  __shared__ float lds[4][WAVES], target;
  const uint32_t tid = threadIdx.x;
  const float eps = a.smoothing, inv_v = 1.f / (float)a.vocab;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int64_t y = target_of(a, r);
    const T* x = static_cast<const T*>(a.logits) + r * a.ld;
    T* dx = a.dlogits ? static_cast<T*>(a.dlogits) + r * a.ldd : nullptr;
    const P p(x, a.vocab);
    const Raw* body = reinterpret_cast<const Raw*>(x + p.head);
    const int mine = p.edge((int)tid);
    // Block b: the pieces b .. b + THREADS - 1, a thread's own one behind a base that all share.
    auto load = [&](int b, bool whole) {
      Raw v;
      if (whole || b + (int)tid < p.n) {
        v = PAST == kPastLoads ? __builtin_nontemporal_load(body + b + tid) : (body + b)[tid];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;   // -inf: adds nothing
      }
      return v;
    };
    auto store = [&](int b, bool whole, const float* v) {
      if (!whole && b + (int)tid >= p.n) return;
      Vec o;
#pragma unroll
      for (int w = 0; w < W; ++w) o[w] = from_f32<T>(v[w]);
      if (same) {
        Vec* to = reinterpret_cast<Vec*>(dx + p.head) + b + tid;
        if (PAST == kPastStores) __builtin_nontemporal_store(o, to);
        else *to = o;
      } else {
#pragma unroll
        for (int w = 0; w < W; ++w) (dx + p.head + b * W)[tid * W + w] = o[w];
      }
    };
    if (y < 0) {
      if (tid == 0) a.loss[r] = 0.f;
      if (dx) {
        const float zero[W] = {};
        for (int b = 0; b < p.n; b += THREADS) store(b, false, zero);
        if (mine >= 0) dx[mine] = from_f32<T>(0.f);
      }
      continue;
    }
    Raw raw[NV];
    const float edge = mine >= 0 ? to_f32(x[mine]) : -INFINITY;
    float m = edge, s = 0.f, lag = 0.f;   // lag: half of the sum of (m - x_j) / V
    for (int c = 0; RES ? c == 0 : c < p.n; c += NV * THREADS) {
#pragma unroll
      for (int i = 0; i < NV; ++i) raw[i] = load(c + i * THREADS, RES && i < NV - 1);
      float top = m;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        unpack_anew<T>(raw[i], top);
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, entry<T>(raw[i], w));
      }
      const float base = exp_base(top);
      s = c == 0 ? exp_less(edge, base) : s * (m == top ? 1.f : exp_less(m, base));
      const float was = m;
      m = top;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        unpack_anew<T>(raw[i], s);
#pragma unroll
        for (int w = 0; w < W; ++w) s += exp_less(entry<T>(raw[i], w), base);
      }
      if (eps != 0.f) {
        if (c == 0) lag = mine >= 0 ? half_gap(base, edge) * inv_v : 0.f;
        else lag += (float)(c / THREADS * W + (mine >= 0)) * inv_v * half_gap(base, exp_base(was));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          unpack_anew<T>(raw[i], lag);
          if ((RES && i < NV - 1) || c + i * THREADS + (int)tid < p.n) {
#pragma unroll
            for (int w = 0; w < W; ++w) lag += half_gap(base, entry<T>(raw[i], w)) * inv_v;
          }
        }
      }
    }
    // Joined over the wave, then over the workgroup.
    float top = wave_max(m), share = 0.f;   // share: entries of those that are joined, over V
    s = wave_sum(s * (m == top ? 1.f : exp_less(m, exp_base(top))));
    if (eps != 0.f) {
      const int own = p.n > (int)tid ? (p.n - (int)tid + THREADS - 1) / THREADS : 0;
      share = (float)(own * W + (mine >= 0)) * inv_v;
      lag = wave_sum(lag + share * half_gap(exp_base(top), exp_base(m)));
      share = wave_sum(share);
    }
    if (tid == 0) target = to_f32(x[y]);   // before anything is written where the logits lie
    if constexpr (WAVES > 1) {
      if ((tid & 63) == 0) { lds[0][tid >> 6] = top; lds[1][tid >> 6] = s; lds[2][tid >> 6] = lag; lds[3][tid >> 6] = share; }
    }
    __syncthreads();
    if constexpr (WAVES > 1) {
      top = lds[0][0];
#pragma unroll
      for (int i = 1; i < WAVES; ++i) top = fmaxf(top, lds[0][i]);
      const float base = exp_base(top);
      if (eps != 0.f && tid < 64)   // the first wave alone, whose thread 0 has the loss
        lag = wave_sum(tid < WAVES ? lds[2][tid] + lds[3][tid] * half_gap(base, exp_base(lds[0][tid])) : 0.f);
      s = 0.f;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) s += lds[1][i] * (lds[0][i] == top ? 1.f : exp_less(lds[0][i], base));
    }
    if (tid == 0) {
      const float log = logf(s);
      float loss = log + (top - target);
      if (eps != 0.f) loss = (eps == 1.f ? 0.f : (1.f - eps) * loss) + (eps * log + 2.f * eps * lag);   // no 0 * inf
      a.loss[r] = loss;
    }
    if (dx) {
      const float g = a.scale ? a.grad_scale * *a.scale : a.grad_scale;
      float by = g / s;
      const float base = exp_base(top), less = g * eps * inv_v, hit = g * (1.f - eps);
      for (int c = 0; RES ? c == 0 : c < p.n; c += NV * THREADS) {
        if constexpr (!RES) {
#pragma unroll
          for (int i = 0; i < NV; ++i) raw[i] = load(c + i * THREADS, false);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int b = c + i * THREADS;
          unpack_anew<T>(raw[i], by);
            float o[W];
#pragma unroll
          for (int w = 0; w < W; ++w) o[w] = exp_less(entry<T>(raw[i], w), base) * by - less;
          const int at = (int)y - p.head - b * W - (int)tid * W;
          if (at >= 0 && at < W) {
#pragma unroll
            for (int w = 0; w < W; ++w) o[w] -= at == w ? hit : 0.f;
          }
          store(b, RES && i < NV - 1, o);
        }
      }
      if (mine >= 0) dx[mine] = from_f32<T>(exp_less(edge, base) * by - less - (mine == (int)y ? hit : 0.f));
    }
    __syncthreads();   // the exchange is used again
  }
}

// out2 = sum of the losses (in 64 bits, rounded once), number of counted rows.
__global__ __launch_bounds__(1024) void loss_sum_kernel(LossArgs a) {
  __shared__ double ss[16];
  __shared__ int sn[16];
  double s = 0.0;
  int n = 0;
  for (int64_t b = threadIdx.x; b < a.rows; b += 8 * 1024) {   // 8 rows of every thread are on their way at once
    float loss[8];
    bool counted[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = b + i * 1024 < a.rows ? b + i * 1024 : b;
      loss[i] = a.loss[r];
      counted[i] = target_of(a, r) >= 0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (b + i * 1024 < a.rows && counted[i]) { s += (double)loss[i]; ++n; }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { s += __shfl_xor(s, o, kWave); n += __shfl_xor(n, o, kWave); }
  if ((threadIdx.x & 63) == 0) { ss[threadIdx.x >> 6] = s; sn[threadIdx.x >> 6] = n; }
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0; n = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) { s += ss[w]; n += sn[w]; }
    a.out2[0] = (float)s; a.out2[1] = (float)n;
  }
}

template <typename T, int WAVES, int NV, bool RES>
void launch_loss_rows(const LossArgs& a, hipStream_t st) {
  const bool same = a.dlogits && (reinterpret_cast<uintptr_t>(a.dlogits) - reinterpret_cast<uintptr_t>(a.logits)) % 16 == 0 && (a.ld - a.ldd) * (int64_t)sizeof(T) % 16 == 0;
  const dim3 grid((unsigned)(a.rows < 1 << 20 ? a.rows : 1 << 20));
  if (!a.dlogits) hipLaunchKernelGGL((cross_entropy_kernel<T, WAVES, NV, RES, kPastLoads>), grid, dim3(64 * WAVES), 0, st, a, same);
  else if (a.rows * a.vocab * (int64_t)sizeof(T) >= kLastLevelCache) hipLaunchKernelGGL((cross_entropy_kernel<T, WAVES, NV, RES, kPastStores>), grid, dim3(64 * WAVES), 0, st, a, same);
  else hipLaunchKernelGGL((cross_entropy_kernel<T, WAVES, NV, RES, kPastNone>), grid, dim3(64 * WAVES), 0, st, a, same);
}
// The kernel that holds a row in `blocks` pieces per thread, LEAST to NV of them.
template <typename T, int WAVES, int LEAST, int NV>
void launch_loss_resident(const LossArgs& a, int blocks, hipStream_t st) {
  if constexpr (NV > LEAST) {
    if (blocks < NV) return launch_loss_resident<T, WAVES, LEAST, NV - 1>(a, blocks, st);
  }
  launch_loss_rows<T, WAVES, NV, true>(a, st);
}

template <typename T>
hipError_t launch_cross_entropy(const LossArgs& a, hipStream_t st) {
  if (a.rows > 0) {
    const int n = a.vocab / (16 / (int)sizeof(T));   // pieces of a row; one that does not begin on 16 bytes has as many or one less
    // Few waves, with 1 to 4 pieces a thread on one, 2 to 8 on four, 5 to 16 on eight, 9 to 16 on sixteen: more of them wait for each other
    // with little to do, and a row that takes more than half of a compute unit's registers leaves no second row to fill its memory's idle
    // time.  us with 1 / 4 / 8 / 16 waves for 48 Mi entries of bf16: rows of 2048 36 / 51 / 89 / 200, 6144 38 / 36 / 46 / 73, 12288 - / 36 /
    // 36 / 51, 24576 - / 39 / 36 / 38, 40960 - / - / 38 / 49, 65536 - / - / 37 / 44; of fp32: 1024 71 / 96 / 163 / 322, 4096 76 / 71 / 70 / 110,
    // 16384 - / 80 / 76 / 74, 32768 - / - / 78 / 81.
    const auto blocks = [n](int waves) { return n < 1 ? 1 : (n + 64 * waves - 1) / (64 * waves); };
    if (n <= 4 * 64) launch_loss_resident<T, 1, 1, 4>(a, blocks(1), st);
    else if (n <= 8 * 256) launch_loss_resident<T, 4, 2, 8>(a, blocks(4), st);
    else if (n <= 16 * 512) launch_loss_resident<T, 8, 5, 16>(a, blocks(8), st);
    else if (n <= 16 * 1024) launch_loss_resident<T, 16, 9, 16>(a, blocks(16), st);
    else launch_loss_rows<T, 16, 8, false>(a, st);
  }
  if (a.out2) hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace varuna
