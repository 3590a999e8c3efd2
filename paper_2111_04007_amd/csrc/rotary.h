// Rotary positions: the pairs (a, b) of a head's first r entries are turned by the angle t = position * frequency of the pair,
//   a' = M (a cos t - b sin t),  b' = M (a sin t + b cos t),
// the transposed turn, sin t -> -sin t, is the gradient.  Pairs are entries (i, i + r/2) or, interleaved, (2i, 2i + 1).  M cos t and M sin t come from
// a table made once with angles in 64 bits (a position of 100000 leaves 32 bits no more than 7 binary digits behind the point).
//
// Bound by memory: every turned entry is read and written once, a row of the table serves all heads of its row and comes from the caches.  A thread turns one piece of
// one head: holding its cosines and sines for 2, 4 or 8 heads was slower (16384 rows of 128 heads of 128 bf16, in place: 198 us; 205, 210, 214).  Past the caches, which that
// call does not fit, it takes 169 us: 6.3 TB/s.
#pragma once
#include "common.h"
#include "layer_ops.h"

namespace varuna {

__global__ __launch_bounds__(256) void rotary_table_kernel(RotaryTableArgs a) {
  const int n = a.r / 2;
  const int64_t all = a.n * n;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < all; k += (int64_t)gridDim.x * 256) {
    const int64_t p = k / n;
    const int i = (int)(k - p * n);
    double s, c;
    sincos((double)p * a.freq[i], &s, &c);
    a.table[p * a.r + i] = (float)(a.magnitude * c);
    a.table[p * a.r + n + i] = (float)(a.magnitude * s);
  }
}

hipError_t launch_rotary_table(const RotaryTableArgs& a, hipStream_t st) {
  const int64_t blocks = (a.n * (a.r / 2) + 255) / 256;
  if (blocks > 0) hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, st, a);
  return hipGetLastError();
}

__device__ __forceinline__ int32_t rotary_position(const RotaryArgs& a, uint32_t t) {
  if (a.positions.p == nullptr) return (int32_t)(t % a.positions.period);
  if (a.positions.wide) {
    const int64_t v = static_cast<const int64_t*>(a.positions.p)[t];
    return v >= 0 && v < a.n_positions ? (int32_t)v : -1;
  }
  const int32_t v = static_cast<const int32_t*>(a.positions.p)[t];
  return v >= 0 && v < a.n_positions ? v : -1;
}

// W pairs per thread, whose sides lie apart or (interleaved) side by side.  slots: pieces of the turned entries of a head, the last of which is the last W pairs where W does not divide
// them (it leaves out those of the piece before it, which that one may have turned in place already), then (out of place) pieces of the entries behind them, which are
// copied.  PAST: past the caches.
template <typename T, int W, bool INTER, bool PAST>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int slots, int turned, int64_t items) {
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < items; k += (int64_t)gridDim.x * 256) {
    const uint32_t q = (uint32_t)(k / slots);   // rows * heads fit 31 bits
    const int slot = (int)(k - (int64_t)q * slots);
    const uint32_t row = q / (uint32_t)a.heads, head = q - row * (uint32_t)a.heads;
    const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.x_row + (int64_t)head * a.x_head;
    T* out = static_cast<T*>(a.out) + (int64_t)row * a.out_row + (int64_t)head * a.out_head;
    if (slot >= turned) {
      const int at = a.r + (slot - turned) * 2 * W, n = a.d - at;
      store_piece<2 * W, PAST>(out + at, n, load_piece<2 * W, PAST>(x + at, n));
      continue;
    }
    const int p = rotary_position(a, row), half = a.r / 2, begin = slot * W, pair = begin + W <= half ? begin : half - W, skip = begin - pair;
    const int at = INTER ? 2 * pair : pair, other = INTER ? W : half;
    if (p < 0 && a.x == a.out) continue;   // a row without a position stays as it is
    const float* table = a.table + (int64_t)(p < 0 ? 0 : p) * a.r + pair;
    const Piece<float, W> c = load_piece<W>(table, W), s = load_piece<W>(table + half, W);
    const Piece<T, W> e = load_piece<W, PAST>(x + at, W), f = load_piece<W, PAST>(x + at + other, W);
    __builtin_amdgcn_sched_barrier(0);   // all loads are under way before the first is waited for (interleaved bf16 193 -> 171 us)
    Piece<T, W> g, b;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      // interleaved: pair i lies at 2i, 2i + 1 of the two pieces side by side
      const float u = to_f32(INTER ? (2 * i < W ? e.v[2 * i % W] : f.v[2 * i % W]) : e.v[i]);
      const float v = to_f32(INTER ? (2 * i + 1 < W ? e.v[(2 * i + 1) % W] : f.v[(2 * i + 1) % W]) : f.v[i]);
      const float si = a.transpose ? -s.v[i] : s.v[i];
      T& first_side = INTER ? (2 * i < W ? g.v[2 * i % W] : b.v[2 * i % W]) : g.v[i];
      T& other_side = INTER ? (2 * i + 1 < W ? g.v[(2 * i + 1) % W] : b.v[(2 * i + 1) % W]) : b.v[i];
      first_side = from_f32<T>(u * c.v[i] - v * si);
      other_side = from_f32<T>(u * si + v * c.v[i]);
    }
    if (p < 0) { g = e; b = f; }
    if (skip == 0) {
      store_piece<W, PAST>(out + at, W, g);
      store_piece<W, PAST>(out + at + other, W, b);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) {   // entries of the pairs from `skip` on
        if ((INTER ? i / 2 : i) >= skip) out[at + i] = g.v[i];
        if ((INTER ? (W + i) / 2 : i) >= skip) out[at + other + i] = b.v[i];
      }
    }
  }
}

// From this many bytes on entries go past the caches.  us in place, through / past, alone and with a pass behind that reads everything: 64 MB 22.4 / 23.8, 42.1 / 44.4; 128 MB 42.4 / 44.6, 88 / 86;
// 192 MB 71.6 / 64.9, 135 / 134; 256 MB 93.6 / 85.4, 184 / 176; 512 MB 185 / 169, 366 / 344.
constexpr int64_t kRotaryPast = 192ll << 20;

template <typename T, int W, bool INTER>
inline void launch_rotary_pieces(const RotaryArgs& a, hipStream_t st) {
  const int turned = (a.r / 2 + W - 1) / W, slots = turned + (a.x == a.out ? 0 : (a.d - a.r + 2 * W - 1) / (2 * W));
  const int64_t items = a.rows * a.heads * slots, blocks = (items + 255) / 256, most = 1 << 22;
  const int64_t bytes = a.rows * a.heads * (a.x == a.out ? a.r : 2 * a.d) * (int64_t)sizeof(T);
  auto kernel = bytes >= kRotaryPast ? rotary_kernel<T, W, INTER, true> : rotary_kernel<T, W, INTER, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a, slots, turned, items);
}

template <typename T>
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t st) {
  if (a.rows > 0 && a.heads > 0) {
    // Pieces of 16 bytes, which are half as many pairs where they lie side by side (16384 rows of 128 heads of 128, us: 188 / 210 with twice as many); fewer pairs than that one by one.
    constexpr int W = 16 / (int)sizeof(T);
    const int half = a.r / 2;
    if (a.interleaved) {
      if (half >= W / 2) launch_rotary_pieces<T, W / 2, true>(a, st);
      else launch_rotary_pieces<T, 1, true>(a, st);
    } else {
      if (half >= W) launch_rotary_pieces<T, W, false>(a, st);
      else launch_rotary_pieces<T, 1, false>(a, st);
    }
  }
  return hipGetLastError();
}

}  // namespace varuna
