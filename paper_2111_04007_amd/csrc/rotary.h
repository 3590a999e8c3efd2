// Rotary positions: the pairs (a, b) of a head's first r entries are turned by the angle t = position * frequency of the pair,
//   a' = M (a cos t - b sin t),  b' = M (a sin t + b cos t),
// the transposed turn, sin t -> -sin t, is the gradient.  Pairs are entries (i, i + r/2) or, interleaved, (2i, 2i + 1).  M cos t and M sin t come from
// a table made once with angles in 64 bits (a position of 100000 leaves 32 bits no more than 7 binary digits behind the point).
//
// Bound by memory: every turned entry is read and written once, a row of the table serves all heads of its row.  A thread holds the
// cosines and sines of one piece of pairs and goes through several heads with them.
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

// W entries of each of a pair's sides per thread (interleaved: W pairs side by side), H heads.  slots: pieces of the turned entries of a
// head, then (out of place) those of the entries behind them, which are copied; groups: heads are h, h + groups, ...
template <typename T, int W, int H, bool INTER>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int slots, int turned, int groups, int64_t items) {
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < items; k += (int64_t)gridDim.x * 256) {
    const int64_t q = k / slots;
    const int slot = (int)(k - q * slots);
    const uint32_t row = (uint32_t)(q / groups);
    const int first = (int)(q - (int64_t)row * groups);
    const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.x_row;
    T* out = static_cast<T*>(a.out) + (int64_t)row * a.out_row;
    if (slot >= turned) {
      const int at = a.r + (slot - turned) * 2 * W, n = a.d - at;
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const int head = first + h * groups;
        if (head < a.heads) store_piece<2 * W>(out + head * a.out_head + at, n, load_piece<2 * W>(x + head * a.x_head + at, n));
      }
      continue;
    }
    const int p = rotary_position(a, row), half = a.r / 2;
    const float* table = a.table + (int64_t)(p < 0 ? 0 : p) * a.r + slot * W;
    const Piece<float, W> c = load_piece<W>(table, W), s = load_piece<W>(table + half, W);
    const int at = INTER ? slot * 2 * W : slot * W;
    if (p < 0 && a.x == a.out) continue;   // a row without a position stays as it is
    const float sign = a.transpose ? -1.f : 1.f;
    Piece<T, W> e[H], f[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int head = first + h * groups;
      if (head >= a.heads) continue;
      const T* from = x + head * a.x_head + at;
      e[h] = load_piece<W>(from, W);
      f[h] = load_piece<W>(from + (INTER ? W : half), W);
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int head = first + h * groups;
      if (head >= a.heads) continue;
      T* to = out + head * a.out_head + at;
      Piece<T, W> g, b;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float u = to_f32(INTER ? (2 * i < W ? e[h].v[2 * i % W] : f[h].v[2 * i % W]) : e[h].v[i]);
        const float v = to_f32(INTER ? (2 * i + 1 < W ? e[h].v[(2 * i + 1) % W] : f[h].v[(2 * i + 1) % W]) : f[h].v[i]);
        const float si = sign * s.v[i];
        const T m = from_f32<T>(u * c.v[i] - v * si), n = from_f32<T>(u * si + v * c.v[i]);
        T& first_side = INTER ? (2 * i < W ? g.v[2 * i % W] : b.v[2 * i % W]) : g.v[i];
        T& other_side = INTER ? (2 * i + 1 < W ? g.v[(2 * i + 1) % W] : b.v[(2 * i + 1) % W]) : b.v[i];
        first_side = m;
        other_side = n;
      }
      if (p < 0) { g = e[h]; b = f[h]; }
      store_piece<W>(to, W, g);
      store_piece<W>(to + (INTER ? W : half), W, b);
    }
  }
}

template <typename T, int W, int H>
inline void launch_rotary_pieces(const RotaryArgs& a, hipStream_t st) {
  const int turned = a.r / 2 / W, slots = turned + (a.x == a.out ? 0 : (a.d - a.r + 2 * W - 1) / (2 * W));
  const int groups = (a.heads + H - 1) / H;
  const int64_t items = a.rows * groups * slots, blocks = (items + 255) / 256;
  const dim3 grid((unsigned)(blocks < (1 << 22) ? blocks : 1 << 22));
  if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<T, W, H, true>), grid, dim3(256), 0, st, a, slots, turned, groups, items);
  else hipLaunchKernelGGL((rotary_kernel<T, W, H, false>), grid, dim3(256), 0, st, a, slots, turned, groups, items);
}

template <typename T>
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t st) {
  if (a.rows > 0 && a.heads > 0) {
    constexpr int W = 16 / (int)sizeof(T);
    const int half = a.r / 2;
    if (half % W == 0) launch_rotary_pieces<T, W, 4>(a, st);
    else launch_rotary_pieces<T, 1, 4>(a, st);
  }
  return hipGetLastError();
}

}  // namespace varuna
