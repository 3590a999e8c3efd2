// What a layer with rotary positions and norms on both sides of its blocks needs beside products and attention, and the update of many
// tensors: what stage.hip's C ABI checks and hands over, layer_ops.hip launches.  Pointers are device memory except where marked host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pipeline_ends.h"

namespace varuna {

// U entries of a row as they lie in memory; vectors need no more than an element's alignment.
template <typename T, int U> struct Piece { T v[U]; };
// p[0 .. U), of which n lie in the row (the rest: 0).  PAST: past the caches.
template <int U, bool PAST = false, typename T>
__device__ __forceinline__ Piece<T, U> load_piece(const T* p, int n) {
  typedef T Any __attribute__((ext_vector_type(U), aligned(sizeof(T))));
  Piece<T, U> e;
  if (n >= U) {
    Any a;
    if constexpr (PAST) a = __builtin_nontemporal_load(reinterpret_cast<const Any*>(p));
    else a = *reinterpret_cast<const Any*>(p);
#pragma unroll
    for (int i = 0; i < U; ++i) e.v[i] = a[i];
  } else {
#pragma unroll
    for (int i = 0; i < U; ++i) e.v[i] = i < n ? p[i] : (T)0.f;
  }
  return e;
}
template <int U, bool PAST = false, typename T>
__device__ __forceinline__ void store_piece(T* p, int n, const Piece<T, U>& e) {
  typedef T Any __attribute__((ext_vector_type(U), aligned(sizeof(T))));
  if (n >= U) {
    Any a;
#pragma unroll
    for (int i = 0; i < U; ++i) a[i] = e.v[i];
    if constexpr (PAST) __builtin_nontemporal_store(a, reinterpret_cast<Any*>(p));
    else *reinterpret_cast<Any*>(p) = a;
  } else {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (i < n) p[i] = e.v[i];
  }
}

// ---- rotary positions -------------------------------------------------------------------
constexpr int kRotaryMost = 512;   // entries of a head that turn: their frequencies travel as kernel arguments
struct RotaryTableArgs {
  double freq[kRotaryMost / 2];
  double magnitude;
  float* table;   // [n, r]: cosines, then sines
  int64_t n;
  int r;
};
hipError_t launch_rotary_table(const RotaryTableArgs& a, hipStream_t st);

struct RotaryArgs {
  const void* x;
  void* out;         // may be x, with its strides
  int64_t x_row, x_head, out_row, out_head;
  IdArgs positions;
  const float* table;
  int64_t rows, n_positions;
  int heads, d, r;
  bool interleaved, transpose;
};
template <typename T> hipError_t launch_rotary(const RotaryArgs& a, hipStream_t st);

// ---- the residual stream between two blocks -----------------------------------------------
constexpr int kNormMost = 16384;   // entries of a row, which is held in registers
struct NormArgs {
  const void *x, *branch, *post_weight, *post_bias, *gate, *weight, *bias;   // x: y in the backward pass
  const void *dz, *dy;
  void *y, *z;              // dx and dbranch in the backward pass
  float *stats, *post_stats;
  float *dweight, *dbias, *dpost_weight, *dpost_bias, *dgate;
  float* scratch;
  int64_t rows, rows_per_gate;
  int h;
  float alpha, beta, eps;
  bool layer, accumulate;
};
template <typename T> hipError_t launch_residual_norm_fwd(const NormArgs& a, hipStream_t st);
template <typename T> hipError_t launch_residual_norm_bwd(const NormArgs& a, hipStream_t st);
// Groups of rows that leave sums of their own.
int64_t residual_norm_bwd_groups(int64_t rows, int64_t h, int64_t rows_per_gate);
size_t residual_norm_bwd_scratch_bytes(int64_t rows, int64_t h, int64_t rows_per_gate);

// ---- AdamW over many tensors ----------------------------------------------------------------
constexpr int kStateBlock = 256;   // entries that share a scale; every tensor's state begins a new one
struct AdamWArgs {
  float one_minus_beta1, one_minus_beta2, beta1, beta2, eps, grad_scale;
  double lr, weight_decay, log2_beta1, log2_beta2, max_norm, clip_eps;
  int64_t step;
  const double* sum_sq;    // may be null
  const double* lr_step;   // may be null: {lr, step}
  const float* skip;       // may be null
  float* master;
  void *m, *v;
  float* scales;           // null: m and v are fp32, otherwise e4m3 codes and two floats a block
};
hipError_t launch_adamw(const TensorSpan& params, const TensorSpan& grads, const float* decays, const AdamWArgs& a, hipStream_t st);

}  // namespace varuna
