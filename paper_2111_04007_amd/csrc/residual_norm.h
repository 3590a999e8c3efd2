// What joins a block to the residual stream and feeds the next block:
//   u = Npost(branch), y = alpha x + beta gate * u, z = Npre(y) of y as it is stored
// with N(v) = (v - mean) rstd * weight + bias, mean 0 for the RMS norm; each norm, the gate and the branch may be missing.  Backward, with gz = dz * weight:
//   d = dy + N'(dz),  N'(dz) = rstd (gz - yhat mean(gz yhat) - [layer] mean(gz))
//   dx = alpha d,  du = beta gate * d,  dbranch = Npost'(du),  dgate = sum of beta d * u,  dweight = sum of dz * yhat, ...
//
// Bound by memory: 4 tensors forward, 6 backward, a row is in registers from its one reading on.  A row's threads, one wave or a workgroup of several,
// meet once for each mean that a norm needs.  The parameters' gradients are summed on the way: a workgroup keeps the sums of its rows in
// registers and leaves them in scratch, a second launch adds the workgroups' in order.
#pragma once
#include "common.h"
#include "layer_ops.h"

namespace varuna {

template <typename T> constexpr int norm_width() { return 16 / (int)sizeof(T); }

// Sums of K values over the threads of a row: one wave, or (MULTI) the workgroup of `waves`.  sh: two sides used in turn, so that one barrier is enough.
template <int K, bool MULTI>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*sh)[16][2], int waves, int& side) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
  if (MULTI) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) sh[side][wave][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = 0.f;
      for (int w = 0; w < waves; ++w) s += sh[side][w][k];
      v[k] = s;
    }
    side ^= 1;
  }
}

// The statistics of a row of which this thread has v[0 .. E), entries beyond the row being 0 and counted by `there`.
template <int NC, int W, bool MULTI>
__device__ __forceinline__ void row_statistics(const float (&v)[NC * W], const int (&there)[NC], int h, bool layer, float eps, float (*sh)[16][2], int waves,
                                               int& side, float& mean, float& rstd) {
  mean = 0.f;
  if (layer) {
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NC * W; ++i) s[0] += v[i];
    row_sums<1, MULTI>(s, sh, waves, side);
    mean = s[0] / (float)h;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float d = i < there[c] ? v[c * W + i] - mean : 0.f;
      q[0] += d * d;
    }
  row_sums<1, MULTI>(q, sh, waves, side);
  rstd = 1.0f / sqrtf(q[0] / (float)h + eps);
}

// Both products rounded by themselves: the norm behind goes by y as it is stored, and without a post norm that is then, bit for bit, what any plain evaluation stores.
__device__ __forceinline__ float residual_sum(float alpha, float x, float by, float u) {
#pragma clang fp contract(off)
  return alpha * x + by * u;
}

// NC pieces of a row per thread.  MULTI: a workgroup for a row, otherwise a wave.
template <typename T, int NC, bool MULTI>
__global__ __launch_bounds__(MULTI ? 1024 : 256) void residual_norm_fwd_kernel(NormArgs a) {
  constexpr int W = norm_width<T>();
  __shared__ float sh[2][16][2];
  const int waves = blockDim.x >> 6, threads = MULTI ? (int)blockDim.x : 64, t = MULTI ? (int)threadIdx.x : (int)(threadIdx.x & 63);
  int side = 0;
  for (int64_t row = MULTI ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * waves + (threadIdx.x >> 6); row < a.rows; row += (int64_t)gridDim.x * (MULTI ? 1 : waves)) {
  const int64_t at = row * a.h;
  int there[NC];
  Piece<T, W> xe[NC], be[NC], ge[NC];
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + row / a.rows_per_gate * a.h : nullptr;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int j = (c * threads + t) * W;
    there[c] = a.h - j;
    xe[c] = load_piece<W>(static_cast<const T*>(a.x) + at + j, there[c]);
    if (a.branch) be[c] = load_piece<W>(static_cast<const T*>(a.branch) + at + j, there[c]);
    if (gate) ge[c] = load_piece<W>(gate + j, there[c]);
  }
  float v[NC * W];
  if (a.branch) {
    float mean = 0.f, rstd = 1.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < W; ++i) v[c * W + i] = to_f32(be[c].v[i]);
    if (a.post_weight) {
      row_statistics<NC, W, MULTI>(v, there, a.h, a.layer, a.eps, sh, waves, side, mean, rstd);
      if (a.post_stats && t == 0) { a.post_stats[row] = mean; a.post_stats[a.rows + row] = rstd; }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int j = (c * threads + t) * W;
      if (a.post_weight) {
        const Piece<T, W> w = load_piece<W>(static_cast<const T*>(a.post_weight) + j, there[c]);
#pragma unroll
        for (int i = 0; i < W; ++i) v[c * W + i] = (v[c * W + i] - mean) * rstd * to_f32(w.v[i]);
        if (a.post_bias) {
          const Piece<T, W> b = load_piece<W>(static_cast<const T*>(a.post_bias) + j, there[c]);
#pragma unroll
          for (int i = 0; i < W; ++i) v[c * W + i] += to_f32(b.v[i]);
        }
      }
      Piece<T, W> e;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        e.v[i] = from_f32<T>(residual_sum(a.alpha, to_f32(xe[c].v[i]), gate ? a.beta * to_f32(ge[c].v[i]) : a.beta, v[c * W + i]));
        v[c * W + i] = i < there[c] ? to_f32(e.v[i]) : 0.f;
      }
      if (a.y) store_piece<W>(static_cast<T*>(a.y) + at + j, there[c], e);
    }
  } else {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < W; ++i) v[c * W + i] = to_f32(xe[c].v[i]);
  }
  if (!a.weight) continue;
  float mean, rstd;
  row_statistics<NC, W, MULTI>(v, there, a.h, a.layer, a.eps, sh, waves, side, mean, rstd);
  if (a.stats && t == 0) { a.stats[row] = mean; a.stats[a.rows + row] = rstd; }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int j = (c * threads + t) * W;
    const Piece<T, W> w = load_piece<W>(static_cast<const T*>(a.weight) + j, there[c]);
    Piece<T, W> b, e;
    if (a.bias) b = load_piece<W>(static_cast<const T*>(a.bias) + j, there[c]);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float n = (v[c * W + i] - mean) * rstd * to_f32(w.v[i]);
      e.v[i] = from_f32<T>(a.bias ? n + to_f32(b.v[i]) : n);
    }
    store_piece<W>(static_cast<T*>(a.z) + at + j, there[c], e);
  }
  }
}

template <typename T, int NC>
inline void launch_residual_norm_fwd_pieces(const NormArgs& a, int waves, hipStream_t st) {
  const int64_t most = 1 << 21, groups = waves == 1 ? (a.rows + 3) / 4 : a.rows;
  const dim3 grid((unsigned)(groups < most ? groups : most));
  if (waves == 1) hipLaunchKernelGGL((residual_norm_fwd_kernel<T, NC, false>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((residual_norm_fwd_kernel<T, NC, true>), grid, dim3(64 * waves), 0, st, a);
}

template <typename T>
hipError_t launch_residual_norm_fwd(const NormArgs& a, hipStream_t st) {
  if (a.rows > 0) {
    const int pieces = (a.h + 64 * norm_width<T>() - 1) / (64 * norm_width<T>());   // of a wave
    int waves = 1;
    while (pieces > 2 * waves) waves *= 2;
    if (waves <= 16) {
      if (pieces <= waves) launch_residual_norm_fwd_pieces<T, 1>(a, waves, st);
      else launch_residual_norm_fwd_pieces<T, 2>(a, waves, st);
    } else {
      launch_residual_norm_fwd_pieces<T, 4>(a, 16, st);
    }
  }
  return hipGetLastError();
}

// ---- backward ---------------------------------------------------------------------------------

// How the rows are shared: segments of rows that have a gate in common (all rows where there is none).  A workgroup takes `chunk` rows of one segment, or, if
// segments are of at most kNormShort rows, `chunk` whole segments, whose gate's gradient is complete where it is summed.
constexpr int kNormShort = 16, kNormGroups = 1024;
struct NormSplit {
  int64_t segment, segments, chunk, per_segment, groups;
  bool whole;
};
inline NormSplit norm_split(int64_t rows, int64_t rows_per_gate) {
  NormSplit s{};
  if (rows < 1) return s;
  s.segment = rows_per_gate > 0 && rows_per_gate < rows ? rows_per_gate : rows;
  s.segments = (rows + s.segment - 1) / s.segment;
  s.whole = s.segments > 1 && s.segment <= kNormShort;
  if (s.whole) {
    s.chunk = (s.segments + kNormGroups - 1) / kNormGroups;
    s.groups = (s.segments + s.chunk - 1) / s.chunk;
    s.per_segment = 0;
  } else {
    const int64_t want = (kNormGroups + s.segments - 1) / s.segments;
    s.chunk = (s.segment + want - 1) / want;
    s.per_segment = (s.segment + s.chunk - 1) / s.chunk;
    s.groups = s.segments * s.per_segment;
  }
  return s;
}

enum NormSum : int { NS_WEIGHT = 0, NS_BIAS = 1, NS_POST_WEIGHT = 2, NS_POST_BIAS = 3, NS_GATE = 4, NS_COUNT = 5 };

int64_t residual_norm_bwd_groups(int64_t rows, int64_t rows_per_gate) { return norm_split(rows, rows_per_gate).groups; }
size_t residual_norm_bwd_scratch_bytes(int64_t rows, int64_t h, int64_t rows_per_gate) {
  return (size_t)norm_split(rows, rows_per_gate).groups * NS_COUNT * (size_t)h * sizeof(float);
}

// NC pieces of a row per thread.  BIASED: a bias' gradient is wanted.
template <typename T, int NC, bool MULTI, bool BIASED, bool POST, bool GATE>
__global__ __launch_bounds__(MULTI ? 1024 : 256) void residual_norm_bwd_kernel(NormArgs a, NormSplit s) {
  constexpr int W = norm_width<T>(), E = NC * W;
  __shared__ float sh[2][16][2];
  __shared__ float joined[MULTI ? 1 : 3][MULTI ? 1 : 64 * E];
  const int waves = blockDim.x >> 6, wave = (int)(threadIdx.x >> 6), threads = MULTI ? (int)blockDim.x : 64, t = MULTI ? (int)threadIdx.x : (int)(threadIdx.x & 63);
  int side = 0;
  const bool pre = a.weight != nullptr;
  int there[NC];
  Piece<T, W> we[NC], pe[NC], pb[NC];
  float dw[E], db[BIASED ? E : 1], dpw[POST ? E : 1], dpb[POST && BIASED ? E : 1], dg[GATE ? E : 1];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int j = (c * threads + t) * W;
    there[c] = a.h - j;
    if (pre) we[c] = load_piece<W>(static_cast<const T*>(a.weight) + j, there[c]);
    if (POST) pe[c] = load_piece<W>(static_cast<const T*>(a.post_weight) + j, there[c]);
    if (POST && GATE && a.post_bias) pb[c] = load_piece<W>(static_cast<const T*>(a.post_bias) + j, there[c]);
  }
#pragma unroll
  for (int i = 0; i < E; ++i) {
    dw[i] = 0.f;
    if (BIASED) db[i] = 0.f;
    if (POST) dpw[i] = 0.f;
    if (POST && BIASED) dpb[i] = 0.f;
    if (GATE) dg[i] = 0.f;
  }
  const int64_t group = blockIdx.x;
  const int workers = MULTI ? 1 : waves, worker = MULTI ? 0 : wave;
  const int64_t seg0 = s.whole ? group * s.chunk + worker : group / s.per_segment;
  int64_t seg1 = s.whole ? (group + 1) * s.chunk : seg0 + 1;
  if (seg1 > s.segments) seg1 = s.segments;
  for (int64_t seg = seg0; seg < seg1; seg += s.whole ? workers : 1) {
    int64_t begin = seg * s.segment, end = begin + s.segment;
    if (end > a.rows) end = a.rows;
    if (!s.whole) {
      begin += (group - seg * s.per_segment) * s.chunk;
      if (end > begin + s.chunk) end = begin + s.chunk;
      begin += worker;
    }
    const T* gate = GATE ? static_cast<const T*>(a.gate) + seg * a.h : nullptr;
    for (int64_t row = begin; row < end; row += s.whole ? 1 : workers) {
      const int64_t at = row * a.h;
      Piece<T, W> ze[NC], ye[NC], de[NC], be[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int j = (c * threads + t) * W;
        if (pre) {
          ze[c] = load_piece<W>(static_cast<const T*>(a.dz) + at + j, there[c]);
          ye[c] = load_piece<W>(static_cast<const T*>(a.x) + at + j, there[c]);
        }
        if (a.dy) de[c] = load_piece<W>(static_cast<const T*>(a.dy) + at + j, there[c]);
        if (POST || GATE) be[c] = load_piece<W>(static_cast<const T*>(a.branch) + at + j, there[c]);
      }
      float d[E];
      if (pre) {
        const float mean = a.layer ? a.stats[row] : 0.f, rstd = a.stats[a.rows + row];
        float k[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const float z = to_f32(ze[c].v[i]), hat = i < there[c] ? (to_f32(ye[c].v[i]) - mean) * rstd : 0.f, g = z * to_f32(we[c].v[i]);
            k[0] += g * hat;
            k[1] += g;
            dw[c * W + i] += z * hat;
            if (BIASED) db[c * W + i] += z;
          }
        if (a.layer) row_sums<2, MULTI>(k, sh, waves, side);
        else { float one[1] = {k[0]}; row_sums<1, MULTI>(one, sh, waves, side); k[0] = one[0]; k[1] = 0.f; }
        k[0] /= (float)a.h;
        k[1] /= (float)a.h;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const float hat = (to_f32(ye[c].v[i]) - mean) * rstd, g = to_f32(ze[c].v[i]) * to_f32(we[c].v[i]);
            d[c * W + i] = rstd * (g - k[1] - hat * k[0]) + (a.dy ? to_f32(de[c].v[i]) : 0.f);
          }
      } else {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < W; ++i) d[c * W + i] = to_f32(de[c].v[i]);
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int j = (c * threads + t) * W;
        Piece<T, W> e;
#pragma unroll
        for (int i = 0; i < W; ++i) e.v[i] = from_f32<T>(a.alpha * d[c * W + i]);
        store_piece<W>(static_cast<T*>(a.y) + at + j, there[c], e);
      }
      if (!POST && !GATE && a.z == nullptr) continue;
      float mean = 0.f, rstd = 1.f;
      if (POST) { mean = a.layer ? a.post_stats[row] : 0.f; rstd = a.post_stats[a.rows + row]; }
      float k[2] = {0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        Piece<T, W> ge;
        if (GATE) ge = load_piece<W>(gate + (c * threads + t) * W, there[c]);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          float du = a.beta * d[c * W + i];
          const float b = POST || GATE ? to_f32(be[c].v[i]) : 0.f, hat = POST ? (i < there[c] ? (b - mean) * rstd : 0.f) : b;
          if (GATE) {
            float u = hat;
            if (POST) { u = hat * to_f32(pe[c].v[i]); if (a.post_bias) u += to_f32(pb[c].v[i]); }
            dg[c * W + i] += du * u;
            du *= to_f32(ge.v[i]);
          }
          if (i >= there[c]) du = 0.f;
          d[c * W + i] = du;
          if (POST) {
            const float g = du * to_f32(pe[c].v[i]);
            k[0] += g * hat;
            k[1] += g;
            dpw[c * W + i] += du * hat;
            if (BIASED) dpb[c * W + i] += du;
          }
        }
      }
      if (POST) {
        if (a.layer) row_sums<2, MULTI>(k, sh, waves, side);
        else { float one[1] = {k[0]}; row_sums<1, MULTI>(one, sh, waves, side); k[0] = one[0]; k[1] = 0.f; }
        k[0] /= (float)a.h;
        k[1] /= (float)a.h;
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        Piece<T, W> e;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          float v = d[c * W + i];
          if (POST) v = rstd * (v * to_f32(pe[c].v[i]) - k[1] - (to_f32(be[c].v[i]) - mean) * rstd * k[0]);
          e.v[i] = from_f32<T>(v);
        }
        store_piece<W>(static_cast<T*>(a.z) + at + (c * threads + t) * W, there[c], e);
      }
    }
    if (GATE && s.whole && a.dgate) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float* to = a.dgate + seg * a.h + (c * threads + t) * W;
        Piece<float, W> e;
        if (a.accumulate) e = load_piece<W>(to, there[c]);
#pragma unroll
        for (int i = 0; i < W; ++i) { e.v[i] = a.accumulate ? e.v[i] + dg[c * W + i] : dg[c * W + i]; dg[c * W + i] = 0.f; }
        store_piece<W>(to, there[c], e);
      }
    }
  }
  // The workgroup's sums: waves that had rows of their own are joined first.
  auto leave = [&](const float* sums, int which) {
    float* to = a.scratch + (group * NS_COUNT + which) * a.h;
    if constexpr (!MULTI) {
      __syncthreads();
      if (wave > 0) {
#pragma unroll
        for (int i = 0; i < E; ++i) joined[wave - 1][i * 64 + t] = sums[i];
      }
      __syncthreads();
      if (wave > 0) return;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      Piece<float, W> e;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        float v = sums[c * W + i];
        if constexpr (!MULTI)
          for (int w = 0; w < 3; ++w) v += joined[w][(c * W + i) * 64 + t];
        e.v[i] = v;
      }
      store_piece<W>(to + (c * threads + t) * W, there[c], e);
    }
  };
  if (a.dweight) leave(dw, NS_WEIGHT);
  if (BIASED && a.dbias) leave(db, NS_BIAS);
  if (POST && a.dpost_weight) leave(dpw, NS_POST_WEIGHT);
  if (POST && BIASED && a.dpost_bias) leave(dpb, NS_POST_BIAS);
  if (GATE && !s.whole && a.dgate) leave(dg, NS_GATE);
}

// Sums of the workgroups' sums: 32 columns, 8 of the workgroups at a time.  A job of `across` column blocks for each parameter's gradient, over all
// workgroups, then for each segment's gate.
__global__ __launch_bounds__(256) void residual_norm_sums_kernel(NormArgs a, NormSplit s, uint32_t across, int64_t blocks) {
  __shared__ float sh[8][32];
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int64_t job = b / across;
    const int col = (int)(b - job * across) * 32 + (int)(threadIdx.x & 31), lane = threadIdx.x >> 5;
    const int which = job < NS_GATE ? (int)job : (int)NS_GATE;
    float* out = job == NS_WEIGHT ? a.dweight : job == NS_BIAS ? a.dbias : job == NS_POST_WEIGHT ? a.dpost_weight : job == NS_POST_BIAS ? a.dpost_bias
                                                                                                                : a.dgate + (job - NS_GATE) * a.h;
    if (!out) continue;
    const int64_t begin = job < NS_GATE ? 0 : (job - NS_GATE) * s.per_segment, end = job < NS_GATE ? s.groups : begin + s.per_segment;
    float v = 0.f;
    if (col < a.h)
      for (int64_t g = begin + lane; g < end; g += 8) v += a.scratch[(g * NS_COUNT + which) * a.h + col];
    sh[lane][threadIdx.x & 31] = v;
    __syncthreads();
    if (lane == 0 && col < a.h) {
      v = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) v += sh[k][threadIdx.x];
      out[col] = a.accumulate ? out[col] + v : v;
    }
    __syncthreads();
  }
}

template <typename T, int NC, bool MULTI>
inline void launch_residual_norm_bwd_pieces(const NormArgs& a, const NormSplit& s, int waves, hipStream_t st) {
  const dim3 grid((unsigned)s.groups), block(MULTI ? 64 * waves : 256);
  const bool biased = a.dbias || a.dpost_bias, post = a.post_weight != nullptr, gate = a.gate != nullptr;
#define VARUNA_NORM_BWD(B, P, G) hipLaunchKernelGGL((residual_norm_bwd_kernel<T, NC, MULTI, B, P, G>), grid, block, 0, st, a, s)
  if (biased) {
    if (post) { if (gate) VARUNA_NORM_BWD(true, true, true); else VARUNA_NORM_BWD(true, true, false); }
    else { if (gate) VARUNA_NORM_BWD(true, false, true); else VARUNA_NORM_BWD(true, false, false); }
  } else {
    if (post) { if (gate) VARUNA_NORM_BWD(false, true, true); else VARUNA_NORM_BWD(false, true, false); }
    else { if (gate) VARUNA_NORM_BWD(false, false, true); else VARUNA_NORM_BWD(false, false, false); }
  }
#undef VARUNA_NORM_BWD
}

template <typename T>
hipError_t launch_residual_norm_bwd(const NormArgs& a, hipStream_t st) {
  constexpr int W = norm_width<T>(), NC = 16 / W;   // 16 entries a thread
  const NormSplit s = norm_split(a.rows, a.gate ? a.rows_per_gate : 0);
  const int pieces = (a.h + 64 * W - 1) / (64 * W);
  int waves = 1;
  while (pieces > NC * waves) waves *= 2;
  if (a.rows < 1) {}
  else if (waves > 1) launch_residual_norm_bwd_pieces<T, NC, true>(a, s, waves, st);
  else if (pieces <= NC / 2) launch_residual_norm_bwd_pieces<T, NC / 2, false>(a, s, 1, st);
  else launch_residual_norm_bwd_pieces<T, NC, false>(a, s, 1, st);
  const bool gates = a.dgate && !s.whole, params = a.dweight || a.dbias || a.dpost_weight || a.dpost_bias;
  const uint32_t across = (uint32_t)(a.h + 31) / 32;
  const int64_t blocks = across * (NS_GATE + (gates ? s.segments : 0)), most = 1 << 22;
  if (gates || params) hipLaunchKernelGGL(residual_norm_sums_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a, s, across, blocks);
  return hipGetLastError();
}

}  // namespace varuna
