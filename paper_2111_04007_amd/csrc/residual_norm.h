// What joins a block to the residual stream and feeds the next block:
//   u = Npost(branch), y = alpha x + beta gate * u, z = Npre(y) of y as it is stored
// with N(v) = (v - mean) rstd * weight + bias, mean 0 for the RMS norm; each norm, the gate and the branch may be missing.  Backward, with gz = dz * weight:
//   d = dy + N'(dz),  N'(dz) = rstd (gz - yhat mean(gz yhat) - [layer] mean(gz))
//   dx = alpha d,  du = beta gate * d,  dbranch = Npost'(du),  dgate = sum of beta d * u,  dweight = sum of dz * yhat, ...
//
// Bound by memory: 4 tensors forward, 6 backward, a row is in registers from its one reading on.  A row's threads, one wave or a workgroup of several,
// meet once for each mean that a norm needs.  The parameters' gradients are summed on the way: a workgroup keeps the sums of its rows in
// registers and shared memory and leaves them in scratch, a second launch adds the workgroups' in order.
// bf16, a norm on both sides: forward 16384x8192 201 us (5.3 TB/s; a large copy moves 4.7), backward 8192x8192 with a gate 171 us (4.7 TB/s, of it the second launch 6); forward
// 4096x1920 14 us, backward 4096x1024 20 us.
#pragma once
#include "common.h"
#include "layer_ops.h"

#include <type_traits>

namespace varuna {

// The sum over 16 lanes, in each of them.
__device__ __forceinline__ float lanes_total(float v) {
  auto dpp = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)); };
  v += dpp(v, std::integral_constant<int, 0xb1>{});    // quad_perm 1 0 3 2
  v += dpp(v, std::integral_constant<int, 0x4e>{});    // quad_perm 2 3 0 1
  v += dpp(v, std::integral_constant<int, 0x141>{});   // row_half_mirror
  v += dpp(v, std::integral_constant<int, 0x140>{});   // row_mirror
  return v;
}
// The sum over a wave, in every lane.
__device__ __forceinline__ float wave_total(float v) {
  v = lanes_total(v);
  auto lane = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return (lane(0) + lane(16)) + (lane(32) + lane(48));
}

// Which entries of a row are thread t's: E consecutive ones from `at` on, of which those in the bits of `own` are its.  The last thread of a row that is no
// multiple of E takes the row's last E entries, so that every load is a whole one, and leaves out those of the thread before it.  Rows have at least E entries.
template <int E> struct Window {
  int at;
  uint32_t own;
  static constexpr uint32_t kAll = (1u << E) - 1;
  __device__ __forceinline__ Window(int t, int h) {
    const int j = t * E;
    at = j + E <= h ? j : h - E;
    own = j >= h ? 0 : kAll << (j - at) & kAll;
  }
};

// E entries of a row as they lie in memory, in whole registers: two bf16 entries to one.  They are unpacked where they are used; keep() stands
// between two uses, or the compiler unpacks once and holds three times the registers in between.
template <typename T, int E> struct Packed {
  static constexpr int N = E * (int)sizeof(T) / 4 > 0 ? E * (int)sizeof(T) / 4 : 1;
  uint32_t v[N];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[i]);
    else return __uint_as_float((i & 1) ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
  }
  __device__ __forceinline__ void keep() {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
  }
  // Entries that are not this thread's become 0.
  __device__ __forceinline__ void clear(uint32_t own) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const bool mine = own >> i & 1;
      if constexpr (sizeof(T) == 4) v[i] = mine ? v[i] : 0u;
      else v[i / 2] = mine ? v[i / 2] : v[i / 2] & ((i & 1) ? 0xffffu : 0xffff0000u);
    }
  }
};
// Vectors need no more than an element's alignment.  PAST: past the caches.
template <int E, bool PAST = false, typename T>
__device__ __forceinline__ Packed<T, E> load_window(const T* row, const Window<E>& w) {
  Packed<T, E> e;
  if constexpr (E * sizeof(T) >= 16) {
    constexpr int U = 16 / (int)sizeof(T);
    typedef T Any __attribute__((ext_vector_type(U), aligned(sizeof(T))));
    typedef T Vec __attribute__((ext_vector_type(U)));
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int k = 0; k < Packed<T, E>::N / 4; ++k) {
      const Any* p = reinterpret_cast<const Any*>(row + w.at) + k;
      Vec v;
      if constexpr (PAST) v = __builtin_nontemporal_load(p);
      else v = *p;
      const Words q = __builtin_bit_cast(Words, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) e.v[4 * k + i] = q[i];
    }
  } else {
    static_assert(E == 1, "whole pieces of 16 bytes, or entries");
    e.v[0] = sizeof(T) == 4 ? __float_as_uint(row[w.at]) : (uint32_t)reinterpret_cast<const uint16_t*>(row)[w.at];
  }
  return e;
}
template <int E, bool PAST = false, typename T>
__device__ __forceinline__ void store_window(T* row, const Window<E>& w, uint32_t own, const float (&v)[E]) {
  constexpr int U = E * sizeof(T) >= 16 ? 16 / (int)sizeof(T) : E;
  T* p = row + w.at;
  if (own == Window<E>::kAll) {
#pragma unroll
    for (int k = 0; k < E; k += U) {
      Piece<T, U> q;
#pragma unroll
      for (int i = 0; i < U; ++i) q.v[i] = from_f32<T>(v[k + i]);
      store_piece<U, PAST>(p + k, U, q);
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (own >> i & 1) p[i] = from_f32<T>(v[i]);
  }
}

// Sums of K values over the `waves` of a row's team, the first of which is wave `first` of the workgroup.  sh: two sides used in turn, so that one barrier is enough.
template <int K>
__device__ __forceinline__ void team_sums(float (&v)[K], float (*sh)[16][2], int first, int waves, int& side) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_total(v[k]);
  if (waves == 1) return;
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) sh[side][threadIdx.x >> 6][k] = v[k];
  }
  __syncthreads();
  const int wave = (int)(threadIdx.x & 15);   // 16 lanes hold the waves' sums
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = lanes_total(wave < waves ? sh[side][first + wave][k] : 0.f);
  side ^= 1;
}

// 1 / sqrt(x): the hardware's, within a step, and one step of Newton's method; below 2^-100 of x 2^100, since the hardware takes what is below 2^-126 for 0.  x = 0: infinity, as the
// formula has it.
__device__ __forceinline__ float inverse_root(float x) {
  const bool tiny = x < 0x1p-100f;
  const float s = tiny ? x * 0x1p100f : x, y = __builtin_amdgcn_rsqf(s), e = __builtin_fmaf(-s * y, y, 1.f), r = s > 0.f && s < INFINITY ? __builtin_fmaf(0.5f * e, y, y) : y;
  return tiny ? r * 0x1p50f : r;
}

// The statistics of a row of which this thread has v[0 .. E), 0 where an entry is not its; takes the mean off them.  per: 1 / h.
template <int E>
__device__ __forceinline__ void row_statistics(float (&v)[E], uint32_t own, const NormArgs& a, float per, float (*sh)[16][2], int waves, int& side, float& mean, float& rstd) {
  float q[1] = {0.f};
  mean = 0.f;
  if (a.layer) {
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < E; ++i) s[0] += v[i];
    team_sums<1>(s, sh, 0, waves, side);
    mean = s[0] / (float)a.h;   // and not times 1 / h: the mean of equal entries is theirs
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] -= mean;
    if (own != Window<E>::kAll) {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = own >> i & 1 ? v[i] : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < E; ++i) q[0] += v[i] * v[i];
  team_sums<1>(q, sh, 0, waves, side);
  rstd = inverse_root(q[0] * per + a.eps);
}

// Both products rounded by themselves: the norm behind goes by y as it is stored, and without a post norm that is then, bit for bit, what any plain evaluation stores.
__device__ __forceinline__ float residual_sum(float alpha, float x, float by, float u) {
#pragma clang fp contract(off)
  return alpha * x + by * u;
}

// Waves that a SIMD of the chip has room for by their registers: of the kernels whose rows are shared by several waves, and the workgroups of the others.
// us, a norm on both sides, bf16, these / a workgroup for every row: 16384 rows, layer norm 8192 wide 207 / 230, RMS norm 12288 wide 328 / 374, 8192 203 / 183, 4096 99 / 91, 2048 45.9 / 44.9,
// 1024 24.3 / 23.1, 333 (1280 workgroups) 12.5 / 12.2; 4096 rows, 8192 wide 44.7 / 48.6, fp32 102 / 120, 2048 wide 13.1 / 12.5, layer norm 1920 wide 17.3 / 16.2.
template <typename T, int E> constexpr int norm_fwd_waves() { return sizeof(T) * E <= 16 ? 8 : 4; }
constexpr int64_t kFwdSingle = 1280;
// From this many bytes of all rows on they are read past the caches, and from twice as many on written past them too.  us of 8192 wide rows / with a pass behind that reads z: 256 MB
// 51.2 / 74.6, read past 46.5 / 66.5, both 48.4 / 71.1; 512 MB 104 / 149, 101 / 146, 95 / 138; 1024 wide 64 MB 15.1 / 21.3, 16.1 / 22.1; 128 MB 25.5 / 37.1, 25.4 / 35.6.
constexpr int64_t kFwdPast = 192ll << 20;

// E entries of a row per thread.  One wave a row and four rows to a workgroup (MULTI false), or a workgroup a row.  No more workgroups than the chip holds: each
// goes through several rows and has the next one on its way while it waits for the sums of this one.  PAST: 1 rows are read past the caches, 2 written too.
template <typename T, int E, bool MULTI, int PAST>
__global__ __launch_bounds__(MULTI ? 1024 : 256, MULTI ? (norm_fwd_waves<T, E>()) : 4) void residual_norm_fwd_kernel(NormArgs a) {
  __shared__ float sh[2][16][2];
  const int waves = MULTI ? (int)(blockDim.x >> 6) : 1, rows = MULTI ? 1 : 4, t = MULTI ? (int)threadIdx.x : (int)(threadIdx.x & 63);
  const Window<E> win(t, a.h);
  const float per = 1.f / (float)a.h;
  int side = 0;
  int64_t row = (int64_t)blockIdx.x * rows + (MULTI ? 0 : threadIdx.x >> 6);
  if (row >= a.rows) return;
  Packed<T, E> pw, w, next_x, next_b;
  if (a.post_weight) pw = load_window<E>(static_cast<const T*>(a.post_weight), win);
  if (a.weight) w = load_window<E>(static_cast<const T*>(a.weight), win);
  next_x = load_window<E, PAST != 0>(static_cast<const T*>(a.x) + row * a.h, win);
  if (a.branch) next_b = load_window<E, PAST != 0>(static_cast<const T*>(a.branch) + row * a.h, win);
  while (row < a.rows) {
    const Packed<T, E> x = next_x;
    Packed<T, E> b = next_b;
    const int64_t here = row, at = here * a.h;
    row += (int64_t)gridDim.x * rows;
    if (row < a.rows) {
      next_x = load_window<E, PAST != 0>(static_cast<const T*>(a.x) + row * a.h, win);
      if (a.branch) next_b = load_window<E, PAST != 0>(static_cast<const T*>(a.branch) + row * a.h, win);
    }
    float v[E], mean = 0.f, rstd = 1.f;
    if (a.branch) {
      if (a.post_weight) {
        if (win.own != Window<E>::kAll) b.clear(win.own);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = b.get(i);
        row_statistics<E>(v, win.own, a, per, sh, waves, side, mean, rstd);
        if (a.post_stats && t == 0) { a.post_stats[here] = mean; a.post_stats[a.rows + here] = rstd; }
        pw.keep();
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = v[i] * rstd * pw.get(i);
        if (a.post_bias) {
          const Packed<T, E> pb = load_window<E>(static_cast<const T*>(a.post_bias), win);
#pragma unroll
          for (int i = 0; i < E; ++i) v[i] += pb.get(i);
        }
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = b.get(i);
      }
      if (a.gate) {
        const Packed<T, E> g = load_window<E>(static_cast<const T*>(a.gate) + (int64_t)((uint32_t)here / (uint32_t)a.rows_per_gate) * a.h, win);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = residual_sum(a.alpha, x.get(i), a.beta * g.get(i), v[i]);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = residual_sum(a.alpha, x.get(i), a.beta, v[i]);
      }
      if (a.y) store_window<E, PAST == 2>(static_cast<T*>(a.y) + at, win, win.own, v);
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = to_f32(from_f32<T>(v[i]));
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = x.get(i);
    }
    if (!a.weight) continue;
    if (win.own != Window<E>::kAll) {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = win.own >> i & 1 ? v[i] : 0.f;
    }
    row_statistics<E>(v, win.own, a, per, sh, waves, side, mean, rstd);
    if (a.stats && t == 0) { a.stats[here] = mean; a.stats[a.rows + here] = rstd; }
    w.keep();
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = v[i] * rstd * w.get(i);
    if (a.bias) {
      const Packed<T, E> pb = load_window<E>(static_cast<const T*>(a.bias), win);
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] += pb.get(i);
    }
    store_window<E, PAST == 2>(static_cast<T*>(a.z) + at, win, win.own, v);
  }
}

// Entries of a row of h that a thread has, E of them making 16 bytes, and how many waves share the row then.
inline int norm_entries(int h, int E) { return h < E ? 1 : h <= 1024 * E ? E : h <= 8192 ? 8 : 16; }
inline int norm_waves(int h, int E) { return (h - 1) / (64 * norm_entries(h, E)) + 1; }

template <typename T, int E>
inline void launch_residual_norm_fwd_entries(const NormArgs& a, int waves, hipStream_t st) {
  const int64_t sets = waves == 1 ? (a.rows + 3) / 4 : a.rows, most = waves == 1 ? kFwdSingle : 256 * (4 * norm_fwd_waves<T, E>() / waves);
  const int64_t each = (sets + most - 1) / most;   // rows of a workgroup
  const dim3 grid((unsigned)((sets + each - 1) / each));
  const int64_t bytes = a.rows * a.h * (int64_t)sizeof(T) * (1 + (a.branch != nullptr) + (a.y != nullptr) + (a.z != nullptr));
  auto launch = [&](auto past) {
    constexpr int P = decltype(past)::value;
    if constexpr (sizeof(T) * E <= 16) {   // more entries are for rows of 16 waves
      if (waves == 1) hipLaunchKernelGGL((residual_norm_fwd_kernel<T, E, false, P>), grid, dim3(256), 0, st, a);
    }
    if constexpr (E > 1) {
      if (waves > 1) hipLaunchKernelGGL((residual_norm_fwd_kernel<T, E, true, P>), grid, dim3(64 * waves), 0, st, a);
    }
  };
  if (bytes >= 2 * kFwdPast) launch(std::integral_constant<int, 2>{});
  else if (bytes >= kFwdPast) launch(std::integral_constant<int, 1>{});
  else launch(std::integral_constant<int, 0>{});
}

template <typename T>
hipError_t launch_residual_norm_fwd(const NormArgs& a, hipStream_t st) {
  if (a.rows > 0) {
    constexpr int E = 16 / (int)sizeof(T);
    const int e = norm_entries(a.h, E), waves = norm_waves(a.h, E);
    if (e == 1) launch_residual_norm_fwd_entries<T, 1>(a, waves, st);
    else if (e == E) launch_residual_norm_fwd_entries<T, E>(a, waves, st);
    else if (e == 8) launch_residual_norm_fwd_entries<T, 8>(a, waves, st);
    else launch_residual_norm_fwd_entries<T, 16>(a, waves, st);
  }
  return hipGetLastError();
}

// ---- backward ---------------------------------------------------------------------------------

// How the rows are shared.  A workgroup of up to 16 waves has `teams` of `waves` waves, a row at a time each.  Segments are rows that have a gate in common (all rows where
// there is none).  A workgroup takes `chunk` rows of one segment; or, if segments are of at most kNormShort rows, a team takes `chunk` whole segments, whose gate's
// gradient is then complete where it is summed.
constexpr int kNormShort = 16, kNormGroups = 256;   // one workgroup for a compute unit: 8192x8192 171 us; 128 224, 512 174; 4096x1024 20.5; 22.2, 27.0
struct NormSplit {
  int64_t segment, segments, chunk, per_segment, groups, pitch;
  int waves, teams;
  bool whole;
};
inline NormSplit norm_split(int64_t rows, int64_t h, int64_t rows_per_gate, int E) {
  NormSplit s{};
  s.pitch = (h + 63) / 64 * 64;
  s.waves = norm_waves((int)h, E);
  s.teams = 16 / s.waves;
  if (rows < 1) return s;
  s.segment = rows_per_gate > 0 && rows_per_gate < rows ? rows_per_gate : rows;
  s.segments = (rows + s.segment - 1) / s.segment;
  s.whole = s.segments > 1 && s.segment <= kNormShort;
  if (s.whole) {
    const int64_t sets = (s.segments + s.teams - 1) / s.teams;
    s.chunk = (sets + kNormGroups - 1) / kNormGroups;
    s.groups = (sets + s.chunk - 1) / s.chunk;
  } else {
    // A segment in as many parts as take the fewest steps in all: rounds of the chip's workgroups times a part's sets of rows, and about two more to begin and end one.
    const int64_t sets = (s.segment + s.teams - 1) / s.teams, first = (s.segments + kNormGroups - 1) / kNormGroups;
    int64_t least = INT64_MAX;
    for (int64_t k = first; k < first + 8; ++k) {
      int64_t parts = k * kNormGroups / s.segments;
      if (parts > sets) parts = sets;
      const int64_t each = (sets + parts - 1) / parts, steps = (s.segments * parts + kNormGroups - 1) / kNormGroups * (each + 2);
      if (steps < least) { least = steps; s.chunk = each * s.teams; }
    }
    s.per_segment = (s.segment + s.chunk - 1) / s.chunk;
    s.groups = s.segments * s.per_segment;
  }
  return s;
}

enum NormSum : int { NS_WEIGHT = 0, NS_BIAS = 1, NS_POST_WEIGHT = 2, NS_POST_BIAS = 3, NS_GATE = 4, NS_COUNT = 5 };

int64_t residual_norm_bwd_groups(int64_t rows, int64_t h, int64_t rows_per_gate) {   // of either type
  const int64_t a = norm_split(rows, h, rows_per_gate, 4).groups, b = norm_split(rows, h, rows_per_gate, 8).groups;
  return a > b ? a : b;
}
size_t residual_norm_bwd_scratch_bytes(int64_t rows, int64_t h, int64_t rows_per_gate) {
  return (size_t)residual_norm_bwd_groups(rows, h, rows_per_gate) * NS_COUNT * (size_t)((h + 63) / 64 * 64) * sizeof(float);
}

// What a thread reads of a row.
template <typename T, int E> struct NormRow {
  Packed<T, E> dz, y, dy, branch;
  float mean, rstd, post_mean, post_rstd;
};
enum NormGate : int { NG_NONE = 0, NG_LONG = 1, NG_SHORT = 2 };   // segments: see NormSplit

// The sums of a thread's columns, in registers or (ASIDE) in shared memory, where its quads lie 1024 apart.
template <int E, bool ASIDE> struct ColumnSums {
  static constexpr int Q = E < 4 ? E : 4;
  float v[ASIDE ? 1 : E];
  floatx4* at;
  __device__ __forceinline__ explicit ColumnSums(floatx4* all) : at(all + threadIdx.x) { clear(); }
  __device__ __forceinline__ void clear() {
    if constexpr (ASIDE) {
#pragma unroll
      for (int q = 0; q < E / 4; ++q) at[q * 1024] = floatx4{0.f, 0.f, 0.f, 0.f};
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = 0.f;
    }
  }
  // Of entries [i, i + Q).
  __device__ __forceinline__ void add(int i, const float (&e)[Q]) {
    if constexpr (ASIDE) {
      floatx4 k = at[i / 4 * 1024];
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] += e[j];
      at[i / 4 * 1024] = k;
    } else {
#pragma unroll
      for (int j = 0; j < Q; ++j) v[i + j] += e[j];
    }
  }
  __device__ __forceinline__ void get(float (&e)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if constexpr (ASIDE) e[i] = at[i / 4 * 1024][i % 4];
      else e[i] = v[i];
    }
  }
};

// E entries of a row per thread.  LEAN: an RMS norm without a bias' gradient.  PAST: rows are read and written past the caches.
// With bhat the normed branch (the branch itself without a post norm), A = sum of d * bhat and C = sum of d over the rows of a segment give all of
// dgate = beta (post_weight A + post_bias C), dpost_weight = beta gate A and dpost_bias = beta gate C: one product and sum an entry for A.
template <typename T, int E, bool LEAN, bool POST, int GATE, bool PAST>
__global__ __launch_bounds__(1024) void residual_norm_bwd_kernel(NormArgs a, NormSplit s) {
  __shared__ float sh[2][16][2];
  __shared__ float joined[E <= 8 ? 1024 * E : 1];   // 16 entries: a workgroup is one team
  constexpr bool SHORT = GATE == NG_SHORT;
  constexpr int Q = E < 4 ? E : 4;
  // Sums that lie in shared memory, in the order in which they go there: the registers of a workgroup that fills its unit hold no five of 8 entries, nor two of 16.  us, in registers (and spilt) / here: layer norm
  // 8192x8192 265 / 175, 4096x4096 with a gate a row 207 / 146; 4096x12288 294 / 169, layer norm 458 / 248.  Two of 8 entries there and the third in registers: 205, 162.
  constexpr int ROOM = E >= 16 ? 2 : E >= 8 ? (LEAN ? SHORT && POST : 3) : E >= 4 ? !LEAN && SHORT && POST : 0, kNever = 9;
  constexpr int kDw = LEAN ? (SHORT ? 1 : 0) : (SHORT ? kNever : 2), kA = LEAN && !SHORT ? 1 : kNever, kDpw = !SHORT ? kNever : LEAN ? 0 : 2;
  constexpr int kDb = LEAN ? kNever : 0, kC = LEAN || SHORT ? kNever : 1, kDpb = LEAN || !SHORT ? kNever : 1;
  __shared__ floatx4 aside[ROOM ? ROOM * (E / 4) * 1024 : 1];
  const int wave = (int)(threadIdx.x >> 6), team = wave / s.waves, first = team * s.waves, threads = s.waves * 64, t = (int)threadIdx.x - first * 64;
  const Window<E> win(t, a.h);
  const bool whole = win.own == Window<E>::kAll, pre = a.weight != nullptr, layer = !LEAN && a.layer;
  const float per = 1.f / (float)a.h;
  int side = 0;
  Packed<T, E> w, pw;
  // Of 16 entries a thread, and of 8 with six sums (layer norm and a gate for every few rows), weights and gates are read when they are used, too (4096x4096 152 -> 106 us;
  // layer norm 4096x12288 327 -> 248, RMS norm 168 -> 171; with a gate a row 475 -> 344).
  constexpr bool KEPT = E < 16 && !(E >= 8 && SHORT && POST && !LEAN);
  auto read_weight = [&](Packed<T, E>& to, const void* from) { to = load_window<E>(static_cast<const T*>(from), win); if (!whole) to.clear(win.own); };
  if (KEPT && pre) read_weight(w, a.weight);
  if (KEPT && POST) read_weight(pw, a.post_weight);

  // Step k of the workgroup: this team's row and whether there is one.  Where there is none the entries of `spare` are read and cleared; its statistics are used, and where they are not
  // finite they leave NaN in the sums: it is a row of the same segment, whose sums are NaN then by the formula too.  Rows fit 31 bits.
  const int64_t group = blockIdx.x;
  int base, end, steps, spare, seg = 0;
  const int segment = (int)s.segment;
  if (GATE == NG_SHORT) {
    seg = (int)(group * s.chunk) * s.teams + team;
    base = seg * segment;
    end = (int)a.rows;
    steps = (int)s.chunk * segment;
    spare = (int)(s.segments - 1) * segment;
  } else {
    seg = (int)(group / s.per_segment);
    const int64_t begin = (int64_t)seg * s.segment + (group - (int64_t)seg * s.per_segment) * s.chunk;
    int64_t last = ((int64_t)seg + 1) * s.segment;
    if (last > a.rows) last = a.rows;
    if (last > begin + s.chunk) last = begin + s.chunk;
    base = (int)begin + team;
    end = (int)last;
    steps = (end - (int)begin + s.teams - 1) / s.teams;
    spare = seg * segment;   // a part of a short last segment may have no row of its own
  }
  Packed<T, E> g;
  auto read_gate = [&](int of) { g = load_window<E>(static_cast<const T*>(a.gate) + (int64_t)of * a.h, win); };
  if (KEPT && GATE == NG_LONG) read_gate(seg);
  // Rows of more entries than a piece of 16 bytes a thread are read when they are used, and again after each sum, which the caches answer: held, or fetched ahead, they
  // would not fit the registers (4096 rows, us: 8192 wide fp32 394 -> 184, 12288 wide bf16 890 -> 344, before their sums left the registers).
  constexpr bool AHEAD = E * sizeof(T) <= 16;
  auto again = [&](int row, NormRow<T, E>& r, bool first) {
    const int64_t at = (int64_t)(row < end ? row : spare) * a.h;
    if (pre && first) {
      r.dz = load_window<E, PAST>(static_cast<const T*>(a.dz) + at, win);
      r.y = load_window<E, PAST>(static_cast<const T*>(a.x) + at, win);
    }
    if (first && a.dy) r.dy = load_window<E, PAST>(static_cast<const T*>(a.dy) + at, win);
    if (POST || GATE) r.branch = load_window<E, PAST>(static_cast<const T*>(a.branch) + at, win);
  };
  auto fetch = [&](int row) {
    NormRow<T, E> r;
    const int64_t k = row < end ? row : spare, at = k * a.h;
    if (pre) {
      if constexpr (!AHEAD) {
        r.dz = load_window<E>(static_cast<const T*>(a.dz) + at, win);
        r.y = load_window<E>(static_cast<const T*>(a.x) + at, win);
      }
      if (layer) r.mean = a.stats[k];
      r.rstd = a.stats[a.rows + k];
    }
    if constexpr (AHEAD) again(row, r, true);
    if (POST) {
      if (layer) r.post_mean = a.post_stats[k];
      r.post_rstd = a.post_stats[a.rows + k];
    }
    return r;
  };

  auto slot = [&](int k) { return aside + (k < ROOM ? k * (E / 4) * 1024 : 0); };
  ColumnSums<E, (kDw < ROOM)> dw(slot(kDw));
  ColumnSums<E, (kA < ROOM)> A(slot(kA));
  ColumnSums<E, (kDpw < ROOM)> dpw(slot(kDpw));
  ColumnSums<E, (kDb < ROOM)> db(slot(kDb));
  ColumnSums<E, (kC < ROOM)> C(slot(kC));
  ColumnSums<E, (kDpb < ROOM)> dpb(slot(kDpb));
  int row = base, left = segment;   // SHORT: rows of the segment that are left
  NormRow<T, E> next;
  if constexpr (AHEAD) next = fetch(row);
  for (int step = 0; step < steps; ++step) {
    NormRow<T, E> r;
    if constexpr (AHEAD) r = next;
    else r = fetch(row);
    const int here = row;
    const uint32_t own = here < end ? win.own : 0u;
    const int64_t at = (int64_t)here * a.h;
    if (GATE == NG_SHORT) {
      if (KEPT && left == segment) read_gate(here < end ? seg : 0);
      row = --left > 0 ? here + 1 : here + 1 + (s.teams - 1) * segment;
    } else {
      row = here + s.teams;
    }
    auto clear = [&] {
      if (own != Window<E>::kAll) {
        if (pre) { r.dz.clear(own); r.y.clear(own); }
        if (a.dy) r.dy.clear(own);
        if (POST || GATE) r.branch.clear(own);
      }
    };
    if constexpr (AHEAD) {
      if (step + 1 < steps) next = fetch(row);
      clear();
    } else if (pre && own != Window<E>::kAll) {
      r.dz.clear(own);
      r.y.clear(own);
    }
    float d[E];
    if (pre) {
      float k[2] = {0.f, 0.f};
      if (!KEPT) read_weight(w, a.weight);
#pragma unroll
      for (int q = 0; q < E; q += Q) {
        float ew[Q], eb[Q];
#pragma unroll
        for (int j = 0; j < Q; ++j) {
          const int i = q + j;
          const float z = r.dz.get(i), c = layer ? r.y.get(i) - r.mean : r.y.get(i), gz = z * w.get(i);
          k[0] += gz * c;
          if (!LEAN) k[1] += gz;
          eb[j] = z;
          ew[j] = z * r.rstd * c;
        }
        dw.add(q, ew);
        if constexpr (!LEAN) db.add(q, eb);
      }
      if (layer) team_sums<2>(k, sh, first, s.waves, side);
      else { float one[1] = {k[0]}; team_sums<1>(one, sh, first, s.waves, side); k[0] = one[0]; k[1] = 0.f; }
      const float by = k[0] * per * r.rstd * r.rstd, all = k[1] * per;
      if constexpr (AHEAD) {
        r.dz.keep();
        r.y.keep();
      } else {
        again(here, r, true);
        clear();
      }
      if (KEPT) w.keep();
      else read_weight(w, a.weight);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float c = layer ? r.y.get(i) - r.mean : r.y.get(i), gz = r.dz.get(i) * w.get(i);
        d[i] = LEAN ? gz - c * by : gz - all - c * by;
        d[i] = a.dy ? r.rstd * d[i] + r.dy.get(i) : r.rstd * d[i];
      }
    } else {
      if constexpr (!AHEAD) {
        again(here, r, true);
        clear();
      }
#pragma unroll
      for (int i = 0; i < E; ++i) d[i] = r.dy.get(i);
    }
    {
      float e[E];
#pragma unroll
      for (int i = 0; i < E; ++i) e[i] = a.alpha * d[i];
      store_window<E, PAST>(static_cast<T*>(a.y) + at, win, own, e);
    }
    if (POST || GATE) {
      float k[2] = {0.f, 0.f};
      if (!KEPT && GATE) read_gate(!SHORT || seg < s.segments ? seg : 0);
      if (!KEPT && POST) read_weight(pw, a.post_weight);
#pragma unroll
      for (int q = 0; q < E; q += Q) {
        float ea[Q], ec[Q];
#pragma unroll
        for (int j = 0; j < Q; ++j) {
          const int i = q + j;
          float b = r.branch.get(i);
          if (POST) b = (layer ? b - r.post_mean : b) * r.post_rstd;
          const float dd = own == Window<E>::kAll ? d[i] : (own >> i & 1 ? d[i] : 0.f);
          ea[j] = dd * b;
          ec[j] = dd;
          d[i] = dd * a.beta;
          if (GATE) d[i] *= g.get(i);
          if (POST) {
            d[i] *= pw.get(i);
            k[0] += d[i] * b;
            if (!LEAN) k[1] += d[i];
          }
        }
        A.add(q, ea);
        if constexpr (!LEAN) C.add(q, ec);
      }
      if (POST) {
        if (layer) team_sums<2>(k, sh, first, s.waves, side);
        else { float one[1] = {k[0]}; team_sums<1>(one, sh, first, s.waves, side); k[0] = one[0]; k[1] = 0.f; }
        const float by = k[0] * per * r.post_rstd, all = k[1] * per;
        if constexpr (AHEAD) {
          r.branch.keep();
        } else {
          again(here, r, false);
          if (own != Window<E>::kAll) r.branch.clear(own);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float c = layer ? r.branch.get(i) - r.post_mean : r.branch.get(i);
          d[i] = r.post_rstd * (LEAN ? d[i] - c * by : d[i] - all - c * by);
        }
      }
      store_window<E, PAST>(static_cast<T*>(a.z) + at, win, own, d);
    } else if (a.z) {
#pragma unroll
      for (int i = 0; i < E; ++i) d[i] *= a.beta;
      store_window<E, PAST>(static_cast<T*>(a.z) + at, win, own, d);
    }
    if constexpr (GATE == NG_SHORT) {
      if (left == 0) {   // the segment is over
        float sa[E], sc[E];
        A.get(sa);
        C.get(sc);
        if (a.dgate && seg < s.segments) {
          Packed<T, E> pb;
          if (!KEPT && POST) read_weight(pw, a.post_weight);
          if (POST && a.post_bias) pb = load_window<E>(static_cast<const T*>(a.post_bias), win);
          float* to = a.dgate + (int64_t)seg * a.h;
          Packed<float, E> old;
          if (a.accumulate) old = load_window<E>(to, win);
          float e[E];
#pragma unroll
          for (int i = 0; i < E; ++i) {
            e[i] = sa[i];
            if (POST) { e[i] *= pw.get(i); if (!LEAN && a.post_bias) e[i] += sc[i] * pb.get(i); }
            e[i] *= a.beta;
            if (a.accumulate) e[i] += old.get(i);
          }
          store_window<E>(to, win, win.own, e);
        }
        if constexpr (POST) {
          if (!KEPT) read_gate(seg < s.segments ? seg : 0);
#pragma unroll
          for (int q = 0; q < E; q += Q) {
            float ew[Q], eb[Q];
#pragma unroll
            for (int j = 0; j < Q; ++j) {
              const float bg = a.beta * g.get(q + j);
              ew[j] = bg * sa[q + j];
              eb[j] = bg * sc[q + j];
            }
            dpw.add(q, ew);
            if constexpr (!LEAN) dpb.add(q, eb);
          }
        }
        A.clear();
        C.clear();
        left = segment;
        seg += s.teams;
      }
    }
  }
  // The workgroup's sums: the teams' joined, in order.
  auto leave = [&](const auto& of, int which) {
    float sums[E];
    if constexpr (std::is_array_v<std::remove_reference_t<decltype(of)>>) {
#pragma unroll
      for (int i = 0; i < E; ++i) sums[i] = of[i];
    } else {
      of.get(sums);
    }
    float* to = a.scratch + (group * NS_COUNT + which) * s.pitch;
    if constexpr (E <= 8) {
      __syncthreads();
      float* mine = joined + team * threads * E + win.at;
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (win.own >> i & 1) mine[i] = sums[i];
      __syncthreads();
      for (int c = (int)threadIdx.x; c < a.h; c += (int)blockDim.x) {
        float v = 0.f;
#pragma unroll 8   // reads under way at once: there are up to 16 teams
        for (int k = 0; k < s.teams; ++k) v += joined[k * threads * E + c];
        to[c] = v;
      }
    } else {
      store_window<E>(to, win, win.own, sums);
    }
  };
  if (a.dweight) leave(dw, NS_WEIGHT);
  if constexpr (!LEAN) { if (a.dbias) leave(db, NS_BIAS); }
  if constexpr (GATE == NG_SHORT) {
    if constexpr (POST) {
      if (a.dpost_weight) leave(dpw, NS_POST_WEIGHT);
      if constexpr (!LEAN) { if (a.dpost_bias) leave(dpb, NS_POST_BIAS); }
    }
  } else {
    float e[E], by[E], sa[E], sc[E];
    if (!KEPT && GATE) read_gate(seg);
    if (!KEPT && POST) read_weight(pw, a.post_weight);
    A.get(sa);
    C.get(sc);
#pragma unroll
    for (int i = 0; i < E; ++i) by[i] = GATE ? a.beta * g.get(i) : a.beta;
    if constexpr (GATE == NG_LONG) {
      if (a.dgate) {
        Packed<T, E> pb;
        if (POST && a.post_bias) pb = load_window<E>(static_cast<const T*>(a.post_bias), win);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          e[i] = sa[i];
          if (POST) { e[i] *= pw.get(i); if (!LEAN && a.post_bias) e[i] += sc[i] * pb.get(i); }
          e[i] *= a.beta;
        }
        leave(e, NS_GATE);
      }
    }
    if constexpr (POST) {
      if (a.dpost_weight) {
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = by[i] * sa[i];
        leave(e, NS_POST_WEIGHT);
      }
      if constexpr (!LEAN) {
        if (a.dpost_bias) {
#pragma unroll
          for (int i = 0; i < E; ++i) e[i] = by[i] * sc[i];
          leave(e, NS_POST_BIAS);
        }
      }
    }
  }
}

// Sums of the workgroups' sums: 64 columns, 16 of the workgroups at a time.  A job of `across` column blocks for each parameter's gradient, over all
// workgroups, then for each segment's gate.
__global__ __launch_bounds__(256) void residual_norm_sums_kernel(NormArgs a, NormSplit s, uint32_t across, int64_t blocks) {
  __shared__ floatx4 sh[16][16];
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int64_t job = b / across;
    const int col = (int)(b - job * across) * 64, lane = (int)(threadIdx.x >> 4), part = (int)(threadIdx.x & 15);
    const int which = job < NS_GATE ? (int)job : (int)NS_GATE;
    float* out = job == NS_WEIGHT ? a.dweight : job == NS_BIAS ? a.dbias : job == NS_POST_WEIGHT ? a.dpost_weight : job == NS_POST_BIAS ? a.dpost_bias
                                                                                                                : a.dgate + (job - NS_GATE) * a.h;
    if (!out) continue;
    const int64_t begin = job < NS_GATE ? 0 : (job - NS_GATE) * s.per_segment, end = job < NS_GATE ? s.groups : begin + s.per_segment;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    const float* from = a.scratch + which * s.pitch + col + part * 4;
#pragma unroll 8
    for (int64_t g = begin + lane; g < end; g += 16) v += *reinterpret_cast<const floatx4*>(from + g * NS_COUNT * s.pitch);
    sh[lane][part] = v;
    __syncthreads();
    const int c = (int)threadIdx.x;
    if (c < 64 && col + c < a.h) {
      float e = 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) e += sh[k][c / 4][c % 4];
      out[col + c] = a.accumulate ? out[col + c] + e : e;
    }
    __syncthreads();
  }
}

// From this many bytes of all rows on they go past the caches.  us of 4096 wide rows / with a pass behind that reads dbranch: 192 MB (2048 wide) 53.0 / 62.5, past 48.0 / 59.9; 384 MB 92.6 / 118,
// 85.3 / 107; 768 MB 170 / 217, 170 / 212; 1024 wide 96 MB 28.1 / 33.7, 28.9 / 36.9.
constexpr int64_t kBwdPast = 160ll << 20;

template <typename T, int E, bool LEAN, bool PAST>
inline void launch_residual_norm_bwd_entries(const NormArgs& a, const NormSplit& s, hipStream_t st) {
  const dim3 grid((unsigned)s.groups), block(64 * s.waves * s.teams);
  auto launch = [&](auto post, auto gate) {
    constexpr bool P = decltype(post)::value;
    constexpr int G = decltype(gate)::value;
    hipLaunchKernelGGL((residual_norm_bwd_kernel<T, E, LEAN, P, G, PAST>), grid, block, 0, st, a, s);
  };
  auto with = [&](auto gate) {
    if (a.post_weight) launch(std::true_type{}, gate);
    else launch(std::false_type{}, gate);
  };
  if (!a.gate) with(std::integral_constant<int, NG_NONE>{});
  else if (s.whole) with(std::integral_constant<int, NG_SHORT>{});
  else with(std::integral_constant<int, NG_LONG>{});
}

template <typename T>
hipError_t launch_residual_norm_bwd(const NormArgs& a, hipStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  const NormSplit s = norm_split(a.rows, a.h, a.gate ? a.rows_per_gate : 0, E);
  if (a.rows > 0) {
    const bool lean = !a.layer && !a.dbias && !a.dpost_bias && !a.post_bias;
    const int64_t bytes = a.rows * a.h * (int64_t)sizeof(T) * (1 + 2 * (a.dz != nullptr) + (a.dy != nullptr) + (a.branch != nullptr) + (a.z != nullptr));
    auto entries = [&](auto e, auto past) {
      constexpr int N = decltype(e)::value;
      constexpr bool P = decltype(past)::value;
      if (lean) launch_residual_norm_bwd_entries<T, N, true, P>(a, s, st);
      else launch_residual_norm_bwd_entries<T, N, false, P>(a, s, st);
    };
    const int e = norm_entries(a.h, E);
    if (e == 1) launch_residual_norm_bwd_entries<T, 1, false, false>(a, s, st);
    else if (e == 16) entries(std::integral_constant<int, 16>{}, std::false_type{});
    else if (e != E) entries(std::integral_constant<int, 8>{}, std::false_type{});
    else if (bytes >= kBwdPast) entries(std::integral_constant<int, E>{}, std::true_type{});
    else entries(std::integral_constant<int, E>{}, std::false_type{});
  }
  const bool gates = a.dgate && !s.whole, params = a.dweight || a.dbias || a.dpost_weight || a.dpost_bias;
  const uint32_t across = (uint32_t)(a.h + 63) / 64;
  const int64_t blocks = across * (NS_GATE + (gates ? s.segments : 0)), most = 1 << 22;
  if (gates || params) hipLaunchKernelGGL(residual_norm_sums_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a, s, across, blocks);
  return hipGetLastError();
}

}  // namespace varuna
