// The first stage's embedding: out[t] = scale * table[id_t] + places[position_t], and the table's fp32 gradient
// dtable[v] (+)= scale * sum of dy[t] over the rows t with id v.
//
// The gradient.  Rows of one id have to meet, in the same order every time.  Three launches:
//   1. embedding_sort_kernel   a stable counting sort of the row numbers by id: `order`, the ids in that order, and where each
//                              id's run begins.  A workgroup owns a range of ids and looks at all ids itself, so that no
//                              workgroup waits for another.
//   2. embedding_sum_kernel    pieces of the sorted order, one wave for a piece and 64 lanes' columns: a run that lies inside
//                              a piece goes to its row of the table, the two ends of a piece that others share go to scratch.
//                              When the gradient is written and not added to, more waves put zeros into the rows of ids that do not occur.
//   3. embedding_join_kernel   the runs that span pieces: their parts summed in order.
// Pieces are cut by position, so a token that fills half of the batch costs what any other rows do.
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

// ---- the gradient ---------------------------------------------------------------------

constexpr int kSortWaves = 16;
constexpr int kSortMaxBits = 9;     // ids of a workgroup: 16 waves' counters of 512 ids are 32 KB of LDS
constexpr int kPiece = 16;          // positions whose rows are in flight together
constexpr int kMaxPieces = 1024;
constexpr int kZeroRows = 16;       // rows of the table looked at together for zeros

struct EmbedScratch {
  int32_t *start, *order, *id;      // [vocab + 1], [rows], [rows]
  float* part;                      // [pieces][2][h]: the first and the last run of a piece, where it shares them with others
  int64_t piece;                    // positions of one
  int pieces;
};
inline size_t embed_align(size_t n) { return (n + 255) / 256 * 256; }
inline EmbedScratch embed_scratch(void* p, int64_t rows, int64_t vocab) {
  EmbedScratch s;
  char* at = static_cast<char*>(p);
  s.start = reinterpret_cast<int32_t*>(at);
  at += embed_align((size_t)(vocab + 1) * 4);
  s.order = reinterpret_cast<int32_t*>(at);
  at += embed_align((size_t)rows * 4);
  s.id = reinterpret_cast<int32_t*>(at);
  at += embed_align((size_t)rows * 4);
  s.part = reinterpret_cast<float*>(at);
  s.piece = ((rows + kMaxPieces - 1) / kMaxPieces + kPiece - 1) / kPiece * kPiece;
  if (s.piece < kPiece) s.piece = kPiece;
  s.pieces = (int)((rows + s.piece - 1) / s.piece);
  return s;
}
size_t embedding_bwd_scratch_bytes(int64_t rows, int64_t h, int64_t vocab) {
  const EmbedScratch s = embed_scratch(nullptr, rows, vocab);
  return embed_align((size_t)(vocab + 1) * 4) + 2 * embed_align((size_t)rows * 4) + (s.pieces > 1 ? (size_t)s.pieces * 2 * (size_t)h * 4 : 0) + 256;
}

// Stable counting sort of the rows whose id lies in [blockIdx.x << bits, (blockIdx.x + 1) << bits).  A wave owns a contiguous
// sixteenth of all rows.  It counts its ids in LDS and, on the way, the rows of lower ids: where the workgroup's own begin.
// After a prefix sum over (id, wave) it walks its rows once more and gives each its place; rows of one id in the same 64 are
// told apart by ballots over the id's bits.
__global__ __launch_bounds__(1024) void embedding_sort_kernel(IdArgs ids, int64_t rows, int64_t vocab, int bits, int32_t* __restrict__ start,
                                                              int32_t* __restrict__ order, int32_t* __restrict__ id_out) {
  extern __shared__ uint32_t counter[];   // [kSortWaves][1 << bits]
  __shared__ uint32_t below[kSortWaves], part[kSortWaves];
  const int own = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t v0 = (int64_t)blockIdx.x << bits;
  uint32_t* mine = counter + wave * own;
  for (int i = threadIdx.x; i < kSortWaves * own; i += 1024) counter[i] = 0;
  __syncthreads();
  const int64_t each = (rows + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
  const int64_t t0 = wave * each, t1 = t0 + each < rows ? t0 + each : rows;
  uint32_t low = 0;
#pragma unroll 4
  for (int64_t t = t0 + lane; t < t1; t += 64) {
    const int64_t v = row_id(ids, t, vocab);
    low += v >= 0 && v < v0;
    if (v >= v0 && v < v0 + own) atomicAdd(&mine[v - v0], 1u);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) low += __shfl_xor(low, o, kWave);
  if (lane == 0) below[wave] = low;
  __syncthreads();
  // Thread i: id i's total, then the prefix over ids, then each wave's first place.
  uint32_t total = 0;
  if ((int)threadIdx.x < own)
    for (int w = 0; w < kSortWaves; ++w) total += counter[w * own + threadIdx.x];
  uint32_t sum = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(sum, o, kWave);
    if (lane >= o) sum += up;
  }
  if (lane == 63) part[wave] = sum;
  __syncthreads();
  uint32_t at = sum - total;
  for (int w = 0; w < kSortWaves; ++w) at += below[w] + (w < wave ? part[w] : 0u);
  if ((int)threadIdx.x < own) {
    const int64_t v = v0 + threadIdx.x;
    if (v < vocab) start[v] = (int32_t)at;
    if (v == vocab - 1) start[vocab] = (int32_t)(at + total);
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t n = counter[w * own + threadIdx.x];
      counter[w * own + threadIdx.x] = at;
      at += n;
    }
  }
  __syncthreads();
  for (int64_t b = t0; b < t1; b += 64) {
    const int64_t t = b + lane;
    const int64_t v = t < t1 ? row_id(ids, t, vocab) : -1;
    const bool in = v >= v0 && v < v0 + own;
    uint64_t same = __ballot(in);
    if (same == 0) continue;
    const uint32_t l = in ? (uint32_t)(v - v0) : 0u;
    for (int k = 0; k < bits; ++k) {
      const uint64_t ones = __ballot((l >> k) & 1);
      same &= (l >> k) & 1 ? ones : ~ones;
    }
    if (in) {
      const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1));
      uint32_t place = 0;
      if (rank == 0) place = atomicAdd(&mine[l], (uint32_t)__popcll(same));
      place = (uint32_t)__shfl((int)place, __builtin_ctzll(same), kWave) + rank;
      order[place] = (int32_t)t;
      id_out[place] = (int32_t)v;
    }
  }
}

// The columns of one lane: K of a wave's 64 K, adjacent where rows lie on 16 bytes (A), 64 apart otherwise.
template <typename T, bool A>
struct Cols {
  static constexpr int K = 16 / (int)sizeof(T);
  typedef T Raw __attribute__((ext_vector_type(K)));
  int at[A ? 1 : K];
  bool in[A ? 1 : K];
  __device__ __forceinline__ Cols(int slice, int lane, int h) {
#pragma unroll
    for (int k = 0; k < (A ? 1 : K); ++k) {
      const int c = A ? (slice * 64 + lane) * K : (slice * K + k) * 64 + lane;
      in[k] = c < h;
      at[k] = in[k] ? c : 0;
    }
  }
  __device__ __forceinline__ Raw load(const T* row) const {
    if constexpr (A) return *reinterpret_cast<const Raw*>(row + at[0]);
    Raw r;
    if constexpr (!A) {
#pragma unroll
      for (int k = 0; k < K; ++k) r[k] = row[at[k]];
    }
    return r;
  }
  __device__ __forceinline__ void load_f32(const float* row, float* v) const {
    if constexpr (A) {
#pragma unroll
      for (int k = 0; k < K; k += 4) {
        const floatx4 q = *reinterpret_cast<const floatx4*>(row + at[0] + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k + e] = q[e];
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = row[at[k]];
    }
  }
  __device__ __forceinline__ void store_f32(float* row, const float* v) const {
    if constexpr (A) {
      if (!in[0]) return;
#pragma unroll
      for (int k = 0; k < K; k += 4) *reinterpret_cast<floatx4*>(row + at[0] + k) = floatx4{v[k], v[k + 1], v[k + 2], v[k + 3]};
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (in[k]) row[at[k]] = v[k];
    }
  }
};

// Zeros into the rows [v0, v0 + kZeroRows) of ids that do not occur, W entries at a time: the wave walks the rows' entries side by side.
template <int W>
__device__ __forceinline__ void embedding_zero_rows(const EmbedGradArgs& a, const int32_t* start, int64_t v0, int lane) {
  const int64_t v = v0 + lane < a.vocab ? v0 + lane : a.vocab;
  const uint64_t none = __ballot(lane < kZeroRows && v < a.vocab && start[v] == start[v < a.vocab ? v + 1 : v]);
  if (none == 0) return;
  const uint32_t per = (uint32_t)a.h / W, rows = (uint32_t)(a.vocab - v0 < kZeroRows ? a.vocab - v0 : kZeroRows);
  float* p = a.dtable + v0 * a.h;
  uint32_t row = lane / per, rest = lane % per;
  const uint32_t step = 64 / per, left = 64 % per;
  for (uint64_t i = lane; row < rows; i += 64) {
    if ((none >> row) & 1) {
      if constexpr (W == 4) reinterpret_cast<floatx4*>(p)[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      else p[i] = 0.f;
    }
    row += step;
    rest += left;
    if (rest >= per) { rest -= per; ++row; }
  }
}

template <typename T, bool A, bool ACC>
__global__ __launch_bounds__(256) void embedding_sum_kernel(EmbedGradArgs a, EmbedScratch s, int slices) {
  typedef Cols<T, A> C;
  constexpr int K = C::K;
  const int lane = threadIdx.x & 63;
  const int64_t job = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t sums = (int64_t)s.pieces * slices;
  if (job >= sums) {
    if (!ACC)
      for (int64_t z = job - sums; z * kZeroRows < a.vocab; z += (int64_t)gridDim.x * 4 - sums) embedding_zero_rows<A ? 4 : 1>(a, s.start, z * kZeroRows, lane);
    return;
  }
  const int piece = (int)(job / slices), slice = (int)(job % slices);
  const int32_t n = s.start[a.vocab];
  const int64_t p0 = piece * s.piece;
  if (p0 >= n) return;
  const int64_t p1 = p0 + s.piece < n ? p0 + s.piece : n;
  const C cols(slice, lane, a.h);
  const T* dy = static_cast<const T*>(a.dy);
  float* part = s.part + (int64_t)piece * 2 * a.h;
  bool shared = p0 > 0 && s.id[p0 - 1] == s.id[p0];   // the run at hand began in an earlier piece
  float sum[K] = {};
  int last = 0, next = -1;
  for (int64_t b = p0; b < p1; b += kPiece) {
    const int64_t q = b + lane;
    const int32_t id_l = q < n && lane <= kPiece ? s.id[q] : -1, row_l = s.order[q < p1 ? q : p1 - 1];
#pragma unroll
    for (int g = 0; g < kPiece; g += 8) {
      if (b + g >= p1) break;
      typename C::Raw raw[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) raw[i] = cols.load(dy + (int64_t)__builtin_amdgcn_readlane(row_l, g + i) * a.h);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (b + g + i < p1) {
          last = __builtin_amdgcn_readlane(id_l, g + i);
          next = __builtin_amdgcn_readlane(id_l, g + i + 1);
#pragma unroll
          for (int k = 0; k < K; ++k) sum[k] += to_f32(raw[i][k]);
          if (last != next) {
#pragma unroll
            for (int k = 0; k < K; ++k) sum[k] *= a.scale;
            if (shared) {
              cols.store_f32(part, sum);
              shared = false;
            } else {
              float* row = a.dtable + (int64_t)last * a.h;
              if (ACC) {
                float old[K];
                cols.load_f32(row, old);
#pragma unroll
                for (int k = 0; k < K; ++k) sum[k] += old[k];
              }
              cols.store_f32(row, sum);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) sum[k] = 0.f;
          }
        }
      }
    }
  }
  if (last == next) {   // the run goes on in the next piece
#pragma unroll
    for (int k = 0; k < K; ++k) sum[k] *= a.scale;
    cols.store_f32(shared ? part : part + a.h, sum);
  }
}

// The run that begins in piece blockIdx.x and ends in a later one: the sum of its parts.  Four waves take them in turn.
template <typename T, bool A, bool ACC>
__global__ __launch_bounds__(256) void embedding_join_kernel(EmbedGradArgs a, EmbedScratch s, int slices) {
  typedef Cols<T, A> C;
  constexpr int K = C::K;
  __shared__ float lds[3][K][64];
  const int32_t n = s.start[a.vocab];
  const int64_t p0 = blockIdx.x * s.piece, p1 = p0 + s.piece;
  if (p1 >= n) return;
  const int32_t id = s.id[p1 - 1];
  if (s.id[p1] != id || s.start[id] < p0) return;
  const int64_t end = (s.start[id + 1] - 1) / s.piece;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t pitch = 2 * (int64_t)a.h;
  for (int slice = blockIdx.y; slice < slices; slice += gridDim.y) {
    const C cols(slice, lane, a.h);
    float sum[K] = {};
#pragma unroll 4
    for (int64_t c = blockIdx.x + wave; c <= end; c += 4) {
      float v[K];
      cols.load_f32(s.part + c * pitch + (c == blockIdx.x ? a.h : 0), v);
#pragma unroll
      for (int k = 0; k < K; ++k) sum[k] += v[k];
    }
    __syncthreads();
    if (wave > 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) lds[wave - 1][k][lane] = sum[k];
    }
    __syncthreads();
    if (wave == 0) {
      float* row = a.dtable + (int64_t)id * a.h;
      float old[K] = {};
      if (ACC) cols.load_f32(row, old);
#pragma unroll
      for (int k = 0; k < K; ++k) sum[k] = ((sum[k] + lds[0][k][lane]) + (lds[1][k][lane] + lds[2][k][lane])) + old[k];
      cols.store_f32(row, sum);
    }
  }
}

template <typename T, bool A, bool ACC>
hipError_t launch_embedding_sums(const EmbedGradArgs& a, const EmbedScratch& s, hipStream_t st) {
  constexpr int cols = Cols<T, A>::K * 64;
  const int slices = (a.h + cols - 1) / cols;
  int64_t zeros = ACC ? 0 : (a.vocab + kZeroRows - 1) / kZeroRows;
  if (zeros > 65536) zeros = 65536;
  const int64_t jobs = (int64_t)s.pieces * slices + zeros;
  hipLaunchKernelGGL((embedding_sum_kernel<T, A, ACC>), dim3((unsigned)((jobs + 3) / 4)), dim3(256), 0, st, a, s, slices);
  if (s.pieces > 1)
    hipLaunchKernelGGL((embedding_join_kernel<T, A, ACC>), dim3(s.pieces - 1, slices < 8 ? slices : 8), dim3(256), 0, st, a, s, slices);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_embedding_bwd(const EmbedGradArgs& a, hipStream_t st) {
  if (a.rows == 0 && a.accumulate) return hipSuccess;
  const EmbedScratch s = embed_scratch(a.scratch, a.rows, a.vocab);
  int bits = 6;   // about as many workgroups as compute units, each with all ids to read
  while (bits < kSortMaxBits && (a.vocab >> bits) >= 256) ++bits;
  const unsigned groups = (unsigned)((a.vocab + (1ll << bits) - 1) >> bits);
  hipLaunchKernelGGL(embedding_sort_kernel, dim3(groups), dim3(1024), (size_t)kSortWaves << (bits + 2), st, a.ids, a.rows, a.vocab, bits, s.start, s.order, s.id);
  const bool whole = a.h % (16 / (int)sizeof(T)) == 0 && reinterpret_cast<uintptr_t>(a.dy) % 16 == 0 && reinterpret_cast<uintptr_t>(a.dtable) % 16 == 0;
  if (whole) return a.accumulate ? launch_embedding_sums<T, true, true>(a, s, st) : launch_embedding_sums<T, true, false>(a, s, st);
  return a.accumulate ? launch_embedding_sums<T, false, true>(a, s, st) : launch_embedding_sums<T, false, false>(a, s, st);
}

}  // namespace varuna
