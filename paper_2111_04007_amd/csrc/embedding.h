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
__device__ __forceinline__ int32_t row_id(const IdArgs& a, uint32_t t, int32_t n) {
  if (a.p == nullptr) return (int32_t)(t % a.period);   // period <= n
  if (a.wide) {
    const int64_t v = static_cast<const int64_t*>(a.p)[t];
    return v >= 0 && v < n ? (int32_t)v : -1;
  }
  const int32_t v = static_cast<const int32_t*>(a.p)[t];
  return v >= 0 && v < n ? v : -1;
}

// A row is moved by `tx` threads in 16-byte pieces (W = 16 / sizeof(T)) where it lies on 16 bytes, else entry by entry; each
// thread has U rows in flight, `apart` rows from one to the next.  Where positions run on their own (SEQ) these are rows of one position in
// U sequences, which read its place once.
template <typename T, int W, int U, bool SEQ, bool PAST>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(EmbedArgs a, int tx_bits, uint32_t apart, uint32_t firsts) {
  typedef T Vec __attribute__((ext_vector_type(W)));
  const int tx = 1 << tx_bits, ty = 256 >> tx_bits, n = a.h / W;
  const bool places = a.places != nullptr;
  const Vec* table = static_cast<const Vec*>(a.table);
  const Vec* place = static_cast<const Vec*>(places ? a.places : a.table);
  const uint32_t rows = (uint32_t)a.rows;
  for (uint32_t i = blockIdx.x * (uint32_t)ty + (threadIdx.x >> tx_bits); i < firsts; i += gridDim.x * (uint32_t)ty) {
    const uint32_t first = i / apart * (apart * U) + i % apart;
    if (first >= rows) continue;
    int64_t id[U], at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t t = u * apart < rows - first ? first + u * apart : first;
      id[u] = row_id(a.ids, t, (int32_t)a.vocab);
      at[u] = SEQ ? (int64_t)(i % apart) : (places ? row_id(a.positions, t, (int32_t)a.n_positions) : -1);
    }
    for (int j = threadIdx.x & (tx - 1); j < n; j += tx) {
      Vec e[U], p[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        e[u] = table[(id[u] < 0 ? 0 : id[u]) * n + j];
        if (SEQ) p[u] = u > 0 ? p[0] : place[at[0] * n + j];
        else if (places) p[u] = place[(at[u] < 0 ? 0 : at[u]) * n + j];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Vec o;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          float v = id[u] < 0 ? 0.f : a.scale * to_f32(e[u][w]);
          if (places && at[u] >= 0) v += to_f32(p[u][w]);
          o[w] = from_f32<T>(v);
        }
        if (u * apart < rows - first) {
          Vec* to = static_cast<Vec*>(a.out) + (int64_t)(first + u * apart) * n + j;
          if (PAST) __builtin_nontemporal_store(o, to);
          else *to = o;
        }
      }
    }
  }
}

template <typename T, int W>
hipError_t launch_embedding_rows(const EmbedArgs& a, hipStream_t st) {
  const int n = a.h / W;
  int bits = 4;
  while (bits < 8 && (1 << bits) < n) ++bits;
  const int64_t ty = 256 >> bits, seq = a.places && !a.positions.p ? a.positions.period : 0;
  // An output larger than the last-level cache is written past the caches, four rows to a thread; where positions run and their table
  // leaves an XCD's L2 (4 MB) by far, these are rows of one position.  us, one row a thread / four / four of one position, all past the caches:
  // 16384 x 8192 over 2048 positions 114 / 112 / 94, 32768 x 8192 222 / 220 / 181, 32768 x 4096 over 1024 94 / 80 / 86, 65536 x 2048 over
  // 2048 106 / 78 / 85; without positions 16384 x 8192 93 / 83, 65536 x 2048 101 / 77 (through the caches 94 at best).  Smaller
  // outputs are faster with one row a thread: 8192 x 4096 23.0 / 25.5, 4096 x 4096 12.2 / 14.5; so are rows of single entries (8201 wide 214 / 350).
  // These go past the caches one row a thread, which pays where nothing reads them soon: us through / past alone, and with a copy of the output behind,
  // bf16 16500 x 8201 210 / 182, 315 / 319; 32768 x 8201 409 / 412, 612 / 626; fp32 9000 x 8201 145 / 147, 257 / 274; 17000 x 4097 140 / 125, 243 / 250.
  const bool past = a.rows * a.h * (int64_t)sizeof(T) >= 256ll << 20, four = past && W > 1;
  const bool share = four && seq > 0 && a.rows >= 4 * seq && seq * a.h * (int64_t)sizeof(T) >= 16 << 20;
  const int64_t u = four ? 4 : 1, apart = share ? seq : ty;
  const int64_t firsts = (a.rows + apart * u - 1) / (apart * u) * apart;   // rows that are some thread's first, to the end of their block
  const int64_t groups = (firsts + ty - 1) / ty;
  const dim3 grid((unsigned)(groups < 1 << 22 ? groups : 1 << 22));
  const uint32_t ap = (uint32_t)apart, fi = (uint32_t)firsts;
  if (!past) hipLaunchKernelGGL((embedding_fwd_kernel<T, W, 1, false, false>), grid, dim3(256), 0, st, a, bits, ap, fi);
  else if constexpr (W == 1) hipLaunchKernelGGL((embedding_fwd_kernel<T, W, 1, false, true>), grid, dim3(256), 0, st, a, bits, ap, fi);
  else if (share) hipLaunchKernelGGL((embedding_fwd_kernel<T, W, 4, true, true>), grid, dim3(256), 0, st, a, bits, ap, fi);
  else hipLaunchKernelGGL((embedding_fwd_kernel<T, W, 4, false, true>), grid, dim3(256), 0, st, a, bits, ap, fi);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_embedding_fwd(const EmbedArgs& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  constexpr int W = 16 / (int)sizeof(T);
  const uintptr_t all = reinterpret_cast<uintptr_t>(a.table) | reinterpret_cast<uintptr_t>(a.places) | reinterpret_cast<uintptr_t>(a.out);
  return a.h % W == 0 && all % 16 == 0 ? launch_embedding_rows<T, W>(a, st) : launch_embedding_rows<T, 1>(a, st);
}

// ---- the gradient ---------------------------------------------------------------------

constexpr int kSortWaves = 16;        // 8 are 1 us faster up to 2048 ids, 50 % slower from 65536 on
constexpr int kSortMaxBits = 9;     // ids of a workgroup: 16 waves' counters of 512 ids are 32 KB of LDS
constexpr int kSortAhead = 8;         // loads of ids under way, per lane
constexpr int kPiece = 16;          // positions whose rows are in flight together
constexpr int kMaxPieces = 1024;
constexpr int kJoinWaves = 8;         // 4: equal, but 16384 rows of two ids 58 us in place of 44
constexpr int kSumWaves = 4096;      // as many waves as pieces and slices of columns are cut for
constexpr int kZeroRows = 16;       // rows of the table looked at together for zeros, fewer where a row is long: 16 KB or one row, whichever is more

// The most pieces that the sorted order of rows h wide is cut into.
inline int64_t embed_most_pieces(int64_t h) {
  const int64_t slices = (h + 511) / 512, most = kSumWaves / slices < kMaxPieces ? kSumWaves / slices : kMaxPieces;
  return most < 64 ? 64 : most;
}
struct EmbedScratch {
  int32_t *start, *order, *id;      // [vocab + 1], [rows], [rows]
  float* part;                      // [pieces][2][h]: the first and the last run of a piece, where it shares them with others
  int64_t piece;                    // positions of one
  int pieces;
};
inline size_t embed_align(size_t n) { return (n + 255) / 256 * 256; }
inline EmbedScratch embed_scratch(void* p, int64_t rows, int64_t h, int64_t vocab) {
  EmbedScratch s;
  char* at = static_cast<char*>(p);
  s.start = reinterpret_cast<int32_t*>(at);
  at += embed_align((size_t)(vocab + 1) * 4);
  s.order = reinterpret_cast<int32_t*>(at);
  at += embed_align((size_t)rows * 4);
  s.id = reinterpret_cast<int32_t*>(at);
  at += embed_align((size_t)rows * 4);
  s.part = reinterpret_cast<float*>(at);
  const int64_t most = embed_most_pieces(h);
  s.piece = ((rows + most - 1) / most + kPiece - 1) / kPiece * kPiece;
  if (s.piece < kPiece) s.piece = kPiece;
  s.pieces = (int)((rows + s.piece - 1) / s.piece);
  return s;
}
size_t embedding_bwd_scratch_bytes(int64_t rows, int64_t h, int64_t vocab) {
  // enough for fewer rows too: their pieces may be more, and shorter
  const int64_t most = embed_most_pieces(h), pieces = (rows + kPiece - 1) / kPiece < most ? (rows + kPiece - 1) / kPiece : most;
  return embed_align((size_t)(vocab + 1) * 4) + 2 * embed_align((size_t)rows * 4) + (size_t)pieces * 2 * (size_t)h * 4 + 256;
}

// LDS written by other lanes of this wave before is read after (the hardware keeps a wave's LDS accesses in order; the compiler has to as well).
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The id of row t as the sort compares it: negative ones and those beyond 32 bits become large numbers, which no range holds.
__device__ __forceinline__ uint32_t sort_id(const IdArgs& a, uint32_t t) {
  if (a.p == nullptr) return t % a.period;
  if (!a.wide) return static_cast<const uint32_t*>(a.p)[t];
  const uint2 v = static_cast<const uint2*>(a.p)[t];
  return v.y == 0 ? v.x : 0xffffffffu;
}

// Stable counting sort of the rows whose id lies in [blockIdx.x << bits, (blockIdx.x + 1) << bits).  A wave owns a contiguous
// sixteenth of all rows.  It counts its ids in LDS and, on the way, the rows of lower ids: where the workgroup's own begin.
// After a prefix sum over (id, wave) it walks its rows once more, gathers those that are its workgroup's, and gives every 64 of
// them their places at once; rows of one id among the 64 are told apart by ballots over the id's bits.  What bounds it is
// instructions: every workgroup looks at every id, with 16 waves on 4 SIMDs, so the walk does little else.  ONE: one id to a
// workgroup, whose lanes would all count in one place; they count for themselves.
template <bool ONE>
__global__ __launch_bounds__(1024) void embedding_sort_kernel(IdArgs ids, uint32_t n, uint32_t vocab, int bits, int32_t* __restrict__ start,
                                                              int32_t* __restrict__ order, int32_t* __restrict__ id_out) {
  extern __shared__ uint32_t counter[];   // [kSortWaves][1 << bits]
  __shared__ uint32_t below[kSortWaves], part[kSortWaves];
  __shared__ uint32_t list_row[kSortWaves][128], list_id[kSortWaves][128];
  const uint32_t own = 1u << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t v0 = blockIdx.x << bits, here = vocab - v0 < own ? vocab - v0 : own;
  uint32_t* mine = counter + wave * own;
  for (uint32_t i = threadIdx.x; i < kSortWaves * own; i += 1024) counter[i] = 0;
  __syncthreads();
  const uint32_t each = (n + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
  const uint32_t t0 = wave * each < n ? wave * each : n, t1 = n - t0 > each ? t0 + each : n;
  uint32_t low = 0, only = 0;
  uint32_t v[kSortAhead];   // ids on their way at once; up to 64 kSortAhead of a wave stay here for the second walk
  auto load = [&](uint32_t b) {
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) v[k] = b + 64 * k + lane < t1 ? sort_id(ids, b + 64 * k + lane) : 0xffffffffu;
  };
  for (uint32_t b = t0; b < t1; b += 64 * kSortAhead) {
    load(b);
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      low += v[k] < v0;
      if (ONE) only += v[k] == v0;
      else if (v[k] - v0 < here) atomicAdd(&mine[v[k] - v0], 1u);
    }
  }
  if (ONE) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) only += __shfl_xor(only, o, kWave);
    if (lane == 0) mine[0] = only;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) low += __shfl_xor(low, o, kWave);
  if (lane == 0) below[wave] = low;
  __syncthreads();
  // Thread i: id i's total, then the prefix over ids, then each wave's first place.
  uint32_t total = 0, of[kSortWaves];
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) of[w] = threadIdx.x < own ? counter[w * own + threadIdx.x] : 0u;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) total += of[w];
  uint32_t sum = total;
#pragma unroll
  for (uint32_t o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(sum, o, kWave);
    if (lane >= o) sum += up;
  }
  if (lane == 63) part[wave] = sum;
  __syncthreads();
  uint32_t at = sum - total;
  for (uint32_t w = 0; w < kSortWaves; ++w) at += below[w] + (w < wave ? part[w] : 0u);
  if (threadIdx.x < here) {
    const uint32_t v = v0 + threadIdx.x;
    start[v] = (int32_t)at;
    if (v == vocab - 1) start[vocab] = (int32_t)(at + total);
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      counter[w * own + threadIdx.x] = at;
      at += of[w];
    }
  }
  __syncthreads();
  uint32_t* rows = list_row[wave];
  uint32_t* keys = list_id[wave];
  uint32_t held = 0;   // gathered and not yet placed: less than 64
  auto place = [&](uint32_t m) {   // the first m of the list, m <= 64
    const bool in = lane < m;
    const uint32_t row = rows[lane], l = in ? keys[lane] : 0u;
    uint64_t same = __ballot(in);
    for (int i = 0; i < bits; ++i) {
      const uint64_t ones = __ballot((l >> i) & 1);
      same &= (l >> i) & 1 ? ones : ~ones;
    }
    if (in) {
      const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1));
      uint32_t first = 0;
      if (rank == 0) first = atomicAdd(&mine[l], (uint32_t)__popcll(same));
      first = (uint32_t)__shfl((int)first, __builtin_ctzll(same), kWave) + rank;
      order[first] = (int32_t)row;
      id_out[first] = (int32_t)(v0 + l);
    }
  };
  for (uint32_t b = t0; b < t1; b += 64 * kSortAhead) {
    if (each > 64 * kSortAhead) load(b);
#pragma unroll
    for (int k = 0; k < kSortAhead; ++k) {
      const bool in = v[k] - v0 < here;
      const uint64_t which = __ballot(in);
      if (which == 0) continue;
      if (in) {
        const uint32_t to = held + (uint32_t)__popcll(which & ((1ull << lane) - 1));
        rows[to] = b + 64 * k + lane;
        keys[to] = v[k] - v0;
      }
      held += (uint32_t)__popcll(which);
      wave_order();
      if (held >= 64) {
        place(64);
        wave_order();
        const uint32_t row = rows[64 + lane], key = keys[64 + lane];
        wave_order();
        rows[lane] = row;
        keys[lane] = key;
        held -= 64;
        wave_order();
      }
    }
  }
  if (held > 0) place(held);
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

// Zeros into those rows of [v0, v0 + rows), rows <= kZeroRows, that `none` has a bit for, W entries at a time: the workgroup walks the
// rows' entries side by side.
template <int W>
__device__ __forceinline__ void embedding_zero_rows(const EmbedGradArgs& a, uint64_t none, int64_t v0, uint32_t rows) {
  if (none == 0) return;
  const uint32_t per = (uint32_t)a.h / W;
  if (a.vocab - v0 < rows) rows = (uint32_t)(a.vocab - v0);
  float* p = a.dtable + v0 * a.h;
  uint32_t row = threadIdx.x / per, rest = threadIdx.x % per;
  const uint32_t step = 256 / per, left = 256 % per;
  for (uint64_t i = threadIdx.x; row < rows; i += 256) {
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
__global__ __launch_bounds__(256) void embedding_sum_kernel(EmbedGradArgs a, EmbedScratch s, int slices, uint32_t zero_rows) {
  typedef Cols<T, A> C;
  constexpr int K = C::K;
  const int lane = threadIdx.x & 63;
  const int64_t job = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t sums = (int64_t)s.pieces * slices;
  if (job >= sums) {
    const int64_t first = (sums + 3) / 4;
    if (!ACC)
      for (int64_t z = blockIdx.x - first; z >= 0 && z * zero_rows < a.vocab; z += gridDim.x - first) {
        const int64_t v = z * zero_rows + lane;
        const uint64_t none = __ballot(lane < (int)zero_rows && v < a.vocab && s.start[v] == s.start[v + 1]);
        embedding_zero_rows<A ? 4 : 1>(a, none, z * zero_rows, zero_rows);
      }
    return;
  }
  const int piece = (int)(job / slices), slice = (int)(job % slices);
  const C cols(slice, lane, a.h);
  const T* dy = static_cast<const T*>(a.dy);
  float* part = s.part + (int64_t)piece * 2 * a.h;
  const int64_t p0 = piece * s.piece;
  const int32_t n = s.start[a.vocab];
  const int32_t before = s.id[p0 > 0 ? p0 - 1 : 0];
  float sum[K] = {};
  bool shared = false, open = false;   // the run at hand began in an earlier piece; it has not ended
  for (int64_t b = p0; b < p0 + s.piece; b += kPiece) {
    // lane i: position b + i (what lies behind the last row that has an id is loaded, so as not to wait for n first, and not used)
    const int64_t q = b + lane < a.rows ? b + lane : a.rows - 1;
    int32_t id_l = s.id[q], row_l = s.order[q];
    const int64_t here = n - b;   // positions from b on
    if (here <= 0) break;
    id_l = lane < here && lane <= kPiece ? id_l : -1;
    row_l = lane < here ? row_l : 0;
    if (b == p0) shared = p0 > 0 && before == __builtin_amdgcn_readlane(id_l, 0);
    typename C::Raw raw[kPiece];
#pragma unroll
    for (int i = 0; i < kPiece; ++i)
      if (i < here) raw[i] = cols.load(dy + (int64_t)__builtin_amdgcn_readlane(row_l, i) * a.h);
    // Positions at which a run ends, and those of them whose sum goes to the table: not that of a run from an earlier piece.
    const int32_t next_l = __shfl_down(id_l, 1, kWave);   // by all lanes: the 16th looks at the 17th
    const uint32_t ends = (uint32_t)__ballot(lane < kPiece && lane < here && id_l != next_l);
    const uint32_t direct = shared ? ends & (ends - 1) : ends;
    if (ends != 0) shared = false;
    // Halves: the rows that are added to are on their way together.
#pragma unroll
    for (int g = 0; g < kPiece; g += kPiece / 2) {
      float old[ACC ? kPiece / 2 : 1][K];
      if (ACC) {
#pragma unroll
        for (int i = 0; i < kPiece / 2; ++i)
          if ((direct >> (g + i)) & 1) cols.load_f32(a.dtable + (int64_t)__builtin_amdgcn_readlane(id_l, g + i) * a.h, old[i]);
      }
#pragma unroll
      for (int i = 0; i < kPiece / 2; ++i) {
        if (g + i < here) {
#pragma unroll
          for (int k = 0; k < K; ++k) sum[k] += to_f32(raw[g + i][k]);
          if ((ends >> (g + i)) & 1) {
#pragma unroll
            for (int k = 0; k < K; ++k) sum[k] *= a.scale;
            if ((direct >> (g + i)) & 1) {
              if (ACC) {
#pragma unroll
                for (int k = 0; k < K; ++k) sum[k] += old[i][k];
              }
              cols.store_f32(a.dtable + (int64_t)__builtin_amdgcn_readlane(id_l, g + i) * a.h, sum);
            } else {
              cols.store_f32(part, sum);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) sum[k] = 0.f;
          }
        }
      }
    }
    open = here >= kPiece && !((ends >> (kPiece - 1)) & 1);
  }
  if (open) {   // the last run goes on in the next piece
#pragma unroll
    for (int k = 0; k < K; ++k) sum[k] *= a.scale;
    cols.store_f32(shared ? part : part + a.h, sum);
  }
}

// The run that begins in piece blockIdx.x and ends in a later one: the sum of its parts.  kJoinWaves waves take them in turn.
template <typename T, bool A, bool ACC>
__global__ __launch_bounds__(64 * kJoinWaves) void embedding_join_kernel(EmbedGradArgs a, EmbedScratch s, int slices) {
  typedef Cols<T, A> C;
  constexpr int K = C::K;
  __shared__ float lds[kJoinWaves - 1][K][64];
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
    for (int64_t c = blockIdx.x + wave; c <= end; c += 4 * kJoinWaves) {   // four parts of every wave are on their way at once
      float v[4][K];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t p = c + i * kJoinWaves <= end ? c + i * kJoinWaves : c;
        cols.load_f32(s.part + p * pitch + (p == blockIdx.x ? a.h : 0), v[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i * kJoinWaves <= end) {
#pragma unroll
          for (int k = 0; k < K; ++k) sum[k] += v[i][k];
        }
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
      for (int w = 0; w < kJoinWaves - 1; ++w) {
#pragma unroll
        for (int k = 0; k < K; ++k) sum[k] += lds[w][k][lane];
      }
#pragma unroll
      for (int k = 0; k < K; ++k) sum[k] += old[k];
      cols.store_f32(row, sum);
    }
  }
}

// How the rows of the table are dealt to workgroups that look for zeros: rows of each, and how many (none where the gradient is added to).
struct ZeroShare { uint32_t rows; int64_t groups; };
inline ZeroShare zero_share(int h, int64_t vocab, bool accumulate) {
  uint32_t rows = (4 << 10) / (uint32_t)h;
  rows = rows < 1 ? 1 : (rows > kZeroRows ? kZeroRows : rows);
  const int64_t groups = accumulate ? 0 : (vocab + rows - 1) / rows;
  return {rows, groups < 65536 ? groups : 65536};
}

template <typename T, bool A, bool ACC>
hipError_t launch_embedding_sums(const EmbedGradArgs& a, const EmbedScratch& s, hipStream_t st) {
  constexpr int cols = Cols<T, A>::K * 64;
  const int slices = (a.h + cols - 1) / cols;
  const ZeroShare zeros = zero_share(a.h, a.vocab, ACC);
  const int64_t groups = ((int64_t)s.pieces * slices + 3) / 4 + zeros.groups;
  hipLaunchKernelGGL((embedding_sum_kernel<T, A, ACC>), dim3((unsigned)groups), dim3(256), 0, st, a, s, slices, zeros.rows);
  if (s.pieces > 1)
    hipLaunchKernelGGL((embedding_join_kernel<T, A, ACC>), dim3(s.pieces - 1, slices < 8 ? slices : 8), dim3(64 * kJoinWaves), 0, st, a, s, slices);
  return hipGetLastError();
}

// Positions that run: the rows of position p are p, p + period, ... and need no sorting.  One wave per position and slice of columns, which sums
// all of a position's rows in order, in fp32: n of them are off by at most n steps of 2^-24 of the sum of their absolute values.
template <typename T, bool A, bool ACC>
__global__ __launch_bounds__(256) void embedding_positions_kernel(EmbedGradArgs a, int slices, uint32_t jobs) {
  typedef Cols<T, A> C;
  constexpr int K = C::K;
  const uint32_t job = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (job >= jobs) return;
  const uint32_t p = job / (uint32_t)slices, period = a.ids.period, rows = (uint32_t)a.rows;
  const C cols((int)(job % (uint32_t)slices), threadIdx.x & 63, a.h);
  const T* dy = static_cast<const T*>(a.dy);
  float* row = a.dtable + (int64_t)p * a.h;
  const uint32_t n = p < period && p < rows ? (rows - p - 1) / period + 1 : 0;
  float sum[K] = {}, old[K] = {};
  if (ACC) cols.load_f32(row, old);
  for (uint32_t b = 0; b < n; b += 8) {
    typename C::Raw raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = cols.load(dy + (int64_t)(p + (b + i < n ? b + i : b) * period) * a.h);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int k = 0; k < K; ++k) sum[k] += b + i < n ? to_f32(raw[i][k]) : 0.f;
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k) sum[k] = sum[k] * a.scale + old[k];
  cols.store_f32(row, sum);
}

// Few rows (up to kFewRows): every wave holds all ids, four of them a lane.  The wave of a row that is the first with its id sums that
// id's rows, the others end at once; more workgroups put zeros into rows of ids that do not occur.  One launch in place of three: us of the
// three / of this, 128 rows of 128 14.6 / 7.4, 256 of 8192 17.8 / 7.5, 250 of 333 19.6 / 7.0.  A run is one wave's, so that 256 rows of one
// id, the worst that can come, are slower: 15 / 27 (512 rows 14 / 50, which is why it ends here).
constexpr int kFewRows = 256;
template <typename T, bool A, bool ACC>
__global__ __launch_bounds__(256) void embedding_few_kernel(EmbedGradArgs a, int slices, uint32_t zero_rows) {
  typedef Cols<T, A> C;
  constexpr int K = C::K, N = kFewRows / 64, AHEAD = 8;
  const uint32_t lane = threadIdx.x & 63, rows = (uint32_t)a.rows, vocab = (uint32_t)a.vocab;
  uint32_t ids[N];
#pragma unroll
  for (int k = 0; k < N; ++k) ids[k] = 64 * k + lane < rows ? sort_id(a.ids, 64 * k + lane) : 0xffffffffu;
  const uint32_t job = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sums = rows * (uint32_t)slices;
  if (job >= sums) {
    const uint32_t first = (sums + 3) / 4;
    if (!ACC && blockIdx.x >= first) {
      for (uint64_t z = blockIdx.x - first; z * zero_rows < vocab; z += gridDim.x - first) {
        const uint32_t v0 = (uint32_t)z * zero_rows;
        uint32_t some = 0;
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (ids[k] - v0 < zero_rows) some |= 1u << (ids[k] - v0);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) some |= __shfl_xor(some, o, kWave);
        embedding_zero_rows<A ? 4 : 1>(a, ~(uint64_t)some, v0, zero_rows);
      }
    }
    return;
  }
  const uint32_t t = job / (uint32_t)slices;
  const uint32_t v = __builtin_amdgcn_readfirstlane(sort_id(a.ids, t));
  if (v >= vocab) return;
  const C cols((int)(job % (uint32_t)slices), (int)lane, a.h);
  const T* dy = static_cast<const T*>(a.dy);
  float* row = a.dtable + (int64_t)v * a.h;
  float sum[K] = {}, old[K] = {};
  uint64_t own[N];
  bool earlier = false;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    own[k] = __ballot(ids[k] == v);
    if (64 * k <= t) earlier = earlier || (own[k] & (t - 64 * k < 64 ? (1ull << (t - 64 * k)) - 1 : ~0ull)) != 0;
  }
  if (earlier) return;
  if (ACC) cols.load_f32(row, old);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    uint64_t left = own[k];
    while (left != 0) {   // AHEAD rows of the id at a time, in order
      typename C::Raw raw[AHEAD];
      uint64_t rest = left;
      int at = 0, n = 0;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (rest != 0) { at = __builtin_ctzll(rest); rest &= rest - 1; ++n; }
        raw[i] = cols.load(dy + (int64_t)(64 * k + at) * a.h);
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (i < n) {
#pragma unroll
          for (int e = 0; e < K; ++e) sum[e] += to_f32(raw[i][e]);
        }
      left = rest;
    }
  }
#pragma unroll
  for (int e = 0; e < K; ++e) sum[e] = sum[e] * a.scale + old[e];
  cols.store_f32(row, sum);
}

// Whether the positions' sums run by themselves: up to 128 rows each, one after the other, or where the waves fill the chip.  us, sorted / by
// themselves, h = 1024: 64 positions of 64 rows 15 / 7, of 128 17 / 11, of 256 23.5 / 21, of 1024 56 / 81; 512 positions of 256 90 / 40;
// 16 of 256 rows 256 wide 15 / 19.
constexpr int kDirectRows = 128, kDirectJobs = 1024;

template <typename T, bool A, bool ACC>
bool launch_embedding_positions(const EmbedGradArgs& a, hipStream_t st) {
  constexpr int cols = Cols<T, A>::K * 64;
  const int slices = (a.h + cols - 1) / cols;
  const int64_t period = a.ids.period < a.rows ? a.ids.period : a.rows;
  const int64_t jobs = (ACC ? period : a.vocab) * slices;
  if (a.ids.p != nullptr || (a.rows > period * kDirectRows && period * slices < kDirectJobs) || jobs == 0 || jobs >= 1 << 24) return false;
  hipLaunchKernelGGL((embedding_positions_kernel<T, A, ACC>), dim3((unsigned)((jobs + 3) / 4)), dim3(256), 0, st, a, slices, (uint32_t)jobs);
  return true;
}

template <typename T, bool A, bool ACC>
hipError_t launch_embedding_few(const EmbedGradArgs& a, hipStream_t st) {
  constexpr int cols = Cols<T, A>::K * 64;
  const int slices = (a.h + cols - 1) / cols;
  const ZeroShare zeros = zero_share(a.h, a.vocab, ACC);
  const int64_t groups = (a.rows * slices + 3) / 4 + zeros.groups;
  hipLaunchKernelGGL((embedding_few_kernel<T, A, ACC>), dim3((unsigned)groups), dim3(256), 0, st, a, slices, zeros.rows);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_embedding_bwd(const EmbedGradArgs& a, hipStream_t st) {
  if (a.rows == 0 && a.accumulate) return hipSuccess;
  const bool whole = a.h % (16 / (int)sizeof(T)) == 0 && reinterpret_cast<uintptr_t>(a.dy) % 16 == 0 && reinterpret_cast<uintptr_t>(a.dtable) % 16 == 0;
  if (whole ? (a.accumulate ? launch_embedding_positions<T, true, true>(a, st) : launch_embedding_positions<T, true, false>(a, st))
            : (a.accumulate ? launch_embedding_positions<T, false, true>(a, st) : launch_embedding_positions<T, false, false>(a, st)))
    return hipGetLastError();
  if (a.rows <= kFewRows) {
    if (whole) return a.accumulate ? launch_embedding_few<T, true, true>(a, st) : launch_embedding_few<T, true, false>(a, st);
    return a.accumulate ? launch_embedding_few<T, false, true>(a, st) : launch_embedding_few<T, false, false>(a, st);
  }
  const EmbedScratch s = embed_scratch(a.scratch, a.rows, a.h, a.vocab);
  int bits = 0;   // about as many workgroups as compute units, each with all ids to read
  while (bits < kSortMaxBits && (a.vocab >> bits) >= 256) ++bits;
  const unsigned groups = (unsigned)((a.vocab + (1ll << bits) - 1) >> bits);
  const size_t lds = (size_t)kSortWaves << (bits + 2);
  const uint32_t rows = (uint32_t)a.rows, vocab = (uint32_t)a.vocab;
  if (bits == 0) hipLaunchKernelGGL(embedding_sort_kernel<true>, dim3(groups), dim3(1024), lds, st, a.ids, rows, vocab, bits, s.start, s.order, s.id);
  else hipLaunchKernelGGL(embedding_sort_kernel<false>, dim3(groups), dim3(1024), lds, st, a.ids, rows, vocab, bits, s.start, s.order, s.id);
  if (whole) return a.accumulate ? launch_embedding_sums<T, true, true>(a, s, st) : launch_embedding_sums<T, true, false>(a, s, st);
  return a.accumulate ? launch_embedding_sums<T, false, true>(a, s, st) : launch_embedding_sums<T, false, false>(a, s, st);
}

}  // namespace varuna
