// The operators at the two ends of a pipeline and the norm that joins its stages: what stage.hip's C ABI checks and hands
// over, pipeline_ends.hip launches.  Pointers are device memory except where marked host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace varuna {

// Ids of table rows, 32 or 64 bits wide; p == nullptr: row t has the id t mod period.
struct IdArgs {
  const void* p;
  bool wide;
  uint32_t period;
};

// out[t] = scale * table[id_t] + places[position_t]; a term whose id lies outside its table is 0, places may be null.
struct EmbedArgs {
  IdArgs ids, positions;
  const void *table, *places;
  void* out;
  int64_t rows, vocab, n_positions;
  int h;
  float scale;
};
template <typename T> hipError_t launch_embedding_fwd(const EmbedArgs& a, hipStream_t st);

// dtable[v] (+)= scale * sum of dy[t] over the rows t with id v, in ascending order of t.
struct EmbedGradArgs {
  IdArgs ids;
  const void* dy;
  float* dtable;
  void* scratch;
  int64_t rows, vocab;
  int h;
  float scale;
  bool accumulate;
};
size_t embedding_bwd_scratch_bytes(int64_t rows, int64_t h, int64_t vocab);
template <typename T> hipError_t launch_embedding_bwd(const EmbedGradArgs& a, hipStream_t st);

struct LossArgs {
  const void *logits, *targets;
  void* dlogits;       // may be null, may be logits
  float *loss, *out2;  // out2 may be null
  const float* scale;  // may be null
  int64_t rows, ld, ldd;
  int vocab;
  bool wide;           // targets of 64 bits
  float smoothing, grad_scale;
};
template <typename T> hipError_t launch_cross_entropy(const LossArgs& a, hipStream_t st);

// Host arrays of n tensors; bf16: the tensor's type (fp32 otherwise).
struct TensorSpan {
  const void* const* p;
  const int32_t* dtype;
  const int64_t* count;
  int32_t n;
};
size_t grad_norm_scratch_bytes(const int64_t* count, int32_t n);
hipError_t launch_grad_norm(const TensorSpan& t, double* sum_sq, float* nonfinite, void* scratch, hipStream_t st);
hipError_t launch_grad_clip(const TensorSpan& dst, const TensorSpan& src, const double* sum_sq, double max_norm, double eps, hipStream_t st);

}  // namespace varuna
