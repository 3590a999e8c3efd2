/*
 * varuna_stage.h -- C ABI of the MI355X (gfx950) pipeline-stage compute library.
 *
 * One pipeline stage's micro-batched training step for a GPT-style transformer:
 * forward for each micro-batch keeping only the stage-input ("boundary")
 * activation; backward first recomputes the stage's internal activations from
 * that stored tensor, then produces the input gradient and the parameter
 * gradients, which accumulate in fp32 over the micro-batches a GPU holds.
 * (Paper: Design Overview, "High-level architecture" -- stage k takes
 * activations from k-1 and gradients from k+1, and recomputes activations from
 * the stored input activation; Background, "Memory optimization" -- gradient
 * checkpointing, forward is about a third of the compute; Job Morphing,
 * "Correctness-preserving morphing" -- gradient accumulation within a GPU.)
 *
 * Conventions
 *   - Every pointer marked "device" is GPU memory owned by the caller (the
 *     caller allocates, e.g. through PyTorch); it must stay valid until
 *     varuna_stage_destroy and be 256-byte aligned.  The library allocates no
 *     device memory in any call.
 *   - hip_stream is a hipStream_t passed as void* (NULL = the default stream).
 *     Every compute call only enqueues work and returns; nothing synchronises
 *     with the host.  All work and all results of a call are ordered on
 *     hip_stream.  The library creates no stream.  One handle is used from one
 *     stream at a time.
 *   - Activations are row-major [T, h], T = micro_batch * seq_len, row index
 *     = batch_index * seq_len + position.  dtype F32: all tensors fp32.
 *     dtype BF16: activations, parameters and dX are bf16; all accumulators,
 *     LayerNorm statistics, log-sum-exp and every parameter gradient are fp32.
 *   - Parameter buffer layout: layers back to back; inside a layer, in this
 *     order, each matrix row-major [out, in]:
 *        ln1_g[h] ln1_b[h] Wqkv[3h,h] bqkv[3h] Wo[h,h] bo[h]
 *        ln2_g[h] ln2_b[h] W1[f,h] b1[f] W2[h,f] b2[h]
 *     Rows of Wqkv are [Q | K | V] blocks of h rows; head j owns rows
 *     j*d .. (j+1)*d-1 of each block (d = h / heads).  The gradient buffer has
 *     the same element order, always fp32.  varuna_stage_param_offset reports
 *     the element offsets.
 *   - Every call returns a varuna_status_t; on failure varuna_last_error()
 *     returns a message (thread-local storage, valid until the next failing
 *     call on that thread).  Argument checks never touch the GPU.
 */
#ifndef VARUNA_STAGE_H
#define VARUNA_STAGE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct varuna_stage varuna_stage_t; /* opaque, host memory owned by the library */

typedef enum {
  VARUNA_OK = 0,
  VARUNA_EINVAL = -1,       /* bad argument or configuration */
  VARUNA_ESTATE = -2,       /* call order violated (e.g. backward before forward of that slot) */
  VARUNA_ENOMEM = -3,       /* host allocation failed */
  VARUNA_EHIP = -4,         /* a HIP runtime call or kernel launch failed */
  VARUNA_EUNSUPPORTED = -5  /* valid but not implemented for this shape */
} varuna_status_t;

typedef enum { VARUNA_F32 = 0, VARUNA_BF16 = 1 } varuna_dtype_t;
typedef enum { VARUNA_I32 = 0, VARUNA_I64 = 1 } varuna_index_t; /* token, position and target ids */

/* Number of parameter tensors per layer and their indices in the layout above. */
#define VARUNA_PARAMS_PER_LAYER 12
enum {
  VARUNA_P_LN1_G = 0, VARUNA_P_LN1_B, VARUNA_P_WQKV, VARUNA_P_BQKV, VARUNA_P_WO, VARUNA_P_BO,
  VARUNA_P_LN2_G, VARUNA_P_LN2_B, VARUNA_P_W1, VARUNA_P_B1, VARUNA_P_W2, VARUNA_P_B2
};

/* Plain data; the library copies it. */
typedef struct {
  int32_t n_layers;        /* L >= 1: transformer layers in this stage */
  int32_t hidden;          /* h */
  int32_t n_heads;         /* a, must divide h */
  int32_t seq_len;         /* s */
  int32_t micro_batch;     /* b: examples per micro-batch (the paper's m) */
  int32_t n_micro_batches; /* M: number of boundary slots (the paper's N_m) */
  int32_t mlp_hidden;      /* f; 0 means 4*h */
  int32_t causal;          /* 1: key index <= query index only; 0: bidirectional */
  int32_t dtype;           /* varuna_dtype_t */
  float ln_eps;            /* 0 means 1e-5 */
  int32_t wgrad_group;     /* G: weight-gradient GEMMs are issued once per G micro-batches with
                              reduction length G*T (0 or 1: after every micro-batch); on the bf16 path
                              G * T * mlp_hidden * 2 bytes must stay below 4 GiB (VARUNA_EUNSUPPORTED) */
  float dropout_p;         /* dropout probability in [0,1), applied as round(256 p)/256; 0: none.
                              See varuna_stage_set_dropout_seed. */
} varuna_stage_config_t;

/* Byte sizes of the four caller-allocated device buffers for this configuration.
 * boundary_bytes = M * T * h * sizeof(activation): one stage-input tensor per
 * micro-batch is all that forward keeps (Design Overview: 3.75 MB per example
 * for h=1920, s=1024 in 16-bit).  Any output pointer may be NULL. */
varuna_status_t varuna_stage_query_sizes(const varuna_stage_config_t* cfg, size_t* param_bytes,
                                         size_t* grad_bytes, size_t* boundary_bytes,
                                         size_t* workspace_bytes);

/* Element offset (from the start of the parameter buffer, equally of the
 * gradient buffer) and element count of parameter tensor `which` of `layer`. */
varuna_status_t varuna_stage_param_offset(const varuna_stage_config_t* cfg, int32_t layer,
                                          int32_t which, size_t* offset_elems, size_t* n_elems);

/* Creates a stage over caller-owned device buffers of the sizes reported by
 * varuna_stage_query_sizes.  params: read-only; grads_f32: accumulators, not
 * cleared here (call varuna_stage_grad_accum_reset); boundary: M slots [T,h];
 * workspace: scratch, contents undefined between calls.  Validates the
 * configuration without touching the GPU. */
varuna_status_t varuna_stage_create(const varuna_stage_config_t* cfg, const void* params /*device*/,
                                    void* grads_f32 /*device*/, void* boundary /*device*/,
                                    void* workspace /*device*/, varuna_stage_t** out);

/* Stage forward for micro-batch slot mb (0 <= mb < M): copies x_in [T,h] into
 * boundary slot mb (skipped when x_in is that slot), runs the L layers, writes
 * the stage output y_out [T,h].  Nothing else is kept.  x_in is read by kernels, as every tensor of these calls is: it has to lie
 * in memory that the GPU of hip_stream can read. */
varuna_status_t varuna_stage_forward(varuna_stage_t* st, int32_t mb, const void* x_in /*device*/,
                                     void* y_out /*device*/, void* hip_stream);

/* Recompute + backward for slot mb: re-derives all internal activations from
 * boundary slot mb (bit-identical to what forward computed), then from the
 * upstream gradient dy_in [T,h] writes the input gradient dx_out [T,h] and adds
 * this micro-batch's parameter gradients into grads_f32 (the four matrix gradients
 * per layer possibly deferred, see varuna_stage_grad_flush).  Requires a forward of
 * slot mb since that slot was last consumed (else VARUNA_ESTATE).  Calls for
 * different slots may be interleaved with forwards in any order.  dy_in is read where it lies by kernels up to the last of the
 * call, so it may be overwritten by work that follows on
 * hip_stream but not by another stream before that; dx_out may be dy_in or overlap it. */
varuna_status_t varuna_stage_backward_recompute(varuna_stage_t* st, int32_t mb,
                                                const void* dy_in /*device*/,
                                                void* dx_out /*device*/, void* hip_stream);

/* Last-stage variant (Design Overview, "Tuning pipeline efficiency": in the paper's schedule
 * the last pipeline stage runs the backward of a micro-batch straight after its forward and
 * therefore never recomputes).  varuna_stage_forward_keep is varuna_stage_forward that also
 * leaves every layer's internal activations of micro-batch mb in the workspace, in exactly
 * the form the recompute pass would leave them (same kernels, same launch geometry);
 * varuna_stage_backward_stored then runs the backward pass of backward_recompute on them
 * without recomputing.  The workspace holds the internals of ONE micro-batch: the pair must
 * be adjacent for a given mb -- any other forward_keep, backward_recompute or
 * grad_accum_reset in between invalidates them (plain varuna_stage_forward calls of other
 * slots do not) and backward_stored then returns VARUNA_ESTATE.  Arguments, layouts, the
 * accumulation into grads_f32 and the wgrad_group deferral are those of the two calls above;
 * outputs and gradients are bit-identical to the forward / backward_recompute pair. */
varuna_status_t varuna_stage_forward_keep(varuna_stage_t* st, int32_t mb, const void* x_in /*device*/,
                                          void* y_out /*device*/, void* hip_stream);
varuna_status_t varuna_stage_backward_stored(varuna_stage_t* st, int32_t mb,
                                             const void* dy_in /*device*/,
                                             void* dx_out /*device*/, void* hip_stream);

/* Optional second stream, created and owned by the caller (default priority; it must outlive
 * the handle or be replaced by NULL first), or NULL (the state after create).  A backward call
 * may run its bias-gradient column sums there, joined back into hip_stream's order before it
 * returns.  The present kernels do not: the sums share a launch with the last LayerNorm of the
 * layer, which is faster at every measured size.  Results are bit-identical either way. */
varuna_status_t varuna_stage_set_side_stream(varuna_stage_t* st, void* side_stream);

/* Dropout (config.dropout_p > 0) acts on the attention probabilities and on the two residual
 * branches (attention-output projection and MLP output, after their bias, before the add).
 * The paper's implementation saves and restores the random-number state so that the
 * recompute pass reproduces the forward pass (Implementation, list of library functions);
 * here every mask is a pure function of (seed, micro-batch slot mb, layer, site, element),
 * so forward, recompute and backward regenerate it and nothing is stored.  Generator:
 * Philox4x32-10, key = (seed mod 2^32, seed div 2^32), counter = (row div 4, column div 4,
 * site + 256*layer, mb); the byte of element (row, column) is byte (column mod 4), little end
 * first, of output word (row mod 4); the element is kept iff byte >= thr = round(256 p) and
 * kept values are multiplied by 256 / (256 - thr).  Sites: 0 = attention probabilities
 * (row = (batch*heads + head)*seq_len + query, column = key), 1 = projection branch,
 * 2 = MLP branch (row = token, column = hidden index).
 * The seed is 0 after create; set a new one per mini-batch.  It must not change between a
 * forward and the backward of the same slot (VARUNA_ESTATE while any slot is forwarded and
 * not yet consumed). */
varuna_status_t varuna_stage_set_dropout_seed(varuna_stage_t* st, uint64_t seed);

/* With wgrad_group G > 1 the operands of the weight-gradient products dW += dY^T X are kept
 * for up to G micro-batches (the workspace holds G slots of them, stacked along the token
 * dimension) and each dW receives ONE GEMM over G*T tokens and one fp32 read-modify-write:
 * gradient accumulation within a GPU (Job Morphing, "Correctness-preserving morphing") with
 * the accumulation partly folded into the GEMM's reduction.  The matrix gradients are then
 * complete only after every G-th backward_recompute call, or after this call, which issues
 * the GEMMs for whatever has been gathered (a no-op when nothing is pending or G <= 1).
 * Bias, gamma and beta gradients are always added per call.  Call it before reading
 * grads_f32 at the end of a mini-batch. */
varuna_status_t varuna_stage_grad_flush(varuna_stage_t* st, void* hip_stream);

/* Zero-fills grads_f32 (start of a mini-batch) and drops any gathered, unflushed operands. */
varuna_status_t varuna_stage_grad_accum_reset(varuna_stage_t* st, void* hip_stream);

/* ---- mini-batch tail: one GPU's share of the optimizer step ------------------------------
 * The paper keeps 16 bytes of state per parameter -- a 16-bit parameter and gradient plus
 * fp32 master weight, momentum and variance (Background, "Memory optimization") -- and
 * synchronises an overflow flag / gradient norm over the stages of a pipeline (Enabling Ease
 * of Programming, "Tracking cross-partition dependencies"; Implementation, "Synchronization
 * of shared state").  These two calls are the per-GPU part; the reduction across GPUs is the
 * caller's.  Both return VARUNA_ESTATE while deferred weight gradients are pending (call
 * varuna_stage_grad_flush first). */

/* out2 (device, 2 floats): [0] = sum of squares of the finite entries of grads_f32,
 * [1] = number of non-finite entries.  Deterministic (fixed reduction order). */
varuna_status_t varuna_stage_grad_stats(varuna_stage_t* st, float* out2 /*device*/, void* hip_stream);

typedef struct {
  float lr, beta1, beta2, eps;
  float weight_decay;  /* decoupled: w -= lr * weight_decay * w */
  float grad_scale;    /* multiplies every gradient first (1/loss scale, 1/M, clip factor) */
  int32_t step;        /* number of this update, >= 1 (bias correction) */
} varuna_adam_t;

/* One Adam update (Kingma & Ba, Algorithm 1, with decoupled weight decay) over all parameters
 * of the stage, element order = parameter layout:  g = grad_scale * grads_f32;
 * m = b1 m + (1-b1) g;  v = b2 v + (1-b2) g^2;
 * master -= lr * ((m / (1-b1^step)) / (sqrt(v / (1-b2^step)) + eps) + weight_decay * master);
 * params_out = master rounded to the stage's storage type (RNE).  master_f32, m_f32, v_f32:
 * caller-owned device buffers of grad_bytes each, 16-byte aligned; params_out: normally the
 * params buffer given to varuna_stage_create.  If skip_if_nonzero (device, may be NULL)
 * points to a non-zero value when the kernel runs, nothing is changed (an overflow anywhere
 * in the pipeline cancels the step). */
varuna_status_t varuna_stage_adam_step(varuna_stage_t* st, const varuna_adam_t* hp, void* params_out /*device*/,
                                       float* master_f32 /*device*/, float* m_f32 /*device*/,
                                       float* v_f32 /*device*/, const float* skip_if_nonzero /*device*/,
                                       void* hip_stream);

/* Releases the host-side handle.  Device buffers stay with the caller. */
varuna_status_t varuna_stage_destroy(varuna_stage_t* st);

const char* varuna_last_error(void);

/* ---- test hooks (not on the timed path) -------------------------------- */

/* Forward that also stores the internal activations of every layer in the
 * workspace, exactly as the recompute pass stores them, so a test can compare
 * the two bit for bit. */
varuna_status_t varuna_stage_debug_forward_save(varuna_stage_t* st, int32_t mb,
                                                const void* x_in /*device*/,
                                                void* y_out /*device*/, void* hip_stream);
/* Byte range of the workspace that holds those stored activations. */
varuna_status_t varuna_stage_debug_saved_region(const varuna_stage_t* st, size_t* offset_bytes,
                                                size_t* n_bytes);

/* Tuning aid: which bf16 MFMA GEMM kernel configuration (the `variant` numbers of varuna_op_gemm)
 * the stage calls use for forward / dgrad / wgrad products on 256x256 and on 128x128 tiles; 0
 * restores the library's choice.  Naming a 128x128 configuration for forward or dgrad also turns
 * off the library's merging of 128x128 tile pairs into one 128x256 / 256x128 tile (configurations
 * 20 / 21), naming one for wgrad its grouping of several weight gradients into one launch; a product of few tiles, which
 * the library gives to smaller tiles (-1), then runs on 128x128 tiles too.  Process-wide, not
 * thread-safe, for same-process A/B timing only: results of every configuration agree to rounding but not bit for bit. */
varuna_status_t varuna_debug_set_gemm_kernels(int32_t fwd256, int32_t dgrad256, int32_t wgrad256,
                                              int32_t fwd128, int32_t dgrad128, int32_t wgrad128);
/* Host only (no GPU call): the kernel configuration of a bf16 product of contiguous, 16-byte aligned operands by the tiles' rounds on the
 * chip alone, op as in varuna_op_gemm (0 forward, 1 dgrad, 2 wgrad): a `variant` number of varuna_op_gemm, -1 for the kernels on small
 * tiles whose waves share the reduction (rows that are not whole 16-byte pieces, and products of few 128x128 tiles), -2 for an
 * invalid argument.  What runs is varuna_debug_gemm_launch's answer. */
int32_t varuna_debug_gemm_choice(int32_t op, int64_t M, int64_t N, int64_t K);
/* The configuration that runs, epi as in varuna_op_gemm: the same, or another one that epilogue and length of the reduction let end sooner. */
int32_t varuna_debug_gemm_launch(int32_t op, int32_t epi, int64_t M, int64_t N, int64_t K);
/* Host only: the configuration (18, 19, 22 or 23) by the tiles' rounds for the weight gradients of n_layers (1 to 4) consecutive
 * bf16 layers over `tokens` stacked tokens (16-byte aligned) in one launch, -1 if they share one launch of the small tiles
 * (at most 128 tiles of 128x128 in all; more layers than that run one by one), 0 if they run one by one, -2 for an invalid argument.  What runs is
 * varuna_debug_wgrad_group_launch's answer. */
int32_t varuna_debug_wgrad_group_choice(int32_t n_layers, int64_t hidden, int64_t mlp, int64_t tokens);
/* What runs: the same, or over long reductions larger tiles (18 or 23). */
int32_t varuna_debug_wgrad_group_launch(int32_t n_layers, int64_t hidden, int64_t mlp, int64_t tokens);

/* ---- per-kernel timing (HIP events on the caller's stream) -------------- */

/* Kernel classes reported by the profiler. */
enum {
  VARUNA_K_GEMM_FWD = 0,  /* Y = X W^T (+bias, GeLU, residual) */
  VARUNA_K_GEMM_DGRAD,    /* dX = dY W (+GeLU') */
  VARUNA_K_GEMM_WGRAD,    /* dW += dY^T X */
  VARUNA_K_ATTN_FWD,
  VARUNA_K_ATTN_BWD,
  VARUNA_K_LN_FWD,
  VARUNA_K_LN_BWD,
  VARUNA_K_COLREDUCE,     /* bias / gamma / beta gradient reductions */
  VARUNA_K_OTHER,         /* copies, fills */
  VARUNA_K_COUNT
};
/* While enabled, each kernel launch is bracketed by HIP events on the stream it
 * runs on.  Events come from a fixed pool created here (no device memory).  Results are
 * bit-identical either way.  A launch that joins work of two classes counts for the one that
 * has its FLOPs (a small fp32 layer's norms are part of the products that follow them); the
 * last LayerNorm of a layer's backward and the column sums, otherwise one launch, are two. */
varuna_status_t varuna_stage_profile_enable(varuna_stage_t* st, int32_t on);
/* Synchronises the recorded events, adds their durations per class into
 * ms[VARUNA_K_COUNT], launches[...] and flops[...] (algorithmic FLOPs of the
 * launches, 0 for memory-bound classes) and bytes[...] (algorithmic HBM bytes),
 * then clears the record. */
varuna_status_t varuna_stage_profile_collect(varuna_stage_t* st, double* ms, int64_t* launches,
                                             double* flops, double* bytes);

/* ---- measurement hook: what the matrix cores sustain when fed from registers ----------
 * Launches compute_units * waves_per_simd workgroups of 4 waves (waves_per_simd = 1 or 2),
 * each wave issuing iters * 8 independent v_mfma_f32_32x32x16_bf16 products on operand
 * fragments it loaded once from `operands` (device, bf16, n_elems a multiple of 8, 16-byte
 * aligned; indices wrap) -- no LDS or memory traffic inside the loop.  pattern selects which
 * of its 4 + 4 fragments consecutive products read: 0 both operands change every product,
 * 1 the first is held for 8 products, 2 the first for 8 and the second for 2 (a 4x2 register
 * tile walked row by row), 3 both always the same, 4 / 5 as 0 with 4 / 2 consecutive products
 * adding to the same accumulator tile, 6 / 7 as 0 / 2 with two v_mfma_f32_16x16x32_bf16 in
 * place of every 32x32x16 product (the same operation count).  The caller times the
 * launch with events on hip_stream; *flops (host, may be NULL) receives the floating-point
 * operations of the launch.  sink: device, compute_units * waves_per_simd * 256 floats,
 * receives accumulator sums (so the products cannot be elided).  The rate depends on the
 * operand data (all-zero operands toggle no multiplier inputs and run at a higher clock
 * than normally distributed ones): it is the measured ceiling a GEMM on the same kind of
 * data sits under, reported beside the nominal peak. */
varuna_status_t varuna_probe_mfma_rate(const void* operands /*device*/, int64_t n_elems, int32_t waves_per_simd,
                                       int32_t pattern, int32_t iters, float* sink /*device*/,
                                       double* flops /*host*/, void* hip_stream);

/* ---- single-operation entry points (unit parity tests, kernel tuning) ---- */

/* C[M,N] = A * B^T style products on device buffers, dtype as varuna_dtype_t.
 * op: 0 forward  (a = X[M,K],  b = W[N,K],  out[M,N]  = X W^T + bias; epi selects
 *                 0 bias, 1 bias+GeLU (aux_out receives pre-GeLU u if not NULL),
 *                 2 bias+residual (aux_in = residual [M,N]))
 *     1 dgrad    (a = dY[M,K], b = W[K,N],  out[M,N]  = dY W; epi 0 plain,
 *                 3 multiply by GeLU'(aux_in[M,N]))
 *     2 wgrad    (a = dY[K,M], b = X[K,N],  out_f32[M,N] += dY^T X)
 * variant: 0 = library's choice; other values force one kernel configuration
 * (VARUNA_EUNSUPPORTED if it cannot run the shape). */
varuna_status_t varuna_op_gemm(int32_t dtype, int32_t op, int32_t epi, int32_t variant, int64_t M,
                               int64_t N, int64_t K, const void* a, const void* b,
                               const void* bias, const void* aux_in, void* out, void* aux_out,
                               void* hip_stream);

/* LayerNorm forward: y = gamma*(x-mean)*rstd+beta on [rows, h]; stats_f32
 * ([2*rows]: mean then rstd) may be NULL. */
varuna_status_t varuna_op_layernorm_fwd(int32_t dtype, int64_t rows, int64_t h, float eps,
                                        const void* x, const void* gamma, const void* beta,
                                        void* y, float* stats_f32, void* hip_stream);
/* LayerNorm backward: dx = res + LN'(dy); dgamma_f32, dbeta_f32 [h] are added to.
 * partial_f32 is scratch of at least varuna_op_colreduce_scratch_bytes(rows, 2*h). */
varuna_status_t varuna_op_layernorm_bwd(int32_t dtype, int64_t rows, int64_t h, const void* dy,
                                        const void* x, const float* stats_f32, const void* gamma,
                                        const void* res, void* dx, float* dgamma_f32,
                                        float* dbeta_f32, float* partial_f32, void* hip_stream);
/* out_f32[n] += sum over rows of a[rows, n]. */
varuna_status_t varuna_op_colsum(int32_t dtype, int64_t rows, int64_t n, const void* a,
                                 float* out_f32, float* partial_f32, void* hip_stream);
size_t varuna_op_colreduce_scratch_bytes(int64_t rows, int64_t n);

/* varuna_op_colsum for callers that cannot allocate device memory and have no workspace to
 * hand over (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): the stage-1 partial sums go to a device array built into the library
 * (varuna_op_colsum_static_max_bytes() = 4 MiB per GPU, held until the process ends), so the
 * call takes inputs and outputs only and calls no allocating routine.  Same kernels, same
 * result bit for bit as varuna_op_colsum.  Shapes whose partial sums
 * (varuna_op_colreduce_scratch_bytes(rows, n)) exceed the built-in array are rejected with
 * VARUNA_EUNSUPPORTED before anything is enqueued.  All calls on one GPU share that array:
 * calls whose kernels may overlap on the GPU (different streams, no ordering between them)
 * race; calls ordered on one stream do not.  The array's address is looked up once per
 * device at the first call on that device (the current device when the call is made). */
varuna_status_t varuna_op_colsum_static(int32_t dtype, int64_t rows, int64_t n, const void* a /*device*/,
                                        float* out_f32 /*device*/, void* hip_stream);
size_t varuna_op_colsum_static_max_bytes(void);

/* Attention forward on qkv [b*s, 3h] -> ctx [b*s, h], lse_f32 [b, heads, s].
 * variant: 0 = library's choice.  bf16: 1 = MFMA kernels on whole tiles (VARUNA_EUNSUPPORTED unless the head dim is
 * 64, 96 or 128 and s a multiple of 128), 2 = their form for any s and head dims that are multiples of 8 up to 128,
 * 3 = fp32 products (head dims up to 128), any other value, and 2 and 3 on other shapes = one wave per row.
 * fp32: -1 = one wave per row, any other value = fp32 products where they take the shape (head dims up to 128, else one wave per row): 4 = in tiles of 16
 * (head dims that are multiples of 4, 16-byte aligned tensors), 5, and 4 on other calls = in tiles of 32, the rest = in the tiles the library would choose. */
varuna_status_t varuna_op_attention_fwd(int32_t dtype, int32_t variant, int32_t b, int32_t s,
                                        int32_t heads, int32_t d, int32_t causal, const void* qkv,
                                        void* ctx, float* lse_f32, void* hip_stream);
/* Attention backward: dqkv [b*s, 3h] from dctx; delta_f32 [b, heads, s] scratch. */
varuna_status_t varuna_op_attention_bwd(int32_t dtype, int32_t variant, int32_t b, int32_t s,
                                        int32_t heads, int32_t d, int32_t causal, const void* qkv,
                                        const void* ctx, const float* lse_f32, const void* dctx,
                                        void* dqkv, float* delta_f32, void* hip_stream);

/* ---- the two ends of a pipeline, and the norm that joins its stages ----------------------
 * What the first and the last stage compute beside their layers, and the quantity that every
 * stage's gradients share (Enabling Ease of Programming, "Tracking cross-partition
 * dependencies": tied embeddings, overflow flag, global norm).  These calls take no handle and
 * keep nothing.  Tensors may begin at any element (those whose rows begin on 16 bytes are moved
 * in 16-byte pieces, the rest in smaller ones); scratch is 256-byte aligned, its contents are
 * undefined before and after, and calls whose kernels may overlap each need their own.  The
 * current device is hip_stream's.  No call reads an id on the host: an id outside its table
 * (-1, say) is no entry of it, which is how padding is marked. */

/* Embedding: out[t] = scale * table[ids[t]] + pos_table[position of t], computed in fp32 and
 * rounded once; scale is finite, out [rows, h], table [vocab, h], pos_table [n_positions, h] in
 * the same dtype.  pos_table NULL: no second term.  positions NULL: the position of row t is t mod seq_len
 * (1 <= seq_len <= n_positions), otherwise positions[t].  ids and positions are of type
 * `index`.  The term of an id or position outside its table is 0.  out overlaps no input. */
varuna_status_t varuna_op_embedding_fwd(int32_t dtype, int32_t index, int64_t rows, int64_t h, int64_t vocab,
                                        const void* ids /*device*/, const void* table /*device*/, float scale,
                                        int64_t seq_len, int64_t n_positions, const void* positions /*device*/,
                                        const void* pos_table /*device*/, void* out /*device*/, void* hip_stream);
/* Gradient of one table: dtable_f32[v] = scale * (sum of dy[t] over the rows t with ids[t] = v),
 * added to what is there if accumulate is 1 (rows of ids that do not occur are not touched), or
 * written, 0 for ids that do not occur, if it is 0.  ids NULL: the id of row t is t mod seq_len,
 * the gradient of a pos_table used with positions NULL (seq_len is not read otherwise).  Rows
 * are summed in an order that depends on the ids alone: the result is the same bit for bit from
 * call to call.  scratch: varuna_op_embedding_bwd_scratch_bytes(rows, h, vocab).  rows below
 * 2^31, vocab up to 2^30, h up to 2^20 (the forward call too). */
varuna_status_t varuna_op_embedding_bwd(int32_t dtype, int32_t index, int64_t rows, int64_t h, int64_t vocab,
                                        const void* ids /*device*/, int64_t seq_len, const void* dy /*device*/,
                                        float scale, int32_t accumulate, float* dtable_f32 /*device*/,
                                        void* scratch /*device*/, void* hip_stream);
size_t varuna_op_embedding_bwd_scratch_bytes(int64_t rows, int64_t h, int64_t vocab);

/* Cross entropy of logits [rows, vocab], whose rows lie ld elements apart, against targets
 * [rows] of type `index`, with label smoothing e in [0, 1]:
 *   loss_f32[r] = (1 - e) (lse - x[y]) + e (lse - mean of x),  lse = log sum exp x
 * and, unless dlogits is NULL, its gradient times g = grad_scale * scale[0] (scale: device, NULL
 * for 1 -- 1 / number of counted rows, or a loss scale, known on the device only):
 *   dlogits[r, j] = g (exp(x[j] - lse) - (1 - e) [j = y] - e / vocab)
 * rounded once; exp is off by up to about 3 (max x - x[j]) 2^-24 of itself and 0 where it is below
 * 2^-126.  dlogits has the dtype of the logits; it is the logits themselves (same ld) or
 * overlaps no input, from the first entry of either to the last; columns from vocab to its own
 * pitch ld_dlogits stay as they are.  A row whose target lies outside [0, vocab) has loss 0 and
 * gradient 0, whatever its logits hold.  Logits of -inf are entries that cannot occur: their
 * probability is 0; with e > 0 the loss is then +inf, as the formula says, and so is that of a
 * target of -inf.  A counted row that has a NaN or a +inf, or -inf only, has NaN throughout.
 * out2 (device, 2 floats, may be NULL): sum of the losses, number of counted rows.  rows up to
 * 2^24, vocab up to 2^30, pitches up to 2^31. */
varuna_status_t varuna_op_cross_entropy(int32_t dtype, int32_t index, int64_t rows, int64_t vocab, int64_t ld,
                                        const void* logits /*device*/, const void* targets /*device*/,
                                        float label_smoothing, float grad_scale, const float* scale /*device*/,
                                        float* loss_f32 /*device*/, int64_t ld_dlogits, void* dlogits /*device*/,
                                        float* out2 /*device*/, void* hip_stream);

/* Global gradient norm over n tensors: sum_sq[0] (device) = sum of squares of their finite
 * entries in 64 bits, nonfinite[0] (device) = number of the others (as a float: what
 * varuna_stage_adam_step takes as skip_if_nonzero).  dtypes, tensors, counts: host arrays of n
 * (varuna_dtype_t, device address, elements), read during the call; n and any count may be 0.
 * Deterministic.  Before the clip call the caller may sum both numbers over the stages.
 * scratch: varuna_op_grad_norm_scratch_bytes(n, counts). */
varuna_status_t varuna_op_grad_norm(int32_t n, const int32_t* dtypes /*host*/, const void* const* tensors /*host*/,
                                    const int64_t* counts /*host*/, double* sum_sq /*device*/,
                                    float* nonfinite /*device*/, void* scratch /*device*/, void* hip_stream);
size_t varuna_op_grad_norm_scratch_bytes(int32_t n, const int64_t* counts /*host*/);
/* Clipping: dst[i] = c * src[i] for n tensors, c = min(1, max_norm / (sqrt(sum_sq[0]) + eps)) in
 * 64 bits and rounded to fp32, the product rounded to dst's type.  A dst is its src (clipped in
 * place; left alone where c is 1) or overlaps no src, for instance its place in the buffer that
 * is exchanged.  Entries that are not finite stay what they are as long as c > 0.  max_norm and
 * eps >= 0; max_norm may be infinite (no clipping).  A sum_sq of NaN clips nothing. */
varuna_status_t varuna_op_grad_clip(int32_t n, const int32_t* dst_dtypes /*host*/, void* const* dst /*host*/,
                                    const int32_t* src_dtypes /*host*/, const void* const* src /*host*/,
                                    const int64_t* counts /*host*/, const double* sum_sq /*device*/,
                                    double max_norm, double eps, void* hip_stream);

/* ---- rotary positions, norms on both sides of a block, AdamW over many tensors --------------
 * What a layer of that form needs beside varuna_op_gemm and varuna_op_attention_*, and one update
 * of all tensors that varuna_op_grad_norm has measured.  As the calls above these take no handle,
 * keep nothing, read no tensor on the host, launch kernels only (all can be captured into a graph),
 * use no floating-point atomics, and take tensors that begin at any element. */

/* Frequencies of rotary positions: frequencies[i] = base^(-2i / rotary_dim) for the rotary_dim / 2
 * pairs, stretched by factor >= 1 for contexts longer than the one trained on:
 *   PLAIN   as they are (factor is not read)
 *   LINEAR  divided by factor
 *   BASE    of the base times factor^(rotary_dim / (rotary_dim - 2)): the slowest by factor, the
 *           fastest not at all (rotary_dim >= 4)
 *   PARTS   by how many turns a pair makes within original_length positions: high_turns and more
 *           as it is, low_turns and fewer divided by factor, between them the mean of both weighted
 *           by the place between (0 <= low_turns < high_turns)
 * Host only.  rotary_dim: even, 2 to 512; base > 0. */
typedef enum { VARUNA_ROTARY_PLAIN = 0, VARUNA_ROTARY_LINEAR = 1, VARUNA_ROTARY_BASE = 2, VARUNA_ROTARY_PARTS = 3 } varuna_rotary_scaling_t;
varuna_status_t varuna_rotary_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor,
                                          double original_length, double low_turns, double high_turns,
                                          double* frequencies /*host, rotary_dim / 2*/);
/* table [n_positions, rotary_dim] fp32: of position p first magnitude * cos(p f_i), then
 * magnitude * sin(p f_i) for the rotary_dim / 2 finite frequencies (host, read during the call).
 * Angles in 64 bits, each value rounded once.  Made once and kept by the caller.  n_positions up to
 * 2^30. */
varuna_status_t varuna_op_rotary_table(int64_t n_positions, int32_t rotary_dim, const double* frequencies /*host*/,
                                       double magnitude, float* table /*device*/, void* hip_stream);
/* Turns the first rotary_dim of the d entries of every head of x [rows, heads, d] by its row's
 * position: pair (a, b) becomes (a cos - b sin, a sin + b cos), computed in fp32 and rounded once;
 * transpose 1: (a cos + b sin, b cos - a sin), the gradient.  Pairs are the entries i and
 * i + rotary_dim / 2, or with interleaved 1 the entries 2i and 2i + 1.  positions NULL: the position
 * of row t is t mod seq_len (1 <= seq_len <= n_positions), otherwise positions[t] of type `index`;
 * a row whose position lies outside [0, n_positions) stays as it is (n_positions at least 1).  Strides in elements: row t,
 * head k begins at x + t * x_row + k * x_head, its entries side by side, so that the query and key
 * heads of the packed qkv of varuna_op_attention_fwd are 2 * heads of one call (x_row 3h, x_head d).
 * out is x with its strides (in place: entries behind rotary_dim are not touched), or another
 * tensor (they are copied), no part of which lies between x's first entry and its last; its heads must not overlap: out_head >= d and
 * out_row over all heads of a row, or out_row >= d and out_head over all rows of a head.  rows, and
 * rows * heads, below 2^31, d up to 65536. */
varuna_status_t varuna_op_rotary(int32_t dtype, int32_t index, int32_t interleaved, int32_t transpose, int64_t rows, int64_t heads,
                                 int64_t d, int32_t rotary_dim, const void* x /*device*/, int64_t x_row, int64_t x_head,
                                 void* out /*device*/, int64_t out_row, int64_t out_head, const void* positions /*device*/,
                                 int64_t seq_len, int64_t n_positions, const float* table /*device*/, void* hip_stream);

typedef enum { VARUNA_NORM_RMS = 0, VARUNA_NORM_LAYER = 1 } varuna_norm_t;
typedef struct {
  int32_t dtype, kind;    /* varuna_dtype_t of all tensors but statistics and parameter gradients; varuna_norm_t of both norms */
  int64_t rows, h;        /* h up to 16384, rows up to 2^30 */
  int64_t rows_per_gate;  /* row t has row t / rows_per_gate of the gate; not read without one */
  float alpha, beta, eps; /* finite, eps >= 0 */
} varuna_residual_norm_t;
/* What joins a block to the residual stream and feeds the next one, rows of h entries:
 *   u = Npost(branch) (branch itself where post_weight is NULL)
 *   y = alpha * x + beta * gate * u (gate NULL: 1), rounded once
 *   z = Npre(y), y as it is stored; NULL with weight NULL: no norm behind
 * N(v) = (v - mean) * rstd * weight + bias in fp32, rstd = 1 / sqrt(mean of (v - mean)^2 + eps),
 * VARUNA_NORM_RMS: mean is 0; a bias may be NULL.  branch NULL: z = Npre(x), with gate, post_weight,
 * post_bias and y NULL too (alpha and beta are not read).  y may be NULL where z is not.  stats and
 * post_stats (fp32 [2*rows]: mean, then rstd; may be NULL) are what the backward call needs.  y and z may each be x
 * or branch itself; otherwise no output overlaps another tensor. */
varuna_status_t varuna_op_residual_norm_fwd(const varuna_residual_norm_t* n, const void* x /*device*/, const void* branch /*device*/,
                                            const void* post_weight /*device*/, const void* post_bias /*device*/,
                                            const void* gate /*device, [rows / rows_per_gate rounded up, h]*/, const void* weight /*device*/,
                                            const void* bias /*device*/, void* y /*device*/, void* z /*device*/, float* post_stats /*device*/,
                                            float* stats /*device*/, void* hip_stream);
/* Its backward: from dz (gradient of z) and dy (what reaches y from behind; NULL: 0), with y the stored one (x where there was no branch)
 *   d = dy + gradient of Npre at y (dy alone where weight is NULL; then dz, y and stats are NULL)
 *   dx = alpha * d, dbranch = gradient of beta * gate * Npost(branch) under d
 *   dx = d where branch and dbranch are both NULL: the gradient of z = Npre(x), alpha and beta are not read.  A branch that was
 *   there and whose gradient is not wanted (dbranch NULL; there is no post norm or gate then) is given for dx to have its alpha
 * each rounded once, and in fp32 dweight, dbias, dpost_weight, dpost_bias [h] and dgate (like gate), any of which
 * may be NULL: added to if accumulate is 1, written if it is 0.  Sums over rows are made in an order that depends on the
 * sizes alone.  What branch holds is read only for a post norm or a gate, and dbranch has to be given with these.  post_bias: read for dgate
 * only.  dx may be dz or dy itself, dbranch may be branch, or dz or dy where dx is not; otherwise no
 * output overlaps another tensor.  scratch: varuna_op_residual_norm_bwd_scratch_bytes(rows, h, rows_per_gate (0 without a gate)), 256-byte aligned (a smaller one is
 * written beyond: the call does not see its size); no rows need none.
 * Gates of more than 16 rows: fewer than 2^22 of them (VARUNA_EUNSUPPORTED, and a size of 0, as for all that the call does not take). */
varuna_status_t varuna_op_residual_norm_bwd(const varuna_residual_norm_t* n, const void* dz /*device*/, const void* dy /*device*/,
                                            const void* y /*device*/, const void* branch /*device*/, const void* post_weight /*device*/,
                                            const void* post_bias /*device*/, const void* gate /*device*/, const void* weight /*device*/,
                                            const float* post_stats /*device*/, const float* stats /*device*/, void* dx /*device*/,
                                            void* dbranch /*device*/, float* dweight /*device*/, float* dbias /*device*/,
                                            float* dpost_weight /*device*/, float* dpost_bias /*device*/, float* dgate /*device*/,
                                            int32_t accumulate, void* scratch /*device*/, void* hip_stream);
size_t varuna_op_residual_norm_bwd_scratch_bytes(int64_t rows, int64_t h, int64_t rows_per_gate);

typedef struct {
  double lr, beta1, beta2, eps, weight_decay; /* betas in [0, 1) */
  double grad_scale;                          /* multiplies every gradient (1/loss scale, 1/M); finite */
  double max_norm, clip_eps;                  /* read with sum_sq only; >= 0, max_norm may be infinite */
  int64_t step;                               /* number of this update, 1 to 2^40 */
  int32_t bits;                               /* of a moment: 32 or 8 */
} varuna_adamw_t;
/* One AdamW update of n tensors, entry by entry in fp32:
 *   g = c * gradient;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
 *   w -= lr * (m / (1 - b1^step) / (sqrt(v / (1 - b2^step)) + eps) + weight_decay * decays[i] * w)
 * An fp32 parameter is w itself; a bf16 one is w rounded, w lying in master.  c = grad_scale, and with
 * sum_sq (device, of varuna_op_grad_norm over these gradients as they are) c = grad_scale * min(1, max_norm / (|grad_scale| sqrt(sum_sq[0]) + clip_eps)) in
 * 64 bits, rounded to fp32; a sum_sq of NaN clips nothing.  skip_if_nonzero (device, may be NULL) as in varuna_stage_adam_step.
 * lr_step (device, 2 doubles, may be NULL): learning rate and step number read on the GPU in the place of lr and step, for a call in a captured
 * graph.  decays (host, may be NULL for 1): factor of each tensor's weight decay.  State: one buffer each of master (fp32; may be NULL if no parameter is
 * bf16), m and v for all tensors, in which tensor i has its counts[i] entries from the end of tensor
 * i-1's on, rounded up to a multiple of 256: varuna_op_adamw_state_entries(n, counts) entries, up to 2^33.  bits 32: m
 * and v are fp32, scales NULL.  bits 8: m and v are e4m3 codes (1 sign, 4 exponent, 3 mantissa bits, no infinities) and scales holds two floats for
 * every 256 entries of the state, powers of two s, s': m = s * code, v = (s' * code)^2.  s = 2^(e-7), e the exponent
 * of the largest finite |m| of the block's entries, at least -119 (s': of sqrt(v)).  A value between two codes becomes the upper one where its
 * distance from the lower, as a share of both codes' distance (v's: of the squares), is above u = frac(i a + step b), i being the entry's place in
 * the state, a = 0xC13FA9A9 / 2^32, b = 0x91E10DA5 / 2^32 (v's: a and b swapped), of which the upper 24 binary digits count; v > 0 becomes the smallest
 * code at least.  A moment that is not finite has the code NaN and no part in its block's scale.  A gradient whose square is beyond fp32
 * makes v infinite, which leaves its entry the decay alone (bits 8: NaN from the next update on).  All zeros is the state before the first step.  State buffers are 16-byte
 * aligned; entries of the state between tensors are not written (scales are).  Parameters and state overlap no tensor. */
varuna_status_t varuna_op_adamw(const varuna_adamw_t* hp, int32_t n, const int32_t* param_dtypes /*host*/, void* const* params /*host*/,
                                const int32_t* grad_dtypes /*host*/, const void* const* grads /*host*/, const int64_t* counts /*host*/,
                                const float* decays /*host*/, float* master /*device*/, void* m /*device*/, void* v /*device*/,
                                float* scales /*device*/, const double* sum_sq /*device*/, const float* skip_if_nonzero /*device*/,
                                const double* lr_step /*device*/, void* hip_stream);
int64_t varuna_op_adamw_state_entries(int32_t n, const int64_t* counts /*host*/); /* -1: invalid */

#ifdef __cplusplus
}
#endif
#endif /* VARUNA_STAGE_H */
