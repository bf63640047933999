/*
 * zoqat.h - C ABI of libzoqat: the forward-only, two-point zeroth-order
 * quantisation-aware training step of ZeroQAT on one NVIDIA B200 (sm_100a).
 *
 * One step (Section 4.1 of the paper):
 *   Eq. (1)  g = [ L(Q(W + eps u); B) - L(Q(W - eps u); B) ] / (2 eps),  u ~ N(0, I), q = 1
 *   Eq. (2)  W <- W - lr * g * u
 * Q is the uniform quantiser of Section 2 (asymmetric, one step size and zero
 * point per group of consecutive input channels for weights; symmetric 8-bit,
 * one step size per token for the inputs of the block linears).  Full-precision
 * masters are kept and only their quantised counterparts enter the forward
 * pass.  The direction u is never stored: element i of tensor t under a 64-bit
 * seed is regenerated from a Philox4x32-10 counter (block i/4, tensor id t)
 * wherever it is needed (both passes and the update).  The lightweight variant
 * of Section 4.3 keeps frozen tensors as packed low-bit codes.
 *
 * Conventions
 *   - Every function returns an int status: ZOQAT_OK (0) or a negative error.
 *     Nothing throws; zoqat_status_string() names a status and
 *     zoqat_last_error() returns the text of the last failure on the calling
 *     thread (arguments are validated on the host before any launch).
 *   - "dev" pointers are device (global) memory of the current CUDA device,
 *     "host" pointers are host memory.  The caller owns all device memory:
 *     masters, packed buffers, workspace, inputs and outputs.  The library owns
 *     only the host-side handle.
 *   - `stream` is a cudaStream_t passed as void* (NULL = default stream).
 *     Calls are asynchronous with respect to the host unless stated otherwise.
 *     One handle may be used from one stream at a time.
 *   - Matrices are row-major; a linear weight is [out_features, in_features]
 *     with quantisation groups contiguous along in_features.
 *   - Device-side waits are bounded; a wait that runs out writes a non-zero
 *     word to the handle's error flag, which zoqat_check() reads.  No kernel
 *     traps the GPU.
 */
#ifndef ZOQAT_H
#define ZOQAT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------- */
#define ZOQAT_OK                     0
#define ZOQAT_ERR_INVALID_ARG       -1
#define ZOQAT_ERR_UNSUPPORTED       -2
#define ZOQAT_ERR_WORKSPACE_SMALL   -3
#define ZOQAT_ERR_CUDA              -4
#define ZOQAT_ERR_BAD_STATE         -5
#define ZOQAT_ERR_TIMEOUT           -6

/* ---- model description --------------------------------------------------- */
#define ZOQAT_ARCH_LLAMA 0   /* RMSNorm, rotary positions, SiLU-gated FFN, no biases   */
#define ZOQAT_ARCH_OPT   1   /* LayerNorm, learned positions, ReLU FFN, linear biases  */

/* Tensor roles.  The first seven are the block linears; their Philox tensor id
 * is 16*(layer+1) + role.  The vocabulary projection has tensor id 0. */
#define ZOQAT_ROLE_WQ            0
#define ZOQAT_ROLE_WK            1
#define ZOQAT_ROLE_WV            2
#define ZOQAT_ROLE_WO            3
#define ZOQAT_ROLE_W_GATE        4   /* OPT: fc1 */
#define ZOQAT_ROLE_W_UP          5   /* LLaMA only */
#define ZOQAT_ROLE_W_DOWN        6   /* OPT: fc2 */
#define ZOQAT_ROLE_ATTN_NORM_G   7
#define ZOQAT_ROLE_ATTN_NORM_B   8   /* OPT only */
#define ZOQAT_ROLE_FFN_NORM_G    9
#define ZOQAT_ROLE_FFN_NORM_B   10   /* OPT only */
#define ZOQAT_ROLE_BQ           11   /* OPT only: biases */
#define ZOQAT_ROLE_BK           12
#define ZOQAT_ROLE_BV           13
#define ZOQAT_ROLE_BO           14
#define ZOQAT_ROLE_B_FC1        15
#define ZOQAT_ROLE_B_FC2        16
#define ZOQAT_ROLE_EMBED        17   /* layer = -1 from here on */
#define ZOQAT_ROLE_POS_EMBED    18   /* OPT only */
#define ZOQAT_ROLE_FINAL_NORM_G 19
#define ZOQAT_ROLE_FINAL_NORM_B 20   /* OPT only */
#define ZOQAT_ROLE_LM_HEAD      21
/* Section 4.2, adaptive outlier smoothing: per-input-channel scale s and shift delta at the four quantised
 * inputs of a layer's linears (point 0: input of q/k/v, 1: input of the output projection, 2: input of
 * gate/up (fc1), 3: input of down (fc2)); fp32 vectors of d_model (d_ffn for point 3) elements, layer >= 0.
 * Role = base + point.  A layer has either all eight or none; with them every block linear of the layer must
 * be TRAINABLE.  They are perturbed and updated like the weights: Philox tensor ids
 * 0x20000 + 16*(layer+1) + point (scale) and 0x30000 + 16*(layer+1) + point (shift). */
#define ZOQAT_ROLE_SMOOTH_SCALE 22   /* .. 25 */
#define ZOQAT_ROLE_SMOOTH_SHIFT 26   /* .. 29 */
#define ZOQAT_ROLE_COUNT        30

/* Tensor flags (linear weights only; every other tensor is frozen fp32). */
#define ZOQAT_TENSOR_TRAINABLE      1u  /* perturbed by +/- eps u in the forward, updated by Eq. (2) */
#define ZOQAT_TENSOR_QUANTIZED      2u  /* forward sees the per-group fake-quantised weight         */
#define ZOQAT_TENSOR_FROZEN_PACKED  4u  /* Section 4.3: forward reads packed codes + (step, zero point) written by
                                           zoqat_prequantize_frozen(); never perturbed, never updated */
#define ZOQAT_TENSOR_ADAPTIVE       8u  /* Section 4.2 adaptive weight quantiser (with TRAINABLE | QUANTIZED): `qparams` holds
                                           one learnable (step, zero point, alpha, beta) per group, code =
                                           clamp(round(w/step) + z, alpha*Q_P, beta*Q_P); perturbed and updated like
                                           the weights under Philox tensor id 0x10000 + the weight's id, element
                                           4*group + {0,1,2,3}.  Codes stay integers in [0, Q_P]: z and the two levels
                                           enter rounded to nearest even, the levels limited to [0, Q_P], upper >= lower */

#define ZOQAT_GEMM_TCGEN05 0   /* tcgen05/TMEM tensor-core kernels (default); GEMM tiles of 256 rows are computed by a
                                  pair of CTAs on two SMs with one cta_group::2 MMA                                  */
#define ZOQAT_GEMM_SIMT    1   /* plain CUDA-core kernels, kept as an on-device cross-check                          */
#define ZOQAT_GEMM_TCGEN05_1CTA 2 /* as 0, but every GEMM tile (128 rows) belongs to a single CTA                    */
#define ZOQAT_GEMM_TCGEN05_I8  3  /* as 0, with every block linear evaluated on integers (appendix on quantisation
                                     settings: one weight scale per output channel, one activation scale per token):
                                       y[t, n] = s_t * (Delta_n * sum_k a[t, k] * (c[n, k] - z_n)) (+ bias),
                                     the sum exact (tcgen05.mma kind::i8 on signed bytes, 32-bit accumulators), which
                                     is Q(x) Q(w)^T of Section 2 with no rounding of the operands; ZOQAT_GEMM_TCGEN05
                                     instead rounds the dequantised weight (c - z) * Delta to bf16.  Needs w_group = 0,
                                     a_bits != 0, w_bits <= 7, every block linear QUANTIZED or FROZEN_PACKED (packed
                                     tensors expand straight into byte operands: no per-step work on their weights
                                     beyond that); the vocabulary projection stays bf16.  A weight row whose c - z leaves [-128, 127]
                                     (zero point far outside the code range) makes the step report status 32 and
                                     zoqat_check() return ZOQAT_ERR_UNSUPPORTED; results of that call are not usable. */

typedef struct zoqat_config {
    int32_t arch;          /* ZOQAT_ARCH_*                                                        */
    int32_t n_layers;
    int32_t d_model;       /* multiple of 64                                                      */
    int32_t n_heads;       /* d_model / n_heads in {32, 64, 128}                                  */
    int32_t d_ffn;         /* multiple of 64                                                      */
    int32_t vocab;
    int32_t max_batch;     /* largest batch ...                                                   */
    int32_t max_seq;       /* ... and sequence length a call will pass                            */
    int32_t w_bits;        /* 2..8 (FROZEN_PACKED tensors: 2, 3 or 4)                             */
    int32_t w_group;       /* 32, 64 or 128 (divides d_model and d_ffn), or 0 = one group per output
                              row ("per-channel" weights; d_model, d_ffn multiples of 128; FROZEN_PACKED
                              tensors then carry one (step, zero point) per row; not in decode)   */
    int32_t a_bits;        /* 4, 6 or 8 = per-token symmetric N-bit codes on block-linear inputs, 0 = none */
    int32_t gemm_impl;     /* ZOQAT_GEMM_*                                                        */
    float   norm_eps;
    float   rope_base;     /* LLaMA only                                                          */
} zoqat_config_t;

typedef struct zoqat_tensor_desc {
    int32_t role;          /* ZOQAT_ROLE_*                                                        */
    int32_t layer;         /* 0..n_layers-1, or -1 for model-level tensors                        */
    uint32_t flags;        /* ZOQAT_TENSOR_* (linear weights)                                     */
    uint32_t reserved;
    void*   data;          /* dev: fp32 values.  For FROZEN_PACKED tensors it is read only by
                              zoqat_prequantize_frozen() and may be freed afterwards.            */
    void*   packed;        /* dev: FROZEN_PACKED only, zoqat_packed_bytes() code bytes             */
    void*   qparams;       /* dev: FROZEN_PACKED: one (float step, float zero point) pair per group;
                              ADAPTIVE: four floats (step, zero point, alpha, beta) per group, 16-byte aligned,
                              updated in place (zoqat_init_qparams() writes the initial values)         */
} zoqat_tensor_desc_t;

typedef struct zoqat_step_result {
    float   loss_plus;     /* L(Q(W + eps u); B)                                                  */
    float   loss_minus;    /* L(Q(W - eps u); B)                                                  */
    float   proj_grad;     /* g of Eq. (1), formed in double precision and rounded                 */
    float   update_scale;  /* lr * g, the factor the update multiplies u by                        */
    int32_t status;        /* 0, or the device error word                                         */
    int32_t n_labels;      /* labelled positions per pass                                         */
} zoqat_step_result_t;

typedef struct zoqat_model zoqat_model_t;

/* ---- the step (Section 4.1, Section 4.3) ---------------------------------- */

/* Bytes of device workspace zoqat_model_create() needs for `cfg` (host only). */
int zoqat_query_workspace(const zoqat_config_t* cfg, size_t* bytes);

/* Sizes of the packed representation of one [rows, cols] tensor: `code_bytes` of
 * codes (rows * cols * bits / 8, rows padded to nothing: cols*bits must be a
 * multiple of 8) and `qparam_bytes` = rows * cols/group * 8. */
int zoqat_packed_bytes(int64_t rows, int64_t cols, int bits, int group,
                       size_t* code_bytes, size_t* qparam_bytes);

/* Builds a handle.  `tensors[0..n)` must name every tensor the architecture has
 * (each role once per layer).  `workspace_dev` (256-byte aligned, `bytes` >=
 * the queried size) is used by every later call on the handle.  Masters flagged
 * TRAINABLE are updated in place by zoqat_step()/zoqat_apply_update(). */
int zoqat_model_create(const zoqat_config_t* cfg, const zoqat_tensor_desc_t* tensors, int n_tensors,
                       void* workspace_dev, size_t bytes, zoqat_model_t** out);
int zoqat_model_destroy(zoqat_model_t* m);

/* Section 4.3: quantises every FROZEN_PACKED tensor from its unperturbed fp32
 * values into `packed` / `qparams`.  Idempotent.  Must run before the first
 * forward when such tensors exist. */
int zoqat_prequantize_frozen(zoqat_model_t* m, void* stream);

/* Optional, after zoqat_prequantize_frozen: expands every FROZEN_PACKED tensor once into the operand the GEMM reads - the
 * bf16 values (code - zero point) * step, or with ZOQAT_GEMM_TCGEN05_I8 the signed bytes code - zero point and the rows'
 * steps - inside `buffer_dev` (caller-owned, 256-byte aligned, zoqat_expand_frozen_bytes() bytes: two bytes per block-linear
 * weight, or one plus four per output row; in use until the handle is destroyed or the call is repeated; buffer_dev = NULL
 * returns to decoding the packed codes on every step).  Afterwards a linear layer whose tensors are all frozen reads them in
 * place, both passes as one product, and a frozen tensor that shares a GEMM with trainable ones (a frozen key projection
 * next to trainable query / value projections) is copied instead of decoded: Section 4.3's frozen tensors then cost no
 * arithmetic per step, at the price of the memory the packed form saves.  Results are bit-identical either way.  With byte
 * operands a row that does not fit a signed byte is reported through zoqat_check() (status 32). */
int zoqat_expand_frozen_bytes(const zoqat_model_t* m, size_t* bytes);
int zoqat_expand_frozen(zoqat_model_t* m, void* buffer_dev, size_t bytes, void* stream);

/* Section 4.2: writes the initial quantiser parameters of every ADAPTIVE tensor - step and zero point of the
 * default min/max scheme on the current (unperturbed) weights, alpha = 0, beta = 1 - at which the adaptive
 * quantiser reproduces the min/max quantiser exactly.  (Smoothing vectors are the caller's to initialise:
 * scale 1 and shift 0 leave the model unchanged.) */
int zoqat_init_qparams(zoqat_model_t* m, void* stream);

/* One forward pass: *loss_out_dev = L(Q(W + signed_eps u(seed)); B), the mean
 * next-token cross-entropy over positions whose label is >= 0 (Eq. (1) argument).
 * signed_eps = 0 gives the unperturbed quantised model.  tokens_dev / labels_dev:
 * int32 [batch, seq] on the device.  Masters are not modified. */
int zoqat_forward_loss(zoqat_model_t* m, const int32_t* tokens_dev, const int32_t* labels_dev,
                       int batch, int seq, uint64_t seed, float signed_eps,
                       float* loss_out_dev, void* stream);

/* One ZO-QAT step: both passes of Eq. (1) (evaluated side by side so that each
 * master and each direction is produced once for the pair), g, and the update
 * of Eq. (2) with the regenerated direction.  No host synchronisation.
 * `result_dev` (device memory) receives the scalars. */
int zoqat_step(zoqat_model_t* m, const int32_t* tokens_dev, const int32_t* labels_dev,
               int batch, int seq, uint64_t seed, float eps, float lr,
               zoqat_step_result_t* result_dev, void* stream);

/* zoqat_step with one learning rate per parameter class (hyperparameter table of the appendix: the weights, the
 * quantiser parameters of ADAPTIVE tensors - its "clipping" rate -, the smoothing vectors).  All classes share the
 * one g of Eq. (1); class c moves by -fl(lr_c * g) u.  zoqat_step(lr) is zoqat_step_rates(lr, lr, lr). */
int zoqat_step_rates(zoqat_model_t* m, const int32_t* tokens_dev, const int32_t* labels_dev,
                     int batch, int seq, uint64_t seed, float eps, float lr, float lr_quant, float lr_smooth,
                     zoqat_step_result_t* result_dev, void* stream);

/* zoqat_step with Eq. (2) deferred: the call returns after both passes and g, and the update W <- W - lr g u is
 * applied by the NEXT zoqat_step_deferred while its operand producers read the masters anyway (one pass over every
 * trainable tensor per step instead of two), or by zoqat_flush_update().  The masters then lag one update behind the
 * returned result until that happens; every other entry point that reads or changes them (zoqat_forward_loss,
 * zoqat_step*, zoqat_apply_update*, zoqat_init_qparams) flushes first, and a caller that reads the master tensors
 * itself calls zoqat_flush_update() before (zoqat_model_destroy() does not: a pending update is dropped with the handle).
 * Same arithmetic, same bits as zoqat_step.  Only the weights wait: the Section 4.2 parameters (quantiser parameters,
 * smoothing vectors) are small and move at once, with their own rates in the _rates form (Appendix hyperparameter
 * table).  With one weight group per output row the pending update is applied by the pass that finds the rows'
 * minima and maxima. */
int zoqat_step_deferred(zoqat_model_t* m, const int32_t* tokens_dev, const int32_t* labels_dev,
                        int batch, int seq, uint64_t seed, float eps, float lr,
                        zoqat_step_result_t* result_dev, void* stream);
int zoqat_step_rates_deferred(zoqat_model_t* m, const int32_t* tokens_dev, const int32_t* labels_dev,
                              int batch, int seq, uint64_t seed, float eps, float lr, float lr_quant, float lr_smooth,
                              zoqat_step_result_t* result_dev, void* stream);
int zoqat_flush_update(zoqat_model_t* m, void* stream);
/* The deferred form of zoqat_step_finish for replicas: forms g from the global sums and leaves Eq. (2) to the next
 * zoqat_step_begin (whose producers apply it) or to zoqat_flush_update(). */
int zoqat_step_finish_deferred(zoqat_model_t* m, const double* sums_dev, uint64_t seed, float eps, float lr,
                               zoqat_step_result_t* result_dev, void* stream);
int zoqat_step_finish_rates_deferred(zoqat_model_t* m, const double* sums_dev, uint64_t seed, float eps, float lr,
                                     float lr_quant, float lr_smooth, zoqat_step_result_t* result_dev, void* stream);

/* Eq. (1) with q = n_dirs directions per step (the paper's estimator averages over q directions u_1..u_q; it never
 * states q): direction i uses seed + i, every g_i is the two-point estimate at the SAME weights, and Eq. (2) then
 * applies W <- W - (lr / q) sum_i g_i u_i, direction by direction in one pass over each trainable tensor.
 * results_dev: n_dirs records (device memory); record i holds L+, L-, g_i and its update factor fl((lr/q) g_i).
 * n_dirs = 1 is zoqat_step.  2 * n_dirs forward passes. */
int zoqat_step_multi(zoqat_model_t* m, const int32_t* tokens_dev, const int32_t* labels_dev,
                     int batch, int seq, uint64_t seed, int n_dirs, float eps, float lr,
                     zoqat_step_result_t* results_dev, void* stream);

/* The step in two halves, for data-parallel replicas that each hold all masters and a
 * shard of the mini-batch (the loss of Eq. (1) is a mean over the mini-batch):
 * zoqat_step_begin runs both passes on the local shard and writes
 * sums_dev = (sum of per-position losses at +eps, the same at -eps, labelled positions)
 * as three doubles; the caller sums sums_dev over replicas (one all-reduce of 24 bytes);
 * zoqat_step_finish forms g from the global sums and applies Eq. (2), so every replica
 * makes the same update and masters stay identical without any weight traffic.
 * zoqat_step is begin + finish on one device. */
int zoqat_step_begin(zoqat_model_t* m, const int32_t* tokens_dev, const int32_t* labels_dev,
                     int batch, int seq, uint64_t seed, float eps, double* sums_dev, void* stream);
int zoqat_step_finish(zoqat_model_t* m, const double* sums_dev, uint64_t seed, float eps, float lr,
                      zoqat_step_result_t* result_dev, void* stream);
int zoqat_step_finish_rates(zoqat_model_t* m, const double* sums_dev, uint64_t seed, float eps, float lr,
                            float lr_quant, float lr_smooth, zoqat_step_result_t* result_dev, void* stream);

/* Same step with HOST inputs and outputs: copies tokens/labels to the device,
 * runs zoqat_step, copies the result back and synchronises the stream. */
int zoqat_step_host(zoqat_model_t* m, const int32_t* tokens_host, const int32_t* labels_host,
                    int batch, int seq, uint64_t seed, float eps, float lr,
                    zoqat_step_result_t* result_host, void* stream);

/* zoqat_step_host around zoqat_step_deferred: the result is back on the host when the call returns, the update of
 * the masters rides on the next step (or zoqat_flush_update()). */
int zoqat_step_host_deferred(zoqat_model_t* m, const int32_t* tokens_host, const int32_t* labels_host,
                             int batch, int seq, uint64_t seed, float eps, float lr,
                             zoqat_step_result_t* result_host, void* stream);

/* Eq. (2) alone: W <- W - scale * u(seed) on every TRAINABLE tensor (and on the Section 4.2 parameters);
 * the _rates form takes one factor per parameter class. */
int zoqat_apply_update(zoqat_model_t* m, uint64_t seed, float scale, void* stream);

/* Eq. (2) for q = n_dirs directions with caller-supplied seeds and factors (Eq. (1) averages over q directions;
 * Appendix G, Proposition 1 (ii): the estimator's error falls like 1/q): W <- W - sum_i scales[i] * u(seeds[i]),
 * applied direction by direction (i = 0, 1, ...: one binary32 fma per element each) in ONE pass over every TRAINABLE
 * tensor and over the Section 4.2 parameters, every class with the same factor.  It is the update half of
 * zoqat_step_multi, for callers that evaluated the directions elsewhere - e.g. q replicas that each ran both passes
 * of one direction on the same batch and exchanged (seed_i, fl((lr/q) g_i)): every replica then applies all q updates
 * and the masters stay bit-identical.  seeds_host: host memory, read before the call returns; scales_dev: device
 * memory, fp32 [n_dirs], read when the kernels run; 1 <= n_dirs <= 64.  A pending deferred update is applied first. */
int zoqat_apply_update_multi(zoqat_model_t* m, const uint64_t* seeds_host, const float* scales_dev, int n_dirs, void* stream);

/* Eq. (1) alone, from the sums zoqat_step_begin produced (all-reduced or not): fills the result record - L+, L-,
 * g = (L+ - L-) / (2 eps), fl(lr * g) - and leaves every master untouched.  With zoqat_apply_update_multi it lets a
 * caller separate the evaluation of a direction from the update (pass lr / q as lr for q directions). */
int zoqat_step_result(zoqat_model_t* m, const double* sums_dev, float eps, float lr, zoqat_step_result_t* result_dev, void* stream);
int zoqat_apply_update_rates(zoqat_model_t* m, uint64_t seed, float scale, float scale_quant, float scale_smooth,
                             void* stream);

/* Synchronises `stream` and returns ZOQAT_OK, ZOQAT_ERR_TIMEOUT if a bounded
 * device wait ran out since the last check, or ZOQAT_ERR_CUDA. */
int zoqat_check(zoqat_model_t* m, void* stream);

/* Number of kernel launches the handle has issued so far. */
int zoqat_launch_count(const zoqat_model_t* m, int64_t* launches);

/* Optional device-side timing by category.  While enabled (on = 1: every category; on = 2: only
 * ZOQAT_PROF_GEMM, a sixth of the event pairs), the launch groups of a forward/step are bracketed by CUDA
 * event pairs on the caller's stream (about 1 % of a 7B step with on = 1);
 * zoqat_profile_read() synchronises `stream`, returns the milliseconds and the number
 * of bracketed intervals accumulated for `category` since its last read, and clears them. */
#define ZOQAT_PROF_GEMM       0   /* linear layers and the fused vocabulary projection / cross-entropy */
#define ZOQAT_PROF_WEIGHT     1   /* perturb + quantise weight operands (and unpacking of frozen codes) */
#define ZOQAT_PROF_ACT        2   /* embedding, norms, activation quantisers, FFN non-linearity         */
#define ZOQAT_PROF_ATTENTION  3
#define ZOQAT_PROF_LOSS       4   /* cross-entropy finalisation                                         */
#define ZOQAT_PROF_UPDATE     5   /* Eq. (2)                                                            */
#define ZOQAT_PROF_COUNT      6
int zoqat_profile_enable(zoqat_model_t* m, int on);
int zoqat_profile_read(zoqat_model_t* m, int category, double* ms, int64_t* intervals, void* stream);

/* Device pointer and size of a workspace buffer holding intermediates of the
 * most recent forward (last layer executed).  Parity hook. */
#define ZOQAT_BUF_RESIDUAL   0   /* fp32 [passes*T, d_model]   residual stream after the last layer */
#define ZOQAT_BUF_QKV        1   /* fp32 [passes*T, 3*d_model] q | k | v of the last layer (before RoPE); only written when
                                    the projection's epilogue does not feed the attention kernel directly (CUDA-core or
                                    single-CTA GEMM, d_model % 256 != 0 or seq % 32 != 0) */
#define ZOQAT_BUF_ATTN       2   /* fp32 [passes*T, d_model]   attention output of the last layer   */
#define ZOQAT_BUF_FFN        3   /* fp32: fc1 output [passes*T, d_ffn] (OPT); LLaMA: silu(gate)*up [passes*T, d_ffn] when
                                    d_ffn is a multiple of 128 with the default GEMM, else gate|up [passes*T, 2*d_ffn] */
#define ZOQAT_BUF_TOKEN_LOSS 4   /* fp32 [passes*T]            per-position cross-entropy            */
int zoqat_debug_buffer(zoqat_model_t* m, int which, void** dev_ptr, size_t* bytes);

/* Parity hook for the activation quantisers as a whole forward runs them (Section 2 symmetric form, Appendix
 * "Quantization settings": per-token activation quantisation at the input of every block linear).  While a capture
 * buffer is set, every forward copies, at each of the four quantisation points of each layer (attn_in, attn_out,
 * ffn_in, ffn_out) and in execution order, one record into `buf_dev`:
 *   input   fp32 [rows, cols]   the value the quantiser saw (after the norm / non-linearity, before the Section 4.2
 *                               shift and scale if the layer has them)
 *   operand bf16 [rows, cols]   what the quantiser wrote for the GEMM (integer codes, or bf16(x) when a_bits = 0); with
 *                               ZOQAT_GEMM_TCGEN05_I8 the block records hold int8 [rows, cols] in the first half of the slot
 *   step    fp32 [rows]         the per-token step
 * each part padded to a multiple of 256 bytes; rows = passes * batch * seq as materialised at that layer (a frozen
 * prefix is evaluated once: rows = batch * seq there), cols = d_model (d_ffn at ffn_out).  One more record follows
 * the last layer: the final norm's output, its bf16 rounding (the vocabulary projection's operand) and steps of 1,
 * rows = passes * batch * seq, cols = d_model.  A forward that would
 * overrun `bytes` fails with ZOQAT_ERR_WORKSPACE_SMALL before launching anything.  buf_dev = NULL switches the hook
 * off.  The caller owns the buffer; zoqat_debug_capture_bytes gives the size one forward of `passes` passes needs. */
int zoqat_debug_capture(zoqat_model_t* m, void* buf_dev, size_t bytes);
int zoqat_debug_capture_bytes(const zoqat_model_t* m, int batch, int seq, int passes, size_t* bytes);

const char* zoqat_status_string(int status);
const char* zoqat_last_error(void);

/* ---- the steps of the path as single operations ---------------------------
 * The same kernels the step launches, callable on raw device buffers so that
 * each can be compared with the oracle at any size.  All asynchronous. */

/* Raw Philox4x32-10 words of counter blocks [blk0, blk0+nblk) of a tensor:
 * counter = (blk_lo, blk_hi, tensor_id, 0), key = (seed_lo, seed_hi).
 * out_dev: uint32 [nblk, 4]. */
int zoqat_op_philox_words(uint64_t seed, uint32_t tensor_id, uint64_t blk0, uint64_t nblk,
                          uint32_t* out_dev, void* stream);

/* u of Eq. (1) for elements [0, n) of a tensor: fp32 [n].  (Test hook: the step
 * itself never writes u to memory.) */
int zoqat_op_normal(uint64_t seed, uint32_t tensor_id, uint64_t n, float* out_dev, void* stream);

/* Weight path of one [rows, cols] tensor (Eq. (1) argument + Section 2
 * quantiser): w' = W + signed_eps u; per group of `group` columns the step,
 * zero point and codes; the bf16 matmul operand (code - zp) * step.
 * bits = 0 skips the quantiser (operand = bf16(w')).  Outputs may be NULL:
 * codes_dev uint8 [rows, cols]; step_dev fp32 and zp_dev int32 [rows, cols/group];
 * operand_dev bf16 [rows, cols]. */
int zoqat_op_weight_quant(const float* w_dev, int64_t rows, int64_t cols, int group, int bits,
                          uint64_t seed, uint32_t tensor_id, float signed_eps,
                          uint8_t* codes_dev, float* step_dev, int32_t* zp_dev, void* operand_dev,
                          void* stream);

/* Both operands of a step from one read of W and one evaluation of u:
 * operand_plus_dev from W + eps u, operand_minus_dev from W - eps u. */
int zoqat_op_weight_operand_pair(const float* w_dev, int64_t rows, int64_t cols, int group, int bits,
                                 uint64_t seed, uint32_t tensor_id, float eps,
                                 void* operand_plus_dev, void* operand_minus_dev, void* stream);

/* The weight producer with the learnable parts of Section 4.2, on one [rows, cols] tensor.
 *   theta_dev (may be NULL = min/max quantiser): fp32 [rows, cols/group, 4] = (step, zero point, alpha, beta) per
 *     group, perturbed by +/- eps u under tensor id 0x10000 + tensor_id.
 *   smooth_dev (may be NULL = no smoothing): fp32 [2][3][cols], the vectors zoqat_op_smooth_perturb wrote: the
 *     quantiser sees scale' (.) w', and bias_dev[sign * rows + r] = bias0_dev[r] (or 0) + sum_k shift'[k] * w'[r, k]
 *     (first equation of Section 4.2: the smoothed bias uses the unscaled, unquantised perturbed weight).
 *   scratch_dev: 18 * rows * cols / group floats, 16-byte aligned (prepared group parameters, bias partial sums).
 * operand_minus_dev may be NULL: one operand (and one bias vector) with eps signed.
 * codes_dev (may be NULL): uint8 [rows, cols] codes of the +eps side.
 * group = 0: one quantisation group per row (cols % 128 == 0; theta_dev then [rows, 1, 4]; theta_dev and
 * smooth_dev may both be NULL: plain min/max over the row); the scratch size is that of group 128. */
int zoqat_op_weight_operand_learned(const float* w_dev, int64_t rows, int64_t cols, int group, int bits,
                                    uint64_t seed, uint32_t tensor_id, float eps,
                                    const float* theta_dev, const float* smooth_dev,
                                    const float* bias0_dev, float* bias_dev, float* scratch_dev,
                                    void* operand_plus_dev, void* operand_minus_dev, uint8_t* codes_dev, void* stream);

/* Perturbed smoothing vectors of one quantisation point (Section 4.2): out_dev fp32 [2][3][cols] =
 * [sign][scale' | shift' | 1/scale'], scale' = scale +/- eps u(seed, scale_id), shift' likewise with shift_id;
 * sign 0 is +eps, sign 1 is -eps.  cols % 4 == 0. */
int zoqat_op_smooth_perturb(const float* scale_dev, const float* shift_dev, int64_t cols, uint64_t seed,
                            uint32_t scale_id, uint32_t shift_id, float eps, float* out_dev, void* stream);

/* zoqat_op_norm_act_operand with the activation side of the smoothing: the quantiser sees
 * (x - shift') * (1/scale') (both operations rounded once) with the vectors of sign 0 of smooth_dev
 * (zoqat_op_smooth_perturb layout) for rows [0, rows_per_pass) and of sign 1 for the rest. */
int zoqat_op_smooth_act_operand(const float* x_dev, int64_t rows, int64_t cols, int norm_kind, const float* gain_dev,
                                const float* bias_dev, float norm_eps, int a_bits, const float* smooth_dev,
                                int64_t rows_per_pass, void* operand_dev, float* row_step_dev, void* stream);

/* Initial quantiser parameters of one tensor (what zoqat_init_qparams writes): theta_dev fp32 [rows, cols/group, 4]
 * (group = 0: [rows, 1, 4], one group per row). */
int zoqat_op_init_qparams(const float* w_dev, int64_t rows, int64_t cols, int group, int bits, float* theta_dev,
                          void* stream);

/* Packing of Section 4.3: quantise W (unperturbed) into packed codes + qparams,
 * and expansion of a packed tensor into the bf16 operand.  group = 0: one group per row
 * (cols % 128 == 0; qparams_dev then holds rows (step, zero point) pairs, zoqat_packed_bytes
 * gives the sizes); zoqat_op_unpack_operand_i8 (group 0 only) expands into the integer GEMM's
 * operand instead: operand_dev int8 [rows, cols] = code - zero point, col_step_dev fp32 [rows]
 * the rows' steps, err_flag_dev (int32, zeroed by the caller) set to 32 if a row does not fit. */
int zoqat_op_pack_frozen(const float* w_dev, int64_t rows, int64_t cols, int group, int bits,
                         void* packed_dev, void* qparams_dev, void* stream);
int zoqat_op_unpack_operand_i8(const void* packed_dev, const void* qparams_dev, int64_t rows, int64_t cols,
                               int bits, void* operand_dev, float* col_step_dev, int32_t* err_flag_dev, void* stream);
int zoqat_op_unpack_operand(const void* packed_dev, const void* qparams_dev, int64_t rows, int64_t cols,
                            int group, int bits, void* operand_dev, void* stream);

/* Eq. (2) on one tensor: w[i] <- w[i] - scale * u_i, i in [0, n). */
int zoqat_op_update(float* w_dev, uint64_t n, uint64_t seed, uint32_t tensor_id, float scale, void* stream);

/* Optional normalisation followed by the activation operand of a linear:
 * norm_kind 0 none, 1 RMSNorm (gain), 2 LayerNorm (gain, bias);
 * a_bits 4 / 6 / 8: per-row symmetric N-bit codes (as bf16 integers) + row step in
 * row_step_dev; a_bits 0: bf16(x), row step 1.  x_dev fp32 [rows, cols];
 * operand_dev bf16 [rows, cols]; row_step_dev fp32 [rows];
 * normed_dev (may be NULL) fp32 [rows, cols] receives the normalised values. */
int zoqat_op_norm_act_operand(const float* x_dev, int64_t rows, int64_t cols, int norm_kind,
                              const float* gain_dev, const float* bias_dev, float norm_eps, int a_bits,
                              void* operand_dev, float* row_step_dev, float* normed_dev, void* stream);

/* FFN activation followed by the activation operand: LLaMA (gated = 1):
 * silu(x[:, :cols]) * x[:, cols:2*cols] from x_dev fp32 [rows, 2*cols];
 * OPT (gated = 0): relu(x) from fp32 [rows, cols]. */
int zoqat_op_ffn_act_operand(const float* x_dev, int64_t rows, int64_t cols, int gated, int a_bits,
                             void* operand_dev, float* row_step_dev, void* stream);

/* out[m, n] (+)= row_step[m] * sum_k A[m, k] * B[n, k] (+ bias[n]), optional ReLU.
 * a_dev bf16 [M, K], b_dev bf16 [N, K], out_dev fp32 [M, N] (ldo = N).
 * row_step_dev / bias_dev may be NULL.  accumulate != 0 adds into out_dev.
 * impl: ZOQAT_GEMM_*.  tcgen05 path: K % 8 == 0. err_flag_dev: int32 device word
 * set non-zero if a bounded wait ran out (may be NULL for the SIMT kernel). */
int zoqat_op_gemm(const void* a_dev, const void* b_dev, int64_t M, int64_t N, int64_t K,
                  const float* row_step_dev, const float* bias_dev, int relu, int accumulate,
                  float* out_dev, int impl, int32_t* err_flag_dev, void* stream);

/* The gate and up projections of a SiLU-gated FFN in one launch, with the non-linearity in the epilogue:
 * act[m, f] = silu(g) * u,  g = row_step[m] * sum_k A[m, k] * B[f, k],  u = row_step[m] * sum_k A[m, k] * B[F + f, k]
 * (the linear layers of the forward pass of Section 4.1; the architecture is the workloads').
 * a_dev bf16 [M, K]; b_dev bf16 [2F, K] = gate rows then up rows; act_dev fp32 [M, F]; row_amax_dev uint32 [M]
 * receives max_f |act[m, f]| as the bit pattern of a float (the per-token quantiser of the next linear starts
 * from it); F % 128 == 0, K % 8 == 0; tcgen05 pair kernel only. */
int zoqat_op_gemm_silu_gate(const void* a_dev, const void* b_dev, int64_t M, int64_t F, int64_t K,
                            const float* row_step_dev, float* act_dev, uint32_t* row_amax_dev,
                            int32_t* err_flag_dev, void* stream);

/* The linear on 8-bit integers (ZOQAT_GEMM_TCGEN05_I8; Section 2 quantisers with one weight group per output row):
 *   out[m, n] (+)= row_step[m] * (col_step[n] * sum_k A[m, k] * B[n, k]) (+ bias[n]),
 * the sum an exact 32-bit integer, converted to fp32 once (round to nearest) before the two multiplications.
 * a_dev int8 [M, K] (activation codes), b_dev int8 [N, K] (weight codes minus zero point), col_step_dev fp32 [N]
 * (required), row_step_dev / bias_dev may be NULL; K % 16 == 0, N % 32 == 0, 16-byte aligned pointers.
 * gated = 1: the SiLU-gated pair of zoqat_op_gemm_silu_gate (N = 2F, b_dev gate rows then up rows, out_dev fp32
 * [M, F], row_amax_dev uint32 [M] required, no accumulation); gated = 0: out_dev fp32 [M, N]. */
int zoqat_op_gemm_i8(const void* a_dev, const void* b_dev, int64_t M, int64_t N, int64_t K,
                     const float* row_step_dev, const float* col_step_dev, const float* bias_dev, int accumulate,
                     int gated, float* out_dev, uint32_t* row_amax_dev, int32_t* err_flag_dev, void* stream);

/* zoqat_op_weight_operand_learned with one group per row, writing the operands of the integer GEMM: operand_plus_dev /
 * operand_minus_dev int8 [rows, cols] = code minus zero point (16-byte aligned; the second may be NULL), col_step_dev
 * fp32 [2][rows] (or [rows]) = the rows' steps per sign.  err_flag_dev (int32, zeroed by the caller) is set to 32 if a
 * row's code minus zero point leaves [-128, 127].  bits 2..7; other arguments as there. */
int zoqat_op_weight_operand_i8(const float* w_dev, int64_t rows, int64_t cols, int bits, uint64_t seed,
                               uint32_t tensor_id, float eps, const float* theta_dev, const float* smooth_dev,
                               const float* bias0_dev, float* bias_dev, float* scratch_dev, void* operand_plus_dev,
                               void* operand_minus_dev, float* col_step_dev, int32_t* err_flag_dev, void* stream);

/* zoqat_op_norm_act_operand writing the per-token codes as signed bytes: operand_dev int8 [rows, cols]; a_bits 4, 6, 8. */
int zoqat_op_norm_act_operand_i8(const float* x_dev, int64_t rows, int64_t cols, int norm_kind,
                                 const float* gain_dev, const float* bias_dev, float norm_eps, int a_bits,
                                 void* operand_dev, float* row_step_dev, void* stream);

/* Causal softmax attention of one layer (the architecture of the workloads; the paper's
 * forward pass of Section 4.1 runs the unmodified decoder between the quantised linears).
 * qkv_dev fp32 [batch*seq, 3*d_model] (q | k | v, heads contiguous inside each); rotary
 * tables cos_dev/sin_dev fp32 [seq, d_head/2] or NULL (no rotation); out_dev fp32
 * [batch*seq, d_model].  All pointers 16-byte aligned.
 * impl ZOQAT_GEMM_TCGEN05: tensor-core kernel; every operand is split into two binary16
 * halves (hi + lo * 2^-11) and every product is formed from three tensor-core products, so
 * the result is binary32-grade; |q|, |k|, |v| must stay below 65504.  Needs scratch_dev
 * (256-byte aligned, zoqat_op_attention_scratch_bytes() bytes) and err_flag_dev (int32, set
 * non-zero if a bounded wait ran out).  impl ZOQAT_GEMM_SIMT: fp32 CUDA-core kernel
 * (cross-check); scratch_dev / err_flag_dev may be NULL. */
int zoqat_op_attention_scratch_bytes(int batch, int seq, int n_heads, int d_head, size_t* bytes);
int zoqat_op_attention(const float* qkv_dev, int batch, int seq, int n_heads, int d_head,
                       const float* cos_dev, const float* sin_dev, float* out_dev,
                       int impl, void* scratch_dev, int32_t* err_flag_dev, void* stream);

/* The q | k | v projection and the attention behind it as the step runs them on the default GEMM: the projection's
 * epilogue applies the rotary embedding, scales q, splits every value into the two binary16 halves and writes the
 * attention kernel's operand layouts itself, so q | k | v never exist as fp32 in memory and no preparation pass
 * runs.  a_dev bf16 [batch*seq, K]; b_dev bf16 [3*d_model, K] (q rows, k rows, v rows; d_model = n_heads*d_head);
 * row_step_dev / bias_dev ([3*d_model]) may be NULL; out_dev fp32 [batch*seq, d_model]; scratch_dev as for
 * zoqat_op_attention.  Needs d_model % 256 == 0, seq % 32 == 0, K % 8 == 0.  Same result as zoqat_op_gemm followed
 * by zoqat_op_attention up to the binary32 rounding of the rotation. */
int zoqat_op_qkv_attention(const void* a_dev, const void* b_dev, int batch, int seq, int n_heads, int d_head, int64_t K,
                           const float* row_step_dev, const float* bias_dev, const float* cos_dev, const float* sin_dev,
                           float* out_dev, void* scratch_dev, int32_t* err_flag_dev, void* stream);

/* Vocabulary projection fused with the cross-entropy: logits = A B^T are never
 * stored.  a_dev bf16 [T, d], b_dev bf16 [V, d], labels_dev int32 [T] (< 0 =
 * ignored); token_loss_dev fp32 [T] (0 where ignored); loss_sum_dev double[1]
 * (sum of the per-position losses) and count_dev int32[1] (labelled positions).
 * scratch_dev: zoqat_op_head_loss_scratch_bytes(T, V) bytes. */
int zoqat_op_head_loss_scratch_bytes(int64_t T, int64_t V, size_t* bytes);
int zoqat_op_head_loss(const void* a_dev, const void* b_dev, const int32_t* labels_dev,
                       int64_t T, int64_t V, int64_t d, float* token_loss_dev,
                       double* loss_sum_dev, int32_t* count_dev, void* scratch_dev,
                       int impl, int32_t* err_flag_dev, void* stream);

/* The same operation as zoqat_op_head_loss for callers that must not allocate device
 * memory and so cannot hand over a scratch buffer.  (The paper has no counterpart: this
 * is a convenience of the library, not a step of the method.)  Typical cases: code that
 * runs after another component has claimed the whole device for its own memory pool, a
 * latency-critical loop in which a cudaMalloc/cudaFree would stall every stream of the
 * device, or a plug-in whose host forbids allocation calls altogether.
 *
 * The scratch is a fixed array of ZOQAT_STATIC_SCRATCH_BYTES inside the library image;
 * every device that loads the library keeps it resident until the process ends.  Inputs
 * and outputs are still the caller's: a_dev bf16 [T, d], b_dev bf16 [V, d], labels_dev
 * int32 [T]; token_loss_dev fp32 [T], loss_sum_dev double[1], count_dev int32[1],
 * err_flag_dev int32[1] (required for ZOQAT_GEMM_TCGEN05) - all device memory.
 *
 *   - Limit: 256-byte-rounded T * ceil(V/128) * 8 plus 256-byte-rounded T * 4 bytes must
 *     fit in the array (T = 4096 with V = 32000 does; T = 8192 with V = 50272 does not).
 *     Larger problems return ZOQAT_ERR_WORKSPACE_SMALL and launch nothing.
 *   - Every call looks up the array's device address for the device (and context) that is
 *     current, so a pointer never outlives the context it came from.  Make the first call on
 *     a device outside any stream capture.
 *   - No cudaMalloc, cudaFree or other allocating routine is called, on any call.
 *   - All calls on a device share the one array, which still holds the previous call's
 *     data; the part that has to start from zero is cleared on `stream` before use.  Two
 *     calls whose kernels can overlap on the GPU (different streams without an ordering
 *     between them, or different host threads doing so) race on it: serialise them. */
#define ZOQAT_STATIC_SCRATCH_BYTES (16u << 20)
int zoqat_op_head_loss_static(const void* a_dev, const void* b_dev, const int32_t* labels_dev,
                              int64_t T, int64_t V, int64_t d, float* token_loss_dev,
                              double* loss_sum_dev, int32_t* count_dev, int impl,
                              int32_t* err_flag_dev, void* stream);

/* ---- decode-time inference over the packed representation -------------------------------
 * The deployment side of the method (the paper's on-device tokens-per-second table): one new
 * token per sequence and call, keys and values cached, every block linear read once per
 * token as stored low-bit codes.  Needs a model whose block linears are all FROZEN_PACKED
 * (zoqat_prequantize_frozen() done), w_bits <= 4 with column groups, d_model and d_ffn
 * multiples of 32 (ZOQAT_ERR_UNSUPPORTED otherwise); batch in {1, 2, 4, 8} sequences advance
 * in lock step.  The kernels of a step are launched as programmatic dependents of one
 * another (each may start while its predecessor drains and reads only constant data until
 * the predecessor has completed); the first kernel of a step is an ordinary launch, so a step
 * is ordered after all earlier work of the stream as usual.
 *
 * Arithmetic: a packed linear is evaluated as an integer runtime does,
 *     y[t, n] = s_t * sum_g Delta[n, g] * ( sum_{k in g} a[t, k] * (c[n, k] - z[n, g]) ) (+ bias),
 * the inner sums exact integers (dp4a), the steps applied in fp32; it differs from the
 * training forward only by that forward's bf16 rounding of (c - z) * Delta.  Weight-only
 * models (a_bits = 0) use the forward's own operands, bf16(x) and bf16((c - z) * Delta),
 * with fp32 accumulation.  Norms,
 * rotary embedding, attention (fp32, over an fp32 cache) and the bf16 vocabulary
 * projection are those of the forward pass.
 *
 * zoqat_decode_begin converts the packed tensors once into `buffer_dev` (zoqat_decode_bytes()
 * bytes, 256-byte aligned, caller-owned, in use until the handle is destroyed or begin is
 * called again): 4-bit nibbles in input-channel order, contiguous group parameters, the
 * vocabulary projection as bf16, and the key/value cache [layer][2][batch][head][max_len][d_head].
 * zoqat_decode_step feeds tokens_dev[batch] at position `pos` (0-based; positions must be fed
 * in order, each overwriting its cache slot) and writes logits_dev fp32 [batch, vocab]
 * and/or next_token_dev int32 [batch] = argmax (lowest index on ties); either may be NULL.
 * Asynchronous, no host synchronisation: a loop of steps can be captured in a CUDA graph. */
int zoqat_decode_bytes(const zoqat_model_t* m, int batch, int max_len, size_t* bytes);
int zoqat_decode_begin(zoqat_model_t* m, void* buffer_dev, size_t bytes, int batch, int max_len, void* stream);
int zoqat_decode_step(zoqat_model_t* m, const int32_t* tokens_dev, int pos, float* logits_dev,
                      int32_t* next_token_dev, void* stream);

/* One packed linear of the decode path on raw buffers: packed_dev / qparams_dev as written by
 * zoqat_op_pack_frozen for a [rows, cols] tensor; act_codes_dev bf16 [batch, cols] integer codes
 * with their steps row_step_dev[batch] (zoqat_op_norm_act_operand output); out_dev fp32
 * [batch, rows] (accumulate != 0 adds); nibble_scratch_dev: rows*cols/2 + 2*batch*cols bytes,
 * 16-byte aligned (the repacked codes, then the activation rows as int8).  batch in
 * {1, 2, 4, 8}; cols % 32 == 0. */
int zoqat_op_decode_gemv(const void* packed_dev, const void* qparams_dev, int64_t rows, int64_t cols, int group, int bits,
                         const void* act_codes_dev, const float* row_step_dev, int batch, const float* bias_dev,
                         int accumulate, float* out_dev, void* nibble_scratch_dev, void* stream);

/* ---- serving drafted tokens over a paged key/value cache ---------------------------------
 * What one step of a batch of requests needs around the linears when every request has a length
 * of its own, brings one or several new tokens (drafts, arranged as a tree) and keeps its keys and
 * values in pages of a shared pool.  (The paper's decode table feeds one token per sequence; this is
 * the deployment side carried on, the operations are those of the forward pass.)  A step calls, in order,
 *     zoqat_op_cache_plan       once: pages, slots, positions and tree masks from the lengths
 *     zoqat_op_cache_append     per layer: rotary embedding, new keys and values into their slots
 *     zoqat_op_tree_attention   per layer: drafts attend to the cached positions and their ancestors
 *     zoqat_op_logit_rules      once: penalties, biases, grammar masks, greedy choice
 * and zoqat_decode_tree_step() is that step for a packed model.  Lengths and tables are device data:
 * no call reads them on the host, so a step can be captured in a CUDA graph and replayed as they change.
 * Inputs that only the device can check are reported in an int32 word (err_flag_dev / status_dev; zeroed by
 * the caller, never cleared here), and the access in question is skipped.  Output buffers must not overlap
 * inputs except where it is said.  All calls are asynchronous. */
#define ZOQAT_TYPE_F32  0
#define ZOQAT_TYPE_BF16 1
#define ZOQAT_TYPE_F16  2

/* One layer's pages.  Element (page, slot, head, i) of K or V is at page * page_stride + slot * slot_stride +
 * head * head_stride + i, in elements: [page][slot][head][d_head] and [page][head][slot][d_head] are both
 * layouts of this form, as is the cache of zoqat_decode_begin (a page per sequence).  Strides are multiples of 16 bytes,
 * k and v 16-byte aligned. */
typedef struct zoqat_paged_cache {
    void*   k;             /* dev */
    void*   v;             /* dev */
    int32_t type;          /* ZOQAT_TYPE_*                                                            */
    int32_t n_pages;
    int32_t page_size;     /* slots per page; n_pages * page_size <= 2^31 - 1                          */
    int32_t n_kv_heads;
    int32_t d_head;        /* 64 or 128                                                               */
    int32_t reserved;
    int64_t page_stride, slot_stride, head_stride;
} zoqat_paged_cache_t;

/* Plan of a step: request b has cached_len_dev[b] tokens in the cache and brings new_len_dev[b] (0: it sits this step out).
 * Pages a request holds already (the first ceil(cached / page_size) entries of its row of block_table_dev [batch, max_pages])
 * are kept; further ones are taken from the end of free_pages_dev[0 .. *n_free_dev), request by request in order, and written
 * behind them (entries beyond stay as they are).  free_capacity: entries of free_pages_dev.  Rows of all requests stand back to
 * back:
 *   kv_len_dev [batch]            cached + new
 *   row_start_dev [batch + 1]     first row of each request; the last entry is the number of rows
 *   row_request_dev, row_pos_dev, slot_dev [max_rows]   request, position (rotary) and slot (page * page_size + offset) of
 *                                 each row; -1 in the rows behind the last
 *   tree_mask_dev [max_rows, mask_words]  bit j: the row sees draft j of its request (itself and its ancestors); 0 behind the
 *                                 last row.  NULL with mask_words = 0: not wanted
 *   n_free_out_dev [1]            pages left (not n_free_dev itself: the call may be repeated on the same inputs)
 * parents_dev [max_rows] (may be NULL: each draft follows the one before it) names each draft's parent by its index within the
 * request, -1 for one that follows the cached context; a parent stands before its children.  position = cached + depth.
 * status_dev is or-ed with 1 (a length negative or too long for the table, more than 32 * mask_words drafts with a mask, more rows
 * than max_rows, a bad *n_free_dev: nothing is planned), 2 (too few pages: nothing is planned), 4 (a page outside [0, n_pages):
 * the row gets slot -1), 8 (a parent not before its child: the walk ends there).  "Nothing is planned" leaves the table as it is,
 * row_start and kv_len are all 0 and every row is padding.  batch <= 16384, mask_words <= 32. */
int zoqat_op_cache_plan(const int32_t* cached_len_dev, const int32_t* new_len_dev, int batch, int page_size, int n_pages,
                        const int32_t* free_pages_dev, int free_capacity, const int32_t* n_free_dev,
                        int32_t* block_table_dev, int max_pages, const int32_t* parents_dev, int max_rows, int mask_words,
                        int32_t* kv_len_dev, int32_t* row_start_dev, int32_t* row_request_dev, int32_t* row_pos_dev,
                        int32_t* slot_dev, uint32_t* tree_mask_dev, int32_t* n_free_out_dev, int32_t* status_dev, void* stream);

/* The new rows of one layer: qkv_dev fp32 [rows, (n_heads + 2 * n_kv_heads) * d_head], rows ld elements apart (16-byte
 * aligned, ld % 4 == 0): q heads, k heads, v heads.  q and k are rotated by the tables' row row_pos_dev[r] (cos_dev / sin_dev fp32
 * [rope_len, d_head / 2], pairs (i, i + d_head / 2); both NULL: no rotation, row_pos_dev unused), rounded once to the cache's
 * type; q goes to q_out_dev (of that type, [rows, n_heads, d_head], rows q_stride elements apart), k and v into slot slot_dev[r].
 * A row with a negative slot is skipped, its q_out row left as it is; so is, whole, a row whose slot or position lies outside the
 * cache / the tables, and it sets *err_flag_dev to 40.  Two rows with the same slot: either may win, element by element.  rows = 0 is
 * allowed (nothing is done). */
int zoqat_op_cache_append(const float* qkv_dev, int64_t ld, const int32_t* row_pos_dev, const int32_t* slot_dev, int rows,
                          int n_heads, const float* cos_dev, const float* sin_dev, int rope_len,
                          const zoqat_paged_cache_t* cache, void* q_out_dev, int64_t q_stride, int32_t* err_flag_dev, void* stream);

/* out[r, h] = softmax(scale * q[r, h] . K) V over what row r sees: with n rows and L = kv_len_dev[b] keys (drafts last, their K
 * and V in the cache already) the keys t < L - n, and draft j (t = L - n + j) if bit j of the row's tree_mask_dev [rows,
 * mask_words] is set (bits beyond mask_words count as 0; tree_mask_dev = NULL: if j is not behind the row).  Query head h reads key
 * head h / (n_heads / n_kv_heads).  A row that sees nothing gives zeros; what a row does not see does not reach it, whatever it
 * holds (NaN, inf).  q_dev and out_dev have the cache's type, [rows, n_heads, d_head] with rows q_stride / out_stride elements
 * apart (16-byte aligned, strides multiples of 16 bytes).  Rows outside row_start_dev's ranges are left as they are.
 * Sums and the softmax are held in fp32; in bf16 / fp16 the softmax weights are rounded to the cache's type for the product with
 * V.  The keys are dealt out evenly over the SMs, long contexts in several pieces that are joined in a fixed order: the same
 * call gives the same bits.  bf16 and fp16 need page_size 8, 16, 32, 64 or a multiple of 128, and with several heads and pages a
 * page_stride that is a multiple of head_stride, fewer than 2^31 strides of a head through all pages and a slot_stride under 2^36
 * (ZOQAT_ERR_UNSUPPORTED otherwise).  scratch_dev:
 * zoqat_op_tree_attention_scratch_bytes() bytes, 256-byte aligned, for one call at a time (calls that may overlap, e.g. two graphs
 * in flight, each need their own).  rows = 0 is allowed (nothing is done).  *err_flag_dev is set to 41 (a request whose lengths or
 * rows contradict each other: it is left out), 42 (a page outside the pool: its keys and values count as zeros), 43 (a bounded
 * device wait ran out). */
int zoqat_op_tree_attention_scratch_bytes(int type, int d_head, size_t* bytes);
int zoqat_op_tree_attention(const void* q_dev, int64_t q_stride, const zoqat_paged_cache_t* cache, const int32_t* block_table_dev,
                            int max_pages, const int32_t* kv_len_dev, const int32_t* row_start_dev, const uint32_t* tree_mask_dev,
                            int mask_words, int batch, int rows, int n_heads, float scale, void* out_dev, int64_t out_stride,
                            void* scratch_dev, size_t scratch_bytes, int32_t* err_flag_dev, void* stream);

/* Rules on logits.  Every pointer is device memory; a NULL group is off. */
typedef struct zoqat_logit_rules {
    const int32_t* row_request;    /* [rows] request of each row, -1: the row is left as it is; NULL: row r is request r */
    const float*   repetition;     /* [batch] fp32; NULL: 1                                                        */
    const float*   presence;       /* [batch] fp32; NULL: 0                                                        */
    const float*   frequency;      /* [batch] fp32; NULL: 0                                                        */
    const int32_t* history;        /* [batch, history_stride <= 2^30] token ids: prompt, then what was generated    */
    const int32_t* history_len;    /* [batch]                                                                      */
    const int32_t* prompt_len;     /* [batch] how many of them are the prompt; NULL: 0                             */
    const int32_t* bias_token;     /* [batch, bias_stride]                                                         */
    const float*   bias_value;     /* [batch, bias_stride]                                                         */
    const int32_t* bias_len;       /* [batch]                                                                      */
    const uint32_t* allowed;       /* [rows, allowed_stride] bit v of a row: token v is allowed                     */
    const int32_t* draft_token;    /* [rows] the token of each row; with row_start and tree_mask a row's ancestors and
                                      itself count as generated (the history does not hold them yet)               */
    const int32_t* row_start;      /* [batch + 1]                                                                  */
    const uint32_t* tree_mask;     /* [rows, mask_words]                                                           */
    int64_t history_stride, allowed_stride;
    int32_t bias_stride, mask_words, batch, reserved;
} zoqat_logit_rules_t;

/* For every row r and token v, each step one fp32 rounding, in this order:
 *   x = logits[r, v];  if v is in the prompt or n > 0: x = x > 0 ? x / repetition : x * repetition, with n = times v was generated;
 *   x -= frequency * n;  if n > 0: x -= presence;  x += the sum of the request's biases for v;  x = -inf if v is not allowed
 * out_dev[r, v] = x in the logits' type (may be logits_dev itself with out_ld == ld; NULL: only the choice is wanted) and
 * token_dev[r] = the lowest v with the largest out value (-1 if none is above -inf; NULL: not wanted).  Tokens outside [0, vocab)
 * in the history, drafts or biases are ignored; NaN logits are never chosen.  type: ZOQAT_TYPE_* of logits and out;
 * rows ld / out_ld elements apart; 1 <= rows <= 65535. */
int zoqat_op_logit_rules(const void* logits_dev, int type, int64_t ld, int rows, int vocab, const zoqat_logit_rules_t* rules,
                         void* out_dev, int64_t out_ld, int32_t* token_dev, void* stream);

/* A step of drafted tokens through a packed model: zoqat_decode_step for requests of different lengths, with their keys and values
 * in pages.  The step's plan (zoqat_op_cache_plan's outputs, device memory): */
typedef struct zoqat_tree_batch {
    const int32_t*  block_table;   /* [batch, max_pages]                                                      */
    const int32_t*  kv_len;        /* [batch]                                                                 */
    const int32_t*  row_start;     /* [batch + 1]                                                             */
    const int32_t*  row_pos;       /* [rows], < max_seq of the model                                          */
    const int32_t*  slot;          /* [rows]                                                                  */
    const uint32_t* tree_mask;     /* [rows, mask_words], or NULL: each draft follows the one before it        */
    int32_t batch, max_pages, mask_words, reserved;
} zoqat_tree_batch_t;

/* Feeds tokens_dev[rows] (rows in {1, 2, 4, 8}; of all requests, back to back; rows behind the last are padding) through the
 * model (a token outside [0, vocab) as an embedding of zeros) and writes logits_dev fp32 [rows, vocab] - row r's prediction of the
 * token after it - and / or next_token_dev int32 [rows]: the greedy choice, under `rules` (zoqat_op_logit_rules, applied to the
 * logits in place) unless that is NULL.
 * caches: n_layers descriptions (host memory, read before the call returns), n_kv_heads = n_heads, any type; the rows' keys and values
 * are written before they are attended to.  Needs zoqat_decode_begin (its batch is the most rows that may leave logits_dev
 * NULL; the cache it lays out is not used).  scratch_dev as for zoqat_op_tree_attention.  Logits of padding rows are unspecified.
 * What the device finds wrong in plan or pages is reported by zoqat_check() as ZOQAT_ERR_INVALID_ARG.  Asynchronous, no host
 * synchronisation; can be captured in a CUDA graph. */
int zoqat_decode_tree_step(zoqat_model_t* m, const int32_t* tokens_dev, int rows, const zoqat_tree_batch_t* plan,
                           const zoqat_paged_cache_t* caches, const zoqat_logit_rules_t* rules, float* logits_dev,
                           int32_t* next_token_dev, void* scratch_dev, size_t scratch_bytes, void* stream);

/* ---- many continuations of one prompt ------------------------------------------------------
 * Beam search, and batches of requests behind one long prompt, over the same pages.  A step of beams, in order:
 *     zoqat_op_cache_plan         once: where the new row of every beam goes (a beam is a request of the plan)
 *     zoqat_op_rotary_append      per layer: norms and rotation of the query and key heads, keys and values into their slots
 *     zoqat_op_prefix_attention   per layer: the keys that all beams of a prompt share are read once for all of them
 *     zoqat_op_beam_select        once: the best continuations of every request's beams
 *     zoqat_op_beam_reorder       once: tables, free pages and token histories follow the beams that go on
 *     zoqat_op_cache_copy         once: what half-filled pages hold is copied for beams that part, in every layer
 * and zoqat_decode_prefix_step() is zoqat_decode_tree_step() with the shared prefixes read once.
 * Conventions as above: device data is read on the device only, words are or-ed or set, never cleared, all calls are asynchronous and
 * can be captured in a CUDA graph. */

/* Angles a position of the pairs of a head whose first `rot` elements are turned: freq_host [rot / 2] (host memory), base^(-2 i / rot)
 * scaled for contexts `factor` times as long as those of the training:
 *   PLAIN   as they are
 *   LINEAR  freq / factor
 *   BASE    the base times factor^(rot / (rot - 2)): the slowest pair slows down by the factor, the fastest is left
 *   PARTS   pairs that turn r = trained_len * freq / (2 pi) times in a training context: freq / factor up to r = 1, freq from r = 32 on, a
 *           linear ramp in r between; *magnitude_host, by which q and k are to be multiplied, is 0.1 ln(factor) + 1 (else 1).  The ramp's ends
 *           are fixed; for one with other ends, or over the numbers of the pairs, fill the frequencies yourself: any [rot / 2] will do */
#define ZOQAT_ROTARY_PLAIN  0
#define ZOQAT_ROTARY_LINEAR 1
#define ZOQAT_ROTARY_BASE   2
#define ZOQAT_ROTARY_PARTS  3
int zoqat_rotary_frequencies(int rot, double base, int kind, double factor, int trained_len, double* freq_host, float* magnitude_host);

/* zoqat_op_cache_append with norms and other rotations: qkv_dev [rows, (n_heads + 2 * n_kv_heads) * d_head] of qkv_type (ZOQAT_TYPE_*; rows
 * ld elements apart, 16-byte aligned).  q heads are multiplied by q_gain / sqrt(mean(x^2) + norm_eps) over the head, k heads with k_gain
 * (fp32 [d_head]; NULL: that head is left as it is), then the first `rot` elements of q and k heads are turned by the angles row_pos_dev[r] *
 * freq_dev[i] (fp64 [rot / 2], radians; rot a multiple of 16, 0: no rotation, freq_dev NULL and row_pos_dev unused): pair i is (i, i + rot /
 * 2), or (2 i, 2 i + 1) with `interleaved`, and multiplied by `magnitude`.  Angles are reduced in 64 bits, so positions may be as far as they like;
 * everything else is fp32, one rounding into the cache's type.  Slots, padding and errors as in zoqat_op_cache_append (a negative position of a live row
 * counts as outside).  rows = 0 is allowed. */
int zoqat_op_rotary_append(const void* qkv_dev, int qkv_type, int64_t ld, const int32_t* row_pos_dev, const int32_t* slot_dev, int rows, int n_heads,
                           const double* freq_dev, int rot, int interleaved, float magnitude, const float* q_gain_dev, const float* k_gain_dev,
                           float norm_eps, const zoqat_paged_cache_t* cache, void* q_out_dev, int64_t q_stride, int32_t* err_flag_dev, void* stream);

/* zoqat_op_tree_attention for requests that share a long prefix: requests group_start_dev[g] .. group_start_dev[g + 1] - 1 ([groups + 1]) form
 * group g, and the first prefix_len_dev[g] keys of each of them that has rows ([groups]) are the same - their rows of block_table name the same pages, or
 * pages that hold the same; request_group_dev [batch] names each request's group.  Requests without rows keep their place: their lengths, rows of
 * block_table and entries of request_group_dev may hold anything.  All keys of the prefix are seen by all rows (prefix_len <= kv_len - rows
 * of the request).  The result is that of zoqat_op_tree_attention up to rounding, the prefix is read once for the whole group (through the table of its first
 * request that has rows and holds it, in whole tiles of 128 keys, fp32 32; what is left of it through each request's own).  Everything else as there, the limits
 * of page sizes and strides among it.  *err_flag_dev is also set to 41 where groups and requests contradict each other: the group or request is left out.  scratch_dev:
 * zoqat_op_prefix_attention_scratch_bytes() bytes for this many rows or fewer, 256-byte aligned, for one call at a time. */
int zoqat_op_prefix_attention_scratch_bytes(int type, int d_head, int rows, int n_heads, size_t* bytes);
int zoqat_op_prefix_attention(const void* q_dev, int64_t q_stride, const zoqat_paged_cache_t* cache, const int32_t* block_table_dev, int max_pages,
                              const int32_t* kv_len_dev, const int32_t* row_start_dev, const int32_t* group_start_dev, const int32_t* prefix_len_dev,
                              const int32_t* request_group_dev, int groups, const uint32_t* tree_mask_dev, int mask_words, int batch, int rows, int n_heads,
                              float scale, void* out_dev, int64_t out_stride, void* scratch_dev, size_t scratch_bytes, int32_t* err_flag_dev, void* stream);

/* Groups of requests that share a prefix, as zoqat_op_prefix_attention takes them (device memory). */
typedef struct zoqat_prefix_groups {
    const int32_t* group_start;    /* [groups + 1]                                                            */
    const int32_t* prefix_len;     /* [groups]                                                                */
    const int32_t* request_group;  /* [batch of the plan]                                                     */
    int32_t groups, reserved;
} zoqat_prefix_groups_t;

/* zoqat_decode_tree_step whose requests share prefixes: beams of a prompt, or requests behind one.  scratch_dev: zoqat_op_prefix_attention_scratch_bytes()
 * bytes for these rows, the model's heads and the caches' type.  Everything else as there. */
int zoqat_decode_prefix_step(zoqat_model_t* m, const int32_t* tokens_dev, int rows, const zoqat_tree_batch_t* plan, const zoqat_prefix_groups_t* groups,
                             const zoqat_paged_cache_t* caches, const zoqat_logit_rules_t* rules, float* logits_dev,
                             int32_t* next_token_dev, void* scratch_dev, size_t scratch_bytes, void* stream);

/* The best continuations: score(b, v) = score_dev[request, b] + logits[request * beams + b, v] - log sum_u exp logits[.., u], formed and
 * compared in 64 bits, ordered from the best down; of equal scores the lower beam, then the larger logit, then the lower token comes first.  Of the
 * beams * (1 + n_eos) best of a request the first `beams` whose token is none of eos_dev [n_eos] (up to 7; n_eos = 0: NULL) go to beam_dev,
 * token_dev, score_out_dev [batch, beams]; those among its first `beams` whose token is one of them to done_beam_dev, done_token_dev,
 * done_score_dev [batch, beams], in the same order; -1 and -inf fill up.  Scores are rounded to fp32 once.  Beams with a score of -inf or NaN (not in use)
 * offer nothing, nor do logits of -inf or NaN, which do not count in the sum either; +inf counts as the largest finite fp32 value.  type:
 * ZOQAT_TYPE_* of the logits, rows ld elements apart (16-byte aligned rows are read fastest).  beams <= 32. */
int zoqat_op_beam_select(const void* logits_dev, int type, int64_t ld, int batch, int beams, int vocab, const float* score_dev, const int32_t* eos_dev,
                         int n_eos, int32_t* beam_dev, int32_t* token_dev, float* score_out_dev, int32_t* done_beam_dev, int32_t* done_token_dev,
                         float* done_score_dev, void* stream);

/* States follow the beams.  Row b * beams + j of the outputs continues row b * beams + parent[b * beams + j] of the inputs (-1: the row
 * ends, its length becomes 0).  A row's keys are in the first ceil(kv_len / page_size) pages of its row of block_table; rows of a request may
 * share pages (in the same column, holding the same), rows of different requests only pages that begin below shared_len of both.
 *   block_table_out [rows, max_pages]   the parent's pages; entries beyond stay as they are.  The page that the parent is still filling (kv_len
 *                       not a multiple of page_size) is kept by the first such row in order; every later row that would share it gets another page, and so
 *                       does the first where a row that goes on is longer and holds that page whole
 *   copy_from, copy_to, copy_len [rows]  what zoqat_op_cache_copy has to copy for such a row (page, page, slots); -1, -1, 0 for the others.  A page
 *                       that begins below shared_len [batch] (NULL: 0) belongs to others too: no row keeps it to fill it, and it never goes back.  So a
 *                       shared_len inside a page is for the one call that parts the rows from that page; from then on they have it as copies of
 *                       their own, and shared_len is to be the length of the whole pages below it
 *   free_pages_out [free_capacity], n_free_out   the free pages afterwards.  Pages that no row of the request holds any more are given back, in the order
 *                       of requests, columns, rows.  A request's new pages are those first; further ones are taken from the end of free_pages[0 ..
 *                       *n_free), request by request, row by row; what is left of the pages given back stands behind the free pages that are left
 *   kv_len_out [rows]   the parent's length
 *   history_out [rows, history_stride], history_len_out [rows]   (history may be NULL) the parent's tokens and, if token [rows] is given, the row's
 *                       token behind them; entries beyond stay as they are
 * status is or-ed with 1 (a length negative or too long for its table or history: it counts as 0; *n_free outside the list, or more pages than the
 * list holds), 2 (too few free pages), 4 (a page outside [0, n_pages): left where it is, neither copied nor given back), 8 (a parent outside [-1, beams): it
 * counts as -1).  With an impossible *n_free or too few pages nothing is reordered: all lengths become 0, there are no copies, the free pages
 * stay, tables and histories are unspecified.  Outputs are other buffers than inputs.  batch <= 16384, beams <= 32; tables and free lists of less than 2^30 entries. */
typedef struct zoqat_beam_reorder {
    const int32_t* parent;        /* [batch * beams]                                                          */
    const int32_t* kv_len;        /* [batch * beams]                                                          */
    const int32_t* block_table;   /* [batch * beams, max_pages]                                               */
    const int32_t* shared_len;    /* [batch], or NULL                                                         */
    const int32_t* free_pages;    /* [free_capacity]                                                          */
    const int32_t* n_free;        /* [1]                                                                      */
    const int32_t* history;       /* [batch * beams, history_stride], or NULL                                 */
    const int32_t* history_len;   /* [batch * beams]                                                          */
    const int32_t* token;         /* [batch * beams], or NULL                                                 */
    int32_t *block_table_out, *kv_len_out, *free_pages_out, *n_free_out, *copy_from, *copy_to, *copy_len, *history_out, *history_len_out;
    int32_t* status;
    int64_t history_stride;
    int32_t batch, beams, page_size, n_pages, max_pages, free_capacity;
} zoqat_beam_reorder_t;
int zoqat_op_beam_reorder_scratch_bytes(int batch, size_t* bytes);
/* r: host memory, read before the call returns.  scratch_dev: 8-byte aligned, for one call at a time. */
int zoqat_op_beam_reorder(const zoqat_beam_reorder_t* r, void* scratch_dev, size_t scratch_bytes, void* stream);

/* For every row r, K and V of the slots [0, len_dev[r]) of page from_dev[r] are copied to the same slots of page to_dev[r], in every one of n_layers
 * caches (host memory, read before the call returns).  len 0: nothing; a page or length outside the cache, or a page onto itself, sets
 * *err_flag_dev to 42 and is skipped.  No page may be written by one row and read or written by another.  rows = 0 is allowed. */
int zoqat_op_cache_copy(const zoqat_paged_cache_t* caches, int n_layers, const int32_t* from_dev, const int32_t* to_dev, const int32_t* len_dev, int rows,
                        int32_t* err_flag_dev, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ZOQAT_H */
