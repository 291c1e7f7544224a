/*
 * moev.h -- C ABI of the B200 (sm_100a) MoE verification layer.
 *
 * One call, moev_verify(), runs the MoE expert layer of the target model's
 * verification pass over the gamma tokens of a speculative draft tree:
 *
 *   router top-k per token  ->  expert union + token->expert grouping
 *   ->  grouped gated-SwiGLU expert FFN over the union, each active expert's
 *       weights read from HBM once  ->  routing-weighted combine,
 *
 * and reports the per-layer active-expert count.
 *
 * Paper passages the operations follow:
 *   - Sec. 1: top-k routing -- the router scores the E experts for every token and the
 *     token is processed by its k best-scoring experts only.
 *   - Eq. 1 (Sec. 3): the verification footprint is the union over the gamma
 *     verified tokens of their expert sets; its size -- not gamma -- drives the
 *     cost, because the verifier fetches every expert of the union from HBM and
 *     reuses it for all tokens routed to it.
 *   - Table 1 / Table 3 metric "average active experts": the size of that union
 *     per MoE layer per verification step (n_active here; shared experts are not
 *     counted, as the autoregressive rows of Table 1 show).
 *   - Table 13: experts per layer, top-k and the always-on shared expert.
 *   - Fig. 1(c): bytes of one expert (moev_expert_bytes).
 * The paper does not print the expert FFN; it is the bias-free gated SwiGLU
 *   FFN_e(x) = W_down,e ( silu(W_gate,e x) * (W_up,e x) ),  silu(z) = z/(1+exp(-z)),
 *   y_t = sum_j w[t,j] FFN_{ids[t,j]}(x_t) + sum_s FFN_shared,s(x_t).
 *
 * Conventions
 *   - No exceptions, aborts or traps cross this boundary: every entry point
 *     returns a moev_status; moev_last_error() gives the text of the last failure.
 *   - Unless a parameter says HOST, pointers are DEVICE pointers, borrowed for the
 *     duration of the call; the library never frees or retains caller memory.
 *   - moev_verify() is asynchronous on the given CUDA stream, allocates nothing
 *     and never synchronises; outputs are valid once the stream reaches that point.
 *   - One context per host thread / stream (calls on one context must not overlap).
 */
#ifndef MOEV_H_
#define MOEV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct moev_ctx moev_ctx; /* opaque; owns the device workspace */

typedef enum {
  MOEV_OK = 0,
  MOEV_EINVAL = 1,       /* bad argument (null, out of range, misaligned, shape granularity) */
  MOEV_EUNSUPPORTED = 2, /* device is not sm_100 */
  MOEV_ECUDA = 3,        /* a CUDA runtime/driver call failed; see moev_last_error */
  MOEV_ENOMEM = 4,       /* workspace allocation failed in moev_create */
  MOEV_ETIMEOUT = 5      /* a bounded device-side wait expired (reported by moev_status_sync) */
} moev_status;

/* Expert-weight storage formats (K = contraction dimension, always contiguous). */
typedef enum {
  MOEV_W_FP32 = 0,         /* float32 */
  MOEV_W_BF16 = 1,         /* bfloat16 */
  MOEV_W_FP8E4M3_B128 = 2, /* e4m3fn codes + float32 scale per 128x128 block: W = code * s */
  MOEV_W_MXFP4 = 3,        /* e2m1 codes, two per byte (even k in the low nibble) + e8m0
                              scale per 32 along K: W = code * 2^(s-127) */
  MOEV_W_INT4 = 4          /* moev_linear_w4 only: 4-bit integers, two per byte (even k in the low
                              nibble) + bfloat16 scale per group along K: W = (code - 8) * s */
} moev_wfmt;

typedef enum { MOEV_ACT_FP32 = 0, MOEV_ACT_BF16 = 1 } moev_afmt;

/* Router weights over the k selected experts (selection itself is always on raw logits,
 * descending, exact ties to the lower expert id):
 *   SOFTMAX: w_j = exp(l_j - l_max) / sum_{j<k} exp(l_j - l_max)
 *   SIGMOID: s_j = 1/(1+exp(-l_j)),  w_j = routed_scale * s_j / (sum_j s_j + 1e-20)      */
typedef enum { MOEV_SCORE_SOFTMAX = 0, MOEV_SCORE_SIGMOID = 1 } moev_score;

/* Which expert-FFN kernels moev_verify uses. */
typedef enum {
  MOEV_IMPL_AUTO = 0,   /* tensor-core (TMA + tcgen05) path when the shape allows, else SIMT */
  MOEV_IMPL_SIMT = 1,   /* CUDA-core kernels (all formats, all shapes) */
  MOEV_IMPL_TCGEN05 = 2 /* tensor-core path; MOEV_EINVAL if the shape does not allow it */
} moev_impl;

/* Expert form.  The paper does not print the FFN; the benchmark configurations use the bias-free
 * gated SwiGLU  down(silu(gate x) * (up x)).  MOEV_FFN_GPTOSS is the published GPT-OSS expert:
 *   g = min(gate x + b_gate, 7),  u = clamp(up x + b_up, -7, 7),
 *   h = g * sigmoid(1.702 g) * (u + 1),  out = down h + b_down   (weighted by the router weight). */
typedef enum { MOEV_FFN_SWIGLU = 0, MOEV_FFN_GPTOSS = 1 } moev_ffn_kind;

/* Group-limited routing (n_group > 0), the rule of the published DeepSeek-V3 models; the paper's
 * routing is the plain top-k.  s_e = sigmoid(logit_e), c_e = s_e + router_bias_e; the E experts
 * form n_group contiguous groups; a group's score is the sum of its two largest c; the topk_group
 * best groups are kept (ties: lower index); among their experts the top_k by c (ties: lower id) are
 * selected and emitted in that order; weights use the unbiased scores:
 * w_j = routed_scale * s_j / (sum_j s_j + 1e-20). */

/* FP8 activations in front of both expert GEMMs (what deployed DeepSeek-V3 inference does; the
 * paper does not print the expert FFN).  The input x of the gate / up projections and the input h
 * of the down projection are quantised on the fly per token and per block of 128 consecutive
 * elements of the contraction axis: amax = max |v| over the block, s = amax / 448 (binary32; with
 * POW2 the smallest power of two that is not below it; 1 for an all-zero block), code = e4m3(v / s)
 * rounded to nearest even, and the GEMM sees decode(code) * s.  The router sees the unquantised x.
 * Tensor-core kernels: MOEV_W_FP8E4M3_B128 with H <= 8192 and I <= 4096; other configurations run
 * on the CUDA-core kernels. */
typedef enum { MOEV_ACTQ_NONE = 0, MOEV_ACTQ_FP8_B128 = 1, MOEV_ACTQ_FP8_B128_POW2 = 2 } moev_act_quant;

typedef struct {
  int32_t H;          /* hidden size; multiple of 32 */
  int32_t I;          /* expert intermediate size; multiple of 32 */
  int32_t E;          /* routed experts, 1..512 */
  int32_t top_k;      /* 1..min(E,32) */
  int32_t n_shared;   /* always-on shared experts (weight 1), >= 0 */
  int32_t max_tokens; /* largest gamma this context will be asked to verify, 1..1024 */
  int32_t wfmt;       /* moev_wfmt */
  int32_t afmt;       /* moev_afmt: type of x and y */
  int32_t score;      /* moev_score */
  int32_t impl;       /* moev_impl */
  float routed_scale; /* c in the SIGMOID rule; ignored for SOFTMAX */
  int32_t ffn_kind;   /* moev_ffn_kind; MOEV_FFN_GPTOSS needs n_shared == 0 */
  int32_t n_group;    /* 0 = plain top-k; > 0: group-limited routing (below), needs MOEV_SCORE_SIGMOID, E % n_group == 0 */
  int32_t topk_group; /* groups kept per token, 1..n_group; top_k <= topk_group * E / n_group */
  int32_t act_quant;  /* moev_act_quant */
} moev_config;

/* One layer's parameters.  Layouts, row-major, last index contiguous:
 *   router_w            [E, H]  float32
 *   w_gate, w_up        [E, I, H]   in wfmt     (K = H)
 *   w_down              [E, H, I]   in wfmt     (K = I)
 *   s_*   FP8 : float32 [E, ceil(N/128), ceil(K/128)]   (N = rows of the matrix)
 *         MXFP4: uint8  [E, N, K/32]                     else NULL
 *   sh_*  the same for the n_shared shared experts (leading dim n_shared), NULL if none.
 * Every pointer must be 16-byte aligned; on the tensor-core path (moev_resolved_impl ==
 * MOEV_IMPL_TCGEN05) the six expert weight tensors w_* and sh_* must be 32-byte aligned (they
 * are read through TMA descriptors).  A misaligned pointer is rejected with MOEV_EINVAL. */
typedef struct {
  const float* router_w;
  const void *w_gate, *w_up, *w_down;
  const void *s_gate, *s_up, *s_down;
  const void *sh_gate, *sh_up, *sh_down;
  const void *sh_s_gate, *sh_s_up, *sh_s_down;
  const float *b_gate, *b_up, *b_down; /* MOEV_FFN_GPTOSS: fp32 biases [E,I], [E,I], [E,H]; NULL = zero */
  const float* router_bias;            /* n_group > 0: fp32 score-correction bias [E]; NULL = zero */
  /* Optional prefetch hint (Sec. 4.1, Eq. 4: the predictor's expert set for this layer): DEVICE list of
   * n_predicted expert ids whose weights the first routing kernel pulls into the L2 while the router
   * runs, next to the shared experts' (only when moev_prefetch_enable switched the prefetch on).  A wrong prediction costs only
   * bandwidth; results never depend on the hint.  At most what fits an 80 MB share of the L2 is taken
   * (the first entries of the list).  NULL / 0 = no hint. */
  const int32_t* predicted_ids;
  int32_t n_predicted;
} moev_layer;

/* Outputs.  y and n_active are required; the others are diagnostics and may be NULL.
 *   y          [gamma, H] in afmt
 *   topk_ids   [gamma, k] int32   expert ids in descending-logit order
 *   topk_w     [gamma, k] float32 router weights
 *   union_ids  [E]        int32   first U entries: active experts, ascending (Eq. 1)
 *   offsets    [E+1]      int32   first U+1 entries: exclusive scan of tokens per active expert
 *   perm       [gamma*k]  int32   assignments a = t*k+j stably sorted by expert id
 *   n_active   [1]        int32   U = size of the union (shared experts not counted)       */
typedef struct {
  void* y;
  int32_t* topk_ids;
  float* topk_w;
  int32_t* union_ids;
  int32_t* offsets;
  int32_t* perm;
  int32_t* n_active;
} moev_out;

/* Create a context for one layer shape on the current CUDA device; allocates the device
 * workspace (router logits, grouping tables, fp32 intermediates).  MOEV_EINVAL on a bad
 * config, MOEV_EUNSUPPORTED when the device is not compute capability 10.x, MOEV_ENOMEM /
 * MOEV_ECUDA on allocation failure.  *out is NULL on failure. */
moev_status moev_create(const moev_config* cfg, moev_ctx** out);

/* Free the workspace.  The caller must have synchronised the streams it used. */
moev_status moev_destroy(moev_ctx* ctx);

/* Verify gamma tokens (1 <= gamma <= max_tokens): x [gamma, H] in afmt (device).
 * Enqueues the whole path on cuda_stream (a cudaStream_t, may be NULL for the default
 * stream) and returns without waiting.  Invalid arguments are rejected with MOEV_EINVAL
 * before anything is launched. */
moev_status moev_verify(moev_ctx* ctx, const moev_layer* layer, const void* x, int32_t gamma,
                        const moev_out* out, void* cuda_stream);

/* The same path for callers whose activations live in HOST memory: x_host [gamma, H]
 * (pinned memory recommended) is copied to the device, the layer runs, and y_host
 * [gamma, H] plus *n_active_host are copied back, all on cuda_stream; the call waits for
 * the stream before returning so the host buffers are valid.  Weights stay on the device. */
moev_status moev_verify_host(moev_ctx* ctx, const moev_layer* layer, const void* x_host,
                             int32_t gamma, void* y_host, int32_t* n_active_host,
                             void* cuda_stream);

/* Wait for cuda_stream and read the device status word: MOEV_OK, or MOEV_ETIMEOUT if a
 * bounded device-side wait gave up (the outputs of that call are then undefined). */
moev_status moev_status_sync(moev_ctx* ctx, void* cuda_stream);

/* Text of the last error on this context ("" if none).  Owned by the context. */
const char* moev_last_error(const moev_ctx* ctx);

/* Bytes of one expert's three matrices including scale factors (Fig. 1(c): the FP8
 * DeepSeek-V3.1 expert is 3*7168*2048 = 44 040 192 code bytes, + 10 752 scale bytes). */
size_t moev_expert_bytes(const moev_config* cfg);

/* Code bytes only (the paper's 44.04 MB figure). */
size_t moev_expert_code_bytes(const moev_config* cfg);

/* Number of kernels one moev_verify call launches on this context (for launch accounting; calls
 * of at most 32 tokens with plain top-k routing take two routing launches, others three -- a
 * context whose max_tokens exceeds 32 reports the larger figure), and which FFN implementation
 * it resolved to (a moev_impl value, never AUTO). */
int32_t moev_launches_per_call(const moev_ctx* ctx);
int32_t moev_resolved_impl(const moev_ctx* ctx);

/* Per-kernel device time of a call, measured with CUDA events recorded on the call's
 * stream between its kernels.  moev_profile_enable(ctx, 1) turns the event records on (at
 * most 512 calls are kept between reads), 0 off.  moev_profile_read waits for the stream and
 * writes mean_us[0..5], the mean duration in microseconds of: router partial logits, top-k
 * with exact refinement, grouping (union / permutation), first FFN kernel (the fused
 * tensor-core kernel, or SIMT gate/up), second FFN kernel (SIMT down; 0 on the fused path),
 * finalize; then the number of calls averaged, and resets the accumulator. */
moev_status moev_profile_enable(moev_ctx* ctx, int32_t on);
moev_status moev_profile_read(moev_ctx* ctx, void* cuda_stream, double* mean_us /*[6]*/,
                              int32_t* calls);

/* Working time of the tensor-core expert kernel inside a call as the call really runs (the event
 * records above switch the dependent launches off, so their interval for a kernel includes its
 * launch gap and its set-up, which a real call hides behind the routing kernels).  With
 * moev_ffn_span_enable(ctx, 1) every CTA of the expert kernel stores the device's global timer when
 * the routing kernels release it and when it leaves (two 8-byte stores per CTA and call; nothing
 * else changes).  moev_ffn_span_read waits for the stream and writes to span_us (host) the time in
 * microseconds from the earliest release to the latest exit in the most recent call, or 0 when no
 * tensor-core expert kernel has run with the stamps on (the CUDA-core path does not stamp).  The
 * paper has no counterpart: a measurement aid for its Fig. 1(a) quantity, latency against the
 * number of active experts. */
moev_status moev_ffn_span_enable(moev_ctx* ctx, int32_t on);
moev_status moev_ffn_span_read(moev_ctx* ctx, void* cuda_stream, double* span_us);

/* Weight prefetch by the first routing kernel (off by default): the shared experts' matrices and
 * those of the layer's predicted_ids are pulled into the L2 while the routing kernels run, so the
 * expert kernel finds them on chip (Sec. 3: the verification cost is expert-weight traffic from
 * HBM; what is known to be needed before the router decides need not wait for it).  Measured on
 * B200 it does not pay: the L2 delivers these bytes only slightly faster than HBM does, and the
 * prefetch traffic delays the latency-bound routing kernels by more than the expert kernel gains. */
moev_status moev_prefetch_enable(moev_ctx* ctx, int32_t on);

/* Several independent layers in one call (multi-layer pipelining; the paper has no counterpart:
 * its prototype runs layer by layer).  Equivalent to n_layers calls of moev_verify on the same
 * stream with layers[l], x[l], outs[l] and the same gamma, except that the first kernel of layer
 * l + 1 is enqueued as a programmatic dependent launch: its CTAs occupy the SMs that layer l's
 * expert kernel has already left, so the router of the next layer overlaps the tail of the
 * previous one.  The inputs x[l] must not depend on the outputs of earlier layers of the same
 * call (independent requests, or hidden states that are already available); results are the same
 * as those of separate calls.  layers / x / outs are HOST arrays of n_layers entries whose
 * pointers are DEVICE pointers.  Errors as moev_verify; nothing is enqueued for layers after the
 * first failing one. */
moev_status moev_verify_pipeline(moev_ctx* ctx, int32_t n_layers, const moev_layer* layers,
                                 const void* const* x, int32_t gamma, const moev_out* outs,
                                 void* cuda_stream);

/* Consecutive dependent layers in one call: layer l + 1 verifies the output of layer l (Sec. 5 /
 * Table 13: a verification pass runs the model's 36 - 94 MoE layers one after another; the
 * attention between them is outside this library and is the identity here).  x0 [gamma, H] is the
 * input of layers[0]; outs[l].y [gamma, H] (afmt, required for every layer) is both the result of
 * layer l and the input of layer l + 1.  Same results as n_layers calls of moev_verify with those
 * inputs; every kernel of the call is a programmatic dependent launch of its predecessor, the
 * first kernel of a layer included: it is scheduled while the previous layer drains, starts the
 * optional weight prefetch at once, and waits for the previous layer's output before it reads it.
 * layers / outs are HOST arrays whose pointers are DEVICE pointers.  Errors as moev_verify. */
moev_status moev_verify_chain(moev_ctx* ctx, int32_t n_layers, const moev_layer* layers, const void* x0,
                              int32_t gamma, const moev_out* outs, void* cuda_stream);

/* Cost-aware draft selection: Algorithm 1 of the paper (Sec. 4.2, Eqs. 7-10), the step that
 * runs between drafting and verification and decides which gamma draft-tree nodes are verified.
 *   n, parent [n]   draft tree in topological order: parent[i] < i, parent[root] = -1
 *   P [n]           cumulative draft probability of every node (float32)
 *   pred [n, W]     predicted expert set of every node as a bitmap over (layer, expert) pairs,
 *                   bit l*E + e, W = ceil(L*E / 32) 32-bit words (Eq. 4)
 *   buffer0 [W]     initial expert buffer B_0, or NULL for the empty set
 *   E_traj(i) = OR of pred along root -> i (Eq. 7);  cost = |E_traj(i) \ B| (Eq. 8);
 *   score = P(i) / (cost + eps) (Eq. 9), evaluated in binary32;  gamma rounds of arg-max
 *   (exact ties: the lowest index, so a parent precedes its children), each followed by
 *   B |= E_traj(chosen).  global_cost != 0 selects the ablation variant of Eq. 10: cost =
 *   |E_traj(i)|, buffer not updated.
 * Outputs: selected [gamma] (first min(gamma, n) entries, in selection order), costs [gamma]
 * (cost of each choice when it was made; may be NULL), buffer_out [W] (final B; may be NULL),
 * n_selected [1] (may be NULL; -1 if a bounded device wait expired).  traj_workspace is
 * caller-provided scratch of n * W + 516 32-bit words (the path footprints, then control words);
 * it must be 16-byte aligned (the control words are accessed as 64-bit and 128-bit quantities),
 * otherwise MOEV_EINVAL.
 * All pointers are DEVICE pointers; one kernel (for bitmaps too long for one CTA's shared memory:
 * one memset and one cooperative kernel over several CTAs) is enqueued on cuda_stream; nothing is
 * allocated.
 * MOEV_EINVAL for n outside 1..4096, W < 1, gamma < 1, eps <= 0, null required pointers, or
 * tables too large for shared memory (3 n + 4 W words above ~50 000). */
moev_status moev_select_drafts(int32_t n, int32_t W, const int32_t* parent, const float* P,
                               const uint32_t* pred, const uint32_t* buffer0, int32_t gamma, float eps,
                               int32_t global_cost, uint32_t* traj_workspace, int32_t* selected,
                               int32_t* costs, uint32_t* buffer_out, int32_t* n_selected,
                               void* cuda_stream);

/* Router top-k without any allocation.  (The paper has no counterpart: this entry point
 * exists for the integration constraints of some callers, not for the method.)
 *
 * Who needs it: code that runs where cudaMalloc is forbidden or unavailable -- inside a
 * memory-pool-managed serving process that has handed all device memory to its own allocator,
 * in a latency-critical thread that may not take the allocator's lock, or before a framework
 * has set up its caching allocator.  Such callers cannot create a moev_ctx (moev_create
 * allocates the workspace), but may still want the routing decision of a layer.
 *
 * Computes, for the gamma tokens x [gamma, H] (afmt of cfg), the same topk_ids [gamma, k] and
 * topk_w [gamma, k] that moev_verify writes for plain top-k routing.  Of cfg it reads H, E,
 * top_k, afmt, score, routed_scale and max_tokens (gamma <= max_tokens); the other fields must
 * merely be valid.  Group-limited routing needs the layer's score-correction bias, which this
 * entry point does not take: cfg->n_group > 0 is rejected with MOEV_EINVAL.  All pointers are
 * DEVICE pointers owned by the caller.  The split-K partial logits live in a fixed 20 MiB array compiled into the
 * library (held by every GPU that loads it until the process exits) instead of a context
 * workspace; moev_route_topk_static_scratch_floats() returns how many of its 5 242 880 floats a
 * problem needs, and problems that need more are rejected with MOEV_EINVAL.  The call itself
 * calls no cudaMalloc/cudaFree and no allocating library routine; it enqueues two kernels on
 * cuda_stream and returns without waiting.
 *
 * The first call on a device looks up the device address of the array (once per device, with
 * that device current); make that first call before starting any stream capture.  All calls
 * share the one array: nothing in it has to be cleared between calls (each call overwrites
 * what it reads), but two calls whose kernels overlap on the GPU (different streams, or
 * several host threads) race on it and give undefined results -- serialise them. */
moev_status moev_route_topk_static(const moev_config* cfg, const float* router_w, const void* x,
                                   int32_t gamma, int32_t* topk_ids, float* topk_w,
                                   void* cuda_stream);
size_t moev_route_topk_static_scratch_floats(int32_t H, int32_t E, int32_t gamma);

/* ======================================================================================
 * The rest of a decoder block.  A verification pass (Sec. 5) runs, between two MoE layers, the
 * residual addition and norm, the projections, and attention of the draft tree over the cached
 * context; the paper takes these from its host framework.  The operators below are stateless like
 * moev_select_drafts: no context, nothing allocated, nothing kept between calls, everything
 * enqueued on cuda_stream of the current device, MOEV_EINVAL before anything is launched.  Row strides are in
 * elements and are not looked at where a tensor has one row; tensors of no rows, and a batch's arrays without sequences, may be NULL.
 * ====================================================================================== */

/* s = x + residual (binary32),  y = s / sqrt(mean(s^2) + eps) * w, and optionally the FP8 1x128
 * quantisation of y (moev_act_quant), from the unrounded y.  residual_out receives s rounded to afmt.
 * Outputs may be the inputs they replace (same pointer, stride and type).  Any H from 1 to 32768 and any stride >= H;
 * rows on 16-byte boundaries with H a multiple of 8 are read and written by full vectors. */
typedef struct {
  int32_t n, H;
  int32_t afmt;            /* moev_afmt of x, residual, residual_out, y */
  int32_t wfmt;            /* moev_afmt of w */
  float eps;
  int32_t act_quant;       /* moev_act_quant; codes and scales are given exactly when it is not NONE */
  const void* x;           /* [n, H] */
  const void* residual;    /* [n, H] or NULL = 0 */
  const void* w;           /* [H] */
  void* residual_out;      /* [n, H] or NULL */
  void* y;                 /* [n, H] or NULL; one of residual_out, y and codes is given */
  uint8_t* codes;          /* [n, H] e4m3 or NULL */
  float* scales;           /* [n, ceil(H / 128)] or NULL */
  int64_t x_stride, residual_stride, residual_out_stride, y_stride, codes_stride;
} moev_norm;
moev_status moev_add_rmsnorm(const moev_norm* p, void* cuda_stream);

/* y [n, N] = x [n, K] W^T + bias for bf16 rows x and a 4-bit weight W [N, K] with group scales:
 *   MOEV_W_INT4   codes uint8 [N, K / 2], scales bfloat16 [N, K / group], group 32, 64 or 128
 *   MOEV_W_MXFP4  codes uint8 [N, K / 2], scales uint8 [N, K / 32], group 32
 * codes on a 4-byte boundary.  K is a multiple of 32 and of group; N is free; MXFP4 scales lie between 2^-100 and 2^100.  moev_w4_pack lays a weight out
 * once in the order in which the kernel streams it (moev_w4_packed_bytes bytes, 16-byte aligned,
 * caller-owned); moev_linear_w4 reads the packed form.  Products are exact (MXFP4: of x held to 2^-40 of the largest of
 * its 128 columns, where that is above 2^-111), sums are binary32; y is yfmt (moev_afmt).
 * Made for the few rows of a draft tree: more than 32 rows are taken 32 at a time, each pass reading the weight. */
typedef struct {
  int32_t N, K, wfmt, group;
} moev_linear;
size_t moev_w4_packed_bytes(const moev_linear* p); /* 0 for an invalid description */
moev_status moev_w4_pack(const moev_linear* p, const void* codes, const void* scales, void* packed, void* cuda_stream);
moev_status moev_linear_w4(const moev_linear* p, const void* packed, const float* bias /* [N] or NULL */, const void* x,
                           int64_t x_stride, int32_t n, void* y, int64_t y_stride, int32_t yfmt, void* cuda_stream);

/* Paged key / value cache in 8 bits.  value = code * scale, one scale per page and kv head for K and
 * one for V, positive, a power of two wherever moev_cache_append wrote it.
 *   k [n_pages, n_kv_heads, page, head_dim] e4m3      v [n_pages, n_kv_heads, head_dim, page] e4m3
 *   k_scale, v_scale [n_pages, n_kv_heads] float32
 * page is 16, 32, 64 or 128, head_dim 64 or 128; k and v on 16-byte boundaries.
 * Every slot below ctx_len counts as context for all drafts, in the order of the slots, and nothing here moves a token to
 * another slot.  After a tree has been verified ctx_len may grow by the length of the accepted path where that is drafts 0, 1, 2,
 * .. in this order (a chain, or the tree's first path).  Any other accepted path has to be written once more, as a chain: with
 * moev_cache_append from the k and v that the caller kept, or by running the accepted tokens through the blocks again
 * (moev_verify_blocks keeps k and v in no form but the cache's). */
typedef struct {
  int32_t n_pages, page, n_kv_heads, head_dim;
  uint8_t *k, *v;
  float *k_scale, *v_scale;
} moev_kv_cache;

/* The drafts of one call.  Sequence b has the token rows cu[b] .. cu[b+1] - 1 (its drafts, in an
 * order in which parents come first) and ctx_len[b] tokens in the cache before them; its page c is
 * page_table[b * table_cols + c]; draft i lives in slot ctx_len[b] + i.  parent [n_tokens]: index of a
 * draft's parent within its sequence, -1 (or anything that is not an earlier draft) for one that
 * continues the context; the position of a draft is ctx_len[b] + the number of its ancestors.  NULL:
 * a chain, draft i continues draft i - 1.  A sequence may have no draft or no context.
 *   max_drafts >= every sequence's drafts (<= 1024 with parents), max_len >= every ctx_len + drafts:
 * host bounds that size the launches.  The arrays are device data: a sequence that breaks the bounds is
 * left out, a page id outside the pool hides its keys, and both raise *status (may be NULL; 1 sequence,
 * 2 page id, 3 position behind the rotation table, 4 a bounded wait of the attention kernel ran out and its
 * outputs are undefined; the largest of what is found and what was there, never cleared).  Rows that belong to no sequence are left as they are. */
typedef struct {
  int32_t n_seq, n_tokens, max_drafts, max_len, table_cols;
  const int32_t *cu, *ctx_len, *page_table, *parent;
  int32_t* status;
} moev_draft_batch;

/* Write the drafts' keys and values (bf16 [n_tokens, n_kv_heads * head_dim], row strides multiples of 8
 * elements, as those of q and q_out) to the cache.  rope [rope_rows, head_dim] float32 (head_dim / 2 cosines, then as many sines,
 * by position), or NULL for no rotation: dimensions i and i + head_dim / 2 of K, and of q where it is
 * given, are rotated in binary32; q_out (may be q) receives the queries in bf16.  A page's scale is the smallest power of
 * two that brings its largest magnitude to 448 or less; a page that held tokens before (ctx_len inside it) keeps
 * the larger of that and its old scale, and its tokens are rescaled when it grows.  The pages that receive tokens belong to
 * one sequence each.  A NaN stays NaN, an infinity becomes the largest finite value.  k, v, q, q_out and rope lie on 16-byte
 * boundaries. */
moev_status moev_cache_append(const moev_kv_cache* cache, const moev_draft_batch* batch, const void* k, int64_t k_stride,
                              const void* v, int64_t v_stride, const float* rope, int32_t rope_rows, const void* q,
                              int64_t q_stride, int32_t n_heads, void* q_out, int64_t q_out_stride, void* cuda_stream);

/* Attention of the drafts over the cache (their own keys are in it).  q, out bf16 [n_tokens, n_heads *
 * head_dim] (row strides multiples of 8 elements), n_heads a multiple of n_kv_heads (query head h reads kv head h / (n_heads / n_kv_heads)).
 * A draft sees the context and, of the drafts, itself and its ancestors; with window > 0 of all these
 * only the last window positions (pages that end before ctx_len + 1 - window may have been given back: their entries in the
 * page table are not looked at).  scores are multiplied by scale (> 0); sinks [n_heads] float32 (or
 * NULL) join the denominator.  lse [n_tokens, n_heads] float32 (or NULL): natural log of the denominator.  q and out lie on
 * 16-byte boundaries.
 * Roundings: q is held to 2^-12 of an element or 2^-18 of its row's largest, whichever is more; scores, sums and lse are
 * binary32; a key's probability times its page's V scale is rounded once to 11 bits (2^-11), or by 2^-28 of the row's largest
 * such product of a key whose V is not all zero, whichever is more (V scales below 2^-48 of the sequence's largest: or
 * by 2^-76 of the largest probability times that scale).  Pages that a row does not see or gives no weight do not enter.
 * workspace: moev_cache_attend_workspace bytes for the same sizes (16-byte aligned; 0 = none needed);
 * its contents do not matter before a call or after it, but calls that may overlap need one each. */
size_t moev_cache_attend_workspace(const moev_kv_cache* cache, const moev_draft_batch* batch, int32_t n_heads, int32_t window);
moev_status moev_cache_attend(const moev_kv_cache* cache, const moev_draft_batch* batch, const void* q, int64_t q_stride,
                              int32_t n_heads, float scale, int32_t window, const float* sinks, void* out,
                              int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Whole decoder blocks of a verification pass: moev_verify_chain with what stands between two MoE layers
 * in the place of the identity.  Per block, on the residual stream h:
 *   x = norm(h, attn_norm);  q | k | v = qkv x;  moev_cache_append;  a = moev_cache_attend;  h += o a;
 *   x = norm(h, ffn_norm);   h += MoE(x)  (moev_verify with ctx)
 * and after the last one, where final_norm is given, final_out = norm(h, final_norm). */
typedef struct {
  const void *attn_norm, *ffn_norm; /* bfloat16 [H], 16-byte aligned as the other norm, hidden and final_out */
  moev_linear qkv, o;               /* [(n_heads + 2 n_kv_heads) head_dim, H] and [H, n_heads head_dim] */
  const void *qkv_packed, *o_packed;
  const float *qkv_bias, *o_bias;   /* or NULL */
  const float* sinks;               /* [n_heads] or NULL */
  int32_t window;                   /* 0: the whole context */
  moev_kv_cache cache;              /* the block's own */
  moev_layer moe;
} moev_block;
typedef struct {
  int32_t n_heads;
  float eps, scale;                 /* norms; attention scores (0 = head_dim ^ -1/2) */
  const float* rope;                /* [rope_rows, head_dim] or NULL */
  int32_t rope_rows;
  const void* final_norm;           /* bfloat16 [H] or NULL */
  void* final_out;                  /* bfloat16 [batch->n_tokens, H], given exactly when final_norm is */
} moev_block_options;

/* hidden bfloat16 [batch->n_tokens, H] (contiguous): h before the first block, overwritten by h after the last.  outs[l].y
 * receives the MoE output of block l; the other fields are diagnostics as in moev_verify.  The context is one for
 * bfloat16 activations with max_tokens >= batch->n_tokens.  Every token row goes through the MoE layers: rows of no
 * sequence (attention output zero) would widen the expert union.  workspace: moev_verify_blocks_workspace bytes for the
 * same sizes (16-byte aligned, contents of no matter), one per call in flight.  blocks and outs are HOST arrays of
 * n_blocks entries whose pointers are DEVICE pointers.  Everything but the MoE layers' own pointers (moev_verify checks those
 * when it is their turn) is checked before the first launch.  Asynchronous on cuda_stream; a time-out of the attention kernel is
 * reported by moev_status_sync like one of the MoE layers'. */
size_t moev_verify_blocks_workspace(const moev_ctx* ctx, int32_t n_blocks, const moev_block* blocks, const moev_draft_batch* batch,
                                    const moev_block_options* options);
moev_status moev_verify_blocks(moev_ctx* ctx, int32_t n_blocks, const moev_block* blocks, const moev_draft_batch* batch,
                               const moev_block_options* options, void* hidden, const moev_out* outs, void* workspace,
                               size_t workspace_bytes, void* cuda_stream);

/* ======================================================================================
 * In front of and behind a verification pass: the prompt's own pass (attention over whole prompts, projections of many rows), the
 * tables that describe a batch, and what is read off the logits.  Stateless as the operators above; the same rules for streams,
 * strides, empty tensors and errors.
 * ====================================================================================== */

/* Packed prompts.  Sequence b has the token rows cu[b] .. cu[b+1] - 1 and the key rows cu_k[b] .. cu_k[b+1] - 1; its tokens are the
 * last of its keys: token i stands at position keys - tokens + i (below 0, where there are fewer keys than tokens, it sees nothing).
 * cu_k NULL: cu, and n_keys = n_tokens.  max_tokens >= every sequence's tokens, and 1 at least, sizes
 * the launch (n_seq * max_tokens rows of tokens, whether they are there or not: one long prompt among many short ones is better a call
 * of its own).  A sequence that breaks
 * the bounds is left out and raises *status (may be NULL) to 1; 4: a bounded wait ran out, outputs are undefined.  Rows that belong to
 * no sequence are left as they are. */
typedef struct {
  int32_t n_seq, n_tokens, n_keys, max_tokens;
  const int32_t *cu, *cu_k;
  int32_t* status;
} moev_prompt_batch;

/* Causal attention over packed prompts.  q, out bfloat16 [n_tokens, n_heads * head_dim], k, v bfloat16 [n_keys, n_kv_heads *
 * head_dim], row strides multiples of 8 elements, on 16-byte boundaries; query head h reads kv head h / (n_heads / n_kv_heads);
 * head_dim 64 or 128.  A token sees the keys of its sequence up to its own position, with window > 0 only the last window of
 * those.  Scores are multiplied by scale (> 0); sinks [n_heads] float32 (or NULL) join the denominator (an infinite one leaves the keys nothing).  lse [n_tokens, n_heads]
 * float32 (or NULL): natural log of the denominator.  A row that sees nothing has output 0 and lse -infinity (or the
 * sink as it is given).  What a row does not see does not reach it, NaN and infinity included.  out overlaps none of the inputs.
 * Rotary positions: moev_cache_append rotates any heads that it is given as q; with q the [query heads | key heads] columns of a fused
 * projection (n_heads + n_kv_heads of them), q_out holds the rotated queries and keys for this call, next to the cache's own.
 * Roundings: scores, sums and lse are binary32, a probability is rounded once to bfloat16 for the product with v.  Sums are taken
 * before they are divided: 2^8 times the sum of the |v| that a row sees has to stay below 2^128. */
typedef struct {
  int32_t n_heads, n_kv_heads, head_dim, window;
  float scale;
  const void *q, *k, *v;
  const float* sinks;
  void* out;
  float* lse;
  int64_t q_stride, k_stride, v_stride, out_stride;
} moev_prompt;
moev_status moev_prompt_attend(const moev_prompt_batch* batch, const moev_prompt* p, void* cuda_stream);

/* Rows of x (xfmt moev_afmt, [n, K]) as 8-bit integers with a scale per row: scale = max |x| / 127 in binary32 (1 for a row of zeros),
 * code = x / scale (binary32), rounded to the nearest integer, ties to even, at most 127 in magnitude.  A row with a NaN or an infinity has scale NaN and codes
 * 0.  K from 1 to 2^24. */
moev_status moev_quant_rows(const void* x, int64_t x_stride, int32_t xfmt, int32_t n, int32_t K, int8_t* codes, int64_t codes_stride, float* scales,
                            void* cuda_stream);

/* y [n, N] = x W^T + bias with W = w * w_scales (int8 [N, K], contiguous on a 16-byte boundary; a scale per channel) and x as
 * moev_quant_rows gives it.  K is a multiple of 16 up to 131056, N is free.  The sums are exact; y = (sum * x_scale) * w_scale + bias
 * in binary32 (the sum rounded to it, the first product rounded, the rest rounded once), then yfmt (moev_afmt).
 * moev_linear_i8 takes codes (row stride a multiple of 16, 16-byte boundary) and scales; moev_linear_w8 takes x (xfmt) and brings it
 * to codes, of more than a row or two in the workspace: moev_linear_w8_workspace bytes (16-byte aligned, contents of no matter), one per call in
 * flight.  y overlaps none of the inputs.
 * *status (may be NULL) is raised to 4 where a bounded wait ran out: y is undefined then. */
typedef struct {
  int32_t N, K;
  const int8_t* w;
  const float *w_scales, *bias; /* [N]; bias may be NULL */
  int32_t* status;
} moev_w8;
moev_status moev_linear_i8(const moev_w8* p, const int8_t* x, int64_t x_stride, const float* x_scales, int32_t n, void* y, int64_t y_stride, int32_t yfmt,
                           void* cuda_stream);
size_t moev_linear_w8_workspace(const moev_w8* p, int32_t n);
moev_status moev_linear_w8(const moev_w8* p, const void* x, int64_t x_stride, int32_t xfmt, int32_t n, void* y, int64_t y_stride, int32_t yfmt,
                           void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Log probabilities under rows of logits z [n, V] (afmt, row stride `stride`; n up to 2^27, V to 2^30), l = scale * z (scale > 0: one over the temperature):
 *   lse = log sum_v exp(l_v)     logprobs[i, j] = l[ids[i, j]] - lse     entropy = lse - sum_v p_v l_v
 *   top_ids[i, 0..k-1]: the k largest z of the row, descending, ties to the lower id; top_logprobs: theirs
 * ids [n, m] int32: an id outside the vocabulary (padding) has -infinity.  ids and logprobs are given exactly with m > 0, top_ids exactly
 * with k > 0 (0 to 32, at most V); entropy, lse and top_logprobs may be NULL.  z of -infinity (masked) has probability 0.  In a row
 * with a NaN or +infinity, or without any finite z, the numbers are NaN (lse of nothing: -infinity); NaNs are no alternatives, a
 * row of fewer than k others ends with id -1 and NaN.  Statistics are binary32, logprobs are taken from them in 64 bits. */
typedef struct {
  int32_t n, V, m, k;
  int32_t afmt;
  float scale;
  const void* logits;
  int64_t stride;
  const int32_t* ids;
  float *logprobs, *entropy, *lse;
  int32_t* top_ids;
  float* top_logprobs;
} moev_logprobs;
moev_status moev_token_logprobs(const moev_logprobs* p, void* cuda_stream);

/* The tables of a batch's next call from the lengths of its sequences, as moev_draft_batch takes them: ctx_len [n_seq] tokens in the
 * cache, new_len [n_seq] tokens to come.
 *   cu [n_seq + 1]: exclusive sums of new_len
 *   page_table [n_seq, table_cols]: sequence b holds columns 0 .. ceil(ctx / page) - 1; the columns from there to ceil((ctx + new) / page) - 1
 *     receive the next pages of the free list, in the order of the sequences; nothing else is written
 *   positions, slots [n_tokens] (either may be NULL): position of a token row in its sequence and its slot in the cache,
 *     page id * page + position % page; -1 in rows behind the last sequence
 *   taken [1] (may be NULL): pages taken
 * free_pages [n_free] from entry *free_first on (NULL: 0).  None of these inputs is changed: a caller that keeps the list on the device
 * adds taken to free_first.  *status (may be NULL, the largest code stays): 1 a sequence of negative length or beyond table_cols
 * pages counts as one of no tokens, 2 the free list is too short or holds a page id that has no slot (entry or slot -1), 3 more tokens than
 * n_tokens (rows beyond are not written).  page is 16, 32, 64 or 128. */
typedef struct {
  int32_t n_seq, n_tokens, page, table_cols, n_free;
  const int32_t *ctx_len, *new_len, *free_pages, *free_first;
  int32_t *page_table, *cu, *slots, *positions, *taken, *status;
} moev_pages;
moev_status moev_build_pages(const moev_pages* p, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* MOEV_H_ */
