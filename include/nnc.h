/*
 * nnc.h -- C ABI of the B200-native Qwen3 forward pass (libnnc.so).
 *
 * The paper frames LLM deployment as "prepare the model once ahead of time, then run a prompt phase followed
 * by token-by-token decoding at batch 1, reporting decode tokens/s" (Section 4, Evaluation; Section 3.3.1 for
 * laying constants out once where the kernels read them).  The three main calls mirror that framing:
 *
 *     nnc_model_create(config, weights)   one-time weight repack + workspace carve-up
 *     nnc_prefill(tokens)                 the prompt phase
 *     nnc_decode_step(token) -> logits    one decoding step (the HBM-bound hot path)
 *
 * Conventions
 *   - Plain C, no exceptions.  Every function that can fail returns an int status: NNC_OK (0) or a negative
 *     nnc_status.  nnc_last_error() gives a human-readable line for the last failure of that model.
 *   - "DEVICE pointer" = CUDA global memory on the device that was current in nnc_model_create.
 *     "HOST pointer" = ordinary host memory.  Unless a parameter says HOST it is a DEVICE pointer.
 *   - The library never allocates or frees device memory: the caller supplies one workspace at create time
 *     (nnc_workspace_bytes tells how large) and owns it; it must stay alive until nnc_model_destroy.
 *   - All work is enqueued on the CUDA stream given at create time (a cudaStream_t passed as void*; NULL =
 *     the legacy default stream) and is asynchronous unless a function says it synchronises.
 *   - Errors that the host can see (bad configuration, null pointers, cache overflow, batch too large,
 *     workspace too small) are returned before anything is launched and leave the model unchanged.  Launch
 *     errors reported by the CUDA runtime are returned as NNC_ERR_CUDA.  Kernels never trap or assert; every
 *     device-side wait is bounded and reports through a status word that nnc_device_status() reads.
 *   - All matrices are bf16, row-major W[out][in] (y = W x); bf16 values are IEEE bfloat16 bit patterns.
 *   - The sequences of a batch advance in lock step: they all hold the same number of cached positions.
 */
#ifndef NNC_H_
#define NNC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    NNC_OK = 0,
    NNC_ERR_INVALID_ARG = -1,   /* null pointer, non-positive size, unsupported shape */
    NNC_ERR_WORKSPACE = -2,     /* workspace smaller than nnc_workspace_bytes(), or misaligned */
    NNC_ERR_CAPACITY = -3,      /* cache length + new tokens > max_seq, batch > max_batch, tokens > max_tokens */
    NNC_ERR_CUDA = -4,          /* a CUDA runtime / driver call failed; see nnc_last_error */
    NNC_ERR_DEVICE_STATUS = -5  /* a kernel reported a bounded wait that ran out, or a cache address out of range */
} nnc_status;

typedef struct nnc_model nnc_model; /* opaque; host struct owned by the library */

/* Model and capacity description.  Supported: head_dim == 128; n_q_heads a multiple of n_kv_heads with at
 * most 8 query heads per KV head; hidden, intermediate multiples of 64; everything positive. */
typedef struct {
    int32_t n_layers, hidden, n_q_heads, n_kv_heads, head_dim, intermediate, vocab;
    int32_t max_seq;        /* KV-cache capacity in positions per sequence */
    int32_t max_batch;      /* sequences held in the cache */
    int32_t max_tokens;     /* most tokens one nnc_prefill call may carry (batch * n_tokens); >= max_batch */
    int32_t tie_embeddings; /* 1: the lm_head is the embedding matrix */
    float rms_eps;          /* 1e-6 for Qwen3 */
    float rope_theta;       /* 1e6 for Qwen3 */
    int32_t tc_operands;    /* operand feed of the tensor-core path (prompt phase, batched decode).  The residual stream
                             * stays fp32 everywhere; this only says how an activation matrix enters a tcgen05.mma.
                             * 0 (default): calls with more than 128 tokens multiply the attention output, the MLP input and
                             *    the SwiGLU output as ONE fp16 term with fp16 copies of Wo, Wgate/up and Wdown (made at
                             *    create time when max_tokens > 128; scaled by a power of two per matrix, exact for bf16
                             *    weights), and the QKV input -- the operand deep models are sensitive to -- as TWO bf16
                             *    terms (value + rounding residual, ~16 mantissa bits).  Calls with at most 128 tokens use
                             *    two bf16 terms throughout (they are bound by streaming the weights, not by the MMAs).
                             * 1: two bf16 terms throughout, no fp16 weight copies (smaller workspace, ~1.8x the tensor work
                             *    of mode 0 in the prompt phase).
                             * 2: one bf16 term throughout (half the tensor work of mode 1; 2^-9 per operand accumulates to
                             *    a few percent of hidden-state error over ~30 layers, outside the parity tolerance). */
    int32_t weight_format;  /* 0 (default): bf16 weights.  1: the second weight precision (the paper evaluates two, Section
                             * 4.1) -- weight-only FP8: at create time every matrix that is multiplied (QKV, O, gate/up,
                             * down, lm_head; a tied embedding is that same matrix) is quantised row by row to E4M3 codes
                             * times a power-of-two scale 2^e per output row (e the smallest integer with max|w| <= 448 *
                             * 2^e, round to nearest even, saturating), and the bf16 copy in the workspace is replaced by
                             * the dequantised values (exact in bf16).  Batch-1 decode streams the codes (half the bytes per
                             * step); the tensor-core paths multiply the dequantised bf16 matrices, so every path computes
                             * the same model: the forward pass on the dequantised weights. */
    int32_t serial_launches; /* 0 (default): kernels are launched with programmatic stream serialization, so a
                             * kernel's set-up and weight prefetch overlap its predecessor's tail.  1: plain stream
                             * order (for debugging and for timing the overlap's worth). */
} nnc_config;

/* Per-layer weights: DEVICE pointers, bf16.  Read only during nnc_model_create (they are repacked into the
 * workspace) and may be freed by the caller afterwards.
 *   wq [n_q_heads*128][hidden]   wk, wv [n_kv_heads*128][hidden]   wo [hidden][n_q_heads*128]
 *   w_gate, w_up [intermediate][hidden]   w_down [hidden][intermediate]
 *   g_in, g_post [hidden] (RMSNorm gains before attention / before the MLP)   g_q, g_k [128] (per-head
 *   query / key RMSNorm gains, shared by the heads of the layer) */
typedef struct {
    const void *wq, *wk, *wv, *wo, *w_gate, *w_up, *w_down;
    const void *g_in, *g_post, *g_q, *g_k;
} nnc_layer_weights;

typedef struct {
    const void *embed;               /* DEVICE [vocab][hidden] */
    const void *lm_head;             /* DEVICE [vocab][hidden]; NULL when tie_embeddings */
    const void *g_final;             /* DEVICE [hidden] */
    const nnc_layer_weights *layers; /* HOST array of n_layers entries (holding DEVICE pointers) */
} nnc_weights;

/* Bytes of workspace nnc_model_create needs for this configuration (repacked weights, KV cache, RoPE table,
 * activations, split-K scratch).  Returns 0 for an invalid configuration.  Pure host arithmetic. */
size_t nnc_workspace_bytes(const nnc_config *config);

/* Ahead-of-time preparation (the paper's "constants laid out once", Section 3.3.1): validates the
 * configuration, carves the workspace (256-byte aligned DEVICE pointer, at least nnc_workspace_bytes), builds
 * the RoPE table on the host in double precision, and repacks the weights on the device: Wq|Wk|Wv are
 * concatenated row-wise, gate/up rows are interleaved pairwise (row 2i = gate_i, row 2i+1 = up_i) so that one
 * warp owns both halves of a SwiGLU output.  Synchronises the stream before returning.  *out is set only on
 * success.  The cache starts empty. */
int nnc_model_create(const nnc_config *config, const nnc_weights *weights, void *workspace,
                     size_t workspace_bytes, void *cuda_stream, nnc_model **out);

/* Releases the host struct, CUDA graphs and tensor maps.  Synchronises the stream.  NULL is ignored. */
void nnc_model_destroy(nnc_model *model);

/* Prompt phase (Section 4: a prompt is processed, then decoding starts).  tokens: int32 [batch][n_tokens],
 * ids in [0, vocab); out-of-range ids are clamped on the device.  The tokens take positions len .. len +
 * n_tokens - 1 of every sequence, their K/V are appended, and len grows by n_tokens.
 * logits: fp32 [batch][vocab] (last position of each sequence), or [batch][n_tokens][vocab] when
 * all_positions != 0; may be NULL to skip the lm_head. */
int nnc_prefill(nnc_model *model, const int32_t *tokens, int32_t batch, int32_t n_tokens, float *logits,
                int32_t all_positions);

/* One decoding step (Section 4: throughput is measured over this stage).  tokens: int32 [batch]; each
 * sequence's token takes position len; len grows by one.  logits: fp32 [batch][vocab].  argmax: int32
 * [batch] or NULL (batch 1 only); lowest index wins ties.  The whole step is one CUDA graph launch, captured on
 * first use for the given buffers and batch size and re-used while they stay the same. */
int nnc_decode_step(nnc_model *model, const int32_t *tokens, int32_t batch, float *logits, int32_t *argmax);

/* End-to-end variants with HOST buffers: copy the tokens to the device, run the step, copy logits (and the
 * argmax, if not NULL) back, and synchronise the stream before returning.  HOST pointers throughout; pinned
 * memory makes the copies faster but is not required.  logits_host may be NULL when only argmax is wanted. */
int nnc_decode_step_host(nnc_model *model, const int32_t *tokens_host, int32_t batch, float *logits_host,
                         int32_t *argmax_host);
int nnc_prefill_host(nnc_model *model, const int32_t *tokens_host, int32_t batch, int32_t n_tokens,
                     float *logits_host, int32_t all_positions);

/* Set the raw cache contents of one layer of one sequence, positions [0, n_pos): k, v DEVICE bf16
 * [n_kv_heads][n_pos][128] (K as the cache stores it: already normalised and rotated).  nnc_set_length then
 * declares how many positions are valid. */
int nnc_kv_import(nnc_model *model, int32_t layer, int32_t batch_index, const void *k, const void *v,
                  int32_t n_pos);
/* Copy the cache of one layer of one sequence, positions [0, n_pos), to k, v (DEVICE, same layout). */
int nnc_kv_export(nnc_model *model, int32_t layer, int32_t batch_index, void *k, void *v, int32_t n_pos);

int nnc_set_length(nnc_model *model, int32_t n_pos); /* cached positions := n_pos (0 empties the cache) */
int32_t nnc_get_length(const nnc_model *model);

/* Parity instrumentation.  taps: DEVICE fp32 [n_layers + 1][rows][hidden] (rows = batch for a decode step,
 * batch * n_tokens for a prefill), receiving the residual stream after the embedding and after every layer of
 * each following call; NULL switches it off.  While a tap is set, decode steps run kernel by kernel instead
 * of through the captured graph (same kernels, same order). */
int nnc_set_hidden_tap(nnc_model *model, float *taps);

/* One decoder layer, one step, batch 1, on a caller-supplied residual-stream vector: x_in, x_out DEVICE fp32
 * [hidden].  The token sits at position len; its K/V are appended to that layer's cache; len is NOT changed
 * (call nnc_set_length to advance). */
int nnc_layer_decode(nnc_model *model, int32_t layer, const float *x_in, float *x_out);

/* Write the ORIGINAL (caller-layout) matrix back from the repacked store: which = 0 wq, 1 wk, 2 wv, 3 wo,
 * 4 w_gate, 5 w_up, 6 w_down; out DEVICE bf16 of that matrix's shape.  Lets a test check that the repack
 * loses nothing (with weight_format 1 the store holds the dequantised values, and those are what comes back). */
int nnc_unrepack(nnc_model *model, int32_t layer, int32_t which, void *out);

/* Reads (and clears) the device status word; synchronises the stream.  0 = no kernel gave up on a wait. */
int nnc_device_status(nnc_model *model, int32_t *status_out /* HOST */);

/* Number of kernels this library launched on behalf of `model` since creation (graph nodes count once per
 * graph launch). */
int64_t nnc_launch_count(const nnc_model *model);

/* Debugging aid.  A library built with -DNNC_BOUNDS_CHECK compares, inside the kernels, the indices that rest on the
 * host's capacity checks (cache positions, matrix row ranges, scratch slots) with their extents; a miss is counted and
 * the access skipped (no trap, no out-of-range access).  This call synchronises the device and returns the number of
 * misses since the last call and the code of the first one (HOST pointers); in a normal build *misses_out is -1.
 * nnc_bounds_check_selftest launches a kernel that touches no memory and, in a checked build, reports one miss with
 * `code` (nothing in a normal build): it shows the counter at work. */
int nnc_bounds_check_report(int32_t *misses_out, int32_t *first_code_out);
int nnc_bounds_check_selftest(int32_t code, void *cuda_stream);

const char *nnc_last_error(const nnc_model *model); /* never NULL; valid until the next call on the model */
const char *nnc_status_string(int status);

/* ---- single operations, exposed for kernel-level tests and isolated timing ----------------------------
 * Each runs on `cuda_stream`, allocates nothing, and returns an nnc_status. */

/* y[T][n_out] = (X + X_lo)[T][n_in] * W[n_out][n_in]^T on the tensor cores (tcgen05, fp32 accumulation in
 * tensor memory).  X, W bf16 row-major (n_in contiguous), n_in a multiple of 64, n_out a multiple of 8.
 * X_lo: NULL, or a second bf16 [T][n_in] matrix (the rounding residual of the activations) multiplied with
 * the same weights into the same accumulator.
 * out_f32 != 0: Y is fp32 (and, if accumulate != 0, Y += product); otherwise Y is bf16. */
int nnc_op_gemm(const void *X, const void *X_lo, const void *W, void *Y, int32_t T, int32_t n_out, int32_t n_in,
                int32_t out_f32, int32_t accumulate, void *cuda_stream);
/* The same product with the SwiGLU epilogue of the MLP: W rows interleaved (row 2i = gate_i, row 2i+1 = up_i),
 * Y bf16 [T][n_out/2], Y[t][i] = silu(gate) * up; n_out a multiple of 16 (rows of Y stay 16-byte aligned). */
int nnc_op_gemm_swiglu(const void *X, const void *X_lo, const void *W, void *Y, void *Y_lo, int32_t T,
                       int32_t n_out, int32_t n_in, void *cuda_stream); /* Y_lo: NULL or the residual of Y */
/* nnc_op_gemm for few tokens (T <= 128), where the product is bound by streaming W: the (output tile, K block)
 * space is cut into one equal contiguous range per SM, so every SM streams the same share of W.  A tile whose K
 * range straddles a cut is finished through fp32 partial tiles in `scratch`: the CTA holding the tile's first K
 * piece waits (bounded; on expiry the status word is set) for the others and adds the pieces in K order
 * (deterministic).  scratch: DEVICE, 256-byte aligned, at least 16 KiB + 2 * 64 KiB * (number of SMs) to cover
 * every T (a smaller one makes large T fall back to whole tiles); its first 16 KiB are flags that must be zero
 * before the first call and are left zero by every call that ends without error.  Calls that share a scratch
 * must not overlap on the device.  With T > 128 it behaves as nnc_op_gemm. */
int nnc_op_gemm_splitk(const void *X, const void *X_lo, const void *W, void *Y, int32_t T, int32_t n_out, int32_t n_in,
                       int32_t out_f32, int32_t accumulate, void *scratch, size_t scratch_bytes, void *cuda_stream);
/* The fp16 forms used by the prompt phase: X fp16 [T][n_in] (T > 128), W fp16 [n_out][n_in], one term.  out_scale: NULL
 * or a DEVICE float multiplied into every accumulator before the epilogue (undoes the scale of an fp16 weight copy).
 * nnc_op_gemm_f16: Y fp32 [T][n_out], Y += product when accumulate != 0.  nnc_op_gemm_swiglu_f16: W rows interleaved
 * gate/up, Y fp16 [T][n_out/2] (values beyond +-65504 saturate). */
int nnc_op_gemm_f16(const void *X, const void *W, float *Y, int32_t T, int32_t n_out, int32_t n_in, int32_t accumulate,
                    const float *out_scale, void *cuda_stream);
int nnc_op_gemm_swiglu_f16(const void *X, const void *W, void *Y, int32_t T, int32_t n_out, int32_t n_in,
                           const float *out_scale, void *cuda_stream);
/* dst (fp16) = src (bf16) * 2^e, n elements (a multiple of 8), with e chosen so that the largest magnitude lands in
 * [2^14, 2^15): exact for every element down to 2^-32 of the largest (smaller ones round with an error below 2^-39 of the largest).  scales: DEVICE float[2] receiving {2^e, 2^-e};
 * scratch_word: DEVICE uint32 used during the call. */
int nnc_op_to_f16_scaled(const void *src, void *dst, size_t n, float *scales, uint32_t *scratch_word, void *cuda_stream);

/* Status word of the nnc_op_* kernels (0 = no tensor-core kernel's bounded wait ran out and no paged-cache kernel met
 * an address out of range: NNC_STATUS_PAGED_ADDRESS, beside the last code); synchronises the device and clears the word.  status_out is a
 * HOST pointer. */
#define NNC_STATUS_PAGED_ADDRESS 0x100
int nnc_op_status(int32_t *status_out);

/* y[n_out] = W[n_out][n_in] x (batch-1 streaming GEMV, fp32 accumulate).  x fp32 [n_in]; y fp32.
 * If gain != NULL (bf16 [n_in]) x is first RMS-normalised with that gain and eps.
 * mode 0: y = Wx;  mode 1: y += Wx (residual);  mode 2: rows interleaved gate/up, y[n_out/2] = silu(g)*u.
 * mode | NNC_GEMV_CHAINED: launch the way the decode step does, with programmatic stream serialization, so that
 * back-to-back calls on one stream overlap the next kernel's weight prefetch with the previous kernel's tail
 * (x and y of consecutive chained calls must then not depend on each other's weights buffer being rewritten). */
#define NNC_GEMV_CHAINED 0x100
int nnc_op_gemv(const void *W, const float *x, float *y, int32_t n_out, int32_t n_in, const void *gain,
                float eps, int32_t mode, void *cuda_stream);

/* FP8 E4M3 row quantisation (nnc_config::weight_format 1): W bf16 [n_out][n_in] -> codes uint8 [n_out][n_in] and
 * scales fp32 [n_out] (= 2^e per row); dequant: NULL, or bf16 [n_out][n_in] receiving code * 2^e (may be W itself).
 * n_in a multiple of 8. */
int nnc_op_quantise_rows_e4m3(const void *W, void *codes, float *scales, void *dequant, int32_t n_out, int32_t n_in,
                              void *cuda_stream);
/* nnc_op_gemv on FP8 weights: y = diag(scales) * codes * x with the same modes, gain and chaining flag; n_in a multiple
 * of 16 (up to 16384; 8192 with mode 2). */
int nnc_op_gemv_fp8(const void *codes, const float *scales, const float *x, float *y, int32_t n_out, int32_t n_in,
                    const void *gain, float eps, int32_t mode, void *cuda_stream);

/* Split-K flash-decode for one query token per sequence over a contiguous cache.
 *   q fp32 [batch][n_q_heads][128] (already normalised and rotated);  kcache, vcache bf16
 *   [batch][n_kv_heads][max_seq][128];  n_ctx positions are attended;  out fp32 [batch][n_q_heads][128].
 *   scratch: DEVICE, at least nnc_attn_scratch_bytes(batch, n_q_heads, n_ctx) bytes, 256-byte aligned. */
size_t nnc_attn_scratch_bytes(int32_t batch, int32_t n_q_heads, int32_t n_ctx);
int nnc_op_attn_decode(const float *q, const void *kcache, const void *vcache, float *out, int32_t batch,
                       int32_t n_q_heads, int32_t n_kv_heads, int32_t max_seq, int32_t n_ctx, void *scratch,
                       void *cuda_stream);

/* Causal attention of the prompt phase for T new tokens per sequence (tcgen05 tensor cores; the score and
 * probability tile stays in tensor memory between the two products, cf. the pass-through layout of Section 3.1.2).
 *   qkv fp32 [batch * T][(n_q_heads + 2 n_kv_heads) * 128]: only the query heads are read (already normalised and
 *   rotated);  kcache, vcache bf16 [batch][n_kv_heads][max_seq][128] must already hold the new tokens' K/V at
 *   positions n_past .. n_past + T - 1;  the query of token s attends to positions 0 .. n_past + s.  Cache rows at
 *   positions >= n_past + T are never read (they may hold anything).
 *   out (and out_lo, NULL or the bf16 rounding residual): bf16 [batch * T][n_q_heads * 128], 16-byte aligned.
 *   n_past: cached positions before these tokens, a host value; n_past + T > max_seq returns NNC_ERR_CAPACITY. */
int nnc_op_attn_prefill(const float *qkv, const void *kcache, const void *vcache, void *out, void *out_lo, int32_t batch,
                        int32_t T, int32_t n_q_heads, int32_t n_kv_heads, int32_t max_seq, int32_t n_past,
                        void *cuda_stream);

/* The one-term form the prompt phase uses: k16, v16 fp16 images of the cache rows (same layout; exact for bf16 values
 * inside the fp16 range), queries and probabilities travel as one fp16 term each (half the tensor-core work of the form
 * above), out fp16 [batch * T][n_q_heads * 128]. */
int nnc_op_attn_prefill_f16(const float *qkv, const void *k16, const void *v16, void *out, int32_t batch, int32_t T,
                            int32_t n_q_heads, int32_t n_kv_heads, int32_t max_seq, int32_t n_past, void *cuda_stream);

/* The same operation for callers that cannot allocate device memory (the paper has no counterpart: this is a
 * deployment convenience of this library).  A plug-in that is handed only its inputs and outputs, or a process
 * whose device memory is owned by another runtime's pool, cannot produce the scratch buffer above; here the
 * scratch lives in a fixed array inside the library image (NNC_ATTN_STATIC_SCRATCH_BYTES per GPU, held from
 * library load until process exit) and the call allocates nothing.
 *   - Needs above that size (nnc_attn_scratch_bytes(batch, n_q_heads, n_ctx) > NNC_ATTN_STATIC_SCRATCH_BYTES,
 *     i.e. roughly batch * n_q_heads > 120) return NNC_ERR_CAPACITY, print one line to stderr, launch nothing.
 *   - Every call on a device shares the array and finds the previous call's contents in it; the call clears
 *     what must start at zero itself.  Calls that overlap on the GPU (two streams, two threads) race on the
 *     array: serialise them.
 *   - The first call on each device looks up the array's device address; issue that first call outside any
 *     stream capture. */
#define NNC_ATTN_STATIC_SCRATCH_BYTES (4u << 20)
int nnc_op_attn_decode_static(const float *q, const void *kcache, const void *vcache, float *out, int32_t batch,
                              int32_t n_q_heads, int32_t n_kv_heads, int32_t max_seq, int32_t n_ctx,
                              void *cuda_stream);

/* ---- rotary positions and the paged key-value cache ------------------------------------------------------
 * Single operations for serving sequences of different lengths: rotate queries and keys (nnc_op_rope), append rows to a
 * cache whose memory is handed out in pages (nnc_op_kv_write_paged), attend from one new token per sequence
 * (nnc_op_attn_decode_paged), read rows back (nnc_op_kv_read_paged).  Positions, sequences, page tables and lengths
 * are DEVICE arrays that a kernel reads when it runs, so a captured graph follows them from replay to replay.  Like
 * the other operations, each launches on `cuda_stream` of the current device, allocates nothing and writes only the
 * rows it names.  Their kernels are launched with programmatic stream serialization and wait for the preceding kernel before
 * they read anything, so consecutive calls overlap their launches and keep their order. */

typedef enum { NNC_F32 = 0, NNC_BF16 = 1, NNC_F16 = 2, NNC_E4M3 = 3 } nnc_type;

/* Angles per position of the rotary pairs: freq[i] (HOST, rotary_dim / 2 doubles) = radians by which pair i turns per
 * position, theta^(-2i / rotary_dim), stretched for contexts longer than the one a model was made for:
 *   NNC_ROPE_PLAIN      unchanged
 *   NNC_ROPE_LINEAR     all divided by `factor`
 *   NNC_ROPE_BASE       theta grown to theta * factor^(rotary_dim / (rotary_dim - 2)): the slowest pair is divided by `factor`
 *   NNC_ROPE_RAMP_TURNS pairs that make at least `fast` turns over `original` positions stay, pairs that make at most
 *                       `slow` are divided by `factor`, between them f * (g + (1 - g) / factor) with g linear in the turns
 *   NNC_ROPE_RAMP_INDEX the same with g linear in the pair's index, between floor(index that makes `fast` turns) and
 *                       ceil(index that makes `slow`), both kept inside [0, rotary_dim - 1]; the upper one is moved 0.001 up
 *                       where they coincide
 * amplitude (HOST, may be NULL): what queries and keys are multiplied by, 0.1 ln(factor) + 1 for the ramp by index (1 for
 * factor <= 1), 1 for the others.  Pure host arithmetic.  rotary_dim even and positive (BASE: at least 4), theta > 0, factor >= 1,
 * original > 0 and 0 < slow < fast where they are used; NNC_ERR_INVALID_ARG otherwise. */
enum { NNC_ROPE_PLAIN = 0, NNC_ROPE_LINEAR = 1, NNC_ROPE_BASE = 2, NNC_ROPE_RAMP_TURNS = 3, NNC_ROPE_RAMP_INDEX = 4 };
int nnc_rope_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor, double original, double slow,
                         double fast, double *freq, float *amplitude);

/* y = the rotation of x by its positions: x, y of `type` (NNC_F32, NNC_BF16 or NNC_F16), element (t, h, i) of token t and head h
 * at t * row_stride + h * head_stride + i (strides in elements, may be 0 or negative for x).  positions: int32 [n_tokens], any value.  freq: DEVICE
 * double [rotary_dim / 2].  The first rotary_dim elements of each head turn (rotary_dim even, 2 <= rotary_dim <=
 * head_dim <= 1024), in pairs (i, i + rotary_dim / 2), or (2i, 2i + 1) with interleaved != 0; the others are copied.
 *   y_a = amplitude * (x_a cos - x_b sin),  y_b = amplitude * (x_b cos + x_a sin),  angle = position * freq[i]
 * inverse != 0 turns the other way: given the gradient with respect to y it is the gradient with respect to x.  The
 * angle is reduced in two doubles (2^-28 turns at any position), the arithmetic is fp32, one rounding to `type` at the end.  y may be x itself (with the
 * same strides); other overlaps of x and y, and rows of y that overlap each other, are not allowed.  n_tokens or n_heads of 0 is a call that
 * does nothing. */
int nnc_op_rope(const void *x, void *y, int32_t type, int32_t n_tokens, int32_t n_heads, int32_t head_dim,
                int64_t x_row_stride, int64_t x_head_stride, int64_t y_row_stride, int64_t y_head_stride,
                const int32_t *positions, const double *freq, int32_t rotary_dim, int32_t interleaved, int32_t inverse,
                float amplitude, void *cuda_stream);

/* A paged cache (HOST struct, DEVICE pointers; the caller owns all memory and hands out the pages).  Position n of
 * sequence s lies in slot n % page_size of page page_table[s * pages_per_seq + n / page_size].
 *   k, v             [n_pages][n_kv_heads][page_size][head_dim] of `type` (NNC_BF16, NNC_F16 or NNC_E4M3), 16-byte aligned
 *   k_scale, v_scale NNC_E4M3 only: one byte a row, [n_pages][n_kv_heads][page_size], 16-byte aligned: the row's values
 *                    are code * 2^(byte - 127), bytes of 67 .. 187 (what nnc_op_kv_write_paged writes).  NULL otherwise.  The attention
 *                    keeps a position's weight to 2^-39 of the largest product of a weight and its value row's scale, rows of zeros
 *                    not counted: scales larger than their rows need cost the other rows' accuracy
 *   page_table       int32 [n_seqs][pages_per_seq]; entries that no call reaches may hold anything.  Sequences may share pages
 *                    (a common prefix) that no call writes
 *   page_size 16, 32, 64, 128 or 256; head_dim 64 or 128.
 * An address that a call reaches and that lies outside (a sequence >= n_seqs, a position >= pages_per_seq * page_size, a
 * page outside [0, n_pages)) is neither read nor written; the call goes on without it and sets NNC_STATUS_PAGED_ADDRESS in
 * nnc_op_status's word. */
typedef struct {
    void *k, *v;
    uint8_t *k_scale, *v_scale;
    const int32_t *page_table;
    int32_t type, n_pages, page_size, n_kv_heads, head_dim, n_seqs, pages_per_seq;
} nnc_paged_kv;

/* Writes the key and value rows of n_tokens tokens: token t goes to position pos[t] of sequence seq[t] (int32 [n_tokens];
 * seq NULL: sequence t, and n_tokens <= n_seqs).  Tokens whose seq or pos is negative are padding and are left out.  No two tokens of
 * a call may name the same slot.  Element (t, h, i) of k and v, of `type` (NNC_F32, NNC_BF16, NNC_F16), lies at t * row_stride +
 * h * head_stride + i.  16-bit caches hold the value rounded to nearest even (a row of the cache's own type is copied); an E4M3
 * row holds codes for the scale 2^e, e the smallest integer with max|x| <= 448 * 2^e over the row's finite values, kept
 * inside [-60, 60] (0 for a row without any but zeros), rounded to nearest even, saturating (infinities too); NaN stays NaN.  Pointers and
 * strides of k and v are multiples of 16 bytes, and they do not overlap the cache. */
int nnc_op_kv_write_paged(const nnc_paged_kv *cache, const void *k, const void *v, int32_t type, int32_t n_tokens,
                          int64_t row_stride, int64_t head_stride, const int32_t *pos, const int32_t *seq, void *cuda_stream);

/* Reads rows back, addressed the same way: the values of position pos[t] of sequence seq[t] to k and v, rounded to `type`
 * (exact for NNC_F32, and for a scaled code in NNC_BF16).  Rows of padding tokens and of addresses out of range are left as
 * they are.  The same position may be read by several tokens. */
int nnc_op_kv_read_paged(const nnc_paged_kv *cache, void *k, void *v, int32_t type, int32_t n_tokens, int64_t row_stride,
                         int64_t head_stride, const int32_t *pos, const int32_t *seq, void *cuda_stream);

/* Attention of one new token per sequence over the paged cache, which already holds that token's own row.
 *   q, out  of `type` (NNC_F32, or the cache's own 16-bit type; NNC_F32, NNC_BF16 or NNC_F16 for an E4M3 cache): row b (of
 *           sequence b, batch <= n_seqs) holds n_q_heads heads of head_dim at b * q_stride / b * out_stride elements.  Query head i
 *           uses KV head i / (n_q_heads / n_kv_heads); any whole ratio
 *   lens    int32 [batch]: sequence b attends to positions max(0, lens[b] - window) .. lens[b] - 1 (window 0: from 0).  Rows of
 *           the cache outside that range are never read into the result (they may hold anything)
 *   scale   multiplies q.k before the softmax
 *   lse     fp32 [batch][n_q_heads] or NULL: log(sum exp) of the scaled scores, natural logarithm
 * Scores are a softmax's whatever their size: -infinity weighs nothing, +infinity or NaN leave a head no number.  Every other
 * attended position has a positive weight, so a column of values with an infinity gives that infinity (both signs, or NaN: NaN).
 * A sequence with nothing to attend to (lens <= 0) gets a row of zeros and lse = -infinity.  A length beyond the table's
 * reach counts as the longest the table holds, and a page out of range as absent; both set the status word.
 * scratch: DEVICE, 256-byte aligned, NNC_ATTN_PAGED_SCRATCH_BYTES; its first NNC_ATTN_PAGED_TICKET_BYTES must be zero before
 * the first call and are left zero by every call.  Calls that share a scratch must not overlap on the device (captured
 * graphs included).  Results do not depend on scheduling: partial results are joined in a fixed order.  q, out and
 * their strides are multiples of 16 bytes.  out may be q itself (with the same strides); other overlaps are not allowed. */
#define NNC_ATTN_PAGED_SCRATCH_BYTES (16u << 20)
#define NNC_ATTN_PAGED_TICKET_BYTES 8192
int nnc_op_attn_decode_paged(const void *q, const nnc_paged_kv *cache, const int32_t *lens, void *out, float *lse, int32_t type,
                             int32_t batch, int32_t n_q_heads, int64_t q_stride, int64_t out_stride, float scale, int32_t window,
                             void *scratch, size_t scratch_bytes, void *cuda_stream);

/* The same where groups of sequences share their first positions (one system prompt, one document): the shared rows are read once for all
 * sequences of a group, not once for each.  Group g is the sequences starts[g] .. starts[g + 1] - 1 (int32 [n_groups + 1], not
 * descending, within 0 .. batch); its sequences have positions 0 .. shared[g] - 1 in common (int32 [n_groups]), which are read
 * through the page table of the group's first sequence, whole pages of them (what is left of the last page counts as each sequence's own).
 * The cache holds all of them, whatever the sequences' lengths; a shorter sequence attends to its first lens[b].  Sequences of
 * no group, and of groups with shared[g] below a page, attend to their own rows alone.  A `starts` that descends or leaves 0 .. batch
 * and a shared[g] outside 0 .. the table's reach are cut to what is allowed and, where the groups are looked at, set the status word.
 * Overlapping groups leave the results of the sequences in them open.  1 <= n_groups <= batch.  n_pages * n_kv_heads * page_size is at most
 * 2^31 - 256 (NNC_ERR_CAPACITY).
 *   q, out, lens, lse, scale, strides: as there, without a window.  A group of few sequences reads each one's own rows (below two, on NNC_E4M3
 *   caches below four; fewer with many query heads per KV head); groups of no sequences cost nothing, so that the arrays of a captured call may
 *   have room for more groups than there are.  Every sequence reads its own rows, and the groups are not looked at, for one sequence, for fp32
 *   queries, fp16 queries on NNC_E4M3 caches, more than 128 query heads per KV head, queries whose rows overlap, and where the table has room
 *   for little: all rows that it could name, whatever the lengths are, times the query heads per KV head in eights are less than 140 MB.
 *   Numerics: fp32 scores, maxima and sums, as there; shared rows of bf16 and NNC_E4M3 caches are weighed by probabilities of 16 bits (two bf16 terms, each
 *   off by at most 2^-16 of itself), of fp16 caches of 22, where nnc_op_attn_decode_paged has 24 and 22.
 * scratch: DEVICE, 256-byte aligned, nnc_attn_prefix_scratch_bytes(batch, n_q_heads, head_dim); its first NNC_ATTN_PAGED_TICKET_BYTES as
 * there.  Up to three launches. */
size_t nnc_attn_prefix_scratch_bytes(int32_t batch, int32_t n_q_heads, int32_t head_dim);
int nnc_op_attn_prefix_paged(const void *q, const nnc_paged_kv *cache, const int32_t *lens, const int32_t *starts, const int32_t *shared,
                             int32_t n_groups, void *out, float *lse, int32_t type, int32_t batch, int32_t n_q_heads, int64_t q_stride,
                             int64_t out_stride, float scale, void *scratch, size_t scratch_bytes, void *cuda_stream);

/* ---- long caches: pages chosen by a score --------------------------------------------------------------------
 * A decoding step that reads part of a long cache: for every page the lowest and the highest of its keys, element by element
 * (nnc_op_page_bounds, after rows were written), the most that a query's product with a key between them can be (nnc_op_score_pages), the
 * pages of the highest scores (nnc_op_select_pages), and the attention over them (nnc_op_attn_selected_paged). */

/* bounds: 16-byte aligned, [n_pages][n_kv_heads][2][head_dim] of the cache's type (NNC_BF16 for an NNC_E4M3 cache, which holds its scaled codes
 * exactly down to 2^-133): lowest, then highest.  Sets them for every page of sequences 0 .. batch - 1 (batch <= n_seqs) that holds a position in
 * [first[b], lens[b]), from all positions of that page below lens[b]; other pages' bounds stay.  lens, first: int32 [batch]; first NULL: 0.
 * NaN where a key is NaN.  Sequences that share such a page give it the same bounds if both have all of it, which shared pages want
 * anyway.  A length beyond the table's reach counts as the longest the table holds, a page out of range is left out; both set the
 * status word. */
int nnc_op_page_bounds(const nnc_paged_kv *cache, void *bounds, const int32_t *lens, const int32_t *first, int32_t batch, void *cuda_stream);

/* scores: fp32 [batch][n_kv_heads][pages_per_seq]: for page n of sequence b the largest, over the query heads of the KV head, of
 * sum_i max(q_i lowest_i, q_i highest_i): no key of the page has a larger product with any of these queries.  -infinity for pages that hold no
 * position below lens[b] and for pages out of range.  A page whose bounds are not all finite scores an infinity or NaN.  q as
 * for nnc_op_attn_decode_paged.  Types other than the bounds' enter as sums of their terms (24 bits, or 22 in fp16); sums
 * are fp32.  n_q_heads / n_kv_heads at most 128. */
int nnc_op_score_pages(const void *q, const nnc_paged_kv *cache, const void *bounds, const int32_t *lens, float *scores, int32_t type,
                       int32_t batch, int32_t n_q_heads, int64_t q_stride, void *cuda_stream);

/* Of the P pages that hold positions below lens[b] (at most n_columns) the n of the highest scores, for each KV head: scores fp32
 * [batch][n_kv_heads][n_columns].  The first `first` and the last `last` pages (first + last <= n) are always among them; NaN is above every
 * number; among equal scores the lowest pages.  pages: int32 [batch][n_kv_heads][n], in ascending order, -1 behind the last; counts: int32
 * [batch][n_kv_heads], min(n, P).  page_size as in the cache. */
int nnc_op_select_pages(const float *scores, const int32_t *lens, int32_t *pages, int32_t *counts, int32_t batch, int32_t n_kv_heads,
                        int32_t n_columns, int32_t page_size, int32_t n, int32_t first, int32_t last, void *cuda_stream);

/* nnc_op_attn_decode_paged over listed pages: the query heads of KV head h of sequence b attend to the positions below lens[b] of the pages
 * pages[b][h][0 .. counts[b][h] - 1] (numbers within the sequence, in any order, none twice; int32 [batch][n_kv_heads][list_len], counts
 * above list_len count as list_len).  A page without such a position adds nothing; one outside [0, pages_per_seq) adds nothing and
 * sets the status word.  Everything else, the scratch among it, is as there. */
int nnc_op_attn_selected_paged(const void *q, const nnc_paged_kv *cache, const int32_t *lens, const int32_t *pages, const int32_t *counts,
                               int32_t list_len, void *out, float *lse, int32_t type, int32_t batch, int32_t n_q_heads, int64_t q_stride,
                               int64_t out_stride, float scale, void *scratch, size_t scratch_bytes, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* NNC_H_ */
