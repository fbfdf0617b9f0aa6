/*
 * spts.h -- C boundary of the SPTS (Self-Predictive Token Skipping) prefill library for
 * NVIDIA B200 (sm_100a).
 *
 * The library runs the token-selective transformer prefill layer of the SPTS paper:
 * Partial Attention Probing (Section 3.2, Eq. 4-5), Low-rank Transformation Probing
 * (Section 3.3, Eq. 12-15), top-k selection, the reduced attention / FFN blocks with
 * residual scatter (Eq. 2, Algorithm 1), Multi-Stage Delayed Pruning (Section 3.4, Eq. 16)
 * and the decode step over the per-layer compressed KV cache.
 *
 * General rules
 *   - Every pointer named in a signature is a DEVICE pointer unless the comment says "host".
 *     Structs (model_desc, layer_weights, kv_layer, layer_plan) live in HOST memory and hold
 *     device pointers.
 *   - The caller owns every buffer, including the workspace given to spts_create().  The
 *     library allocates no device memory and frees nothing.
 *   - All work is enqueued on the context's CUDA stream and returns without synchronising.
 *     Sizes (N, k, m_attn, m_ffn, n_next) are host integers: Algorithm 1 fixes them from the
 *     schedule (M^l = min(|T^l|, M_fixed), Section 3.4), so no call reads a count back.
 *   - Storage type: dtype SPTS_BF16 (bf16 in HBM, fp32 accumulation, tensor-core kernels) or
 *     SPTS_FP32 (verification mode: fp32 storage and CUDA-core fp32 arithmetic).  Scores,
 *     softmax statistics and norms are fp32 in both modes.
 *   - Weight matrices are row-major [out_features, in_features].  RMSNorm gains are expected
 *     to be folded into the columns of the matrices that consume the normalised rows
 *     (spts_fold_norm_gain()); with unit gains nothing needs to be done.
 *   - Index lists are int32, strictly ascending.  Ties in a top-k go to the lower index.
 *   - Errors detectable on the host (null pointer, k > N, unsupported shape, workspace too
 *     small, misalignment) are returned before anything is launched.  Device-side problems
 *     (a bounded wait that expired, a non-finite score) set a status word that
 *     spts_last_device_status() returns after synchronising the stream; kernels never trap.
 *   - Pointers must be 16-byte aligned; rows of X, K, V are contiguous.
 *   - A context is bound to one device and one stream and is not thread-safe: calls on one context must
 *     not overlap on the host.  Contexts on different streams are independent (each has its workspace).
 *     spts_layer_prefill_skip() and spts_prefill() use the context's workspace for every intermediate
 *     (K of all candidates, the selected rows' Q, the attention output, the SwiGLU intermediate, scores,
 *     index lists), so the workspace grows with max_seq: about 24 KiB per candidate at the 8B shape plus 0.55 GB (of
 *     which 0.47 GB is the SwiGLU intermediate of one 16384-row chunk): 1.37 GB at 32768 candidates, 3.75 GB at 131072.
 */
#ifndef SPTS_H_
#define SPTS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SPTS_OK = 0,
  SPTS_ERR_INVALID_ARG = 1,
  SPTS_ERR_SHAPE = 2,
  SPTS_ERR_WORKSPACE = 3,
  SPTS_ERR_CUDA = 4,
  SPTS_ERR_TIMEOUT = 5,
  SPTS_ERR_NONFINITE = 6,
  SPTS_ERR_UNSUPPORTED = 7,
  SPTS_ERR_INDEX = 8      /* SPTS_DEBUG_CHECKS: an index list was out of range or not strictly ascending */
} spts_status;

enum { SPTS_BF16 = 0, SPTS_FP32 = 1 };

/* flags */
enum {
  SPTS_FORCE_LAST = 1u,   /* the last candidate is always selected (it carries the output state) */
  SPTS_REFERENCE_KERNELS = 2u, /* spts_set_option: run the plain CUDA-core kernels also in bf16 mode */
  SPTS_PAP_WINDOW = 8u,        /* spts_set_option: value = number of trailing queries the probe score averages over
                                  (1..64; 1 = last token only, Eq. 4; larger windows are the query-length ablation of
                                  Appendix C: every query attends causally, K and the queries are taken as stored) */
  SPTS_DEBUG_CHECKS = 32u,     /* spts_set_option: after every selection a small kernel checks the index list
                                  (0 <= idx < N, strictly ascending) and records SPTS_ERR_INDEX in the device status
                                  word; nothing traps.  Off by default (one extra launch per selection) */
  SPTS_FFN_SCORE_PAP_ONLY = 16u /* spts_set_option: T_f = TopK(S_mha, m_ffn) -- the FFN block selects by the attention
                                  probe's score alone (Eq. 4) and the proxy FFN of Eq. 12-14 is not evaluated: the
                                  criterion the paper's proxy-network ablation (Table 4) compares Eq. 14 against */
};

typedef struct {
  int32_t hidden;      /* D */
  int32_t n_q_heads;   /* H */
  int32_t n_kv_heads;  /* Hkv, divides H */
  int32_t head_dim;    /* d */
  int32_t ffn_dim;     /* Dff */
  int32_t ltp_dlow;    /* D_low of the proxy FFN (Eq. 12) */
  int32_t ltp_rank;    /* r of the proxy FFN */
  int32_t n_layers;
  int32_t vocab;
  float rms_eps;
  float rope_theta;
  int32_t dtype;       /* SPTS_BF16 or SPTS_FP32 */
} spts_model_desc;

/* Device pointers, each [out, in] row-major in the model's storage type. */
typedef struct {
  const void* wq;      /* [H*d, D]   */
  const void* wk;      /* [Hkv*d, D] */
  const void* wv;      /* [Hkv*d, D] */
  const void* wo;      /* [D, H*d]   */
  const void* w_gate;  /* [Dff, D]   */
  const void* w_up;    /* [Dff, D]   */
  const void* w_down;  /* [D, Dff]   */
  const void* ug;      /* [r, D]      U_gate^T  */
  const void* vg;      /* [Dlow, r]   V_gate^T  */
  const void* uu;      /* [r, D]      U_up^T    */
  const void* vu;      /* [Dlow, r]   V_up^T    */
  const void* vd;      /* [r, Dlow]   V_down    */
  const void* ud;      /* [D, r]      U_down    */
  const void* prepared; /* optional: the layer's buffer filled by spts_prepare_layer() (NULL: the proxy factors are
                           repacked inside every call that evaluates Eq. 12-14) */
} spts_layer_weights;

/* One layer's KV cache: k, v are [capacity, Hkv, d] in the storage type (K after RoPE),
 * pos [capacity] holds the original position of every cached token.  `len` is host state. */
typedef struct {
  void* k;
  void* v;
  int32_t* pos;
  int32_t len;
  int32_t capacity;
} spts_kv_layer;

/* Per-layer entry of the MSDP schedule (Section 3.4): active budgets already clipped to the
 * candidate count, and the candidate count to prune to after this layer (0 = not a stage end). */
typedef struct {
  int32_t m_attn;
  int32_t m_ffn;
  int32_t prune_to;
} spts_layer_plan;

/* One stage of the MSDP schedule (Section 3.4; the settings of Section 4.1 are given in this form): the last
 * layer of the stage (0-indexed), the fixed active budgets M_fixed of its attention and FFN blocks (<= 0: that
 * block runs on every candidate in this stage) and the candidate count N_{s+1} the stage end prunes to by
 * Eq. 16 (<= 0: the stage end does not prune). */
typedef struct {
  int32_t last_layer;
  int32_t m_attn_fixed;
  int32_t m_ffn_fixed;
  int32_t n_next;
} spts_msdp_stage;

typedef struct {
  const spts_layer_weights* layers; /* host array [n_layers] */
  const void* lm_head;              /* [vocab, D] */
  const void* embed;                /* [vocab, D], used by spts_decode_step */
} spts_model_weights;

/* Operation tags of the per-operation timer (spts_profile_begin / spts_profile_end). */
enum {
  SPTS_OP_PREP = 1,        /* row RMS statistics, rotary table, last-token query            */
  SPTS_OP_KPROJ = 2,       /* K projection of all candidates + RoPE + PAP logits (Eq. 4)   */
  SPTS_OP_PAP_SOFTMAX = 3, /* head-mean softmax of Eq. 4                                    */
  SPTS_OP_TOPK = 4,        /* Eq. 5 / 15 / 16                                               */
  SPTS_OP_KV_GATHER = 5,   /* K^ = K[T_a], cache positions                                  */
  SPTS_OP_QVPROJ = 6,      /* gathered Q (RoPE) and V projections                           */
  SPTS_OP_ATTN = 7,        /* causal GQA attention among the active rows                    */
  SPTS_OP_OPROJ = 8,       /* O projection + residual scatter                               */
  SPTS_OP_LTP = 9,         /* proxy FFN chain, row norms and score fusion (Eq. 12-14)       */
  SPTS_OP_GATEUP = 10,     /* gathered gate/up GEMM + SwiGLU                                */
  SPTS_OP_DOWN = 11,       /* down GEMM + residual scatter                                  */
  SPTS_OP_COMPACT = 12,    /* stage-end row compaction (Eq. 16)                             */
  SPTS_OP_HEAD = 13,       /* final norm, LM head, argmax                                   */
  SPTS_OP_DECODE = 14,     /* all layers of one decode step                                 */
  SPTS_OP_COUNT = 16
};

typedef struct spts_ctx spts_ctx;

/* Bytes of device workspace spts_create() needs for sequences of up to max_seq candidates. */
size_t spts_workspace_bytes(const spts_model_desc* desc, int max_seq);

/* Creates a context.  `workspace` is caller-owned device memory of at least
 * spts_workspace_bytes() bytes, 256-byte aligned; `cuda_stream` is a cudaStream_t (may be 0).
 * Must be called with the target device current.  Returns SPTS_ERR_SHAPE for shapes the
 * kernels do not cover (head_dim must be 64 or 128, H a multiple of Hkv, dimensions
 * multiples of 8; bf16 tensor-core mode additionally needs head_dim 128 and hidden, ffn_dim,
 * ltp_dlow multiples of 64, ltp_rank a multiple of 16). */
spts_status spts_create(const spts_model_desc* desc, int max_seq, void* workspace,
                        size_t workspace_bytes, void* cuda_stream, spts_ctx** out);
void spts_destroy(spts_ctx* ctx);

/* Sets SPTS_REFERENCE_KERNELS, SPTS_FFN_SCORE_PAP_ONLY or SPTS_DEBUG_CHECKS on/off
 * (value 0/1), or SPTS_PAP_WINDOW (value 1..64).  A context whose shape or storage type has no
 * tensor-core kernels for the prefill runs it on the plain ones whatever the option says and
 * answers value 0 with SPTS_ERR_UNSUPPORTED; in bf16 SPTS_REFERENCE_KERNELS still selects the
 * kernels of its 4-bit calls and of spts_paged_*, and value 0 after 1 takes that back with SPTS_OK. */
spts_status spts_set_option(spts_ctx* ctx, uint32_t option, int value);

/* Synchronises the context's stream and returns the device status word (then clears it).  The word holds the first problem since it was
 * read last.  After SPTS_ERR_TIMEOUT outputs of that call are incomplete, and calls that are joined by the block that comes last (those of
 * spts_paged_*, spts_token_logprobs, spts_kv4_attention, spts_process_logits) can go wrong until the word is read: reading a word that is not
 * SPTS_OK also clears what they count on, so the context is as before. */
spts_status spts_last_device_status(spts_ctx* ctx);

/* Guard bands (the paper has no counterpart: a stand-in for a memory checker).  Every slice the library carves out
 * of the caller's workspace is followed by a 256-byte band that spts_create() fills with a fixed pattern and no
 * kernel has any business writing.  spts_check_guards synchronises the stream, reads the bands back and stores the
 * number of bands that no longer hold the pattern in *n_corrupt (HOST memory); a non-zero count means some kernel
 * wrote past the end of its slice. */
spts_status spts_check_guards(spts_ctx* ctx, int32_t* n_corrupt);

/* The check SPTS_DEBUG_CHECKS runs after every selection, on a list the caller provides: idx [n] (device) must lie
 * in [0, N) and ascend strictly, otherwise SPTS_ERR_INDEX is recorded in the device status word (read it with
 * spts_last_device_status).  The kernel only reads the n entries; it never dereferences them. */
spts_status spts_debug_check_index_list(spts_ctx* ctx, const int32_t* idx, int n, int N);

/* Exercises the give-up path of the bounded waits (again no counterpart in the paper).  Every mbarrier wait of the
 * tensor-core kernels ends after a time limit: the waiting thread raises a CTA-wide flag, the other roles see it
 * and return from their own waits, the CTA lets copies in flight land, records SPTS_ERR_TIMEOUT in the device
 * status word and exits normally.  This call launches one tiny CTA that runs exactly that code on two barriers
 * nobody ever arrives on, with the limit shortened to limit_us microseconds (1..100000), so a test can see the
 * status come back and the context stay usable.  The production kernels are not involved; what those of spts_paged_* and
 * spts_token_logprobs count on is left as by a call that gave up, until the status is read. */
spts_status spts_selftest_wait_timeout(spts_ctx* ctx, uint32_t limit_us);

/* Number of kernels the library has launched on this context so far. */
int64_t spts_launch_count(const spts_ctx* ctx);

/* Per-operation timing with CUDA events recorded on the context's stream (the paper has no
 * counterpart; this is measurement plumbing).  spts_profile_begin starts recording event pairs
 * around every operation with tag `op` (-1: every tagged operation); spts_profile_end stops,
 * synchronises the stream and fills four host arrays of SPTS_OP_COUNT entries indexed by tag:
 * elapsed milliseconds, number of timed operations, algorithmic FLOPs and algorithmic bytes. */
spts_status spts_profile_begin(spts_ctx* ctx, int op);
spts_status spts_profile_end(spts_ctx* ctx, float* ms, int64_t* calls, double* flops, double* bytes);

/* W[o, i] *= g[i], in place, rounded to the storage type: folds an RMSNorm gain g [in] into a
 * weight matrix [out, in] that consumes the normalised rows (pre-norm block placement; the
 * paper's Algorithm 1 leaves normalisation out). */
spts_status spts_fold_norm_gain(spts_ctx* ctx, void* W, const float* g, int out_features,
                                int in_features);

/* Partial Attention Probing, Eq. 4 / Algorithm 1 "K <- X W_K, q <- X_N W_Q; S_MHA":
 * K_out[n] = RoPE(rmsnorm(X[n]) W_K, pos[n]) for all N candidates (storage type, [N,Hkv,d]),
 * q = RoPE(rmsnorm(X[N-1]) W_Q, pos[N-1]),
 * S_mha_out[n] = (1/H) sum_h softmax_n(q_h . K_{h / (H/Hkv)} / sqrt(d))[n]   (fp32, [N]).
 * The logits are taken from the unrounded fp32 keys.  K_out may be NULL (workspace is used). */
spts_status spts_pap_score(spts_ctx* ctx, const spts_layer_weights* w, const void* X,
                           const int32_t* pos, int N, void* K_out, float* S_mha_out);

/* One-time repacking of a layer's proxy-FFN factors (Eq. 12) into the operand layouts the probe's GEMM chain reads,
 * so that nothing of it is left on the per-layer path: U_gate^T stacked over U_up^T (one [2r, D] matrix: the
 * residual stream is then read once for both), V_gate^T and V_up^T zero-padded to [D_low, 2r] each, and the Gram
 * matrix G = U_down^T U_down [r, r] split into a high and a low part: since ||t U_down^T||^2 = t G t^T, Eq. 13's
 * norm needs an [N, r] x [r, 2r] product instead of the [N, r] x [r, D] one.  `prepared` is caller-owned device
 * memory of spts_prepared_bytes(desc) bytes, 256-byte aligned; put its address into spts_layer_weights.prepared.
 * It must be redone when ug, uu, vg, vu or ud change.  Results are bit-identical with and without it. */
size_t spts_prepared_bytes(const spts_model_desc* desc);
spts_status spts_prepare_layer(spts_ctx* ctx, const spts_layer_weights* w, void* prepared, size_t prepared_bytes);

/* Low-rank Transformation Probing, Eq. 12-14: C[n] = || f(rmsnorm(X[n])) ||_2 with
 * f(x) = (silu(x Ug Vg) * (x Uu Vu)) Vd^T Ud^T, and S_ffn[n] = C[n] * S_mha[n].
 * C_out may be NULL.  X is the residual stream the FFN block would see. */
spts_status spts_ltp_score(spts_ctx* ctx, const spts_layer_weights* w, const void* X,
                           const float* S_mha, int N, float* C_out, float* S_ffn_out);

/* TopK of Eq. 5 / 15 / 16: the k largest of scores[0..N), written ascending by index.
 * Order: score descending, then index ascending; -0.0 equals +0.0; NaN ranks last (and sets
 * SPTS_ERR_NONFINITE in the device status).  flags: SPTS_FORCE_LAST.  1 <= k <= N. */
spts_status spts_topk_select(spts_ctx* ctx, const float* scores, int N, int k, uint32_t flags,
                             int32_t* idx_out);

/* The same selection for callers that cannot allocate device memory (the paper has no counterpart:
 * this exists for hosts whose device memory is planned and frozen before inference starts, or that are
 * only ever handed input and output buffers -- they can neither allocate the workspace spts_create()
 * needs nor let a library allocate behind their back).  It needs no context and no workspace: its
 * scratch is a fixed array of SPTS_TOPK_STATIC_SCRATCH_BYTES inside the library, resident on every GPU
 * that loads the library until the process exits.  Same result as spts_topk_select (same ordering rule,
 * ascending output, SPTS_FORCE_LAST); NaN scores rank last but are not reported, there being no context
 * to hold a status word.  Work is enqueued on `cuda_stream` (a cudaStream_t, may be 0) of the current
 * device and the call does not synchronise.
 *   - 1 <= k <= N <= SPTS_TOPK_STATIC_MAX_N, else SPTS_ERR_INVALID_ARG / SPTS_ERR_SHAPE before any launch.
 *   - The first call on each device looks up the array's device address (a synchronous runtime query,
 *     made with that device current); make that first call before any stream capture begins.
 *   - All calls on one device share the array.  Each call clears the counters it needs, so calls that
 *     are ordered on the GPU (same stream, or dependent streams) are fine; calls that may overlap on
 *     the GPU race on the scratch and give undefined index lists.
 *   - It calls no cudaMalloc / cudaFree or other allocating routine. */
#define SPTS_TOPK_STATIC_MAX_N 8388608
#define SPTS_TOPK_STATIC_SCRATCH_BYTES 36928
spts_status spts_topk_select_static(const float* scores, int N, int k, uint32_t flags, int32_t* idx_out,
                                    void* cuda_stream);

/* One decoder layer of Algorithm 1 in the prefill phase, in place on X [N, D]:
 *   S_mha (Eq. 4) -> T_a = TopK(S_mha, m_attn) -> Q, V projected for the rows in T_a, K rows
 *   reused -> cache <- (K^, V^, pos[T_a]) -> causal GQA attention among the active rows ->
 *   X[T_a] += O W_O (Eq. 2); then C, S_ffn (Eq. 12-14) on the updated X -> T_f =
 *   TopK(S_ffn, m_ffn) -> X[T_f] += FFN(rmsnorm(X[T_f])) (Eq. 6).  Rows outside T_a and T_f
 *   are not written.  m_attn == N / m_ffn == N run that block densely without probing.
 * cache->len is set to m_attn (capacity must be >= m_attn).  S_mha_out [N], idx_attn_out
 * [m_attn], idx_ffn_out [m_ffn] are optional outputs (NULL to skip; S_mha is still computed
 * when a selection needs it).  flags: SPTS_FORCE_LAST. */
spts_status spts_layer_prefill_skip(spts_ctx* ctx, const spts_layer_weights* w, void* X,
                                    const int32_t* pos, int N, int m_attn, int m_ffn,
                                    uint32_t flags, spts_kv_layer* cache, float* S_mha_out,
                                    int32_t* idx_attn_out, int32_t* idx_ffn_out);

/* The attention step of the reduced MHA on its own (Algorithm 1: O^ <- F_MHA(Q^, K^, V^), before W_O): causal
 * grouped-query attention among m rows in their compact order, row i attending to rows j <= i,
 *   O[i, h] = softmax_j(Q[i, h] . K[j, h / (H/Hkv)] / sqrt(d)) V[j, h / (H/Hkv)].
 * Q [m, H, d] and K [m, Hkv, d] are taken as given (after RoPE), V [m, Hkv, d]; O_out [m, H*d]; all in the storage
 * type, 16-byte aligned, none aliasing another.  1 <= m <= max_seq.  This is the kernel spts_layer_prefill_skip
 * runs between the Q/V projections and the O projection; the call exists so that it can be checked and timed on
 * operands of the caller's choosing. */
spts_status spts_reduced_attention(spts_ctx* ctx, const void* Q, const void* K, const void* V, int m, void* O_out);

/* The same layer for several independent prompts packed row after row into X [total, D] (the paper evaluates one
 * prompt at a time; Algorithm 1 applies to each prompt on its own, and that is what this call computes):
 * sequence b owns rows [seq_start[b], seq_start[b + 1]) of X and pos, has its own budgets m_attn[b], m_ffn[b]
 * (1 <= m <= its length) and its own cache caches[b].  seq_start [n_seq + 1], m_attn [n_seq], m_ffn [n_seq] and the
 * caches array are HOST memory; seq_start[0] == 0 and total = seq_start[n_seq] <= max_seq.
 * Everything that Eq. 4, 5 and 15 define per prompt stays per prompt: the probe uses each sequence's own last
 * token, its softmax runs over that sequence's candidates, TopK selects within the sequence (SPTS_FORCE_LAST keeps
 * each sequence's last row), attention is causal within the sequence.  The row normalisation, the K projection
 * (every row probed with its own sequence's last-token query), the per-sequence softmax and TopK, the Q / V / O
 * projections of all selected rows, the proxy FFN of Eq. 12-14 and the selected rows' SwiGLU FFN (Eq. 6) each run once
 * over the packed rows -- gathered GEMMs with ragged index lists, the attention kernel over a table of all
 * sequences' query tiles (tensor-core mode, up to 1024 sequences of up to 8192 rows each, probe window 1; other
 * batches run the attention blocks one sequence after the other).  Every row gets the bits the single-sequence call
 * gives it.
 * Optional outputs: S_mha_out [total]; idx_attn_out [sum m_attn] and idx_ffn_out [sum m_ffn], sequence after
 * sequence, each numbered from the sequence's own first row. */
spts_status spts_layer_prefill_skip_batch(spts_ctx* ctx, const spts_layer_weights* w, void* X, const int32_t* pos,
                                          int n_seq, const int32_t* seq_start, const int32_t* m_attn,
                                          const int32_t* m_ffn, uint32_t flags, spts_kv_layer* caches,
                                          float* S_mha_out, int32_t* idx_attn_out, int32_t* idx_ffn_out);

/* Stage-end pruning, Eq. 16 / Algorithm 1 "X <- X[T^{l+1}, :]": keeps the
 * n_next = min(N, N_{s+1}) candidates with the largest S_mha, in token order.  Out of place:
 * X_out [n_next, D], pos_out, orig_out [n_next] must not alias the inputs; idx_out [n_next]
 * (optional) receives the kept candidate indices.  flags: SPTS_FORCE_LAST. */
spts_status spts_msdp_compact(spts_ctx* ctx, const void* X_in, const int32_t* pos_in,
                              const int32_t* orig_in, const float* S_mha, int N, int n_next,
                              uint32_t flags, void* X_out, int32_t* pos_out, int32_t* orig_out,
                              int32_t* idx_out);

/* The budget rule of Multi-Stage Delayed Pruning (Section 3.4: M^l = min(|T^l|, M^l_fixed); Algorithm 1's
 * "M <- min(N, M_fix)" lines and the candidate update of Eq. 16), evaluated on the host: fills plan_out [n_layers]
 * (HOST memory) for a prompt of n_prompt tokens.  `stages` [n_stages] (HOST memory) is ordered by last_layer;
 * layer l belongs to the first stage whose last_layer >= l, layers after the last boundary to the last stage (they
 * keep its budgets).  Layers before `skip_from` run densely (m_attn = m_ffn = current candidate count) as the
 * paper's shallow layers do.  A stage's last layer gets prune_to = n_next when that is positive and smaller than
 * the current candidate count, and the later layers see that many candidates.  Optional outputs (host):
 * *n_final = candidates left after the last layer; *kv_token_layers = sum of m_attn over the layers, the number
 * of (token, layer) pairs the prefill leaves in the KV caches.  Pure host arithmetic: needs no context and no GPU.
 * Errors: SPTS_ERR_INVALID_ARG for null pointers, n_layers / n_prompt / n_stages < 1, stages out of order. */
spts_status spts_msdp_plan(int n_layers, int n_prompt, int skip_from, const spts_msdp_stage* stages, int n_stages,
                           spts_layer_plan* plan_out, int32_t* n_final, int64_t* kv_token_layers);

/* Offline construction of the low-rank proxy FFN of one layer (Section 3.3, "Low-rank Proxy FFN"):
 *   z(x) = |silu(x W_gate) * (x W_up)| for every calibration token x (rows of calib [n_cal, D], the hidden states
 *   preceding the FFN block, storage type; they are RMS-normalised like the FFN's input);
 *   I_j = mean of the max(1, floor(rho * n_cal)) largest z(x)[j] over the calibration tokens;
 *   C = TopK(I, D_low) (ascending, ties to the lower channel);  W' = W[:, C] for W_gate, W_up, W_down;
 *   W' ~ U V by truncated SVD of rank r (U has orthonormal columns, V carries the singular values).
 * Outputs, in the layouts spts_layer_weights expects (storage type): ug, uu [r, D]; vg, vu [D_low, r];
 * vd [r, D_low]; ud [D, r].  Optional: importance_out [Dff] fp32, channels_out [D_low] int32,
 * sigma_out [3, D_low] fp32 (singular values of the reduced gate, up, down matrices, descending).
 * `scratch` is caller-owned device memory of spts_proxy_scratch_bytes(desc, n_cal) bytes, 256-byte aligned.
 * Needs ltp_dlow <= ffn_dim, ltp_dlow even, ltp_rank <= min(ltp_dlow, hidden); 0 < rho <= 1.
 * Runs off the inference path (a few hundred small launches per matrix); asynchronous like every other call. */
size_t spts_proxy_scratch_bytes(const spts_model_desc* desc, int n_cal);
spts_status spts_proxy_build(spts_ctx* ctx, const spts_layer_weights* w, const void* calib, int n_cal, double rho,
                             void* scratch, size_t scratch_bytes, float* importance_out, int32_t* channels_out,
                             void* ug, void* vg, void* uu, void* vu, void* vd, void* ud, float* sigma_out);

/* End of prefill (the output of Algorithm 1 feeds next-token prediction): RMSNorm of one
 * hidden row x [D], logits = lm_head x (fp32 [vocab], optional), token = argmax (lowest index). */
spts_status spts_first_token(spts_ctx* ctx, const void* x_row, const void* lm_head,
                             float* logits_out, int32_t* token_out);

/* Whole prefill (Algorithm 1, prefill phase) over n_layers layers following `plan` (host
 * array [n_layers]).  X [N, D] is updated in place; at every stage end the survivors are
 * compacted into X_alt and the two buffers swap roles, likewise pos/orig with pos_alt/orig_alt
 * (each sized for N entries).  *n_final (host) receives the final candidate count and
 * *final_in_alt (host) tells which buffer holds the result.  token_out (device, optional)
 * receives the first generated token. */
spts_status spts_prefill(spts_ctx* ctx, const spts_model_weights* mw, const spts_layer_plan* plan,
                         void* X, int32_t* pos, int32_t* orig, void* X_alt, int32_t* pos_alt,
                         int32_t* orig_alt, int N, uint32_t flags, spts_kv_layer* caches,
                         int32_t* n_final, int32_t* final_in_alt, int32_t* token_out);

/* One decode step (Algorithm 1 outside the prefill phase: no skipping).  The new token's
 * embedding row is x_in [D] (if NULL, row token_in of mw->embed is used); it runs every layer
 * densely against that layer's cache plus itself at position `pos`, appends its K/V to every
 * cache (len += 1; capacity must allow it), then the first-token head.  x_out [D] optional. */
spts_status spts_decode_step(spts_ctx* ctx, const spts_model_weights* mw, spts_kv_layer* caches,
                             const void* x_in, int32_t token_in, int32_t pos, void* x_out,
                             float* logits_out, int32_t* token_out);

/* ---------------------------------------------------------------------------------------------------------------
 * Generation with 4-bit weights and a 4-bit KV cache (the paper's decode phase reads every weight and every cached
 * row once per token; these calls are the same phase with both held in 4 bits, and the rules a generation puts on
 * its logits).
 *
 * A 4-bit group is 32, 64 or 128 elements that share a bf16 pair (scale, mid); a code c in 0..15 stands for
 *   scale * (c - 8) + mid
 * with a scale of either sign (the quantisers here make none below zero).
 * Quantising a group x (all in 64 bits; bf16() rounds to fp32 and from there to bf16, to nearest even both times):
 *   scale = bf16((max x - min x) / 15),  mid = bf16((max x + min x) / 2 + scale / 2),
 *   c = clamp(rint((x - mid) / scale) + 8, 0, 15), ties to even;  scale == 0: c = 8.
 * A group with a NaN or an infinity in it is stored as scale 0, mid NaN, and SPTS_ERR_NONFINITE goes to the device
 * status word.
 *
 * None of these calls reads anything back or depends on the host's view of a length, so all of them can be captured
 * into a CUDA graph; like every call they use the context's workspace, so two captured graphs of one context must
 * not run at the same time.  They take either storage type; SPTS_REFERENCE_KERNELS selects the plain kernels. */

/* A weight matrix [out, in] in 4 bits: byte i of a row holds element 2i in its low and 2i + 1 in its high nibble. */
typedef struct {
  const void* codes;      /* [out, in / 2] bytes, 16-byte aligned          */
  const void* params;     /* [out, in / group, 2] bf16 (scale, mid), 16-byte aligned */
  int32_t out_features;
  int32_t in_features;    /* a multiple of group                           */
  int32_t group;          /* 32, 64 or 128                                 */
} spts_w4;

/* Quantises W [out, in] (storage type) into codes and params as above. */
spts_status spts_w4_quantize(spts_ctx* ctx, const void* W, int out_features, int in_features, int group, void* codes,
                             void* params);

enum {
  SPTS_W4_NORM = 1u,      /* x is RMS-normalised first (rms_eps of the context; gains folded into W): y *= 1 / rms(x) */
  SPTS_W4_FP32_OUT = 2u   /* Y is fp32 whatever the storage type (logits) */
};
#define SPTS_W4_MAX_N 32
#define SPTS_W4_MAX_IN 131072
#define SPTS_W4_MAX_OUT (1 << 30)

/* Y[t] = X[t] W^T for n tokens, 0 <= n <= SPTS_W4_MAX_N, in_features <= SPTS_W4_MAX_IN (the codes are read once for all
 * tokens up to 32768 features, beyond that once for every 24, 16 or 8; the plain kernels read them once for every four tokens).
 *   w2 given: Y[t] = silu(X[t] W^T) * (X[t] W2^T) (gate and up projection; same shape and group)
 *   residual given: Y[t] = residual[t] + X[t] W^T (Y may be the residual itself; not with w2 or SPTS_W4_FP32_OUT)
 * X [n, in], residual and Y [n, out] in the storage type with row strides ldx, ldr, ldy in elements; X 16-byte aligned,
 * ldx a multiple of 8 (n > 1); Y lies apart from X.  Sums in fp32, one rounding at the end; in bf16 storage an element of x below
 * 2^-26 of its token's largest one is rounded first, by up to 2^-34 of that one (not by the plain kernels).  A token that holds an
 * infinity or a NaN gets outputs that are infinite or NaN; the other tokens' are what they are without it. */
spts_status spts_w4_gemv(spts_ctx* ctx, const spts_w4* w, const spts_w4* w2, const void* X, int64_t ldx, int n,
                         const void* residual, int64_t ldr, uint32_t flags, void* Y, int64_t ldy);

/* One layer's KV cache of n_seq sequences in 4 bits, head-major: the rows of one KV head of one sequence are
 * contiguous.  Inside a row of d codes (two to a byte, low nibble first) storage position p holds
 *   keys    dim 32 t + 8 c + j at p = (c * d / 32 + t) * 8 + j   (c < 4, j < 8)
 *   values  dim 32 t + 4 g + j at p = (g * d / 32 + t) * 4 + j   (g < 8, j < 4)
 * (the order in which the attention kernel's matrix fragments want them).  Groups run along the dims of a head.
 * Rows at and behind len[b] are never read as data: they may hold anything. */
typedef struct {
  void* k_codes;          /* [n_seq, Hkv, capacity, d / 2] bytes              */
  void* v_codes;
  void* k_params;         /* [n_seq, Hkv, capacity, d / group, 2] bf16        */
  void* v_params;
  int32_t* pos;           /* [n_seq, capacity] original positions, optional   */
  int32_t* len;           /* DEVICE [n_seq]: rows held by each sequence       */
  int32_t n_seq;
  int32_t capacity;       /* a multiple of 32                                 */
  int32_t group;          /* 32, 64 or 128, at most d                         */
} spts_kv4_cache;

/* Quantises n_rows rows of K and V [n_rows, Hkv, d] (K after RoPE; row strides ldk, ldv in elements) into the cache.
 * Sequence b owns rows [row_start[b], row_start[b + 1]) (device [n_seq + 1]; NULL: n_rows == n_seq, one row each);
 * they go to slots at[b], at[b] + 1, ... (device [n_seq]; NULL: behind the rows held, at = len), and len[b] becomes
 * at[b] + the sequence's number of rows.  Rows behind row_start[n_seq] (padding) are ignored.  Starts ascend within
 * [0, n_rows]; of a sequence that claims rows outside only those that there are count, and starts that break the rule
 * put SPTS_ERR_INDEX into the device status word.  A slot outside
 * [0, capacity) is not written, len is clipped to the capacity, and SPTS_ERR_WORKSPACE goes to the device status word.
 * pos [n_rows] is stored where the cache has positions.  K_read, V_read [n_rows, Hkv, d] (storage type, optional):
 * the values that the cache now stands for; padding rows of them are left as they were.  K_read may be K and V_read V, where
 * their rows are packed; they overlap nothing else. */
spts_status spts_kv4_append(spts_ctx* ctx, const spts_kv4_cache* cache, const void* K, int64_t ldk, const void* V,
                            int64_t ldv, const int32_t* pos, const int32_t* row_start, const int32_t* at, int n_rows,
                            void* K_read, void* V_read);

/* Attention of one query per sequence over what its cache holds: O[b, h] = softmax_j(Q[b, h] . K[b, j] / sqrt(d))
 * V[b, j], j < len[b], KV head h / (H / Hkv).  Q [n_seq, H, d] and O [n_seq, H * d] in the storage type, row strides
 * ldq, ldo in elements; O lies apart from Q, whose elements are below 2^100 (small ones beside large ones of a query are rounded as
 * in spts_w4_gemv).  In bf16 storage the weights meet V's scales in fp16 and V's mids in two bf16 pieces (2^-12 and 2^-17 relative).
 * Infinities and NaN in the params of a row held make the outputs that they reach infinite or NaN.
 * A sequence with len[b] <= 0 gets zeros; len[b] beyond the capacity counts as the capacity.  n_seq <= SPTS_KV4_MAX_SEQ. */
#define SPTS_KV4_MAX_SEQ 1024
spts_status spts_kv4_attention(spts_ctx* ctx, const spts_kv4_cache* cache, const void* Q, int64_t ldq, void* O_out,
                               int64_t ldo);

/* Rules for the logits of n rows.  Every pointer is a device pointer and may be NULL (the rule is off).
 * The lists are packed: row b's tokens are history[history_start[b]] .. history[history_start[b + 1] - 1] and of them
 * those from index generated_start[b] on were generated (NULL: all); its biases are the entries bias_start[b] ..
 * bias_start[b + 1] - 1.  Tokens outside [0, vocab) are ignored, and so is what a start puts outside its list. */
#define SPTS_LOGITS_MAX_LIST (1 << 29)   /* entries of a list  */
#define SPTS_LOGITS_MAX_VOCAB (1 << 30)
typedef struct {
  const int32_t* history;          /* [n_history]  */
  const int32_t* history_start;    /* [n + 1]      */
  const int32_t* generated_start;  /* [n]          */
  const float* repetition;         /* [n] > 0      */
  const float* presence;           /* [n]          */
  const float* frequency;          /* [n]          */
  const int32_t* bias_token;       /* [n_bias]     */
  const float* bias_value;         /* [n_bias]     */
  const int32_t* bias_start;       /* [n + 1]      */
  const uint32_t* mask;            /* [n, ld_mask] words; bit (v % 32) of word v / 32 set: token v is allowed */
  int64_t ld_mask;
  int32_t n_history;
  int32_t n_bias;
} spts_logits_rules;

/* For every row b and token v, each step one fp32 operation:
 *   a token of the history:  l = l > 0 ? l / repetition[b] : l * repetition[b]
 *   a generated token:       l = l - frequency[b] * (times generated);  l = l - presence[b]
 *   l = l + bias (of several entries for one token the last one counts)
 *   l = -inf where the mask does not allow the token
 * out [n, vocab] (row stride ldo; may be the logits themselves; NULL: not written) and token_out [n] (optional) = the
 * lowest index of the largest l; NaN never wins; -1 where no token is left above -inf. */
spts_status spts_process_logits(spts_ctx* ctx, const float* logits, int64_t ld, int n, int vocab,
                                const spts_logits_rules* rules, float* out, int64_t ldo, int32_t* token_out);

/* One layer's weights in 4 bits: the projections of q, k and v stacked row after row, the others as in spts_layer_weights.
 * RMSNorm gains are folded into the columns (spts_fold_norm_gain) before quantising. */
typedef struct {
  spts_w4 wqkv;    /* [(H + 2 Hkv) * d, D] */
  spts_w4 wo;      /* [D, H * d]           */
  spts_w4 w_gate;  /* [Dff, D]             */
  spts_w4 w_up;    /* [Dff, D], the group of w_gate */
  spts_w4 w_down;  /* [D, Dff]             */
} spts_layer_weights4;

typedef struct {
  const spts_layer_weights4* layers; /* host array [n_layers] */
  spts_w4 lm_head;                   /* [vocab, D]            */
  const void* embed;                 /* [vocab, D] in the storage type, used with token_in */
} spts_model_weights4;

/* One decode step with 4-bit weights and caches for all sequences of the caches (Algorithm 1 outside the prefill phase: no
 * skipping): one new token each, at most SPTS_W4_MAX_N and max_seq sequences.  `caches` is a host array [n_layers] with the
 * same n_seq.  The tokens' rows are x_in [n_seq, D], or, if that is NULL, rows token_in[b] (DEVICE [n_seq]) of mw->embed (a
 * token outside the vocabulary gives a row of zeros and SPTS_ERR_INDEX in the device status word).  pos (DEVICE [n_seq]) are
 * their original positions.  Every layer appends the token's K / V to its cache (len grows on the device) and attends to what
 * the cache then holds.  x_out [n_seq, D] optional.  logits_out [n_seq, vocab] fp32 receives the head's logits, with the rules
 * applied where there are any (rules without logits_out are refused); token_out [n_seq] (optional, needs logits_out) the largest
 * one's token as in spts_process_logits.  A step that is refused leaves the caches as they were.  Everything that changes from
 * step to step lies on the device, so one captured step can be replayed: token_out may be the next step's token_in. */
spts_status spts_decode_step4(spts_ctx* ctx, const spts_model_weights4* mw, const spts_kv4_cache* caches, const void* x_in,
                              const int32_t* token_in, const int32_t* pos, const spts_logits_rules* rules, void* x_out,
                              float* logits_out, int32_t* token_out);

/* ---------------------------------------------------------------------------------------------------------------
 * Serving over a paged KV cache in the storage type (the paper keeps one contiguous cache per layer, of another length in every
 * layer; pages let many sequences and layers of different lengths share one pool), with chunks of new tokens: the next turn of a
 * conversation, drafted tokens that are verified, or one token each.
 *
 * As in the calls above nothing is read back and everything that changes from call to call lies on the device, so the calls can be
 * captured into a CUDA graph; two captured graphs of one context must not run at the same time. */

#define SPTS_PAGED_MAX_SEQ 1024
#define SPTS_PAGED_MAX_ROWS (1 << 25)    /* rows of one sequence: max_pages * page_size */

/* One layer's cache.  Row j of sequence b lies in page table[b, j / page_size] at j % page_size; len[b] rows are held (a length
 * beyond max_pages * page_size counts as that, one below 0 as 0).  What lies behind a sequence's rows and in pages of no sequence may
 * hold anything.  Sequences may share pages that no call writes: an append writes the pages of the new rows, spts_paged_weights and
 * spts_paged_evict those of all rows.  An entry of the table that a held or new row needs and that is outside [0, n_pages) puts
 * SPTS_ERR_INDEX into the device status word; its rows read as zeros and are not written, and an eviction ranks them last. */
typedef struct {
  void* k;                /* [n_pages, page_size, Hkv, d] in the storage type (K after RoPE), 16-byte aligned */
  void* v;
  int32_t* pos;           /* [n_pages, page_size] original positions, optional      */
  float* weight;          /* [n_pages, page_size] gathered attention weight, optional */
  const int32_t* table;   /* [n_seq, max_pages]                                     */
  int32_t* len;           /* DEVICE [n_seq]                                         */
  int32_t n_pages;
  int32_t page_size;      /* 16, 32, 64, 128 or 256                                 */
  int32_t max_pages;
  int32_t n_seq;          /* at most SPTS_PAGED_MAX_SEQ                             */
} spts_paged_kv;

/* Copies n_rows rows of K and V [n_rows, Hkv, d] (row strides ldk, ldv in elements) into the cache; they overlap none of its
 * buffers.  Sequence b owns rows [row_start[b], row_start[b + 1]) (device [n_seq + 1]; NULL: n_rows == n_seq, one row each); they
 * become its rows at[b], at[b] + 1, ... (device [n_seq]; NULL: behind the rows held), and len[b] becomes at[b] + their number.
 * Rows behind row_start[n_seq] (padding) are ignored.  Starts ascend within [0, n_rows]; of a sequence that claims rows outside only
 * those that there are count, and starts that break the rule put SPTS_ERR_INDEX into the device status word.  A row that would lie
 * outside [0, max_pages * page_size) is not written, len is clipped to that range, and SPTS_ERR_WORKSPACE goes to the device status
 * word.  pos [n_rows] is stored where the cache has positions (NULL: they stay as they were); the weight of a new row is 0. */
spts_status spts_paged_append(spts_ctx* ctx, const spts_paged_kv* cache, const void* K, int64_t ldk, const void* V, int64_t ldv,
                              const int32_t* pos, const int32_t* row_start, const int32_t* at, int n_rows);

/* Attention of a chunk of new tokens over the cache that holds them already (append first).  Sequence b owns the queries
 * [row_start[b], row_start[b + 1]) (as in spts_paged_append); they are its last n rows, and query i of n sees the rows j <= len[b] - n + i:
 *   O[i, h] = softmax_j(Q[i, h] . K[j, h / (H / Hkv)] / sqrt(d)) V[j, h / (H / Hkv)],   lse[i, h] = log sum_j exp(Q[i, h] . K[j] / sqrt(d)).
 * Q [n_rows, H, d] and O [n_rows, H * d] in the storage type, row strides ldq, ldo in elements, O apart from Q; lse_out fp32
 * [n_rows, H], optional.  A query that sees no row gets zeros and -inf; queries behind row_start[n_seq] (padding) are left as they were.
 * What a query does not see does not reach it, whatever it holds.  In bf16 storage the weights are rounded to bf16 before they meet V. */
spts_status spts_paged_attention(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start,
                                 int n_rows, void* O_out, int64_t ldo, float* lse_out);

/* The attention weight that the rows of the cache get from the queries of spts_paged_attention, gathered in cache->weight:
 *   weight[j] = decay * weight[j] + 1 / H sum_i sum_h exp(Q[i, h] . K[j, h / (H / Hkv)] / sqrt(d) - lse[i, h])
 * over the queries i that see row j (the mean over heads of Eq. 4, summed over the queries), for all rows held by all sequences.
 * lse is what spts_paged_attention gave for these queries.  decay >= 0: 1 adds up over calls, 0 forgets what was there (whatever it
 * was).  The last rows of a prompt are a window of queries as well: row_start then counts those alone. */
spts_status spts_paged_weights(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start,
                               int n_rows, const float* lse, float decay);

/* Cuts every sequence that holds more than keep[b] rows (DEVICE [n_seq]; below 0: the sequence is left alone) down to keep[b].
 * The rows at positions pos < n_sink and pos > p - n_recent, p being the largest position that the sequence holds, stay before all
 * others, the others by the largest weight; ties go to the row that comes first in the cache, a weight that is NaN ranks last
 * (SPTS_ERR_NONFINITE in the device status word, also for a row that stays before all others).  Rows that stay and lie among the first keep[b] are not moved: the r-th place among those that
 * an evicted row leaves takes the r-th of the staying rows that lie behind, with its K, V, position and weight.  So the rows
 * are no longer in the order of their positions, which attention does not ask for.  len[b] becomes keep[b]; the pages behind the
 * rows left are free.  cache->weight is needed, cache->pos where n_sink > 0 or n_recent > 0. */
spts_status spts_paged_evict(spts_ctx* ctx, const spts_paged_kv* cache, const int32_t* keep, int n_sink, int n_recent);

/* What a row of logits says about a token: for each of n rows, l = logits[row] (fp32, row stride ld),
 *   logprob = l[target] - log sum_v exp(l[v]),   entropy = - sum_v p[v] log p[v],   rank = number of tokens before the target,
 *   top_logprob, top_token [n, n_top] = the n_top largest tokens in order
 * where a token comes before another if its logit is larger, or equal and its index lower.  targets and all outputs are device pointers; each
 * output may be NULL (logprob_out and rank_out need targets).  A token at -inf has no share and is no alternative: places that are left get -inf and
 * token -1.  A row with no token above -inf: logprob -inf, entropy 0.  A target outside [0, vocab) (padding): logprob 0,
 * rank -1.  A row that holds a NaN or +inf: logprob, entropy and the log probabilities of its alternatives are NaN; NaN is never an alternative and
 * never before a target. */
#define SPTS_LOGPROBS_MAX_TOP 32
spts_status spts_token_logprobs(spts_ctx* ctx, const float* logits, int64_t ld, int n, int vocab, const int32_t* targets, int n_top,
                                float* logprob_out, int32_t* rank_out, float* entropy_out, float* top_logprob_out,
                                int32_t* top_token_out);

#ifdef __cplusplus
}
#endif
#endif /* SPTS_H_ */
