/*
 * earlytom.h — C boundary of the MI355X (gfx950) EarlyTom vision-encoder library.
 *
 * The library runs a pre-LayerNorm ViT encoder (SigLIP layout) over the frames of a
 * video clip and applies the paper's early token compression once, inside the encoder:
 * adjacent-frame similarity (Sec. 3.2) -> segment boundaries (Eq. 1, alpha = 1) ->
 * per-position mean over each segment (Sec. 3.2, simplified whole-segment merge) ->
 * per-frame top-k token selection (Eq. 4; score = squared L2 norm, ties to the lower
 * position) -> gather in original order (Eq. 7) -> remaining blocks on the kept tokens.
 *
 * Conventions
 *   - Pointers named *_dev are DEVICE memory owned by the caller; pointers without the
 *     suffix are HOST memory.  The library never frees caller memory and returns nothing
 *     the caller must free, except the opaque encoder (et_encoder_destroy).
 *   - All device activations are bfloat16 (bit patterns, uint16_t), row-major; index and
 *     offset data are int32.
 *   - Every function returning int returns ET_OK (0) or a negative ET_ERR_* code; the
 *     message of the last failure on the calling thread is available from et_last_error().
 *     Arguments are validated before any device work is issued.
 *   - `hip_stream` is a hipStream_t passed as void* (NULL = the default stream).  All
 *     work is enqueued on it.  One encoder must be used by one stream at a time; different
 *     encoders share no state and may be driven at once from different host threads and streams.
 *   - No exceptions cross this boundary.
 */
#ifndef EARLYTOM_H
#define EARLYTOM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ET_OK 0
#define ET_ERR_INVALID_ARG (-1) /* null pointer, size or parameter out of range          */
#define ET_ERR_WORKSPACE (-2)   /* workspace_bytes smaller than the required size        */
#define ET_ERR_HIP (-3)         /* a HIP runtime call or kernel launch failed            */
#define ET_ERR_ALLOC (-4)       /* host or device allocation failed (create only)        */
#define ET_ERR_UNSUPPORTED (-5) /* a shape the kernels are not instantiated for          */

typedef struct et_encoder et_encoder; /* opaque; owns the packed device weights */

/* Encoder shape.  Tokens per frame L = (image_h / patch) * (image_w / patch); pixels past the
 * last whole patch are ignored.  head_dim = d_model / n_heads must be 16, 32, 64, 72, 80, 96
 * or 128; d_model must be a multiple of 64, at most 4096. */
typedef struct {
  int32_t n_layers, d_model, n_heads, d_mlp, patch, image_h, image_w, channels;
  float ln_eps;
  int32_t has_final_ln;
} et_config;

/* HOST float32 weights, row-major, read only during et_encoder_create (converted once to
 * bfloat16 with round-to-nearest-even; LayerNorm gains/biases and linear biases stay fp32).
 * Linear layers are y = x * W^T + b with W stored out-features major. */
typedef struct {
  const float *patch_w; /* [D, C*P*P], patch vector flattened in (c, py, px) order        */
  const float *patch_b; /* [D]                                                            */
  const float *pos_emb; /* [L, D], token l = gy * (image_w / patch) + gx                  */
  /* per-layer tables: n_layers host pointers each */
  const float *const *ln1_g, *const *ln1_b; /* [D]                                        */
  const float *const *wqkv, *const *bqkv;   /* [3D, D] rows q | k | v; head h = rows h*hd.. */
  const float *const *wo, *const *bo;       /* [D, D], [D]                                */
  const float *const *ln2_g, *const *ln2_b; /* [D]                                        */
  const float *const *w1, *const *b1;       /* [Mh, D], [Mh]                              */
  const float *const *w2, *const *b2;       /* [D, Mh], [D]                               */
  const float *final_ln_g, *final_ln_b;     /* [D]; may be NULL iff !has_final_ln         */
} et_weights;

/* Outputs.  Every *_dev buffer is caller-allocated with the stated capacity (in elements). */
typedef struct {
  uint16_t *tokens_dev;   /* bf16, capacity T*L*D; written [n_tokens, D], frame-major      */
  int32_t *kept_idx_dev;  /* capacity T*L; written [n_tokens]: spatial position l of each
                             output token, ascending inside a frame                        */
  int32_t *cu_tokens_dev; /* capacity T+1; written [n_frames_out+1]: token offset of each
                             output frame                                                  */
  int32_t *seg_start_dev; /* capacity T+1; written [n_frames_out+1]: first input frame of
                             each segment, last entry = T                                  */
  float *frame_sim_dev;   /* capacity max(T-1,1); written s_t for t = 1..T-1; may be NULL  */
  int32_t n_frames_out;   /* HOST, valid on return: number of segments N                   */
  int32_t n_tokens;       /* HOST, valid on return: N * k                                  */
} et_output;

/* ---- the hot path ------------------------------------------------------------------- */

/* Pack `weights` for `config` onto the current HIP device.  max_frames bounds T of later
 * calls.  On success *out receives the encoder.  The two LayerNorms of every block are folded
 * into the QKV and fc1 weights here (gamma scales the weight columns, each folded row is centred
 * so that the row mean of the input drops out, beta goes into the bias), so the blocks compute
 * only the row scale 1 / sqrt(var + eps) and apply it in the GEMM epilogue; the folded weights are
 * rounded to bfloat16 with error diffusion along each row.  Errors: INVALID_ARG, UNSUPPORTED,
 * ALLOC, HIP. */
int et_encoder_create(const et_config *config, const et_weights *weights, int32_t max_frames,
                      et_encoder **out);
void et_encoder_destroy(et_encoder *enc); /* NULL is allowed */

/* Bytes of device workspace et_encode_clip needs for a clip of T frames (0 on bad arguments). */
size_t et_workspace_bytes(const et_encoder *enc, int32_t T);

/* Encode one clip.
 *   frames_dev   float32 [T, C, image_h, image_w] (NCHW), device.
 *   merge_layer  m: compression acts on the residual stream after m blocks have run,
 *                0 <= m <= n_layers (m = n_layers: after the last block, before the final
 *                LayerNorm).  m < 0 disables compression (plain encoder: N = T, k = L).
 *   sim_threshold  tau of Eq. 1: frame t opens a new segment iff s_t < tau (NaN s_t also
 *                opens one).  +INFINITY makes every frame its own segment.  NaN is rejected.
 *   keep_ratio   in (0, 1]; k = et_keep_count(L, keep_ratio) tokens are kept per output frame.
 * The host waits twice: in the middle for an event on `hip_stream` (N is copied to pinned memory
 * of the encoder right after the boundary scan, so the blocks that follow are enqueued while the
 * merge, selection and compaction still run) and for the whole stream before returning.
 * Blocks that run on fewer than 8192 rows (those after the selection) have their weights read
 * ahead by small kernels on a stream the encoder owns (default priority), released by an event on
 * `hip_stream` and joined to it before the call returns; they read encoder memory only.  One
 * encoder therefore serves one encode call at a time.
 * Errors: INVALID_ARG (incl. T < 1 or T > max_frames), WORKSPACE, HIP. */
int et_encode_clip(et_encoder *enc, const float *frames_dev, int32_t T, int32_t merge_layer,
                   float sim_threshold, float keep_ratio, void *workspace_dev,
                   size_t workspace_bytes, void *hip_stream, et_output *out);

/* The compression stage alone on caller-supplied hidden states x_dev (bf16 [T, L, D],
 * D a multiple of 8, T >= 1): similarity, boundary scan, segment mean, top-k, compaction.
 * out->tokens_dev receives the packed merged tokens [N*k, D].  Needs
 * et_merge_workspace_bytes(T, L, D) bytes of workspace.  Synchronises the stream once
 * before returning. */
int et_merge_select(const uint16_t *x_dev, int32_t T, int32_t L, int32_t D, float sim_threshold,
                    float keep_ratio, void *workspace_dev, size_t workspace_bytes,
                    void *hip_stream, et_output *out);
size_t et_merge_workspace_bytes(int32_t T, int32_t L, int32_t D);

/* et_merge_select for callers that cannot allocate or hand over a workspace (a stage under HIP graph
 * capture set-up, a tight serving loop, a harness that forbids hipMalloc): same arguments minus the
 * workspace, same kernels, same results bit for bit.  The scratch the kernels need (cosines, their
 * partial sums, scores, the merged frames, counters) lives in a device array that is part of the
 * library's code object, ET_STATIC_SCRATCH_BYTES large, one copy per GPU for the life of the process;
 * its address is looked up once per device, on the first call there.  The call allocates nothing and
 * frees nothing.  Shapes with et_merge_workspace_bytes(T, L, D) above ET_STATIC_SCRATCH_BYTES (e.g. more
 * than 39 frames of 729 x 1152) are rejected with ET_ERR_WORKSPACE before any device work.  Every call
 * on a GPU uses that GPU's one array: calls that overlap on one GPU (from several threads or streams)
 * race; nothing in it has to start at zero, so a call is not affected by what the previous one left.
 * Synchronises the stream once before returning, like et_merge_select. */
#define ET_STATIC_SCRATCH_BYTES (64u << 20)
int et_merge_select_static(const uint16_t *x_dev, int32_t T, int32_t L, int32_t D, float sim_threshold,
                           float keep_ratio, void *hip_stream, et_output *out);

/* k = clamp(floor(keep_ratio * L + 1e-4), 1, L); 0 on bad arguments.  (The paper floors
 * window sizes in Eq. 6 but does not state the rounding for top-K; this rule is this
 * library's reading.) */
int32_t et_keep_count(int32_t L, float keep_ratio);

const char *et_last_error(void); /* thread-local, never NULL */

/* ---- the paper-exact compression forms -------------------------------------------------
 * A policy selects, per stage, between the simple form used by et_encode_clip / et_merge_select
 * and the form the paper describes:
 *   merge_mode   ET_MERGE_MEAN: a segment becomes one frame (per-position mean).
 *                ET_MERGE_ALG1: Alg. 1 — head and tail frame of a segment are kept, middle frames
 *                are walked left to right and (F_i, F_{i+1}) are fused with weights
 *                (s_i, s_{i+1}) / (s_i + s_{i+1}) iff s_i > tau_merge and s_i > s_{i+1} (Eq. 2-3),
 *                s_i = Sim(F_i, F_{i+1}); a pair is eligible only if both are middle frames.
 *   select_mode  ET_SELECT_UNIFORM: every output frame keeps k = et_keep_count(L, ratio) tokens.
 *                ET_SELECT_DECOUPLED: Alg. 2 — head/tail ("dynamic") frames keep the top r_hat
 *                tokens, r_hat = clamp(floor(ratio*T*L/N + 0.5), 1, L) (this library's reading of
 *                Eq. 5: `ratio` is the overall retention relative to the T*L input tokens); other
 *                ("static") frames keep the arg-max of each of ceil(L / w) windows of
 *                w = floor(L / r_hat) consecutive positions (Eq. 6).
 *   alpha        smoothing factor of Eq. 1 in (0, 1]; the smoothed similarity restarts at every
 *                segment start.  tau_seg: segment threshold.  tau_merge: Eq. 2 threshold.
 *   score_mode   ET_SCORE_L2NORM: a token's score is its squared L2 norm (as on the simple path).
 *                ET_SCORE_ATTENTION: the attention the token receives in the encoder block just
 *                before the selection (Sec. 3.3 and Alg. 2 rank by a score per token taken from the
 *                encoder's attention without defining it; this library's reading): the mean over heads and over the queries
 *                of its frame of softmax(Q K^T / sqrt(hd))[query][token].  Needs a block before
 *                the selection (select layer >= 1) whose input is what the selection sees, so no
 *                merge may run at the select layer itself; only et_encode_clip_multi accepts it.
 * Tie-breaks and ordering are those of the simple path.  With these forms output frames
 * keep different token counts: cu_tokens_dev is ragged, seg_start_dev has n_segments + 1 entries
 * and n_frames_out counts output frames (>= segments). */
enum { ET_MERGE_MEAN = 0, ET_MERGE_ALG1 = 1 };
enum { ET_SELECT_UNIFORM = 0, ET_SELECT_DECOUPLED = 1 };
enum { ET_SCORE_L2NORM = 0, ET_SCORE_ATTENTION = 1 };
typedef struct {
  int32_t merge_mode, select_mode;
  float alpha, tau_seg, tau_merge, ratio;
  int32_t score_mode;
} et_policy;

/* Optional description of the output frames (device arrays of capacity T, or NULL). */
typedef struct {
  int32_t *frame_first_dev;   /* first ORIGINAL input frame behind output frame n              */
  int32_t *frame_count_dev;   /* number of consecutive original frames behind it               */
  int32_t *frame_dynamic_dev; /* 1 = head or tail frame of its segment ("dynamic"), 0 = static */
  int32_t n_segments;         /* HOST, valid on return                                         */
} et_plan_out;

/* et_merge_select / et_encode_clip under a policy.  Same buffers, workspace sizes and
 * synchronisation as the simple entry points; `plan` may be NULL.  Errors as there, plus
 * INVALID_ARG for alpha outside (0, 1], NaN thresholds, ratio outside (0, 1] or unknown modes. */
int et_merge_select_policy(const uint16_t *x_dev, int32_t T, int32_t L, int32_t D, const et_policy *policy,
                           void *workspace_dev, size_t workspace_bytes, void *hip_stream, et_output *out,
                           et_plan_out *plan);
int et_encode_clip_policy(et_encoder *enc, const float *frames_dev, int32_t T, int32_t merge_layer,
                          const et_policy *policy, void *workspace_dev, size_t workspace_bytes,
                          void *hip_stream, et_output *out, et_plan_out *plan);

/* ---- per-kernel timing (optional) ----------------------------------------------------
 * With profiling on, et_encode_clip brackets every kernel launch with HIP events on
 * `hip_stream` and accumulates elapsed time and launch counts per kernel kind.  Off by
 * default (events cost a little host time).  An encoder of width 64, at most 64 tokens per frame and an MLP of at most 256
 * runs all blocks between two stages as one launch, under ET_K_MISC. */
enum {
  ET_K_IM2COL = 0, ET_K_GEMM_PATCH, ET_K_LAYERNORM, ET_K_GEMM_QKV, ET_K_ATTENTION,
  ET_K_GEMM_OUT, ET_K_GEMM_FC1, ET_K_GEMM_FC2, ET_K_SIMILARITY, ET_K_SCAN, ET_K_MERGE,
  ET_K_SELECT, ET_K_COMPACT, ET_K_MISC, ET_K_SCORE, ET_K_COUNT
};
int et_profile_enable(et_encoder *enc, int32_t on);
/* Reads the accumulators into ms[2 * ET_K_COUNT] and launches[2 * ET_K_COUNT]: entry
 * kind + ET_K_COUNT * phase, phase 0 = launches on all T*L tokens (up to and including the
 * compression stage), phase 1 = launches on the kept tokens; clears them if `reset` != 0. */
int et_profile_read(et_encoder *enc, double *ms, int64_t *launches, int32_t reset);
const char *et_kernel_name(int32_t kind);
/* The same for the stand-alone stage: with on = 1, et_merge_select and et_merge_select_static bracket
 * the whole launch sequence with two HIP events on `hip_stream`; with on = 2 also every launch (which
 * lengthens the sequence by the events' own cost).  The read fills
 * ms[ET_K_COUNT] / launches[ET_K_COUNT] per kernel kind, *total_ms with the summed time between the
 * first launch's start and the last launch's end (launch gaps included, the final device-to-host copy
 * and stream wait excluded) and *calls.  Process-wide state, not thread-safe; off by default. */
int et_merge_profile_enable(int32_t on);
int et_merge_profile_read(double *ms, int64_t *launches, double *total_ms, int64_t *calls, int32_t reset);

/* ---- single steps (the device code of the hot path, one step per call; for parity tests and
 *      micro-benchmarks).  All asynchronous on `hip_stream` unless stated.  On narrow rows the hot path
 *      runs selection and gather (et_topk_select + et_compact_tokens) as ONE launch on the same select
 *      routine; the two calls below launch them separately. ------------- */

/* Sec. 3.2: cos_dev [T-1, L] float32 per-position cosine similarities of frames t and t-1,
 * sim_dev [T-1] their mean over positions.  x_dev bf16 [T, L, D]. */
int et_frame_similarity(const uint16_t *x_dev, int32_t T, int32_t L, int32_t D, float *cos_dev,
                        float *sim_dev, void *hip_stream);

/* Eq. 1 (alpha = 1): seg_start_dev [capacity T+1] and *n_seg_dev (one int32) from sim_dev [T-1]. */
int et_segment_scan(const float *sim_dev, int32_t T, float sim_threshold, int32_t *seg_start_dev,
                    int32_t *n_seg_dev, void *hip_stream);

/* Segment mean and score: merged_dev bf16 [N, L, D] (capacity T*L*D), score_dev float32
 * [N, L] (capacity T*L); N and the ranges are read from the device arrays. */
int et_segment_mean(const uint16_t *x_dev, int32_t T, int32_t L, int32_t D,
                    const int32_t *seg_start_dev, const int32_t *n_seg_dev, uint16_t *merged_dev,
                    float *score_dev, void *hip_stream);

/* Eq. 4: for each of n_rows rows of score_dev [n_rows, L] (float32, non-negative or NaN), the
 * k positions that come first in the order (score descending, position ascending), written
 * ascending to kept_idx_dev [n_rows, k]. */
int et_topk_select(const float *score_dev, int32_t n_rows, int32_t L, int32_t k,
                   int32_t *kept_idx_dev, void *hip_stream);

/* Eq. 7: out_dev[(n*k + j), :] = merged_dev[n, kept_idx_dev[n*k + j], :], n < n_rows. */
int et_compact_tokens(const uint16_t *merged_dev, const int32_t *kept_idx_dev, int32_t n_rows,
                      int32_t L, int32_t D, int32_t k, uint16_t *out_dev, void *hip_stream);

/* LayerNorm over rows: y = (x - mean) / sqrt(var + eps) * gamma + beta; x, y bf16 [rows, D]
 * (may alias), gamma/beta float32 [D] on the device. */
int et_layernorm(const uint16_t *x_dev, const float *gamma_dev, const float *beta_dev, float eps,
                 int32_t rows, int32_t D, uint16_t *y_dev, void *hip_stream);

/* C[M, N] = A[M, K] * W[N, K]^T + bias, bf16 in / fp32 accumulate / bf16 out, with an
 * epilogue: 0 bias only, 1 bias + GELU-tanh, 2 bias + residual (res_dev bf16 [M, N], may
 * alias c_dev).  bias_dev float32 [N].  Standalone form for tests: any M >= 1, N and K
 * multiples of 8; allocates and frees padded copies of the operands itself and synchronises.
 * tile_config: -1 = the library's choice (which may also split the last tile rows or a thin last
 * column off into a launch of its own), else one workgroup tiling: 0 = 256 x 256 with 8 wavefronts
 * and 1 = 128 x 128 with 4 (persistent kernel), 2 = 64 x 64 with 4, 3 = 128 x 64 and 4 = 128 x 128
 * with 8 (kernels that split K over the wavefronts of a workgroup, for few rows), 5 = 256 x 128
 * with 8. */
int et_gemm_bf16(const uint16_t *a_dev, const uint16_t *w_dev, const float *bias_dev,
                 const uint16_t *res_dev, int32_t M, int32_t N, int32_t K, int32_t epilogue,
                 int32_t tile_config, uint16_t *c_dev, void *hip_stream);

/* Per-frame multi-head attention on a fused projection buffer qkv_dev bf16 [rows, 3D]
 * (q | k | v, head h at columns h*hd): out_dev bf16 [rows, D].  cu_tokens_dev [n_frames+1]
 * gives each frame's row range; max_len >= the longest frame. */
int et_attention(const uint16_t *qkv_dev, const int32_t *cu_tokens_dev, int32_t n_frames,
                 int32_t max_len, int32_t n_heads, int32_t head_dim, uint16_t *out_dev,
                 void *hip_stream);

/* The same attention for frames of equal length `len` (frame f = rows f*len .. f*len+len-1),
 * which is what the hot path runs; same kernels (K tiles stream through LDS by direct global -> LDS
 * loads, V^T fragments by LDS transpose reads; few queries: key tiles split over groups of wavefronts;
 * many: a wavefront owns two blocks of 32 queries). */
int et_attention_uniform(const uint16_t *qkv_dev, int32_t n_frames, int32_t len, int32_t n_heads,
                         int32_t head_dim, uint16_t *out_dev, void *hip_stream);

/* The start of encoder block `layer` on caller-supplied hidden states x_dev (bf16 [rows, D]), with the
 * bits that et_encode_clip gets: the row scales 1 / sqrt(var + eps) of LayerNorm 1 into rstd_dev
 * (float32 [rows]) and the fused projection with the LayerNorm folded in into qkv_dev (bf16
 * [rows, 3D], q | k | v).  Lets a test rank attention-received scores on the very q and k the
 * encoder used.  Errors: INVALID_ARG, HIP. */
int et_encoder_block_qkv(et_encoder *enc, int32_t layer, const uint16_t *x_dev, int32_t rows,
                         float *rstd_dev, uint16_t *qkv_dev, void *hip_stream);

/* Stage I at several encoder layers, Stage II once (the paper merges at three layers, e.g. 6, 14,
 * 20, and selects after the encoder; Table 8).  At every layer of merge_layers[0..n_merge_layers)
 * (strictly ascending, each <= select_layer) the adjacent-frame similarity of the CURRENT frames
 * drives Eq. 1 and the merge of policy->merge_mode; frames keep all L tokens.  At select_layer
 * (after that layer's merge if they coincide) the selection of policy->select_mode runs once:
 * dynamic flags come from the most recent merge (all frames dynamic if n_merge_layers = 0), the
 * re-scaled count of Eq. 5 uses the original T.  seg_start_dev and the plan's frame ranges are in
 * original frame indices.  Synchronises the stream once per merge / select layer and at the end;
 * frame_sim_dev receives the similarities of the first merge layer only. */
int et_encode_clip_multi(et_encoder *enc, const float *frames_dev, int32_t T, const int32_t *merge_layers,
                         int32_t n_merge_layers, int32_t select_layer, const et_policy *policy,
                         void *workspace_dev, size_t workspace_bytes, void *hip_stream, et_output *out,
                         et_plan_out *plan);

/* Attention-received scores (ET_SCORE_ATTENTION) of equal-length frames: score_dev float32
 * [n_frames, L], each row summing to 1, from the q and k thirds of qkv_dev bf16 [n_frames * L,
 * 3 * n_heads * head_dim] (the layout et_attention reads).  scratch_dev: at least
 * et_attention_scores_scratch_bytes(n_frames, L, n_heads) bytes.  head_dim a multiple of 8, <= 128. */
size_t et_attention_scores_scratch_bytes(int32_t n_frames, int32_t L, int32_t n_heads);
int et_attention_scores(const uint16_t *qkv_dev, int32_t n_frames, int32_t L, int32_t n_heads,
                        int32_t head_dim, void *scratch_dev, float *score_dev, void *hip_stream);

/* ---- the projector that follows the encoder (Sec. 3.1: vision encoder -> projector -> language
 *      model) -------------------------------------------------------------------------------------
 * A two-layer MLP on the kept tokens, out = W2 * gelu_tanh(W1 * x + b1) + b2, so that the time of
 * encoder plus everything done to the visual tokens can be taken as one figure when the selection sits after the
 * encoder (merge_layer = n_layers, where the paper places Stage II).  The paper does not describe the
 * projector; the two-layer form and the GELU are this library's reading, the widths are arguments.
 * Weights: HOST float32, out-features major (w1 [d_hidden, d_in], w2 [d_out, d_hidden]), converted once
 * to bfloat16.  d_in a multiple of 64; d_hidden and d_out multiples of 8. */
typedef struct et_projector et_projector;
int et_projector_create(int32_t d_in, int32_t d_hidden, int32_t d_out, const float *w1, const float *b1,
                        const float *w2, const float *b2, et_projector **out);
void et_projector_destroy(et_projector *proj); /* NULL is allowed */
size_t et_projector_workspace_bytes(const et_projector *proj, int32_t rows);
/* tokens_dev bf16 [rows, d_in] -> out_dev bf16 [rows, d_out]; asynchronous on `hip_stream`.
 * Errors: INVALID_ARG, WORKSPACE, HIP. */
int et_project_tokens(et_projector *proj, const uint16_t *tokens_dev, int32_t rows, void *workspace_dev,
                      size_t workspace_bytes, uint16_t *out_dev, void *hip_stream);

/* ---- the key-value cache of the language model behind the projector ------------------------------
 * The kept tokens end up as keys and values in a cache that every later token of the answer reads.  The cache is paged:
 * `n_pages` pages of `page_size` tokens in one device buffer that the caller owns, and a page table that
 * gives each sequence its pages.  These calls store new keys and values (in 8 or 4 bits if asked to), read them
 * back, and compute the attention of one new token for each sequence.
 *
 * A page is et_kv_page_bytes() bytes, one key-value head after the other; a head's part holds
 *     keys [page_size, head_dim] | values [page_size, head_dim] | key maxima [page_size] | value maxima [page_size],
 * so pages can be copied, shared and moved as they are.  ET_KV_BF16: keys and values in bfloat16, no maxima.  ET_KV_INT8 and
 * ET_KV_E4M3: one byte per value (two's complement; OCP 8-bit float with 4 exponent bits); a row x of
 * head_dim values is held as its largest magnitude m (bfloat16, exact) and the codes round(x * Q / m), ties to even, Q = 127
 * or 448; it stands for code * m / Q.  A row with an infinity or a NaN has m = NaN and reads back as NaN throughout.
 * ET_KV_MXFP4: 4 bits per value and one exponent for 32 of them (4.25 bits in all where head_dim is a multiple of 32, 4.3 for 80).
 * A head's part holds
 *     keys [page_size, head_dim / 2] | values [page_size, head_dim / 2] | key exponents [page_size, blocks] | value exponents [blocks, page_size],
 * blocks = ceil(head_dim / 32) (the last of 80 has 16 dimensions), an exponent being the byte e + 127, two codes a byte, the even
 * dimension in the low half: the sign (8) and the number (0 to 7) of one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, times 2^e.  e is the
 * smallest with which the block's largest magnitude is at most 7 * 2^e, within -125 .. 125; the nearest value is taken, ties to the even code,
 * and magnitudes past 6 * 2^e become 6 * 2^e.  A block with an infinity or a NaN has the byte 255 and codes 0, and reads back as NaN; the
 * row's other blocks keep their values.  Every value is exact in bfloat16.
 *
 * Token `pos` of sequence b is token pos % page_size of page page_table[b * table_stride + pos / page_size].  An
 * entry outside [0, n_pages) is no page: nothing is stored there, it reads back as zeros, and attention leaves its tokens out;
 * so do the calls with positions past pages_per_seq * page_size.  All of this is checked on the device; lengths and
 * tables stay there, so the calls can be captured into a graph and replayed as the sequences grow.
 * Sequences may share pages that they only read.  Two rows of one et_kv_append that come to lie in the same place leave
 * either's values there, and not necessarily those of one row alone.
 *
 * Rows: et_kv_append and et_kv_read take the new (or wanted) tokens of all sequences as consecutive rows; rows
 * cu_rows[b] .. cu_rows[b + 1] are the LAST tokens of sequence b, i.e. row cu_rows[b + 1] - 1 is position kv_len[b] - 1
 * (kv_len counts the new tokens).  cu_rows_dev = NULL: one row for each sequence (rows = n_seqs).  Rows outside
 * cu_rows[0] .. cu_rows[n_seqs], such as padding behind the last sequence, are neither read nor written; a row whose
 * position would be negative (an idle slot of kv_len 0) is not stored and reads back as zeros. */
enum { ET_KV_BF16 = 0, ET_KV_E4M3 = 1, ET_KV_INT8 = 2, ET_KV_MXFP4 = 4 };
typedef struct {
  void *data_dev;              /* n_pages * et_kv_page_bytes bytes, aligned to 16                    */
  int32_t n_pages, page_size;  /* page_size 16, 32, 64, 128 or 256                                   */
  int32_t n_kv_heads, head_dim; /* head_dim 64, 80, 96, 128 or 256                                   */
  int32_t format;
} et_kv_cache;
typedef struct {
  const int32_t *page_table_dev; /* [n_seqs, table_stride], of which pages_per_seq columns are used  */
  int32_t table_stride, pages_per_seq; /* pages_per_seq * page_size at most 2^30                     */
  const int32_t *kv_len_dev; /* [n_seqs]                                                             */
  int32_t n_seqs;
} et_kv_seqs;

/* Bytes of one page; 0 on bad arguments. */
size_t et_kv_page_bytes(int32_t page_size, int32_t n_kv_heads, int32_t head_dim, int32_t format);

/* Store rows of k_dev and v_dev, bf16 [rows, n_kv_heads * head_dim] with row strides in elements (multiples of 8, pointers
 * aligned to 16 bytes; columns of a fused projection can be passed as they lie); rows at most 2^30 - 64.  Asynchronous on `hip_stream`.  Errors:
 * INVALID_ARG, UNSUPPORTED (page_size, head_dim), HIP. */
int et_kv_append(const et_kv_cache *cache, const et_kv_seqs *seqs, const int32_t *cu_rows_dev, int32_t rows,
                 const uint16_t *k_dev, int64_t k_stride, const uint16_t *v_dev, int64_t v_stride, void *hip_stream);

/* The same for rows whose places the caller has: row i goes to token slots_dev[i] % page_size of page slots_dev[i] / page_size;
 * a negative slot, or one past the last page, is no place and its row is not stored.  (int64: et_kv_resize makes them.)  Slots that
 * are places differ from one another: where they do not, that token holds a mixture of their rows. */
int et_kv_append_slots(const et_kv_cache *cache, const int64_t *slots_dev, int32_t rows, const uint16_t *k_dev, int64_t k_stride,
                       const uint16_t *v_dev, int64_t v_stride, void *hip_stream);

/* The inverse: the values that the cache's rows stand for, rounded to bf16 once.  Same rows, same strides, same errors. */
int et_kv_read(const et_kv_cache *cache, const et_kv_seqs *seqs, const int32_t *cu_rows_dev, int32_t rows,
               uint16_t *k_out_dev, int64_t k_stride, uint16_t *v_out_dev, int64_t v_stride, void *hip_stream);

/* Attention of one new token per sequence over its cached tokens (its own among them, once et_kv_append has stored it):
 *   out[b, h] = sum over t of softmax_t(scale * q[b, h] . k[t, h'])  v[t, h'],   h' = h / (n_heads / n_kv_heads),
 * t running over the last `window` positions below kv_len[b] (window = 0: all of them) that have a page.  A head
 * that no token is left for, or whose logits are all minus infinity, gets zeros.  q_dev bf16 [n_seqs, n_heads *
 * head_dim] with row stride q_stride (a multiple of 8; aligned to 16 bytes); out_dev bf16 [n_seqs, n_heads * head_dim],
 * contiguous, not q_dev.  max_len: a bound of every kv_len that the host knows (positions from max_len on are left out).  The tokens
 * of all sequences are shared out evenly over the chip's workgroups on the device, by the lengths it finds there; sequences that are
 * short by their bound, or more than 4096, are one part each.  A bound far above the lengths costs nothing where these are long;
 * short sequences take a second launch by it (1 x 197 tokens 7.7 instead of 4.8 us, 256 x 500 58 instead of 50, 1024 x 60 97 instead
 * of 33).  Two equal calls give equal bits; a sequence beside others, or under another bound, may be split elsewhere, which moves
 * its result within the rounding.
 * Logits, their maximum, the sums and the products' accumulators are float32, the weights within 2^-15 of that.  Values are summed
 * before the division by the weights' sum, and in 8 bits a query's products with the codes before the row's factor, so values and
 * queries beyond 2^100 can overflow; in 8 bits the weights carry the value rows' maxima, so those below 2^-90 lose bits.  Keys
 * and values in 4 bits enter both products as the exact numbers that they stand for.
 * workspace: et_attention_paged_workspace_bytes with the same arguments (0 where max_len is at most 512), contents arbitrary, aligned
 * to 16 bytes; calls that run at the same time need one each.  n_seqs * n_heads at most 2^24 (2^24 - 2^19 where every query head
 * has its own key-value head), n_seqs * max_len at most 2^36.  Asynchronous on `hip_stream`.  Errors: INVALID_ARG, UNSUPPORTED
 * (page_size, head_dim), WORKSPACE, HIP. */
size_t et_attention_paged_workspace_bytes(const et_kv_cache *cache, const et_kv_seqs *seqs, int32_t n_heads,
                                          int32_t max_len, int32_t window);
int et_attention_paged(const et_kv_cache *cache, const et_kv_seqs *seqs, const uint16_t *q_dev, int64_t q_stride,
                       int32_t n_heads, int32_t max_len, int32_t window, float scale, void *workspace_dev,
                       size_t workspace_bytes, uint16_t *out_dev, void *hip_stream);

/* ---- pages for sequences that grow, shrink and end ------------------------------------------------
 * The cache's free pages lie in a ring of n_pages cells; state = { first, free, missing, 0 }: `free` pages from cell `first` on.
 * et_kv_resize takes every sequence b from kv_len[b] to new_len[b] tokens (negative lengths count as 0).  With pages(n) =
 * min(ceil(n / page_size), pages_per_seq):
 *   - entries pages(kv_len) .. pages(new_len) of its table row get pages from the ring's front, sequence by sequence and entry by entry;
 *     once the ring is empty they get -1 (no page), and `missing` of the new state counts those;
 *   - entries pages(new_len) .. pages(kv_len), of a sequence that shrinks or ends, give their pages back behind the ring's last one, in the same
 *     order, to be taken from the next call on.  Entries that are no page give nothing, nor do pages for which the ring has no room.
 * The new tokens of all sequences are consecutive rows, sequence by sequence: cu_rows [n_seqs + 1] their ranges (as et_kv_append takes
 * them, with new_len as lengths), positions [rows] the place of each in its sequence, slots [rows] page * page_size + place in the page, or -1
 * where there is no page (a missing one, or past pages_per_seq).  positions_dev and slots_dev may be NULL; `rows` is how many
 * rows they have, and may be a bound: rows past that are not written, and those behind the last sequence's get position 0 and slot -1, so
 * that et_kv_append_slots stores nothing for them (pool->keep_rest = 1: they stay as they are, which may be places of an earlier
 * call).  cu_rows stops at 2^31 - 1.
 * kv_len, new_len and everything else of the table stay as they are, and so do the ring's pages that were free: with another buffer as state_out_dev
 * (state_out_dev = state_dev is allowed) a call is taken back by going on with the old state and the old lengths, as when
 * pages are missing.  A page must be in one place, a table's live entry or a free cell of the ring; sequences that share pages are the
 * caller's to keep apart.  Whatever state, ring, lengths and table hold, nothing outside them is touched.
 * state_dev and state_out_dev int32 [4], aligned to 16 bytes; n_seqs at most 2^20, n_seqs * pages_per_seq below 2^31.  workspace:
 * et_kv_resize_workspace_bytes (0 up to 4096 sequences), aligned to 16 bytes, contents arbitrary.  Calls on the same ring,
 * state or table follow each other in one stream.  Asynchronous on `hip_stream`; can be captured.  Errors: INVALID_ARG, WORKSPACE, HIP. */
typedef struct {
  int32_t *ring_dev;           /* [n_pages]                                                          */
  int32_t n_pages, page_size;  /* page_size 16, 32, 64, 128 or 256                                   */
  int32_t keep_rest;           /* 1: rows behind the last sequence's stay as they are; 0 otherwise   */
} et_kv_pool;
size_t et_kv_resize_workspace_bytes(int32_t n_seqs);
int et_kv_resize(const et_kv_pool *pool, const int32_t *state_dev, int32_t *state_out_dev, int32_t *page_table_dev,
                 int32_t table_stride, int32_t pages_per_seq, const int32_t *kv_len_dev, const int32_t *new_len_dev,
                 int32_t n_seqs, int32_t rows, int32_t *cu_rows_dev, int32_t *positions_dev, int64_t *slots_dev,
                 void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* ---- rotary positions of queries and keys ----------------------------------------------------------
 * Pair i = 0 .. rot_dim / 2 - 1 of a head, dimensions (a, b) = (i, i + rot_dim / 2) (ET_ROTARY_HALF) or (2 i, 2 i + 1)
 * (ET_ROTARY_INTERLEAVED), becomes  A (a cos t - b sin t, b cos t + a sin t),  t = position * f_i;  dimensions from rot_dim on stay
 * as they are.  f_i = base^(-2 i / rot_dim), changed for contexts that are longer than those a model was trained with:
 *   ET_ROTARY_LINEAR: f_i / factor.      ET_ROTARY_NTK: base * factor^(rot_dim / (rot_dim - 2)) in the place of base.
 *   ET_ROTARY_YARN: f_i / factor * r + f_i * (1 - r), r rising from 0 to 1 between the pairs (whole numbers outwards) that turn `fast` and
 *     `slow` times (32 and 1, usually) over original_len positions, i.e. i = rot_dim ln(original_len / (2 pi turns)) / (2 ln base);
 *     A = 0.1 ln(factor) + 1.
 *   ET_ROTARY_TURNS: the same mix, r falling from 1 to 0 as the number of turns original_len f_i / (2 pi) goes from `slow` to `fast` (1 and 4,
 *     usually).
 * A = 1 but for ET_ROTARY_YARN.  et_rotary_steps (host only) writes f_i as fractions of a turn, steps[i] = 2^64 f_i / (2 pi), within two,
 * [rot_dim / 2], and A; the caller puts the steps on the device.  position * steps[i] mod 2^64 is then the angle of any int32
 * position, negative ones too, within 2^-29 radians.  base in [1, 1e30], factor in [1, 1e9]; scaling NULL: none.  Errors: INVALID_ARG. */
enum { ET_ROTARY_HALF = 0, ET_ROTARY_INTERLEAVED = 1 };
enum { ET_ROTARY_PLAIN = 0, ET_ROTARY_LINEAR = 1, ET_ROTARY_NTK = 2, ET_ROTARY_YARN = 3, ET_ROTARY_TURNS = 4 };
typedef struct {
  int32_t kind;
  double factor, original_len, slow, fast; /* the last three: ET_ROTARY_YARN and ET_ROTARY_TURNS     */
} et_rotary_scaling;
int et_rotary_steps(const et_rotary_scaling *scaling, int32_t rot_dim, double base, uint64_t *steps, float *amplitude);

typedef struct {
  const uint64_t *steps_dev; /* [rot_dim / 2]                                                        */
  int32_t head_dim, rot_dim, layout; /* even, rot_dim <= head_dim <= 512                             */
  float amplitude;
} et_rotary;
typedef struct {
  const uint16_t *in_dev; /* bf16 [rows, n_heads * head_dim], row stride in_stride (elements)        */
  int64_t in_stride;
  uint16_t *out_dev; /* may be in_dev, with the same stride; otherwise apart from all of q and k     */
  int64_t out_stride;
  int32_t n_heads;
} et_rotary_rows;
/* Turns rows of queries and (k NULL or n_heads 0: none) keys by positions_dev int32 [rows].  transpose = 1: by the transposed matrix, the
 * way back where A = 1, and a gradient's way through.  Products and sums are float32, results rounded once; cosine and sine are within
 * 2^-22 of A.  Any strides and alignments; 16 bytes and pairs in whole eighths (half: rot_dim a multiple of 16) are fastest.  rows at
 * most 2^27 - 8.  Asynchronous on `hip_stream`.  Errors: INVALID_ARG, HIP. */
int et_rotary_apply(const et_rotary *rotary, const int32_t *positions_dev, int32_t rows, const et_rotary_rows *q,
                    const et_rotary_rows *k, int32_t transpose, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* EARLYTOM_H */
