/*
 * hippo.h -- C ABI of the MI355X (gfx950) implementation of HIPPO's data-parallel hot path:
 * semantic-aware visual-token scoring and selection, construction of the pruned draft KV cache,
 * and the two attention calls that video parallel speculative decoding overlaps (draft decode over
 * the pruned cache, target verification of gamma+1 tokens over the full cache).
 *
 * The hot path proper:   hippo_score_tokens, hippo_select_gather_kv, hippo_draft_attention,
 *                        hippo_verify_attention (+ hippo_workspace_bytes, hippo_status_string).
 * Built around it:       hippo_score_tokens_layers (Eq. 2's layer sum in one call),
 *                        hippo_*_attention_append, hippo_*_attention_paged and
 *                        hippo_*_attention_fp8kv with hippo_quantize_kv_e4m3 (cache-format variants),
 *                        hippo_spec_verify (the speculative-sampling verdict of Eq. 1),
 *                        hippo_*_attention_mass with hippo_evict_kv (a draft cache that stays within a budget),
 *                        hippo_token_logprobs (log probabilities of an answer's words),
 *                        hippo_prefill_attention* (prompts, packed or over pages), hippo_tree_attention* (trees of drafted
 *                        tokens), hippo_plan_pages and hippo_write_kv_paged (what fills a paged cache),
 *                        hippo_vpsd_* (host-side control of the parallel decoding rounds).
 *
 * Conventions common to every entry point
 *  - All data pointers are DEVICE pointers owned and allocated by the caller.  The library never
 *    allocates or frees device memory and never synchronises: it validates its arguments on the
 *    host, enqueues kernels on `stream` (a hipStream_t passed as void*, NULL = default stream)
 *    and returns.  Outputs are valid once the caller has synchronised that stream.  Calls on
 *    different streams may run concurrently as long as their outputs and workspaces are distinct.
 *  - The descriptor structs are HOST pointers, read before the call returns.
 *  - Every call returns a status (HIPPO_OK = 0).  Validation happens before any kernel is
 *    launched: on a non-zero status nothing has been enqueued and no output was touched.  No
 *    exception crosses the boundary.
 *  - `workspace` is device scratch of at least hippo_workspace_bytes(...) bytes, 256-byte aligned,
 *    private to the call until the stream has passed it.
 *  - Data pointers must be 16-byte aligned; strides are in elements and must keep every row
 *    16-byte aligned (multiples of 8 for bf16, of 4 for fp32).  head_dim is 64 or 128.
 *  - dtype: HIPPO_DTYPE_F32 or HIPPO_DTYPE_BF16 for q / K / V / emb / attention outputs (plus the
 *    8-bit cache type of the *_fp8kv calls and the gather, see enum hippo_dtype).  Scores,
 *    attention mass and log-sum-exp are always fp32, indices int32.  Accumulation is fp32;
 *    bf16 outputs are rounded to nearest even.
 */
#ifndef HIPPO_H_
#define HIPPO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum hippo_status {
  HIPPO_OK = 0,
  HIPPO_ERR_NULL_ARG = 1,            /* a required pointer is NULL */
  HIPPO_ERR_BAD_SHAPE = 2,           /* a size, count, stride or index range is invalid */
  HIPPO_ERR_BAD_DTYPE = 3,           /* dtype is not one the call supports */
  HIPPO_ERR_BAD_ALIGN = 4,           /* a pointer or stride breaks the 16-byte rule */
  HIPPO_ERR_WORKSPACE_TOO_SMALL = 5, /* workspace_bytes below hippo_workspace_bytes(...) */
  HIPPO_ERR_HIP = 6,                 /* a HIP runtime call (launch) failed */
  HIPPO_ERR_STATIC_SCRATCH_LIMIT = 7 /* hippo_verify_attention_static: the shapes need more scratch
                                        than hippo_static_scratch_bytes() */
};

enum hippo_dtype {
  HIPPO_DTYPE_F32 = 0,
  HIPPO_DTYPE_BF16 = 1,
  /* 8-bit floating-point CACHE elements (E4M3, see hippo_verify_attention_fp8kv): one byte each.
   * Accepted by the *_fp8kv attention calls, by hippo_select_gather_kv (rows are byte copies) and by
   * hippo_workspace_bytes for those calls; every other call answers BAD_DTYPE. */
  HIPPO_DTYPE_FP8_E4M3 = 2
};

enum hippo_call {
  HIPPO_CALL_SCORE_TOKENS = 0,
  HIPPO_CALL_SELECT_GATHER_KV = 1,
  HIPPO_CALL_DRAFT_ATTENTION = 2,
  HIPPO_CALL_VERIFY_ATTENTION = 3
};

/* which terms of the holistic score are enabled (the paper's ablation removes one at a time) */
enum hippo_score_flags {
  HIPPO_SCORE_ATTN = 1u,            /* global semantic relevance, Eq. 2 */
  HIPPO_SCORE_TEMP = 2u,            /* inter-frame temporal redundancy, Eq. 3-4 */
  HIPPO_SCORE_SPA = 4u,             /* intra-frame spatial redundancy, Eq. 5-6 */
  HIPPO_SCORE_ALL = 7u,
  HIPPO_SCORE_ACCUMULATE_ONLY = 8u  /* add this layer's attention mass into attn_mass_inout and stop
                                       (the outer layer sum of Eq. 2); no other output is written */
};

/* A K or V cache (or the q/out heads that go with it).
 * Element (b, hk, n, c) of a cache lives at base + b*stride_b + hk*stride_h + n*stride_n + c. */
typedef struct hippo_kv_desc {
  int32_t batch;
  int32_t n_q_heads;   /* H; multiple of n_kv_heads.  Query head h reads KV head h / (H / H_kv) */
  int32_t n_kv_heads;  /* H_kv */
  int32_t head_dim;    /* d_k: 64 or 128 */
  int32_t dtype;       /* enum hippo_dtype */
  int64_t stride_b, stride_h, stride_n;  /* elements; stride_n >= head_dim */
} hippo_kv_desc;

/* Where the video sits inside the sequence and how its tokens are arranged.
 * Visual token j = f*grid_h*grid_w + y*grid_w + x is cache row vis_offset + j.
 * Crops (Eq. 5-6) are non-overlapping crop_h x crop_w tiles of each frame anchored at (0,0);
 * tiles cut by the right / bottom edge keep the tokens they have. */
typedef struct hippo_video_desc {
  int32_t n_frames, grid_h, grid_w;
  int32_t vis_offset;
  int32_t crop_h, crop_w;           /* the paper uses 5 x 5; crop_h*crop_w <= 64 */
} hippo_video_desc;

const char* hippo_status_string(int status);

/* Bytes of workspace `call` needs for these shapes; never 0 for valid arguments, 0 if they are
 * invalid.  n_rows = l_txt for SCORE_TOKENS, q_len for the attention calls, ignored otherwise;
 * seq_len = number of valid cache rows (ctx_len + q_len for attention); k = tokens kept (select);
 * num_splits as passed to the attention call (0 = library's choice). */
size_t hippo_workspace_bytes(int32_t call, const hippo_kv_desc* kv, const hippo_video_desc* vid,
                             int32_t n_rows, int32_t seq_len, int32_t k, int32_t num_splits);

/*
 * Semantic-aware token scoring (Method, "Semantic-aware Token Preservation", Eq. 2-7).
 *   s_attn[j] = 1/(H l_txt) sum_h sum_i softmax_j(q_txt[i,h] . K_vid[j] / sqrt(d_k))      (Eq. 2,
 *               softmax over the N_v visual keys; one layer per call)
 *   s_temp[j] = 1 - mean over existing neighbour frames f-1, f+1 of the cosine between token j and
 *               the token at the same grid position there (1 if the video has one frame) (Eq. 3-4)
 *   s_spa[j]  = population variance over the tokens k of j's crop of cos(emb_j, emb_k)    (Eq. 5-6)
 *   scores[j] = sum over enabled terms of (s - mean_f) / std_f, statistics per frame, population
 *               std, a term with std_f = 0 contributes 0                                   (Eq. 7)
 * An embedding without a positive norm (of zeros, or with a NaN) has cosine 0 with everything.
 *
 * q_txt   [B, l_txt, H, d] contiguous, dtype kv->dtype: the text-prompt queries.
 * k_cache the cache whose keys guide pruning; rows [vis_offset, vis_offset + N_v) are read.
 * emb     [B, N_v, emb_dim] with token stride emb_stride_tok (batch stride N_v*emb_stride_tok),
 *         dtype kv->dtype, or NULL: then token j's embedding is its key vectors of all KV heads
 *         concatenated in head order (emb_dim, emb_stride_tok ignored).
 * attn_mass_inout [B, N_v] fp32 or NULL.  If non-NULL it holds the sum of s_attn over the layers
 *         already processed; this call adds its layer's s_attn to it and, unless ACCUMULATE_ONLY is
 *         set, uses the accumulated value as the attention term (a positive factor such as 1/N_L
 *         does not change Eq. 7's normalised value).
 * scores_out [B, N_v] fp32 (required unless ACCUMULATE_ONLY).
 * components_out optional [3, B, N_v] fp32: raw s_attn (this call's, or accumulated), s_temp, s_spa.
 * Errors: NULL_ARG, BAD_SHAPE (l_txt < 1, N_v < 1, vis_offset + N_v > seq_len, crop too large,
 *         no term enabled; beyond the launch limits: B * layers > 65535, more than 65535 frames,
 *         N_v > 65535 * 256 tokens in bf16, 65535 * 128 in fp32), BAD_DTYPE, BAD_ALIGN, WORKSPACE_TOO_SMALL, HIP.
 */
int hippo_score_tokens(const void* q_txt, int32_t l_txt,
                       const void* k_cache, const hippo_kv_desc* kv, int32_t seq_len,
                       const hippo_video_desc* vid,
                       const void* emb, int32_t emb_dim, int64_t emb_stride_tok,
                       uint32_t flags,
                       float* attn_mass_inout, float* scores_out, float* components_out,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same with Eq. 2's outer sum over layers done inside the call: the attention term is
 * sum over the n_layers given layers of that layer's s_attn (queries and keys of layer l from
 * q_txt_layers[l], k_cache_layers[l]; all layers share kv's shape and strides), swept in ONE launch per
 * pass instead of one call per layer.  q_txt_layers and k_cache_layers are HOST arrays of n_layers
 * device pointers (1 <= n_layers <= 64), read before the call returns.  When emb is NULL the
 * embedding terms use the keys of layer emb_layer.  attn_mass_inout, if given, is added to (and
 * updated with) the call's layer sum, exactly as for single calls.  hippo_score_tokens is this call
 * with one layer.  Workspace: hippo_score_layers_workspace_bytes(kv, vid, l_txt, n_layers).
 */
size_t hippo_score_layers_workspace_bytes(const hippo_kv_desc* kv, const hippo_video_desc* vid,
                                          int32_t l_txt, int32_t n_layers);
int hippo_score_tokens_layers(int32_t n_layers, const void* const* q_txt_layers, int32_t l_txt,
                              const void* const* k_cache_layers, int32_t emb_layer,
                              const hippo_kv_desc* kv, int32_t seq_len, const hippo_video_desc* vid,
                              const void* emb, int32_t emb_dim, int64_t emb_stride_tok,
                              uint32_t flags,
                              float* attn_mass_inout, float* scores_out, float* components_out,
                              void* workspace, size_t workspace_bytes, void* stream);

/*
 * Top-k retention and draft-cache construction (Method, end of "Holistic Score Fusion": keep the
 * top-k visual tokens by score; App. "Details of Experimental Setups": the pruned video features
 * are removed from the draft model's input, everything that is not video is kept whole).
 *   idx_out[b, :] = the k visual-token indices with the largest scores[b, :], listed in ascending
 *                   index order.  Equal scores (-0 == +0): the lower index wins.  NaN ranks below
 *                   every number.
 *   dst rows      = src rows [0, vis_offset) | src rows vis_offset + idx_out[b, .] | src rows
 *                   [vis_offset + N_v, src_len), for K and V and every KV head, bit copies.
 * scores [B, N_v] fp32.  1 <= k <= N_v.  src/dst descriptors must agree in batch, n_kv_heads,
 * head_dim and dtype (strides may differ); dst holds src_len - N_v + k rows.  k_src/v_src may be a
 * different model's cache than the one that was scored, and may be an 8-bit cache
 * (HIPPO_DTYPE_FP8_E4M3: the kept rows' codes are copied; the per-head multipliers stay valid).  k_dst/v_dst may be NULL together to get
 * the indices only.  src and dst must not overlap.
 * Errors: NULL_ARG, BAD_SHAPE (k out of range, video span outside src_len, descriptor mismatch),
 *         BAD_DTYPE, BAD_ALIGN, WORKSPACE_TOO_SMALL, HIP.
 */
int hippo_select_gather_kv(const float* scores, int32_t k,
                           const void* k_src, const void* v_src, const hippo_kv_desc* src,
                           int32_t src_len, const hippo_video_desc* vid,
                           void* k_dst, void* v_dst, const hippo_kv_desc* dst,
                           int32_t* idx_out,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * Eviction from a cache that has outgrown its budget, by accumulated attention weight (hippo_*_attention_mass): what a draft
 * cache needs that is pruned once, at prefill, and then grows with the answer.  Every (batch element, KV head) chooses for
 * itself; of its src_len rows these `keep` stay:
 *   the first n_first, the last n_recent, and of those between the keep - n_first - n_recent with the largest mass
 *   (equal ones, -0 == +0: the lower row; NaN ranks below every number).
 *   idx_out[b, hk, :] = the rows that stay, ascending
 *   dst row j of (b, hk) = src row idx_out[b, hk, j] for K and V, bit copies;  mass_dst likewise
 * A row of dst is not at its old position: attention over dst takes ctx_len = keep, and a model's position embedding goes on from
 * the old length, as it does behind a pruned cache.
 * mass: element (b, hk, n) at b * mass_stride_b + hk * mass_stride_h + n, fp32; only rows between are read for the choice.
 * src and dst may be 8-bit caches (codes are copied; the per-head multipliers stay valid); they agree in batch, n_kv_heads,
 * head_dim and dtype.  k_dst/v_dst may be NULL together (indices and mass only, k_src/v_src are then not read), mass_dst may be
 * NULL.  Rows of dst and mass_dst from `keep` on are left as they were, so that a decoding loop appends behind them.
 * src and dst, and mass and mass_dst, must not overlap.  1 <= keep <= src_len <= 2^30, n_first + n_recent <= keep.  Deterministic.
 * Errors: NULL_ARG, BAD_SHAPE (also dst on src, and strides by which rows of dst or of mass_dst would meet), BAD_DTYPE, BAD_ALIGN, WORKSPACE_TOO_SMALL, HIP.
 */
size_t hippo_evict_kv_workspace_bytes(const hippo_kv_desc* src, int32_t src_len, int32_t keep);
int hippo_evict_kv(const float* mass, int64_t mass_stride_b, int64_t mass_stride_h,
                   int32_t keep, int32_t n_first, int32_t n_recent,
                   const void* k_src, const void* v_src, const hippo_kv_desc* src, int32_t src_len,
                   void* k_dst, void* v_dst, const hippo_kv_desc* dst,
                   float* mass_dst, int64_t mass_dst_stride_b, int64_t mass_dst_stride_h,
                   int32_t* idx_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Target verification attention (Preliminaries, "Speculative Decoding": the target model takes the
 * prefix plus the gamma draft tokens and emits p_0..p_gamma; Method, "Adaptive Decoding Strategy
 * Switching": in conservative mode it verifies x_1 alone, so any q_len >= 1 is accepted).
 *   out[b, i, h, :] = sum_n softmax_n(softmax_scale * q[b,i,h,:] . K[b,h/G,n,:]) V[b,h/G,n,:],
 *   n in [0, ctx_len + i]   -- the cache already holds the q_len new rows' own K/V at rows
 *   ctx_len .. ctx_len + q_len - 1, and new row i sees the context and new rows 0..i.
 * q, out [B, q_len, H, d] contiguous, dtype kv->dtype.  lse_out optional [B, H, q_len] fp32: natural
 * log of the softmax denominator (of the scaled logits).  softmax_scale <= 0 means 1/sqrt(d).
 * num_splits: how many slices the KV range is cut into (flash-decoding style), 0 = library's
 * choice; the result does not depend on it beyond rounding (fp32 caches: fp32 throughout; 16- and 8-bit
 * caches: each slice's output reaches the merge rounded to bf16 or finer, its statistics in fp32).
 * ctx_len >= 0, q_len >= 1.
 * Workspace: hippo_workspace_bytes.  With num_splits 0 it does not grow with seq_len once that gives
 * every compute unit a slice, with one exception: 65 to 96 query rows a KV head (q_len H / H_kv) of bf16
 * caches of more than 256 MiB (K and V) need about twice as much.  Such a call also takes a workspace of
 * half that, as hippo_workspace_bytes says for a shorter cache, and is then 10 to 30 % slower.
 * Errors: NULL_ARG, BAD_SHAPE, BAD_DTYPE, BAD_ALIGN, WORKSPACE_TOO_SMALL, HIP.
 */
int hippo_verify_attention(const void* q, int32_t q_len,
                           const void* k_cache, const void* v_cache, const hippo_kv_desc* kv,
                           int32_t ctx_len, float softmax_scale, int32_t num_splits,
                           void* out, float* lse_out,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * Draft-decode attention over the pruned cache (Preliminaries, "Speculative Decoding": the draft
 * model is invoked gamma times, one new token per forward).  Same contract, arguments, kernels (padded
 * to one 16-row block at G = 7 or 8 rows) and split heuristic as hippo_verify_attention; the one
 * difference is that its waves do not raise their issue priority, so a verification running beside it
 * keeps the right of way.  Running it on the cache hippo_select_gather_kv built with k = N_v equals
 * attention over the unpruned cache.
 */
int hippo_draft_attention(const void* q, int32_t q_len,
                          const void* k_cache, const void* v_cache, const hippo_kv_desc* kv,
                          int32_t ctx_len, float softmax_scale, int32_t num_splits,
                          void* out, float* lse_out,
                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * hippo_verify_attention for callers that can neither allocate device memory nor pass a workspace:
 * code running under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, result and errors as hippo_verify_attention minus the workspace pair; the split partials
 * live in an array that is part of the library's device image (hippo_static_scratch_bytes() = 8 MiB on
 * every GPU the library is used on, held until the process ends).  The call allocates and frees
 * nothing.  Shapes whose partials exceed the array (hippo_workspace_bytes(HIPPO_CALL_VERIFY_ATTENTION,
 * ...) > hippo_static_scratch_bytes(), e.g. many sequences with num_splits forced high) are refused
 * with HIPPO_ERR_STATIC_SCRATCH_LIMIT before anything is enqueued.  Every call on a GPU uses that
 * GPU's one array: calls must not overlap in time on one GPU (same stream, or ordered by events), or
 * they race.  Nothing in the array has to be cleared between calls, whatever the previous call left.
 * The array's device address is looked up on the first call on each device; hippo_static_scratch_init()
 * does that lookup for the current device ahead of time (call it before capturing a graph).
 */
size_t hippo_static_scratch_bytes(void);
int hippo_static_scratch_init(void);
int hippo_verify_attention_static(const void* q, int32_t q_len,
                                  const void* k_cache, const void* v_cache, const hippo_kv_desc* kv,
                                  int32_t ctx_len, float softmax_scale, int32_t num_splits,
                                  void* out, float* lse_out, void* stream);

/*
 * The same two attention calls with the append of the new rows folded in (a cache-format variant for
 * decode loops: the gamma+1 rows the target verifies, or the one row the draft model decodes, come
 * straight from the K/V projection and would otherwise need a copy kernel of their own before the
 * attention launch).  k_new, v_new [B, q_len, H_kv, d] contiguous, dtype kv->dtype: the new rows'
 * keys and values.  The result is exactly that of hippo_verify_attention / hippo_draft_attention on
 * a cache whose rows ctx_len .. ctx_len + q_len - 1 hold them; the call also WRITES those rows into
 * k_cache / v_cache (bit copies), so the next call finds them there.  Rows below ctx_len are read
 * only.  k_new / v_new must not overlap the caches.  Everything else as above.
 * Errors: as above, plus NULL_ARG / BAD_ALIGN for k_new, v_new.
 */
int hippo_verify_attention_append(const void* q, int32_t q_len, const void* k_new, const void* v_new,
                                  void* k_cache, void* v_cache, const hippo_kv_desc* kv,
                                  int32_t ctx_len, float softmax_scale, int32_t num_splits,
                                  void* out, float* lse_out,
                                  void* workspace, size_t workspace_bytes, void* stream);
int hippo_draft_attention_append(const void* q, int32_t q_len, const void* k_new, const void* v_new,
                                 void* k_cache, void* v_cache, const hippo_kv_desc* kv,
                                 int32_t ctx_len, float softmax_scale, int32_t num_splits,
                                 void* out, float* lse_out,
                                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same two attention calls with the weight that every cache row was given: what an eviction goes by (hippo_evict_kv).
 *   mass_out[b, hk, n] = (n < ctx_len ? mass_in[b, hk, n] : 0)
 *                        + sum over the new rows i and the query heads h of KV head hk of softmax_n(...)[b, i, h],
 *   n in [0, ctx_len + q_len); a new row i gives nothing to rows behind ctx_len + i.
 * out and lse_out as without mass (over bf16 caches, of probabilities rounded to bf16: lse_out is within 2^-8 of the unrounded
 * one's), but that the slices' outputs reach the merge in fp32.  The weights are fp32 from fp32 logits, of the probabilities before
 * any rounding; sums run in a fixed order.
 * Several new rows are those that a draft model takes in at once, such as the words that a verification accepted.  Every row's
 * weights are added: there is no call that takes back the share of rows that are dropped afterwards (their own rows' mass is written
 * anew with the rows), so a chain that may still be rejected is best attended to without mass.
 * mass: `in` may be NULL (nothing accumulated yet) or `out` (in place, the same strides), and does not overlap it otherwise; element
 * (b, hk, n) lies at b * stride_b + hk * stride_h + n.  Elements of `out` from ctx_len + q_len on are left as they were.
 * k_new, v_new: both NULL (the caches hold the new rows), or the rows to append, as in the *_append calls.  Caches: F32 or BF16,
 * contiguous.  Workspace: hippo_attention_mass_workspace_bytes, with seq_len = ctx_len + q_len; it grows with seq_len times the
 * query rows.
 * Errors: as the *_append calls, plus NULL_ARG for mass or its out, BAD_SHAPE for mass strides of rows that would meet.
 */
typedef struct hippo_mass_desc {
  const float* in;
  float* out;
  int64_t in_stride_b, in_stride_h, out_stride_b, out_stride_h;   /* elements */
} hippo_mass_desc;

size_t hippo_attention_mass_workspace_bytes(const hippo_kv_desc* kv, int32_t q_len, int32_t seq_len, int32_t num_splits);
int hippo_verify_attention_mass(const void* q, int32_t q_len, const void* k_new, const void* v_new,
                                void* k_cache, void* v_cache, const hippo_kv_desc* kv,
                                int32_t ctx_len, float softmax_scale, int32_t num_splits,
                                void* out, float* lse_out, const hippo_mass_desc* mass,
                                void* workspace, size_t workspace_bytes, void* stream);
int hippo_draft_attention_mass(const void* q, int32_t q_len, const void* k_new, const void* v_new,
                               void* k_cache, void* v_cache, const hippo_kv_desc* kv,
                               int32_t ctx_len, float softmax_scale, int32_t num_splits,
                               void* out, float* lse_out, const hippo_mass_desc* mass,
                               void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same two attention calls over a cache stored in 8-bit floating point (a cache-format variant
 * the paper does not discuss: it halves the bytes these bandwidth-bound calls stream).  k_codes /
 * v_codes hold E4M3 codes (1 sign, 4 exponent, 3 mantissa bits, bias 7, finite-only: no infinities,
 * 0x7f / 0xff are NaN), one byte per element, laid out as kv describes with strides counted in
 * elements = bytes (multiples of 16).  k_scale / v_scale are DEVICE arrays [B, H_kv] of fp32
 * multipliers, all > 0: the cache entry is multiplier * decoded code.  kv->dtype must be
 * HIPPO_DTYPE_FP8_E4M3, the type of the cache; q and out are bf16.  The result is that of hippo_verify_attention /
 * hippo_draft_attention on the dequantised cache, computed with the same arithmetic as the bf16 path
 * (codes convert to bf16 exactly; the K multiplier joins the softmax scale, the V multiplier the
 * output).  Workspace: hippo_workspace_bytes with the same kv.  Caches are read only.
 * Errors: as hippo_verify_attention, plus NULL_ARG for the multipliers, BAD_DTYPE for any other
 * cache type.
 */
int hippo_verify_attention_fp8kv(const void* q, int32_t q_len, const void* k_codes, const void* v_codes,
                                 const float* k_scale, const float* v_scale, const hippo_kv_desc* kv,
                                 int32_t ctx_len, float softmax_scale, int32_t num_splits,
                                 void* out, float* lse_out,
                                 void* workspace, size_t workspace_bytes, void* stream);
int hippo_draft_attention_fp8kv(const void* q, int32_t q_len, const void* k_codes, const void* v_codes,
                                const float* k_scale, const float* v_scale, const hippo_kv_desc* kv,
                                int32_t ctx_len, float softmax_scale, int32_t num_splits,
                                void* out, float* lse_out,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * Writer of that 8-bit cache format: rows [0, n_rows) of a bf16 or fp32 cache become E4M3 codes and
 * one multiplier per (batch element, KV head), separately for K and V:
 *     multiplier = max|x| / 448 over the head's n_rows x d entries (fp32; 1 when the maximum is 0)
 *     code       = the E4M3 value nearest to x / multiplier (fp32 division), ties to the even code
 * so the largest entry of every head maps to the largest code and nothing overflows.  src describes
 * k_src / v_src (dtype F32 or BF16), dst the code arrays (dtype FP8_E4M3, strides in bytes); both
 * agree in batch, n_kv_heads, head_dim.  k_scale / v_scale [B, H_kv] fp32 are OUTPUTS.  Inputs must
 * be finite (a NaN or infinity gives unspecified codes for its head).  The outputs must not overlap the
 * sources.  Deterministic.  Workspace: hippo_quantize_kv_workspace_bytes(src, n_rows).
 * Errors: NULL_ARG, BAD_DTYPE, BAD_SHAPE (descriptor mismatch, n_rows < 1), BAD_ALIGN,
 *         WORKSPACE_TOO_SMALL, HIP.
 */
size_t hippo_quantize_kv_workspace_bytes(const hippo_kv_desc* src, int32_t n_rows);
int hippo_quantize_kv_e4m3(const void* k_src, const void* v_src, const hippo_kv_desc* src, int32_t n_rows,
                           void* k_codes, void* v_codes, const hippo_kv_desc* dst,
                           float* k_scale, float* v_scale,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same two attention calls over a PAGED cache (a cache-format variant for serving stacks that
 * allocate the cache in fixed-size pages).  k_pool / v_pool are page pools; cache row n of sequence
 * b and KV head hk lives at element
 *     block_table[b * max_pages + n / page_size] * stride_page + (n % page_size) * stride_n + hk * stride_h
 * (+ c for head-dim element c), e.g. a [n_pool_pages, page_size, H_kv, d] pool has stride_page =
 * page_size * H_kv * d, stride_n = H_kv * d, stride_h = d.  block_table is a DEVICE array of int32,
 * [B, max_pages]; entries outside [0, n_pool_pages) are clamped into the pool (the result is then
 * meaningless, but no access leaves the pool).  page_size is a power of two, 16..256.  The result
 * is bit-identical to the contiguous call on the same rows.  A block stages the page numbers of its
 * KV slice in LDS, which bounds a slice to about 1000 pages: with num_splits forced very low on a
 * long cache the call returns BAD_SHAPE.  Use hippo_workspace_bytes with a hippo_kv_desc of the same
 * batch / heads / head_dim / dtype for the workspace size.
 * Errors: as hippo_verify_attention, plus BAD_SHAPE for a page size, table width or pool size
 * that does not fit, BAD_ALIGN for strides that break the 16-byte rule.
 */
typedef struct hippo_paged_kv_desc {
  int32_t batch, n_q_heads, n_kv_heads, head_dim, dtype;
  int32_t page_size;        /* tokens per page */
  int32_t max_pages;        /* columns of block_table; >= ceil((ctx_len + q_len) / page_size) */
  int32_t n_pool_pages;     /* pages in the pool */
  int64_t stride_page, stride_n, stride_h;   /* elements */
} hippo_paged_kv_desc;

int hippo_verify_attention_paged(const void* q, int32_t q_len, const void* k_pool, const void* v_pool,
                                 const int32_t* block_table, const hippo_paged_kv_desc* kv,
                                 int32_t ctx_len, float softmax_scale, int32_t num_splits,
                                 void* out, float* lse_out,
                                 void* workspace, size_t workspace_bytes, void* stream);
int hippo_draft_attention_paged(const void* q, int32_t q_len, const void* k_pool, const void* v_pool,
                                const int32_t* block_table, const hippo_paged_kv_desc* kv,
                                int32_t ctx_len, float softmax_scale, int32_t num_splits,
                                void* out, float* lse_out,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * Speculative-sampling verification of one chain of gamma draft tokens per sequence
 * (Preliminaries, "Speculative Decoding": Eq. 1, the resampling rule below it, and the extra token
 * after a full acceptance; Method, "Adaptive Decoding Strategy Switching": conservative mode
 * verifies x_1 alone, i.e. gamma = 1).
 *   p_i = softmax(p_logits[b, i, :] / temperature), i = 0..gamma    target rows
 *   q_i = softmax(q_logits[b, i, :] / temperature), i = 0..gamma-1  draft rows; draft token
 *         x_i = draft_tokens[b, i] was sampled from q_i and is verified against p_i
 *   alpha_i = 1 if p_i[x_i] >= q_i[x_i] else p_i[x_i] / q_i[x_i]                          (Eq. 1)
 *   token i is accepted iff u_accept[b, i] < alpha_i; n_accept_out[b] = j = the first rejected
 *   position (gamma if none).  next_token_out[b] is drawn with u_sample[b] from
 *   max(0, p_j - q_j) / sum (from p_j if that sum is 0) after a rejection, from p_gamma otherwise:
 *   the first word t whose running sum r_0 + .. + r_t exceeds u_sample * sum(r), in index order.
 *   The caller emits x_0 .. x_{j-1} followed by next_token.
 * temperature == 0 is greedy decoding (the paper's evaluation setting): p_i is one-hot at the first
 *   maximum of its row, q_i one-hot at x_i, so alpha_i = [x_i == argmax p_i] and next_token is the
 *   argmax of row j; q_logits, u_accept and u_sample are not read and may be NULL.
 * alpha_out (optional) [B, gamma] fp32: alpha_i for every position, also after the first rejection.
 * A draft token outside [0, vocab) is rejected (alpha 0).  Logits may be -inf (masked words) but
 * not NaN or +inf, and every row needs a finite entry.  The uniforms are the caller's, in [0, 1).
 *
 * p_logits [B, gamma+1, p_stride_row], q_logits [B, gamma, q_stride_row], dtype F32 or BF16, row
 * strides in elements, >= vocab and keeping rows 16-byte aligned; the first `vocab` entries of a
 * row are read.  draft_tokens [B, gamma] int32, u_accept [B, gamma] fp32, u_sample [B] fp32,
 * outputs int32 [B].  0 <= gamma <= 64 (gamma = 0 just draws from p_0), vocab <= 2^20.
 * Sums are fp32; a word that the exact arithmetic would draw can be replaced by a neighbour in
 * the running sum only when u_sample * sum lies within fp32 rounding of the boundary between them.
 * Errors: NULL_ARG, BAD_SHAPE, BAD_DTYPE, BAD_ALIGN, WORKSPACE_TOO_SMALL, HIP.
 */
size_t hippo_spec_verify_workspace_bytes(int32_t batch, int32_t gamma, int32_t vocab, int32_t dtype);
int hippo_spec_verify(const void* p_logits, const void* q_logits, int32_t dtype,
                      int64_t p_stride_row, int64_t q_stride_row,
                      const int32_t* draft_tokens, const float* u_accept, const float* u_sample,
                      int32_t batch, int32_t gamma, int32_t vocab, float temperature,
                      int32_t* n_accept_out, int32_t* next_token_out, float* alpha_out,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * Log probabilities of given words under rows of logits, with each row's entropy and its most likely words: what an answer's
 * tokens were worth (for a verified chain, row i of hippo_spec_verify's p_logits judges token i).
 *   y = logits[r, :vocab] / temperature,  log p_v = y_v - log sum_u exp(y_u)
 *   logprob_out[r] = log p of tokens[r];  entropy_out[r] = - sum_v p_v log p_v  (natural logarithms)
 *   top_ids_out[r, :], top_logprobs_out[r, :]: the n_top words with the largest logits, the largest first, equal ones by
 *   the lower word first (-0 == +0), and their log p.  NULL for n_top = 0.
 * Logits may be -inf (masked words: p = 0, log p = -inf, nothing added to the entropy).  A row of -inf alone has log p = -inf for
 * every word and entropy 0.  A row with a NaN gives NaN, one with +inf unspecified values; the words named are in the vocabulary
 * all the same.  A token outside [0, vocab) has log p = -inf.
 * logits [rows, stride_row], dtype F32 or BF16, rows 16-byte aligned, stride_row >= vocab; the first `vocab` entries of a row
 * are read.  tokens [rows] int32; outputs fp32 [rows], int32 and fp32 [rows, n_top].  1 <= rows <= 2^22, vocab <= 2^20,
 * 0 <= n_top <= 32 and <= vocab, temperature > 0 and finite (at least 1e-38).  Sums are fp32, of the words other than
 * the largest, so that a row whose best word has nearly all the weight keeps its entropy (words below 2^-126 of the best one's weight
 * add nothing to the sums).  Deterministic.
 * Errors: NULL_ARG, BAD_SHAPE, BAD_DTYPE, BAD_ALIGN, WORKSPACE_TOO_SMALL, HIP.
 */
size_t hippo_token_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t dtype, int32_t n_top);
int hippo_token_logprobs(const void* logits, int32_t dtype, int64_t stride_row, const int32_t* tokens, int32_t rows,
                         int32_t vocab, float temperature, int32_t n_top,
                         float* logprob_out, float* entropy_out, int32_t* top_ids_out, float* top_logprobs_out,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * Attention of whole prompts, or of their next pieces: what fills a model's hidden states behind the rows that verification and draft
 * decoding start from.  The sequences' rows lie one behind the other, without padding.
 *   sequence b: query rows cu_q[b] .. cu_q[b+1] - 1 and key rows cu_k[b] .. cu_k[b+1] - 1 (len_q and len_k of them), the last ones
 *   of both being the same tokens
 *   out[cu_q[b] + i, h, :] = sum_n softmax_n(softmax_scale * q[cu_q[b] + i, h, :] . K[cu_k[b] + n, h/G, :]) V[cu_k[b] + n, h/G, :],
 *   n in [0, len_k - len_q + i]
 * cu_q, cu_k [n_seqs + 1] int32 on the DEVICE, ascending, within [0, total_q] and [0, total_k]; cu_k = cu_q for whole prompts.
 * Sequences may be empty.  Rows of q that belong to no sequence are not read, and their rows of out and lse_out are left as
 * they were.  (Offsets outside the buffers are cut off at their ends, and of a descending pair no row is taken: the
 * result is then meaningless, but no access leaves the buffers.)
 * A row that sees nothing (len_q > len_k), or whose logits are all -inf, gives zeros and lse -inf.  What K and V hold at rows that a
 * query row does not see, infinities and NaN included, does not reach that row.
 * q [total_q, H, d], k and v [total_k, H_kv, d], with the strides of desc: slices of one fused projection's output will do.  out
 * [total_q, H, d] contiguous, dtype desc->dtype (F32 or BF16); lse_out optional [H, total_q] fp32.  softmax_scale <= 0 means
 * 1/sqrt(d).  num_splits: blocks that share a tile of query rows (up to 64, and up to total_k / 64), 0 = library's choice; the result does not
 * depend on it beyond rounding.  fp32 throughout, but that over bf16 the probabilities are rounded to bf16 before their product with V (and summed as
 * rounded: lse_out is within 2^-8 of the unrounded one's, and goes with out where outputs are joined by it).  total_q = 0 does nothing.
 * Workspace: hippo_prefill_workspace_bytes with paged 0.  It holds the parts of tiles that blocks share, and may be larger for a smaller call, which
 * needs more blocks a tile to fill the device: ask for each.  The lengths are on the device; the library's choice takes them as alike.
 * Errors: NULL_ARG, BAD_SHAPE (also more than 65535 sequences or query heads, 2^30 query rows times heads, 0x7fffff00 rows of K and V,
 *         strides of their rows above 2^24 elements, or 2^23 blocks and more: (total_q * H / H_kv / 256 + n_seqs) * H_kv, in fp32 with
 *         head_dim 64 total_q * H / H_kv / 128), BAD_DTYPE, BAD_ALIGN, WORKSPACE_TOO_SMALL, HIP.
 */
typedef struct hippo_packed_desc {
  int32_t n_q_heads, n_kv_heads, head_dim, dtype;
  int64_t q_stride_n, q_stride_h;     /* elements, from token to token and from head to head */
  int64_t kv_stride_n, kv_stride_h;   /* of k and v alike */
} hippo_packed_desc;

size_t hippo_prefill_workspace_bytes(const hippo_packed_desc* desc, int32_t total_q, int32_t total_k, int32_t n_seqs, int32_t paged,
                                     int32_t num_splits);
int hippo_prefill_attention(const void* q, int32_t total_q, const void* k, const void* v, int32_t total_k,
                            const hippo_packed_desc* desc, const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs,
                            float softmax_scale, int32_t num_splits, void* out, float* lse_out,
                            void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same over a paged cache (hippo_paged_kv_desc, with batch = n_seqs) that already holds the new rows: sequence b's key row n lies
 * where block_table says, and len_k = kv_lens[b] (int32 on the device, cut off at max_pages * page_size).  Pools of at most 2^22 pages, here and in
 * the tree's and the write's calls.  Workspace: hippo_prefill_workspace_bytes with total_k = max_pages * page_size and paged 1.
 * num_splits 0 takes a row of the table as full: beside a table much wider than the lengths a tile gets blocks without work, whose parts take
 * memory and are merged.  num_splits 1 has none.
 */
int hippo_prefill_attention_paged(const void* q, int32_t total_q, int64_t q_stride_n, int64_t q_stride_h,
                                  const void* k_pool, const void* v_pool, const int32_t* block_table,
                                  const hippo_paged_kv_desc* kv, const int32_t* cu_q, const int32_t* kv_lens,
                                  float softmax_scale, int32_t num_splits, void* out, float* lse_out,
                                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * Verification of a tree of drafted tokens: where a chain's node sees everything before it, a tree's sees the context, its ancestors
 * and itself.
 *   out[b, i, h, :] as hippo_verify_attention's, over n in [0, ctx) and ctx + j for every node j on the way from node i to the root
 *   parents[b, i]: the parent of node i, a node before it; -1: the context's last token.  Anything else (-2, say): there is no
 *   such node (a batch's smaller trees are padded with them), nor its descendants: its row of out is zeros, its lse -inf, and no
 *   node sees it, whatever its rows of K and V hold.
 * n_nodes 1 .. 64.  The cache holds node j's own K and V at row ctx + j, at ctx + n_nodes rows in all.  ctx is ctx_lens[b] (int32
 * [B] on the DEVICE: every sequence has its own length, and a captured graph follows them; cut off at seq_len - n_nodes), or ctx_len where
 * ctx_lens is NULL.  seq_len: rows that the cache has room for.  parents [B, n_nodes] int32 on the device, parents_stride_b
 * elements from one batch element to the next (0: one tree for all).  q, out [B, n_nodes, H, d] contiguous; lse_out optional [B, H, n_nodes].
 * softmax_scale, num_splits (up to seq_len / 64; of 2 to 64 sequences with ctx_lens the average: long ones get more, short ones fewer), rounding,
 * lse, unseen rows as hippo_prefill_attention; num_splits 0 takes a cache of one or of more than 64 sequences as full.  Workspace: hippo_tree_workspace_bytes (which does not look at kv's strides).
 * The accepted path's rows are afterwards moved to ctx, ctx + 1, ...: over pages by hippo_plan_pages (which gives the tree's
 * rows back) and hippo_write_kv_paged (which picks rows).
 * Errors: NULL_ARG, BAD_SHAPE (also more than 65535 sequences or KV heads, 4096 query heads to one of them, 2^30 nodes times query heads of the
 *         batch, 0x7fffff00 rows, row strides above 2^24 elements, or 2^23 blocks and more: ceil(n_nodes * H / H_kv / 256) * batch * H_kv, in fp32 with
 *         head_dim 64 / 128), BAD_DTYPE, BAD_ALIGN, WORKSPACE_TOO_SMALL, HIP.
 */
size_t hippo_tree_workspace_bytes(const hippo_kv_desc* kv, int32_t n_nodes, int32_t seq_len, int32_t num_splits);
int hippo_tree_attention(const void* q, int32_t n_nodes, const void* k_cache, const void* v_cache, const hippo_kv_desc* kv,
                         int32_t seq_len, const int32_t* parents, int64_t parents_stride_b,
                         const int32_t* ctx_lens, int32_t ctx_len, float softmax_scale, int32_t num_splits,
                         void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream);
/* over pages: seq_len = max_pages * page_size (in hippo_tree_workspace_bytes too) */
int hippo_tree_attention_paged(const void* q, int32_t n_nodes, const void* k_pool, const void* v_pool, const int32_t* block_table,
                               const hippo_paged_kv_desc* kv, const int32_t* parents, int64_t parents_stride_b,
                               const int32_t* ctx_lens, int32_t ctx_len, float softmax_scale, int32_t num_splits,
                               void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The pages of a step, from the requests' lengths, without the host: request b has ctx_lens[b] rows in the cache and gets new_lens[b]
 * more, or gives its last -new_lens[b] back (rejected drafts; all of them: the request is done).  All pointers are device int32.
 *   1. given back: the pages behind ceil((ctx + new) / page_size) of every request with new < 0 go on the stack of free pages
 *      (free_pages[0 .. n_free[0]) are free, the last is on top), request by request, each in the order of its table row
 *   2. admitted: request b with new >= 0 if its rows fit its row of the table and, where it needs pages or slots at all, the pages
 *      that the requests with new >= 0 up to and with b need are free and their new rows at most max_tokens
 *   3. the admitted requests take their new pages off the stack, top first, in their order, into the next entries of their row
 * kv_lens_out[b] = the rows that b has then: ctx where it was not admitted.
 * cu_q_out [batch + 1]: offsets of the admitted new rows, 0 for the requests that bring none (hippo_prefill_attention_paged's cu_q)
 * slots_out [max_tokens]: new row t's place in the pool, page * page_size + row in the page; positions_out: its row of the request.
 *   Both are -1 from cu_q_out[batch] on, and a slot is where its page is none of the pool's.
 * n_free_out [1]: how many pages are free then.  free_pages [n_pool_pages] and block_table [batch, max_pages] are written in place:
 * new entries only, those given back stay where they stood.  (So a call may be repeated: as long as n_free and the lengths are
 * the old ones it finds the same.)  ctx_lens, new_lens and n_free may not share memory with anything that is written (BAD_SHAPE).
 * Negative ctx_lens count as 0, n_free as at most n_pool_pages.  page_size a power of two, 16..256; batch <= 4096; max_tokens,
 * n_pool_pages and max_pages <= 2^22, batch * max_pages <= 2^30.  Deterministic.
 * Errors: NULL_ARG, BAD_SHAPE, BAD_ALIGN, HIP.
 */
int hippo_plan_pages(const int32_t* ctx_lens, const int32_t* new_lens, int32_t batch,
                     int32_t* block_table, int32_t max_pages, int32_t* free_pages, int32_t n_pool_pages, const int32_t* n_free,
                     int32_t page_size, int32_t max_tokens, int32_t* slots_out, int32_t* positions_out, int32_t* cu_q_out,
                     int32_t* kv_lens_out, int32_t* n_free_out, void* stream);

/*
 * K and V rows into the pages: row rows[t] (t where rows is NULL) of k_new and v_new goes to slot slots[t], t < n_tokens, for every KV
 * head, bit copies.  Tokens whose slot is outside the pool or whose row is outside [0, n_rows) are skipped, so that a step padded
 * to a fixed size needs no count.  A slot that is named twice holds pieces of either row.
 * k_new, v_new: element (row, hk, c) at row * stride_n + hk * stride_h + c, dtype kv->dtype (F32 or BF16); kv's batch, n_q_heads and
 * max_pages are not looked at.  slots, rows: int32 [n_tokens] on the device.  The pools must not overlap k_new, v_new or each
 * other.  n_tokens = 0 does nothing.
 * Errors: NULL_ARG, BAD_SHAPE (also a pool whose rows would meet, more than 2^31 pieces of 16 bytes in all or 2^20 a token, of K), BAD_DTYPE,
 *         BAD_ALIGN, HIP.
 */
int hippo_write_kv_paged(const void* k_new, const void* v_new, int32_t n_rows, int64_t stride_n, int64_t stride_h,
                         const int32_t* slots, const int32_t* rows, int32_t n_tokens,
                         void* k_pool, void* v_pool, const hippo_paged_kv_desc* kv, void* stream);

/* ------------------------------------------------------------------------------------------
 * Host-side control of video parallel speculative decoding (Method, "Video Parallel Speculative
 * Decoding").  No device work and no device pointers: every argument here is a HOST pointer.
 *
 * A round launches one target verification and, concurrently on another stream, draft decoding:
 *   optimistic mode   (the previous batch was fully accepted, or a prefill buffer exists): the target
 *                     verifies all n_pending buffered draft tokens while the draft model generates the
 *                     next gamma.  Full acceptance emits the verified tokens and the new batch becomes
 *                     the buffer (the extra token of serial speculative decoding is not taken: the draft
 *                     has already continued past it).  A rejection emits the accepted prefix plus the
 *                     target's replacement and discards every other draft; mode becomes conservative.
 *   conservative mode (a rejection occurred, nothing buffered): the draft model generates x_1; then
 *                     the target verifies x_1 alone while the draft generates x_2..x_gamma.  If x_1
 *                     is rejected drafting is aborted, the replacement is emitted and the mode stays;
 *                     if accepted, x_1 is emitted, x_2..x_gamma become the buffer and the mode becomes
 *                     optimistic.
 * (The paper fixes neither what happens to the extra token in the parallel modes nor how many
 * buffered tokens one verification takes; the above is this library's reading.)
 */
enum hippo_vpsd_mode { HIPPO_VPSD_CONSERVATIVE = 0, HIPPO_VPSD_OPTIMISTIC = 1 };
enum hippo_vpsd_policy { HIPPO_POLICY_AUTOREGRESSIVE = 0, HIPPO_POLICY_SERIAL_SD = 1, HIPPO_POLICY_VPSD = 2 };

typedef struct hippo_vpsd_state {
  int32_t gamma;            /* draft tokens per batch, 1..64 */
  int32_t mode;             /* enum hippo_vpsd_mode */
  int32_t n_pending;        /* drafted tokens waiting for verification */
  int32_t reserved;
  int64_t n_emitted;        /* tokens committed to the output so far */
  int64_t n_rounds, n_target_calls;
  int64_t n_draft_tokens;   /* draft forward passes so far (prefill buffer included) */
  int64_t n_draft_wasted;   /* draft tokens generated and then discarded */
  int64_t n_mode_switches;
} hippo_vpsd_state;

typedef struct hippo_vpsd_round {
  int32_t mode;             /* the mode this round runs in */
  int32_t draft_serial;     /* draft tokens to generate BEFORE the parallel phase (1 in conservative mode) */
  int32_t verify_len;       /* draft tokens the target verifies: hippo_verify_attention q_len = verify_len + 1,
                               hippo_spec_verify gamma = verify_len */
  int32_t draft_parallel;   /* draft tokens to generate concurrently with that verification */
} hippo_vpsd_round;

typedef struct hippo_vpsd_result {
  double time;              /* modelled wall time, in the unit of t_draft / t_target */
  double speedup;           /* n_emitted * t_target / time: against one target forward per token */
  int64_t n_emitted, n_rounds, n_target_calls, n_draft_tokens, n_draft_wasted, n_mode_switches;
  int64_t n_flags_used;
} hippo_vpsd_result;

/* Tokens the draft model can decode while the target model is still in prefill ("Synchronous
 * Draft-Target Prefill"): floor((t_prefill_target - t_prefill_draft) / t_draft_token), 0 if the
 * target is not slower; the paper's example (0.8 s, 0.2 s, 50 ms) gives 12.  -1 on invalid times. */
int32_t hippo_vpsd_prefill_buffer(double t_prefill_target, double t_prefill_draft, double t_draft_token);

/* Start of generation: n_prefill_buffer (0..64) draft tokens already buffered; optimistic if any. */
int hippo_vpsd_init(hippo_vpsd_state* state, int32_t gamma, int32_t n_prefill_buffer);
/* What to enqueue in the next round.  Does not change the state. */
int hippo_vpsd_plan(const hippo_vpsd_state* state, hippo_vpsd_round* round_out);
/* Account for the round's outcome: n_accept in [0, verify_len] as hippo_spec_verify reports it,
 * n_drafted_parallel = draft tokens actually produced concurrently (= draft_parallel unless
 * drafting was cut short by a rejection).  Errors: NULL_ARG, BAD_SHAPE (a round that is not the
 * one planned for this state, counts out of range, a fully accepted round whose new batch is
 * incomplete). */
int hippo_vpsd_commit(hippo_vpsd_state* state, const hippo_vpsd_round* round, int32_t n_accept,
                      int32_t n_drafted_parallel);

/* Timing model of a generation of at least n_tokens tokens under `policy`, with one draft forward
 * costing t_draft, one target forward (any verify width: it is memory-bound) t_target, and the
 * i-th verified draft token accepted iff accept[i] != 0 (flags beyond n_flags count as accepted;
 * one flag is consumed per token looked at, the rejected one included).
 *   AUTOREGRESSIVE: n_tokens target forwards.
 *   SERIAL_SD: per round gamma draft forwards, then one verification; emits n_accept + 1 tokens
 *     (Motivated Experiments, "Non-negligible Draft Latency": with t_target = 3 t_draft and gamma = 3
 *     the speedup is 2 when everything is accepted and 0.5 when every first token is rejected).
 *   VPSD: the state machine above; a fully accepted round costs draft_serial * t_draft +
 *     max(t_target, draft_parallel * t_draft), a round with a rejection draft_serial * t_draft +
 *     t_target (drafting is cut when the verdict arrives). */
int hippo_vpsd_simulate(int32_t policy, int32_t gamma, double t_draft, double t_target,
                        int32_t n_prefill_buffer, const uint8_t* accept, int64_t n_flags,
                        int64_t n_tokens, hippo_vpsd_result* result_out);

#ifdef __cplusplus
}
#endif
#endif /* HIPPO_H_ */
