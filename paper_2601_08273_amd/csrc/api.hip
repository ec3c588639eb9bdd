// extern "C" boundary: argument validation, launch heuristics and workspace carving.  No kernel
// lives here.  Every check runs before the first launch, so a non-zero status means nothing was
// enqueued.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "rows_attention.h"

using namespace hippo;

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int elem_bytes(int dtype) {
  return dtype == HIPPO_DTYPE_FP8_E4M3 ? 1 : (dtype == HIPPO_DTYPE_BF16 ? 2 : 4);
}

// allow_fp8: the call takes 8-bit caches (the fp8 attention calls, the gather, their workspace query)
int check_heads(const hippo_kv_desc* kv, bool allow_fp8) {
  if (kv == nullptr) return HIPPO_ERR_NULL_ARG;
  if (kv->dtype != HIPPO_DTYPE_F32 && kv->dtype != HIPPO_DTYPE_BF16 &&
      !(allow_fp8 && kv->dtype == HIPPO_DTYPE_FP8_E4M3))
    return HIPPO_ERR_BAD_DTYPE;
  if (kv->batch < 1 || kv->n_kv_heads < 1 || kv->n_q_heads < 1) return HIPPO_ERR_BAD_SHAPE;
  if (kv->n_q_heads % kv->n_kv_heads != 0) return HIPPO_ERR_BAD_SHAPE;
  if (kv->head_dim != 64 && kv->head_dim != 128) return HIPPO_ERR_BAD_SHAPE;
  if (kv->batch > 65535 || kv->n_kv_heads > 65535) return HIPPO_ERR_BAD_SHAPE;
  return HIPPO_OK;
}

int check_kv(const hippo_kv_desc* kv, bool allow_fp8 = false) {
  const int rc = check_heads(kv, allow_fp8);
  if (rc != HIPPO_OK) return rc;
  if (kv->stride_n < kv->head_dim || kv->stride_h < 0 || kv->stride_b < 0) return HIPPO_ERR_BAD_SHAPE;
  if (kv->stride_n > (1ll << 24)) return HIPPO_ERR_BAD_SHAPE;   // row offsets inside a tile stay 32-bit
  const int per16 = 16 / elem_bytes(kv->dtype);
  if (kv->stride_n % per16 || kv->stride_h % per16 || kv->stride_b % per16) return HIPPO_ERR_BAD_ALIGN;
  return HIPPO_OK;
}

// Blocks of `len` elements at d[0].stride i + d[1].stride j + d[2].stride k, i < d[0].count and so on: whether two of them share an
// element, that is, whether len exceeds the size of some sum of the strides, each up to count - 1 times and in either direction.
// The wider strides come first: what the narrower ones reach leaves few multiples of a wider one to try, and none but 0 of the
// layouts in which a dimension steps over the ones inside it.
struct Spaced {
  long long count, stride;
};
bool blocks_meet(const Spaced* d, int n, __int128 at, bool moved, long long len) {
  if (n == 0) return moved && at < len && -at < len;
  __int128 reach = len - 1;
  for (int i = 1; i < n; ++i) reach += (__int128)(d[i].count - 1) * d[i].stride;
  if (d->count <= 1) return blocks_meet(d + 1, n - 1, at, moved, len);
  const __int128 most = d->count - 1, s = d->stride;             // s >= len > 0, see rows_meet
  __int128 lo = -((reach + at) / s), hi = (reach - at) / s;
  // (a distance and its opposite are of the same two blocks)
  for (__int128 i = std::max(lo, moved ? -most : (__int128)0); i <= std::min(hi, most); ++i)
    if (blocks_meet(d + 1, n - 1, at + i * s, moved || i != 0, len)) return true;
  return false;
}
bool rows_meet(Spaced a, Spaced b, Spaced c, long long len) {
  if (len < 1) return false;
  Spaced d[3] = {a, b, c};
  for (const Spaced& x : d)
    if (x.count > 1 && x.stride < len) return true;
  std::sort(d, d + 3, [](const Spaced& x, const Spaced& y) { return x.stride > y.stride; });
  return blocks_meet(d, 3, 0, false, len);
}

int check_video(const hippo_video_desc* v) {
  if (v == nullptr) return HIPPO_ERR_NULL_ARG;
  if (v->n_frames < 1 || v->grid_h < 1 || v->grid_w < 1 || v->vis_offset < 0) return HIPPO_ERR_BAD_SHAPE;
  if ((long long)v->n_frames * v->grid_h * v->grid_w > (1ll << 30)) return HIPPO_ERR_BAD_SHAPE;
  if (v->n_frames > 65535) return HIPPO_ERR_BAD_SHAPE;   // frames are a y dimension of the crop kernels' grids
  return HIPPO_OK;
}

// ---- attention planning -------------------------------------------------------------------------
constexpr size_t kStaticScratchBytes = 8u << 20;   // hippo_verify_attention_static's array

struct AttnPlan {
  int R, row_chunk, n_chunks, S;
  bool wide;                               // 65 to 96 bf16 rows in one block
  size_t off_m, off_l, off_e, bytes;
};

// mass: for a call that sums its weights
int plan_attention(int call, const hippo_kv_desc* kv, int q_len, int n_total, int num_splits, AttnPlan* pl,
                   bool may_be_wide = true, bool mass = false) {
  (void)call;   // draft and verify share one launch heuristic (they differ in wave priority only)
  if (q_len < 1 || n_total < q_len || num_splits < 0) return HIPPO_ERR_BAD_SHAPE;
  const int G = kv->n_q_heads / kv->n_kv_heads;
  if ((long long)G * q_len > 4096) return HIPPO_ERR_BAD_SHAPE;
  pl->R = G * q_len;
  const bool f32 = kv->dtype == HIPPO_DTYPE_F32;
  // A block takes at most 64 rows of a 16- or 8-bit cache (96 of a large bf16 one, below): more go in equal chunks, the same
  // slices and tiles in every cache format (chunks of 64 and a rest -> equal ones, us a call with K and V in the last-level
  // cache / from HBM, before one block took up to 96 rows of the large ones: 33K x 4
  // heads, 91 rows 23.3 -> 21.0 / 28.0 -> 26.4; 8K, 91 rows 14.4 -> 13.6 / 14.5 -> 13.6; 2 x 8 heads x 20K, 72 rows 40.1 -> 35.9 /
  // 54.2 -> 53.4; 8-bit 33K, 91 rows 24.6 -> 20.7 / 25.2 -> 21.5).  The fp32 kernel takes 65 to 128 in one chunk: two chunks
  // stream the whole cache twice and give every slice half the compute units (a call over 70K x 2 heads x 64 channels, 70 rows: 43 us in one chunk, 52 in two; four
  // sequences x 9K, 91 rows: 28.9 and 33.6).  Not where a slice per compute unit leaves units idle, which the two chunks
  // then have to themselves (1K x 4 heads x 128, 77 rows: 16.4 in one, 15.0 in two); nor where it means more than 64
  // slices, the most the merge takes in one step, of under eight tiles (64 channels x 2 heads, 91 rows, 4K: 14.9 in one
  // and 128 slices, 12.9 in two; 16K: 22.0 and 21.2).  Beyond 128 rows a block has no waves left for one chunk.
  const int n_tiles = (n_total + 31) / 32;
  const long long heads = (long long)kv->batch * kv->n_kv_heads;
  // The library's choice never takes more slices than the static array has room for (one excepted), so that the static
  // call serves it with the same slices and hence the same bits.  A slice per compute unit of up to 124 fp32 rows of 64
  // channels fits, of 65 rows of 128 channels does not: those go in two chunks (33K x 4 heads, 91 rows: 92 us; 95 in one
  // chunk of as many slices as fit, 74 in one of a slice per compute unit).
  const size_t slice_bytes = (size_t)heads * pl->R * (kv->head_dim * (f32 ? sizeof(float) : 2) + 2 * sizeof(float));
  const long long fit = std::max<long long>(1, (long long)((kStaticScratchBytes - 3 * 256) / slice_bytes));
  const bool one_chunk = f32 && pl->R > 64 && pl->R <= 128 && n_tiles * heads > kNumCU &&
                         (kNumCU <= 64 * heads || n_tiles * heads >= 8 * kNumCU) &&
                         (num_splits > 0 || kNumCU / heads <= fit);
  // 65 to 96 rows of a bf16 cache that no cache of the chip holds go in one block too: the second chunk's blocks keep half the
  // transfers in flight on what the first chunk's fetch.  us a call from a graph over two caches in turn, two chunks -> one:
  // 4 x 8 heads x 128 x 37000, 72 rows 130 -> 108, from pages 149 -> 112; 37127, 96 rows 130 -> 108, from pages 152 -> 116;
  // 4 x 4 x 33000, 70 rows 62 -> 52, from pages 72 -> 58; 64 channels, 4 x 8 x 37000, 72 rows 86 -> 76, from pages 95 -> 78.
  // Of a cache that the last-level cache can hold not: 33K x 4 heads, 91 rows of eight layers in turn 24.9 and 24.8, from
  // pages 27.4 and 25.7, but of one layer 27.1 against 29.8; 16K 16.4 against 19.3.
  // Nor where the heads (batch elements x KV heads) come in a second round and the chunks of a head on one XCD, at the same
  // time, so that its L2 serves the second chunk: KV heads a multiple of 8, up to 160, of 64 channels (two chunks' time = 1: 264 to
  // 384 heads 1.02 to 1.25, 38 x 8 x 9359, 77 rows 214 -> 258 us; 400 to 512 0.90 to 1.05; 528 to 640 1.04 to 1.18; more 0.97 to 1.13;
  // KV heads of 192 and more, or 12, 20, 36 0.72 to 0.99), up to 32 of 128 channels, up to 384 heads (0.94 to 1.07; of 40 to 96 0.80 to
  // 0.99, 400 heads and more, two rounds for four of chunks, 0.79 to 0.94).  Up to 256 heads 0.68 to 1.00.
  // A slice of each head has to fit the static array: 128 channels, 96 rows up to 321 heads, 64 channels 606; more take two chunks.
  const bool shared = heads > kNumCU && kv->n_kv_heads % 8 == 0 &&
                      (kv->head_dim == 64 ? kv->n_kv_heads <= 160 : kv->n_kv_heads <= 32 && heads <= 384);
  const long long fit_wide = (long long)((kStaticScratchBytes - 4 * 256) / (slice_bytes + (size_t)heads * pl->R * 2 * sizeof(float)));
  const bool wide = pl->wide = may_be_wide && kv->dtype == HIPPO_DTYPE_BF16 && pl->R > 64 && pl->R <= 96 && num_splits == 0 &&
                    !shared && fit_wide >= 1 && 2 * heads * n_total * kv->head_dim * 2 > (256ll << 20);
  const int n_equal = (pl->R + 63) / 64;
  pl->row_chunk = wide ? 96 : one_chunk ? (pl->R <= 96 ? 96 : 128) : f32 && pl->R > 64 ? 64 : ((pl->R + n_equal - 1) / n_equal + 15) / 16 * 16;
  // short caches are bound by latency, not bytes: thin slices on many compute units win (bf16, 1896 rows, 7 query
  // rows: 59 slices of 32 rows beat 14 of 128 by 9 %)
  pl->n_chunks = (pl->R + pl->row_chunk - 1) / pl->row_chunk;
  if ((long long)kv->batch * pl->n_chunks > 65535) return HIPPO_ERR_BAD_SHAPE;
  int S = num_splits;
  if (S == 0) {
    // one block per compute unit (measured at the 16K configuration: 48 or 80-128 slices per KV head
    // are all slower than 64), but never slices thinner than one 32-token tile
    const long long per_split = (long long)kv->batch * kv->n_kv_heads * pl->n_chunks;
    S = (int)(kNumCU / per_split);          // rounded down: a block beyond the last compute unit would share one
    if (S < 1) S = 1;
    if (S > fit) S = (int)fit;
    if (wide) S = (int)std::max<long long>(1, std::min<long long>(kNumCU / heads, fit_wide));   // (the exponents fit too)
    // A cache of a few tiles under up to 16 query rows goes in one slice, whose block writes the output itself: no merge
    // launch.  Where the line lies, us a call in a graph, slices and merge -> one slice (eager 10.7 -> 8): bf16, 7 rows,
    // 4 heads x 128: 100 rows 6.2 -> 4.1, 250 6.2 -> 5.3, 500 6.3 -> 8.3; 8 bits: 100 6.5 -> 4.8, 200 6.6 -> 6.4, 256 6.5 -> 6.4
    // (2 heads x 64: 256 rows bf16 5.9 -> 4.5, 8 bits 6.0 -> 5.0); fp32: 100 8.1 -> 7.1, 250 8.0 -> 10.8; bf16, 35 rows: 100
    // 6.7 -> 5.5, 250 6.9 -> 7.6.
    const int few_tiles = pl->R > 16 ? 0 : f32 ? 4 : 8;
    if (n_tiles <= few_tiles) S = 1;
  }
  if (S > n_tiles) S = n_tiles;
  if (S < 1) S = 1;
  if (S > 1024) S = 1024;
  pl->S = S;
  const size_t slots = (size_t)kv->batch * kv->n_kv_heads * S;
  // the bf16 kernel hands its slices' outputs to the merge as bf16, the fp32 kernel and the one for attention mass as fp32
  const size_t o_bytes = align_up(slots * pl->R * kv->head_dim * (f32 || mass ? sizeof(float) : 2), 256);
  const size_t ml_bytes = align_up(slots * pl->R * sizeof(float), 256);
  pl->off_m = o_bytes;
  pl->off_l = o_bytes + ml_bytes;
  pl->off_e = o_bytes + 2 * ml_bytes;
  pl->bytes = pl->off_e + (wide ? align_up(slots * pl->R * 2 * sizeof(float), 256) : 0);
  return HIPPO_OK;
}

// What a call that sums its weights needs beside that: the slices' second denominators, and the logits.
struct MassPlan {
  AttnPlan attn;
  int logits_ld;
  size_t off_f, off_logits, bytes;
};

int plan_mass(int call, const hippo_kv_desc* kv, int q_len, int n_total, int num_splits, MassPlan* pl) {
  const int rc = plan_attention(call, kv, q_len, n_total, num_splits, &pl->attn, false, true);
  if (rc != HIPPO_OK) return rc;
  const size_t heads = (size_t)kv->batch * kv->n_kv_heads;
  pl->logits_ld = (int)align_up((size_t)n_total, 64);
  pl->off_f = pl->attn.bytes;
  pl->off_logits = pl->off_f + align_up(heads * pl->attn.S * pl->attn.R * sizeof(float), 256);
  pl->bytes = pl->off_logits + heads * pl->attn.R * pl->logits_ld * sizeof(float);
  return HIPPO_OK;
}

// what the cache-format variants add to a plain attention call
struct AttnExtra {
  bool append = false;
  const void* k_new = nullptr;
  const void* v_new = nullptr;
  const int32_t* block_table = nullptr;     // paged
  int page_size = 0, max_pages = 0, n_pool_pages = 0;
  long long page_stride = 0;
  bool fp8 = false;                         // E4M3 cache with per-(b, hk) multipliers
  const float* k_scale = nullptr;
  const float* v_scale = nullptr;
  bool mass = false;                        // sums of the weights
  const float* mass_in = nullptr;
  float* mass_out = nullptr;
  long long mass_isb = 0, mass_ish = 0, mass_osb = 0, mass_osh = 0;
};

int attention_entry(int call, const void* q, int32_t q_len, const void* k_cache, const void* v_cache,
                    const hippo_kv_desc* kv, int32_t ctx_len, float softmax_scale, int32_t num_splits,
                    void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream,
                    const AttnExtra& ex = AttnExtra()) {
  const bool append = ex.append;
  const void* k_new = ex.k_new;
  const void* v_new = ex.v_new;
  if (q == nullptr || k_cache == nullptr || v_cache == nullptr || out == nullptr || workspace == nullptr)
    return HIPPO_ERR_NULL_ARG;
  if (append && (k_new == nullptr || v_new == nullptr)) return HIPPO_ERR_NULL_ARG;
  if (ex.fp8 && (ex.k_scale == nullptr || ex.v_scale == nullptr)) return HIPPO_ERR_NULL_ARG;
  int rc = check_kv(kv, ex.fp8);
  if (rc != HIPPO_OK) return rc;
  if (ex.fp8 != (kv->dtype == HIPPO_DTYPE_FP8_E4M3)) return HIPPO_ERR_BAD_DTYPE;
  if (ctx_len < 0 || q_len < 1 || (long long)ctx_len + q_len > 0x7fffff00ll) return HIPPO_ERR_BAD_SHAPE;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return HIPPO_ERR_BAD_ALIGN;
  if (append && (!aligned16(k_new) || !aligned16(v_new))) return HIPPO_ERR_BAD_ALIGN;
  AttnPlan pl;
  MassPlan mp;
  rc = ex.mass ? plan_mass(call, kv, q_len, ctx_len + q_len, num_splits, &mp)
               : plan_attention(call, kv, q_len, ctx_len + q_len, num_splits, &pl);
  if (rc != HIPPO_OK) return rc;
  if (ex.mass) {
    pl = mp.attn;
    pl.bytes = mp.bytes;
  }
  // One block for 65 to 96 rows needs twice the workspace of two chunks.  A loop that sized its own before the cache grew past
  // that line, or for more query rows, goes on in two chunks.
  if (workspace_bytes < pl.bytes && pl.wide) rc = plan_attention(call, kv, q_len, ctx_len + q_len, num_splits, &pl, false);
  if (rc != HIPPO_OK) return rc;
  if (workspace_bytes < pl.bytes) return HIPPO_ERR_WORKSPACE_TOO_SMALL;
  int page_shift = 0;
  if (ex.block_table != nullptr) {
    while ((1 << page_shift) < ex.page_size) ++page_shift;
    // a block keeps the page numbers of its slice in LDS: bound the slice (32-token tiles, a ragged
    // tile at either end) by the staging area
    const long long tiles32 = ((long long)ctx_len + q_len + 31) / 32;
    const long long slice_tokens = (tiles32 / pl.S + 2) * 32;
    if (slice_tokens / ex.page_size + 2 > kMaxSlicePages) return HIPPO_ERR_BAD_SHAPE;
  }

  AttnParams p;
  p.q = q; p.k = k_cache; p.v = v_cache; p.out = out; p.lse = lse_out;
  p.part_o = workspace;
  p.part_m = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.off_m);
  p.part_l = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.off_l);
  p.part_e = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.off_e);
  p.B = kv->batch; p.q_len = q_len; p.H = kv->n_q_heads; p.Hkv = kv->n_kv_heads;
  p.G = kv->n_q_heads / kv->n_kv_heads; p.R = pl.R;
  p.ctx_len = ctx_len; p.n_total = ctx_len + q_len;
  p.sb = kv->stride_b; p.sh = kv->stride_h; p.sn = kv->stride_n;
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)kv->head_dim);
  p.scale_log2 = scale * kLog2e;
  p.S = pl.S; p.row_chunk = pl.row_chunk; p.n_chunks = pl.n_chunks;
  p.wave_prio = call == HIPPO_CALL_VERIFY_ATTENTION ? 1 : 0;
  p.phase_per_head = 1.0f / (float)((long long)kv->batch * kv->n_kv_heads);
  p.k_new = append ? k_new : nullptr; p.v_new = append ? v_new : nullptr;
  p.k_w = const_cast<void*>(k_cache); p.v_w = const_cast<void*>(v_cache);
  p.block_table = ex.block_table; p.page_shift = page_shift; p.max_pages = ex.max_pages;
  p.n_pool_pages = ex.n_pool_pages; p.page_stride = ex.page_stride;
  p.k_scale = ex.fp8 ? ex.k_scale : nullptr; p.v_scale = ex.fp8 ? ex.v_scale : nullptr;
  if (ex.mass) {
    MassParams m;
    static_cast<AttnParams&>(m) = p;
    char* ws = static_cast<char*>(workspace);
    // (fp32 probabilities are not rounded: one denominator serves both)
    m.part_f = kv->dtype == HIPPO_DTYPE_F32 ? p.part_l : reinterpret_cast<float*>(ws + mp.off_f);
    m.logits = reinterpret_cast<float*>(ws + mp.off_logits);
    m.logits_ld = mp.logits_ld;
    m.mass_in = ex.mass_in; m.mass_out = ex.mass_out;
    m.mass_isb = ex.mass_isb; m.mass_ish = ex.mass_ish; m.mass_osb = ex.mass_osb; m.mass_osh = ex.mass_osh;
    const hipError_t e = launch_attention_mass(m, kv->dtype, kv->head_dim, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
  }
  // q and out of the 8-bit cache calls are bf16
  const int io_dtype = ex.fp8 ? (int)HIPPO_DTYPE_BF16 : kv->dtype;
  const hipError_t e = launch_attention(p, io_dtype, kv->head_dim, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

// ---- scoring planning ---------------------------------------------------------------------------
struct ScorePlan {
  int n_tile, n_rsplit;
  bool once;
  size_t off_word, off_bin, off_flags, off_arrived, clear_bytes, off_redo;   // one sweep: all but the last are cleared together
  size_t off_row_l, off_row_lse, off_col, off_sa, off_st, off_ss, bytes;
};

// finer: the finer cuts of short videos (see score_row_splits)
int plan_score(const hippo_kv_desc* kv, const hippo_video_desc* vid, int l_txt, int n_layers, ScorePlan* pl, bool finer = true) {
  if (l_txt < 1 || l_txt > (1 << 20)) return HIPPO_ERR_BAD_SHAPE;
  if (n_layers < 1 || n_layers > kMaxScoreLayers || (long long)kv->batch * n_layers > 65535) return HIPPO_ERR_BAD_SHAPE;
  const long long Nv = (long long)vid->n_frames * vid->grid_h * vid->grid_w;
  const int tile = score_token_tile(kv->dtype);
  pl->n_tile = (int)((Nv + tile - 1) / tile);
  if (pl->n_tile > 0x7fffffff / 2) return HIPPO_ERR_BAD_SHAPE;
  const size_t rows = (size_t)kv->batch * n_layers * kv->n_q_heads * l_txt;
  const size_t row_part = align_up(rows * pl->n_tile * sizeof(float), 256);
  const size_t row_lse = align_up(rows * sizeof(float), 256);
  const int rows_per_kv_head = l_txt * (kv->n_q_heads / kv->n_kv_heads);
  pl->once = score_once(kv->dtype, Nv, rows_per_kv_head);
  pl->n_rsplit = score_row_splits(kv->dtype, (long long)pl->n_tile * kv->n_kv_heads * kv->batch * n_layers,
                                  rows_per_kv_head, kv->head_dim, pl->once, finer, kv->n_kv_heads * n_layers);
  // launch limits of the sweeps (KV heads on grid x, key tiles on y, row runs x (layer, batch element) on z) and of
  // the row merge (32 rows per block)
  if (pl->n_tile > 65535 || (long long)kv->batch * n_layers * pl->n_rsplit > 65535 || kv->n_kv_heads > 65535 ||
      rows / 32 >= (1ull << 31))
    return HIPPO_ERR_BAD_SHAPE;
  const size_t col = align_up((size_t)kv->batch * n_layers * kv->n_kv_heads * pl->n_rsplit * Nv * sizeof(float), 256);
  const size_t vec = align_up((size_t)kv->batch * Nv * sizeof(float), 256);
  size_t o = 0;
  o += row_part;            pl->off_row_l = o;
  o += row_part;            pl->off_row_lse = o;
  o += row_lse;             pl->off_col = o;
  o += col;                 pl->off_sa = o;
  o += vec;                 pl->off_st = o;
  o += vec;                 pl->off_ss = o;
  o += vec;
  const size_t heads = (size_t)kv->n_kv_heads * kv->batch * n_layers, runs = heads * pl->n_rsplit;
  const size_t once_rows = heads * score_once_rows(rows_per_kv_head) * sizeof(unsigned long long);
  const size_t words = once_rows * kScoreOnceWords, bins = once_rows * kScoreOnceBins;
  // (its launches are one-dimensional: a grid's threads stay below 2^32)
  pl->once = pl->once && runs * pl->n_tile < (1u << 22) && words + bins < (1ull << 34);
  if (pl->once) {
    pl->off_word = o;       o += align_up(words, 256);
    pl->off_bin = o;        o += align_up(bins, 256);
    pl->off_flags = o;      o += align_up(runs * 2 * sizeof(unsigned), 256);
    pl->off_arrived = o;    o += align_up(runs * sizeof(int), 256);
    pl->clear_bytes = o - pl->off_word;
    pl->off_redo = o;       o += align_up(runs * pl->n_tile * sizeof(int), 256);
  }
  pl->bytes = o;
  return HIPPO_OK;
}

int check_crop(const hippo_video_desc* vid) {
  if (vid->crop_h < 1 || vid->crop_w < 1 || (long long)vid->crop_h * vid->crop_w > 64) return HIPPO_ERR_BAD_SHAPE;
  return HIPPO_OK;
}

// ---- speculative-sampling verification planning -------------------------------------------------
struct SpecPlan {
  int n_seg, n_rows;
  size_t off_cells, off_arrived, bytes;
};

int plan_spec(int batch, int gamma, int vocab, int dtype, SpecPlan* pl) {
  if (dtype != HIPPO_DTYPE_F32 && dtype != HIPPO_DTYPE_BF16) return HIPPO_ERR_BAD_DTYPE;
  if (batch < 1 || batch > 65535 || gamma < 0 || gamma > kSdMaxGamma || vocab < 1 || vocab > kSdMaxVocab)
    return HIPPO_ERR_BAD_SHAPE;
  pl->n_seg = (vocab + kSdSeg - 1) / kSdSeg;
  pl->n_rows = 2 * gamma + 1;
  const size_t stats = align_up((size_t)batch * pl->n_rows * pl->n_seg * sizeof(SegStat), 256);
  const size_t cells = align_up((size_t)batch * 2 * pl->n_seg * spec_cells_per_segment(dtype) * sizeof(float), 256);
  pl->off_cells = stats;
  pl->off_arrived = stats + cells;
  pl->bytes = stats + cells + align_up((size_t)batch * sizeof(int), 256);
  return HIPPO_OK;
}

// ---- attention of many rows: planning -------------------------------------------------------------
constexpr int kMaxRowSplits = 64;   // the merge keeps a split's statistics in a lane

// The blocks that a call can be cut into: row blocks, made in pairs (launch_rows_rb's).
struct RowsBlock {
  int rb;
  bool pair;
};
const RowsBlock kRowsBlocks[] = {{8, false}, {4, false}, {4, true}, {2, false}, {1, false}};
// What a block takes, in us: `fixed` (its start, its masked stages and its end) and `pace` for 64 tokens; beside another one on its compute unit,
// where it leaves room for one (pace_beside 0: it does not).  Pace 0: there is no such block (fp32 x 64: pairs take 4 to 40 % less than 256
// rows a block).  bf16: fitted to 492 calls of prompts (1 to 200 of 4 to 16384 rows, 1 to 4096 over up to 30000) and 112 of trees (1 to 128 of
// 1 to 64 nodes over 30 to 30000 rows), each timed with every block and, trees, 1 to 48 blocks a tile, by random steps that lower the mean
// logarithm of (time of the block that this chooses) / (least time): 1.2 and 2.2 % (prompts, 64 and 128 channels), 2.7 and 2.2 % (trees), at
// worst 44 %.  The times are in profiles/rows_blocks_timings.txt; caches and tables with much more room than rows are not among them.
// fp32: from 64 nodes over 16640 rows of 28 x 128, 16 over 2000 of 14 x 64, prompts of 32 to 16384 rows.
struct RowsCost {
  double fixed, pace, fixed_beside, pace_beside;
};
const RowsCost kRowsCost[2][2][2][5] = {      // [trees][bf16][head_dim 128], as kRowsBlocks
    {{{{0, 0}, {7.0, 4.4}, {3.5, 4.6, 3.5, 8.1}, {4.5, 2.3}, {4.0, 1.45}}, {{7.0, 16.0}, {7.0, 8.2}, {0, 0}, {4.5, 4.8}, {0, 0}}},
     {{{7.0, 1.01}, {4.5, 0.65}, {3.7, 0.98, 3.0, 1.23}, {4.5, 0.32}, {4.0, 0.34}},
      {{7.0, 1.40}, {6.5, 0.79}, {3.5, 1.37, 3.4, 1.61}, {3.6, 1.1, 3.5, 1.1}, {5.1, 0.80}}}},
    {{{{0, 0}, {5.0, 4.4}, {4.5, 4.6, 4.5, 8.1}, {4.9, 2.3}, {4.3, 1.45}}, {{5.5, 16.0}, {5.0, 8.2}, {0, 0}, {4.9, 4.8}, {0, 0}}},
     {{{6.2, 1.0}, {6.5, 0.62}, {4.7, 1.04, 2.5, 1.7}, {6.0, 0.36}, {5.2, 0.37}},
      {{8.0, 1.38}, {7.0, 0.83}, {5.5, 1.23, 4.8, 2.15}, {5.4, 1.03, 5.4, 1.45}, {5.7, 0.69}}}}};

// How to cut a call: the rows of a block and the blocks that share a tile's tokens, by the time that they are going to take.
//   a block: its fixed time besides its tokens, one on a compute unit at a time, or two
//   a call:  the longest block of all, or all blocks on all compute units: as many rounds as that takes, a last one in proportion where
//            the blocks' sizes are spread (short ones fill it up)
//   blocks that share tiles: a merge, kMergeUs and kMergeMbUs for a megabyte of parts
// rows: query rows of a KV head of one sequence, on average; seen, seen_least: the tokens that the last and the first of them see; tree:
// a sequence's tiles are its own; num_splits: the caller's, who may know that one of the sequences is much longer than the others: as many
// blocks as `longest`, the most tokens that one can have, has stages for.
constexpr double kMergeUs = 3.0, kMergeMbUs = 0.75;
void cut_rows(RowsPlan* pl, int dtype, int head_dim, double rows, double n_seqs, double seen, double seen_least, double longest, bool tree,
              int Hkv, double part_bytes, int num_splits) {
  static const int splits[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64};
  double best = 1e30;
  for (int b = 0; b < 5; ++b) {
    const RowsBlock& of = kRowsBlocks[b];
    const RowsCost& cost = kRowsCost[tree][dtype == HIPPO_DTYPE_BF16][head_dim == 128][b];
    if (cost.pace == 0) continue;
    const double tiles = n_seqs * (tree ? ceil(rows / (32 * of.rb)) : std::max(1.0, rows / (32 * of.rb) + 0.5)) * Hkv;
    for (int S : splits) {
      if (num_splits > 0 ? S != 1 : S > 1 && seen < 64.0 * S) break;
      const double n = num_splits > 0 ? num_splits : S;
      const bool two = cost.pace_beside > 0, beside = two && tiles * n > kNumCU;
      const double fixed = beside ? cost.fixed_beside : cost.fixed, pace = beside ? cost.pace_beside : cost.pace;
      const double longest = fixed + seen / 64 / n * pace, mean = fixed + (seen + seen_least) / 128 / n * pace;
      const double rounds = tiles * n / (two ? 2 * kNumCU : kNumCU), alike = (fixed + seen_least / 64 / n * pace) / longest;
      const double t = std::max(longest, (rounds + alike * (ceil(rounds) - rounds)) * mean) +
                       (n > 1 ? kMergeUs + kMergeMbUs * n * part_bytes * 1e-6 : 0.0);
      if (t < best * 0.999) {
        best = t;
        pl->rb = of.rb;
        pl->pair = of.pair;
        pl->S = S;
      }
    }
  }
  if (num_splits > 0) pl->S = num_splits;
  pl->S = (int)std::max(1.0, std::min<double>(std::min(pl->S, kMaxRowSplits), ((num_splits > 0 ? longest : seen) + 63) / 64));
}

// A launch numbers its threads along a dimension in 32 bits, and a block has up to 512.  What is too much for the block that was chosen by
// time goes in larger ones: tiles(rows of a block) is how many a KV head has then.
constexpr long long kMostBlocks = (1ll << 32) / 512 - 1;
template <typename Tiles>
bool fit_rows(RowsPlan* pl, int dtype, int head_dim, int Hkv, Tiles tiles) {
  while (tiles(32 * pl->rb) * Hkv > kMostBlocks) {
    int larger = -1;
    for (int b = 0; b < 5; ++b)                               // (from the largest down)
      if (kRowsBlocks[b].rb > pl->rb && !kRowsBlocks[b].pair && kRowsCost[0][dtype == HIPPO_DTYPE_BF16][head_dim == 128][b].pace != 0) larger = b;
    if (larger < 0) return false;
    pl->rb = kRowsBlocks[larger].rb;
    pl->pair = false;
  }
  return true;
}

void carve_plan(RowsPlan* pl, int head_dim, long long tokens, int H) {
  if (tokens * H > (1 << 25)) pl->S = 1;                      // (the merge's launch: 64 threads a row and head, below 2^32)
  const size_t slots = pl->S > 1 ? (size_t)pl->S * tokens * H : 0;
  pl->off_m = align_up(slots * head_dim * sizeof(float), 256);
  pl->off_l = pl->off_m + align_up(slots * sizeof(float), 256);
  pl->bytes = std::max<size_t>(256, pl->off_l + align_up(slots * sizeof(float), 256));
}

int check_packed(const hippo_packed_desc* d) {
  if (d == nullptr) return HIPPO_ERR_NULL_ARG;
  if (d->dtype != HIPPO_DTYPE_F32 && d->dtype != HIPPO_DTYPE_BF16) return HIPPO_ERR_BAD_DTYPE;
  if (d->n_kv_heads < 1 || d->n_q_heads < 1 || d->n_q_heads % d->n_kv_heads != 0) return HIPPO_ERR_BAD_SHAPE;
  if (d->n_q_heads > 65535 || (d->head_dim != 64 && d->head_dim != 128)) return HIPPO_ERR_BAD_SHAPE;
  if (d->q_stride_n < 0 || d->q_stride_h < 0 || d->kv_stride_n < 0 || d->kv_stride_h < 0) return HIPPO_ERR_BAD_SHAPE;
  if (d->kv_stride_n > (1ll << 24)) return HIPPO_ERR_BAD_SHAPE;   // row offsets inside a transfer stay 32-bit
  const int per16 = 16 / elem_bytes(d->dtype);
  if (d->q_stride_n % per16 || d->q_stride_h % per16 || d->kv_stride_n % per16 || d->kv_stride_h % per16) return HIPPO_ERR_BAD_ALIGN;
  return HIPPO_OK;
}

// total_k: rows of packed K and V, or the most that a sequence's pages hold
int plan_prefill(const hippo_packed_desc* d, bool paged, int total_q, int total_k, int n_seqs, int num_splits, RowsPlan* pl) {
  if (total_q < 0 || total_k < 0 || n_seqs < 1 || n_seqs > 65535 || num_splits < 0) return HIPPO_ERR_BAD_SHAPE;
  const int G = d->n_q_heads / d->n_kv_heads;
  const long long rows = (long long)total_q * G;
  // (block and thread numbers of the launches, and a merge's wave for every row of q and query head)
  if (rows > (1 << 30) || (long long)total_q * d->n_q_heads > (1 << 30) || total_k > 0x7fffff00) return HIPPO_ERR_BAD_SHAPE;
  // (the lengths are on the device: taken as equal, each seeing what is there beside the others)
  const double len_q = std::max(1.0, (double)total_q / n_seqs), seen = std::max(len_q, paged ? (double)total_k : (double)total_k / n_seqs);
  cut_rows(pl, d->dtype, d->head_dim, len_q * G, std::min<double>(n_seqs, std::max(1, total_q)), seen, seen - len_q, total_k,
           false, d->n_kv_heads, (double)total_q * d->n_q_heads * d->head_dim * 4, num_splits);
  pl->deal = 0;
  auto tiles = [&](int block) { return rows / block + n_seqs; };
  if (!fit_rows(pl, d->dtype, d->head_dim, d->n_kv_heads, tiles)) return HIPPO_ERR_BAD_SHAPE;
  pl->n_tiles = (int)tiles(32 * pl->rb);
  carve_plan(pl, d->head_dim, total_q, d->n_q_heads);
  return HIPPO_OK;
}

// by_length: the sequences have lengths of their own
int plan_tree(const hippo_kv_desc* kv, int nodes, long long seq_len, bool by_length, int num_splits, RowsPlan* pl) {
  if (nodes < 1 || nodes > 64 || seq_len < nodes || seq_len > 0x7fffff00ll || num_splits < 0) return HIPPO_ERR_BAD_SHAPE;
  const int G = kv->n_q_heads / kv->n_kv_heads;
  if (G > 4096) return HIPPO_ERR_BAD_SHAPE;
  const long long tokens = (long long)kv->batch * nodes;
  cut_rows(pl, kv->dtype, kv->head_dim, G * nodes, kv->batch, (double)seq_len, (double)seq_len, (double)seq_len, true,
           kv->n_kv_heads, (double)tokens * kv->n_q_heads * kv->head_dim * 4, num_splits);
  if (tokens * kv->n_q_heads > (1 << 30)) return HIPPO_ERR_BAD_SHAPE;
  auto tiles = [&](int block) { return (long long)((G * nodes + block - 1) / block) * kv->batch; };
  if (!fit_rows(pl, kv->dtype, kv->head_dim, kv->n_kv_heads, tiles)) return HIPPO_ERR_BAD_SHAPE;
  pl->n_tiles = (int)tiles(32 * pl->rb);
  pl->deal = 0;
  if (pl->S > 1 && by_length && kv->batch > 1 && kv->batch <= 64) {
    pl->deal = pl->S * kv->batch;
    pl->S = std::min(2 * pl->S, kMaxRowSplits);
  }
  carve_plan(pl, kv->head_dim, tokens, kv->n_q_heads);
  if (pl->S == 1) pl->deal = 0;
  return HIPPO_OK;
}

// A pool as the kernels take it: every element of a page lies inside the page's stride, so that a clamped page number keeps every
// access inside the pool.  (The stride of a single page is nobody's.)
int check_pool(const hippo_paged_kv_desc* pd) {
  if (pd == nullptr) return HIPPO_ERR_NULL_ARG;
  if (pd->dtype != HIPPO_DTYPE_F32 && pd->dtype != HIPPO_DTYPE_BF16) return HIPPO_ERR_BAD_DTYPE;
  if (pd->n_kv_heads < 1 || pd->n_kv_heads > 65535 || (pd->head_dim != 64 && pd->head_dim != 128)) return HIPPO_ERR_BAD_SHAPE;
  if (pd->page_size < 16 || pd->page_size > 256 || (pd->page_size & (pd->page_size - 1))) return HIPPO_ERR_BAD_SHAPE;
  if (pd->n_pool_pages < 1 || pd->n_pool_pages > kPlanMost) return HIPPO_ERR_BAD_SHAPE;
  if (pd->stride_n < pd->head_dim || pd->stride_n > (1ll << 24) || pd->stride_h < 0) return HIPPO_ERR_BAD_SHAPE;
  if (pd->n_pool_pages > 1 &&
      (long long)(pd->page_size - 1) * pd->stride_n + (long long)(pd->n_kv_heads - 1) * pd->stride_h + pd->head_dim > pd->stride_page)
    return HIPPO_ERR_BAD_SHAPE;
  const int per16 = 16 / elem_bytes(pd->dtype);
  if (pd->stride_n % per16 || pd->stride_h % per16 || (pd->n_pool_pages > 1 && pd->stride_page % per16)) return HIPPO_ERR_BAD_ALIGN;
  return HIPPO_OK;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

void carve_rows(RowsParams* p, const RowsPlan& pl, void* workspace) {
  p->S = pl.S;
  p->n_tiles = pl.n_tiles;
  p->deal = pl.deal;
  p->tiles_per_seq = std::max(1, pl.n_tiles / p->n_seq);
  p->by_heads = divisor(p->Hkv); p->by_group = divisor(p->G); p->by_tiles = divisor(p->tiles_per_seq);
  p->part_o = static_cast<float*>(workspace);
  p->part_m = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.off_m);
  p->part_l = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.off_l);
}

float scale_or_default(float softmax_scale, int head_dim) {
  return (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim)) * kLog2e;
}

// ---- log probabilities: planning ------------------------------------------------------------------
struct LogprobPlan {
  int n_range, range_words;
  bool wide;
  size_t off_best, bytes;
};

int plan_logprobs(int rows, int vocab, int dtype, int n_top, LogprobPlan* pl) {
  if (dtype != HIPPO_DTYPE_F32 && dtype != HIPPO_DTYPE_BF16) return HIPPO_ERR_BAD_DTYPE;
  if (rows < 1 || rows > (1 << 22) || vocab < 1 || vocab > kLpMaxVocab || n_top < 0 || n_top > kLpMaxTop || n_top > vocab)
    return HIPPO_ERR_BAD_SHAPE;
  logprob_plan(rows, vocab, &pl->n_range, &pl->range_words, &pl->wide);
  const size_t ranges = pl->n_range > 1 ? (size_t)rows * pl->n_range : 0;
  pl->off_best = align_up(ranges * kLpStatBytes, 256);
  pl->bytes = std::max<size_t>(256, pl->off_best + align_up(ranges * n_top * sizeof(unsigned long long), 256));
  return HIPPO_OK;
}

}  // namespace

// ---- scratch for callers that cannot allocate -----------------------------------------------------
// One array per GPU, part of the loaded code object: it exists from the moment the library is loaded on
// a device until the process ends.  In host code the name `scratch` is only a handle for the runtime's
// symbol lookup, never an address a kernel could use; the per-device address comes from
// hipGetSymbolAddress and is what every launch receives.
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];

namespace {

constexpr int kMaxDevices = 64;
std::atomic<void*> g_scratch_ptr[kMaxDevices];   // zero-initialised: not looked up yet

// address of the current device's copy of the array (looked up once per device), or null with *status set
void* static_scratch(int* status) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) {
    *status = HIPPO_ERR_HIP;
    return nullptr;
  }
  void* ptr = g_scratch_ptr[dev].load(std::memory_order_acquire);
  if (ptr == nullptr) {
    if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)) != hipSuccess || ptr == nullptr) {
      *status = HIPPO_ERR_HIP;
      return nullptr;
    }
    g_scratch_ptr[dev].store(ptr, std::memory_order_release);   // every thread finds the same address
  }
  *status = HIPPO_OK;
  return ptr;
}

}  // namespace

extern "C" {

const char* hippo_status_string(int status) {
  switch (status) {
    case HIPPO_OK: return "ok";
    case HIPPO_ERR_NULL_ARG: return "a required pointer is NULL";
    case HIPPO_ERR_BAD_SHAPE: return "invalid size, count, stride or index range";
    case HIPPO_ERR_BAD_DTYPE: return "unsupported dtype";
    case HIPPO_ERR_BAD_ALIGN: return "pointer or stride is not 16-byte aligned (workspace: 256)";
    case HIPPO_ERR_WORKSPACE_TOO_SMALL: return "workspace smaller than hippo_workspace_bytes()";
    case HIPPO_ERR_HIP: return "HIP runtime error at kernel launch";
    case HIPPO_ERR_STATIC_SCRATCH_LIMIT:
      return "the call needs more scratch than the library's static array holds (hippo_static_scratch_bytes())";
    default: return "unknown status";
  }
}

size_t hippo_workspace_bytes(int32_t call, const hippo_kv_desc* kv, const hippo_video_desc* vid,
                             int32_t n_rows, int32_t seq_len, int32_t k, int32_t num_splits) {
  (void)k;
  if (check_kv(kv, call != HIPPO_CALL_SCORE_TOKENS) != HIPPO_OK) return 0;
  switch (call) {
    case HIPPO_CALL_SCORE_TOKENS: {
      ScorePlan pl;
      if (check_video(vid) != HIPPO_OK || plan_score(kv, vid, n_rows, 1, &pl) != HIPPO_OK) return 0;
      return pl.bytes;
    }
    case HIPPO_CALL_SELECT_GATHER_KV:
      return 256;   // the selection keeps its state in LDS; a token amount keeps the contract uniform
    case HIPPO_CALL_DRAFT_ATTENTION:
    case HIPPO_CALL_VERIFY_ATTENTION: {
      AttnPlan pl;
      if (plan_attention(call, kv, n_rows, seq_len, num_splits, &pl) != HIPPO_OK) return 0;
      return pl.bytes;
    }
    default:
      return 0;
  }
}

size_t hippo_score_layers_workspace_bytes(const hippo_kv_desc* kv, const hippo_video_desc* vid, int32_t l_txt,
                                          int32_t n_layers) {
  ScorePlan pl;
  if (check_kv(kv) != HIPPO_OK || check_video(vid) != HIPPO_OK || plan_score(kv, vid, l_txt, n_layers, &pl) != HIPPO_OK)
    return 0;
  return pl.bytes;
}

// polls: see ScoreOnce.  Not in hippo.h: it lets the tests end every wait at once, which a GPU to itself hardly ever does.
int hippo_score_tokens_layers_polls(int32_t n_layers, const void* const* q_txt_layers, int32_t l_txt,
                                    const void* const* k_cache_layers, int32_t emb_layer, const hippo_kv_desc* kv,
                                    int32_t seq_len, const hippo_video_desc* vid, const void* emb, int32_t emb_dim,
                                    int64_t emb_stride_tok, uint32_t flags, float* attn_mass_inout, float* scores_out,
                                    float* components_out, void* workspace, size_t workspace_bytes, void* stream,
                                    int32_t polls) {
  if (q_txt_layers == nullptr || k_cache_layers == nullptr || workspace == nullptr) return HIPPO_ERR_NULL_ARG;
  if (n_layers < 1 || n_layers > kMaxScoreLayers || emb_layer < 0 || emb_layer >= n_layers) return HIPPO_ERR_BAD_SHAPE;
  for (int l = 0; l < n_layers; ++l)
    if (q_txt_layers[l] == nullptr || k_cache_layers[l] == nullptr) return HIPPO_ERR_NULL_ARG;
  int rc = check_kv(kv);
  if (rc != HIPPO_OK) return rc;
  if ((rc = check_video(vid)) != HIPPO_OK) return rc;
  if ((rc = check_crop(vid)) != HIPPO_OK) return rc;
  const bool acc_only = (flags & HIPPO_SCORE_ACCUMULATE_ONLY) != 0;
  if (flags & ~(HIPPO_SCORE_ALL | HIPPO_SCORE_ACCUMULATE_ONLY)) return HIPPO_ERR_BAD_SHAPE;
  if (!acc_only && (flags & HIPPO_SCORE_ALL) == 0) return HIPPO_ERR_BAD_SHAPE;
  if (acc_only && attn_mass_inout == nullptr) return HIPPO_ERR_NULL_ARG;
  if (!acc_only && scores_out == nullptr) return HIPPO_ERR_NULL_ARG;
  const long long Nv = (long long)vid->n_frames * vid->grid_h * vid->grid_w;
  if (seq_len < 1 || (long long)vid->vis_offset + Nv > seq_len) return HIPPO_ERR_BAD_SHAPE;
  const int per16 = 16 / elem_bytes(kv->dtype);
  if (emb != nullptr) {
    if (emb_dim < 1 || emb_stride_tok < emb_dim) return HIPPO_ERR_BAD_SHAPE;
    if (emb_dim % per16) return HIPPO_ERR_BAD_SHAPE;
    if (emb_stride_tok % per16 || !aligned16(emb)) return HIPPO_ERR_BAD_ALIGN;
  }
  for (int l = 0; l < n_layers; ++l)
    if (!aligned16(q_txt_layers[l]) || !aligned16(k_cache_layers[l])) return HIPPO_ERR_BAD_ALIGN;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return HIPPO_ERR_BAD_ALIGN;
  ScorePlan pl;
  if ((rc = plan_score(kv, vid, l_txt, n_layers, &pl)) != HIPPO_OK) return rc;
  // A short video's finer cut can need more than a longer one's: a workspace sized for that one serves without it.
  if (workspace_bytes < pl.bytes && (rc = plan_score(kv, vid, l_txt, n_layers, &pl, false)) != HIPPO_OK) return rc;
  if (workspace_bytes < pl.bytes) return HIPPO_ERR_WORKSPACE_TOO_SMALL;

  ScoreParams p;
  p.q_txt = q_txt_layers[0]; p.k_cache = k_cache_layers[emb_layer]; p.emb = emb;
  p.n_layers = n_layers; p.Bz = kv->batch * n_layers;
  for (int l = 0; l < kMaxScoreLayers; ++l) {
    p.q_layers[l] = l < n_layers ? q_txt_layers[l] : nullptr;
    p.k_layers[l] = l < n_layers ? k_cache_layers[l] : nullptr;
  }
  p.B = kv->batch; p.L = l_txt; p.H = kv->n_q_heads; p.Hkv = kv->n_kv_heads;
  p.G = kv->n_q_heads / kv->n_kv_heads; p.D = kv->head_dim; p.dtype = kv->dtype;
  p.sb = kv->stride_b; p.sh = kv->stride_h; p.sn = kv->stride_n;
  p.F = vid->n_frames; p.gh = vid->grid_h; p.gw = vid->grid_w; p.P = vid->grid_h * vid->grid_w;
  p.Nv = (int)Nv; p.vis_off = vid->vis_offset; p.ch = vid->crop_h; p.cw = vid->crop_w;
  p.emb_dim = emb_dim; p.emb_stride_tok = emb_stride_tok; p.emb_stride_b = Nv * emb_stride_tok;
  p.flags = flags;
  p.attn_mass_inout = attn_mass_inout; p.scores_out = scores_out; p.components_out = components_out;
  char* ws = static_cast<char*>(workspace);
  p.row_m = reinterpret_cast<float*>(ws);
  p.row_l = reinterpret_cast<float*>(ws + pl.off_row_l);
  p.row_lse = reinterpret_cast<float*>(ws + pl.off_row_lse);
  p.col_part = reinterpret_cast<float*>(ws + pl.off_col);
  p.s_attn = reinterpret_cast<float*>(ws + pl.off_sa);
  p.s_temp = reinterpret_cast<float*>(ws + pl.off_st);
  p.s_spa = reinterpret_cast<float*>(ws + pl.off_ss);
  p.n_tile = pl.n_tile;
  p.n_rsplit = pl.n_rsplit;
  ScoreOnce once{};
  once.polls = polls;
  if (pl.once) {
    once.row_word = reinterpret_cast<unsigned long long*>(ws + pl.off_word);
    once.row_bin = reinterpret_cast<unsigned long long*>(ws + pl.off_bin);
    once.run_flags = reinterpret_cast<unsigned*>(ws + pl.off_flags);
    once.run_arrived = reinterpret_cast<int*>(ws + pl.off_arrived);
    once.tile_redo = reinterpret_cast<int*>(ws + pl.off_redo);
    once.clear_bytes = pl.clear_bytes;
  }
  const hipError_t e = launch_score(p, once, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

int hippo_score_tokens_layers(int32_t n_layers, const void* const* q_txt_layers, int32_t l_txt,
                              const void* const* k_cache_layers, int32_t emb_layer, const hippo_kv_desc* kv,
                              int32_t seq_len, const hippo_video_desc* vid, const void* emb, int32_t emb_dim,
                              int64_t emb_stride_tok, uint32_t flags, float* attn_mass_inout, float* scores_out,
                              float* components_out, void* workspace, size_t workspace_bytes, void* stream) {
  return hippo_score_tokens_layers_polls(n_layers, q_txt_layers, l_txt, k_cache_layers, emb_layer, kv, seq_len, vid, emb,
                                         emb_dim, emb_stride_tok, flags, attn_mass_inout, scores_out, components_out,
                                         workspace, workspace_bytes, stream, -1);
}

int hippo_score_tokens(const void* q_txt, int32_t l_txt, const void* k_cache, const hippo_kv_desc* kv,
                       int32_t seq_len, const hippo_video_desc* vid, const void* emb, int32_t emb_dim,
                       int64_t emb_stride_tok, uint32_t flags, float* attn_mass_inout, float* scores_out,
                       float* components_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (q_txt == nullptr || k_cache == nullptr) return HIPPO_ERR_NULL_ARG;
  const void* qs[1] = {q_txt};
  const void* ks[1] = {k_cache};
  return hippo_score_tokens_layers(1, qs, l_txt, ks, 0, kv, seq_len, vid, emb, emb_dim, emb_stride_tok, flags,
                                   attn_mass_inout, scores_out, components_out, workspace, workspace_bytes, stream);
}

int hippo_select_gather_kv(const float* scores, int32_t k, const void* k_src, const void* v_src,
                           const hippo_kv_desc* src, int32_t src_len, const hippo_video_desc* vid,
                           void* k_dst, void* v_dst, const hippo_kv_desc* dst, int32_t* idx_out,
                           void* workspace, size_t workspace_bytes, void* stream) {
  if (scores == nullptr || idx_out == nullptr || workspace == nullptr) return HIPPO_ERR_NULL_ARG;
  int rc = check_video(vid);
  if (rc != HIPPO_OK) return rc;
  const long long Nv = (long long)vid->n_frames * vid->grid_h * vid->grid_w;
  if (k < 1 || k > Nv) return HIPPO_ERR_BAD_SHAPE;
  const bool do_gather = (k_dst != nullptr) || (v_dst != nullptr);
  if (do_gather && (k_dst == nullptr || v_dst == nullptr || k_src == nullptr || v_src == nullptr))
    return HIPPO_ERR_NULL_ARG;
  if (src == nullptr) return HIPPO_ERR_NULL_ARG;
  if ((rc = check_kv(src, true)) != HIPPO_OK) return rc;
  if (workspace_bytes < 256) return HIPPO_ERR_WORKSPACE_TOO_SMALL;
  SelectParams p;
  p.scores = scores; p.B = src->batch; p.Nv = (int)Nv; p.k = k; p.idx_out = idx_out;
  p.k_src = k_src; p.v_src = v_src; p.k_dst = nullptr; p.v_dst = nullptr;
  p.Hkv = src->n_kv_heads; p.D = src->head_dim; p.elem_bytes = elem_bytes(src->dtype);
  p.ssb = src->stride_b; p.ssh = src->stride_h; p.ssn = src->stride_n;
  p.dsb = p.dsh = p.dsn = 0;
  p.src_len = src_len; p.dst_len = 0; p.vis_off = vid->vis_offset;
  if (do_gather) {
    if (dst == nullptr) return HIPPO_ERR_NULL_ARG;
    if ((rc = check_kv(dst, true)) != HIPPO_OK) return rc;
    if (dst->batch != src->batch || dst->n_kv_heads != src->n_kv_heads || dst->head_dim != src->head_dim ||
        dst->dtype != src->dtype)
      return HIPPO_ERR_BAD_SHAPE;
    if (src_len < 1 || (long long)vid->vis_offset + Nv > src_len) return HIPPO_ERR_BAD_SHAPE;
    if (!aligned16(k_src) || !aligned16(v_src) || !aligned16(k_dst) || !aligned16(v_dst))
      return HIPPO_ERR_BAD_ALIGN;
    p.k_dst = k_dst; p.v_dst = v_dst;
    p.dsb = dst->stride_b; p.dsh = dst->stride_h; p.dsn = dst->stride_n;
    p.dst_len = (int)(src_len - Nv + k);
  }
  const hipError_t e = launch_select_gather(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

size_t hippo_evict_kv_workspace_bytes(const hippo_kv_desc* src, int32_t src_len, int32_t keep) {
  if (check_kv(src, true) != HIPPO_OK || src_len < 1 || src_len > (1 << 30) || keep < 1 || keep > src_len) return 0;
  return 256;   // the selection keeps its state in LDS; a token amount keeps the contract uniform
}

int hippo_evict_kv(const float* mass, int64_t mass_stride_b, int64_t mass_stride_h, int32_t keep, int32_t n_first,
                   int32_t n_recent, const void* k_src, const void* v_src, const hippo_kv_desc* src, int32_t src_len,
                   void* k_dst, void* v_dst, const hippo_kv_desc* dst, float* mass_dst, int64_t mass_dst_stride_b,
                   int64_t mass_dst_stride_h, int32_t* idx_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (mass == nullptr || idx_out == nullptr || workspace == nullptr || src == nullptr) return HIPPO_ERR_NULL_ARG;
  int rc = check_kv(src, true);
  if (rc != HIPPO_OK) return rc;
  if (src_len < 1 || src_len > (1 << 30) || n_first < 0 || n_recent < 0 || keep < 1 || keep > src_len) return HIPPO_ERR_BAD_SHAPE;
  if ((long long)n_first + n_recent > keep) return HIPPO_ERR_BAD_SHAPE;
  if (mass_stride_b < 0 || mass_stride_h < 0) return HIPPO_ERR_BAD_SHAPE;
  if ((reinterpret_cast<uintptr_t>(mass) & 3u) || (reinterpret_cast<uintptr_t>(idx_out) & 3u) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return HIPPO_ERR_BAD_ALIGN;
  EvictParams p;
  p.mass = mass; p.mass_sb = mass_stride_b; p.mass_sh = mass_stride_h;
  p.n_src = src_len; p.n_first = n_first; p.n_between = src_len - n_first - n_recent;
  p.k = keep - n_first - n_recent; p.keep = keep;
  p.idx_out = idx_out;
  p.k_src = k_src; p.v_src = v_src; p.k_dst = nullptr; p.v_dst = nullptr;
  p.mass_dst = mass_dst; p.mass_dsb = mass_dst_stride_b; p.mass_dsh = mass_dst_stride_h;
  p.B = src->batch; p.Hkv = src->n_kv_heads; p.D = src->head_dim; p.elem_bytes = elem_bytes(src->dtype);
  p.ssb = src->stride_b; p.ssh = src->stride_h; p.ssn = src->stride_n;
  p.dsb = p.dsh = p.dsn = 0;
  // every (batch element, KV head) writes rows of its own: those of different heads must not meet
  if (mass_dst != nullptr) {
    if (mass_dst == mass) return HIPPO_ERR_BAD_SHAPE;
    if (reinterpret_cast<uintptr_t>(mass_dst) & 3u) return HIPPO_ERR_BAD_ALIGN;
    if (rows_meet({p.B, mass_dst_stride_b}, {p.Hkv, mass_dst_stride_h}, {1, 0}, keep)) return HIPPO_ERR_BAD_SHAPE;
  }
  if (k_dst != nullptr || v_dst != nullptr) {
    if (k_dst == nullptr || v_dst == nullptr || k_src == nullptr || v_src == nullptr || dst == nullptr) return HIPPO_ERR_NULL_ARG;
    if ((rc = check_kv(dst, true)) != HIPPO_OK) return rc;
    if (dst->batch != src->batch || dst->n_kv_heads != src->n_kv_heads || dst->head_dim != src->head_dim ||
        dst->dtype != src->dtype || k_dst == k_src || v_dst == v_src || k_dst == v_src || v_dst == k_src || k_dst == v_dst)
      return HIPPO_ERR_BAD_SHAPE;
    if (!aligned16(k_src) || !aligned16(v_src) || !aligned16(k_dst) || !aligned16(v_dst)) return HIPPO_ERR_BAD_ALIGN;
    if (rows_meet({p.B, dst->stride_b}, {p.Hkv, dst->stride_h}, {keep, dst->stride_n}, p.D)) return HIPPO_ERR_BAD_SHAPE;
    p.k_dst = k_dst; p.v_dst = v_dst;
    p.dsb = dst->stride_b; p.dsh = dst->stride_h; p.dsn = dst->stride_n;
  }
  if (workspace_bytes < 256) return HIPPO_ERR_WORKSPACE_TOO_SMALL;
  const hipError_t e = launch_evict(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

int hippo_verify_attention(const void* q, int32_t q_len, const void* k_cache, const void* v_cache,
                           const hippo_kv_desc* kv, int32_t ctx_len, float softmax_scale, int32_t num_splits,
                           void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  return attention_entry(HIPPO_CALL_VERIFY_ATTENTION, q, q_len, k_cache, v_cache, kv, ctx_len, softmax_scale,
                         num_splits, out, lse_out, workspace, workspace_bytes, stream);
}

int hippo_draft_attention(const void* q, int32_t q_len, const void* k_cache, const void* v_cache,
                          const hippo_kv_desc* kv, int32_t ctx_len, float softmax_scale, int32_t num_splits,
                          void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  return attention_entry(HIPPO_CALL_DRAFT_ATTENTION, q, q_len, k_cache, v_cache, kv, ctx_len, softmax_scale,
                         num_splits, out, lse_out, workspace, workspace_bytes, stream);
}

size_t hippo_static_scratch_bytes(void) { return kStaticScratchBytes; }

int hippo_static_scratch_init(void) {
  int rc = HIPPO_OK;
  static_scratch(&rc);
  return rc;
}

int hippo_verify_attention_static(const void* q, int32_t q_len, const void* k_cache, const void* v_cache,
                                  const hippo_kv_desc* kv, int32_t ctx_len, float softmax_scale,
                                  int32_t num_splits, void* out, float* lse_out, void* stream) {
  // every argument check that needs no device comes before the scratch lookup; the size check uses the
  // same plan as the launch
  if (q == nullptr || k_cache == nullptr || v_cache == nullptr || out == nullptr) return HIPPO_ERR_NULL_ARG;
  int rc = check_kv(kv);
  if (rc != HIPPO_OK) return rc;
  if (ctx_len < 0 || q_len < 1 || (long long)ctx_len + q_len > 0x7fffff00ll) return HIPPO_ERR_BAD_SHAPE;
  AttnPlan pl;
  if ((rc = plan_attention(HIPPO_CALL_VERIFY_ATTENTION, kv, q_len, ctx_len + q_len, num_splits, &pl)) != HIPPO_OK)
    return rc;
  if (pl.bytes > kStaticScratchBytes) return HIPPO_ERR_STATIC_SCRATCH_LIMIT;
  void* ws = static_scratch(&rc);
  if (ws == nullptr) return rc;
  // the split partials are written in full before the merge reads them: nothing has to start at zero
  return attention_entry(HIPPO_CALL_VERIFY_ATTENTION, q, q_len, k_cache, v_cache, kv, ctx_len, softmax_scale,
                         num_splits, out, lse_out, ws, kStaticScratchBytes, stream);
}

size_t hippo_spec_verify_workspace_bytes(int32_t batch, int32_t gamma, int32_t vocab, int32_t dtype) {
  SpecPlan pl;
  return plan_spec(batch, gamma, vocab, dtype, &pl) == HIPPO_OK ? pl.bytes : 0;
}

int hippo_spec_verify(const void* p_logits, const void* q_logits, int32_t dtype, int64_t p_stride_row,
                      int64_t q_stride_row, const int32_t* draft_tokens, const float* u_accept,
                      const float* u_sample, int32_t batch, int32_t gamma, int32_t vocab, float temperature,
                      int32_t* n_accept_out, int32_t* next_token_out, float* alpha_out, void* workspace,
                      size_t workspace_bytes, void* stream) {
  SpecPlan pl;
  int rc = plan_spec(batch, gamma, vocab, dtype, &pl);
  if (rc != HIPPO_OK) return rc;
  if (!(temperature >= 0.f) || isinf(temperature)) return HIPPO_ERR_BAD_SHAPE;
  const bool greedy = temperature == 0.f;
  if (p_logits == nullptr || n_accept_out == nullptr || next_token_out == nullptr || workspace == nullptr)
    return HIPPO_ERR_NULL_ARG;
  if (gamma > 0 && (draft_tokens == nullptr || (!greedy && (q_logits == nullptr || u_accept == nullptr))))
    return HIPPO_ERR_NULL_ARG;
  if (!greedy && u_sample == nullptr) return HIPPO_ERR_NULL_ARG;
  if (p_stride_row < vocab || (gamma > 0 && !greedy && q_stride_row < vocab)) return HIPPO_ERR_BAD_SHAPE;
  const int per16 = 16 / elem_bytes(dtype);
  if (p_stride_row % per16 || !aligned16(p_logits) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return HIPPO_ERR_BAD_ALIGN;
  if (gamma > 0 && !greedy && (q_stride_row % per16 || !aligned16(q_logits))) return HIPPO_ERR_BAD_ALIGN;
  if (workspace_bytes < pl.bytes) return HIPPO_ERR_WORKSPACE_TOO_SMALL;

  SpecParams p;
  p.p_logits = p_logits; p.q_logits = q_logits; p.tokens = draft_tokens;
  p.u_accept = u_accept; p.u_sample = u_sample;
  p.B = batch; p.gamma = gamma; p.V = vocab; p.n_rows = pl.n_rows; p.n_seg = pl.n_seg;
  p.p_stride = p_stride_row; p.q_stride = q_stride_row;
  p.c = greedy ? 0.f : kLog2e / temperature;
  p.inv_temperature = greedy ? 0.0 : 1.0 / (double)temperature;
  p.n_accept = n_accept_out; p.next_token = next_token_out; p.alpha_out = alpha_out;
  char* ws = static_cast<char*>(workspace);
  p.stats = reinterpret_cast<SegStat*>(ws);
  p.cells = reinterpret_cast<float*>(ws + pl.off_cells);
  p.arrived = reinterpret_cast<int*>(ws + pl.off_arrived);
  const hipError_t e = launch_spec_verify(p, dtype, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

size_t hippo_token_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t dtype, int32_t n_top) {
  LogprobPlan pl;
  return plan_logprobs(rows, vocab, dtype, n_top, &pl) == HIPPO_OK ? pl.bytes : 0;
}

int hippo_token_logprobs(const void* logits, int32_t dtype, int64_t stride_row, const int32_t* tokens, int32_t rows,
                         int32_t vocab, float temperature, int32_t n_top, float* logprob_out, float* entropy_out,
                         int32_t* top_ids_out, float* top_logprobs_out, void* workspace, size_t workspace_bytes, void* stream) {
  LogprobPlan pl;
  const int rc = plan_logprobs(rows, vocab, dtype, n_top, &pl);
  if (rc != HIPPO_OK) return rc;
  if (!(temperature > 0.f) || isinf(temperature) || isinf(kLog2e / temperature)) return HIPPO_ERR_BAD_SHAPE;
  if (logits == nullptr || tokens == nullptr || logprob_out == nullptr || entropy_out == nullptr || workspace == nullptr)
    return HIPPO_ERR_NULL_ARG;
  if (n_top > 0 && (top_ids_out == nullptr || top_logprobs_out == nullptr)) return HIPPO_ERR_NULL_ARG;
  if (stride_row < vocab) return HIPPO_ERR_BAD_SHAPE;
  if (stride_row % (16 / elem_bytes(dtype)) || !aligned16(logits) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return HIPPO_ERR_BAD_ALIGN;
  for (const void* p : {(const void*)tokens, (const void*)logprob_out, (const void*)entropy_out, (const void*)top_ids_out,
                        (const void*)top_logprobs_out})
    if (reinterpret_cast<uintptr_t>(p) & 3u) return HIPPO_ERR_BAD_ALIGN;
  if (workspace_bytes < pl.bytes) return HIPPO_ERR_WORKSPACE_TOO_SMALL;

  LogprobParams p;
  p.logits = logits; p.stride = stride_row; p.tokens = tokens; p.R = rows; p.V = vocab; p.n_top = n_top;
  p.n_range = pl.n_range; p.range_words = pl.range_words; p.wide = pl.wide;
  p.c = kLog2e / temperature; p.inv_t = 1.0f / temperature;
  p.logprob = logprob_out; p.entropy = entropy_out; p.top_ids = top_ids_out; p.top_logprobs = top_logprobs_out;
  p.stats = workspace;
  p.best = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + pl.off_best);
  const hipError_t e = launch_logprobs(p, dtype, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

int hippo_verify_attention_append(const void* q, int32_t q_len, const void* k_new, const void* v_new,
                                  void* k_cache, void* v_cache, const hippo_kv_desc* kv, int32_t ctx_len,
                                  float softmax_scale, int32_t num_splits, void* out, float* lse_out,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  if (k_new == nullptr || v_new == nullptr) return HIPPO_ERR_NULL_ARG;
  AttnExtra ex;
  ex.append = true; ex.k_new = k_new; ex.v_new = v_new;
  return attention_entry(HIPPO_CALL_VERIFY_ATTENTION, q, q_len, k_cache, v_cache, kv, ctx_len, softmax_scale,
                         num_splits, out, lse_out, workspace, workspace_bytes, stream, ex);
}

int hippo_draft_attention_append(const void* q, int32_t q_len, const void* k_new, const void* v_new,
                                 void* k_cache, void* v_cache, const hippo_kv_desc* kv, int32_t ctx_len,
                                 float softmax_scale, int32_t num_splits, void* out, float* lse_out,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (k_new == nullptr || v_new == nullptr) return HIPPO_ERR_NULL_ARG;
  AttnExtra ex;
  ex.append = true; ex.k_new = k_new; ex.v_new = v_new;
  return attention_entry(HIPPO_CALL_DRAFT_ATTENTION, q, q_len, k_cache, v_cache, kv, ctx_len, softmax_scale,
                         num_splits, out, lse_out, workspace, workspace_bytes, stream, ex);
}

static int mass_entry(int call, const void* q, int32_t q_len, const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                      const hippo_kv_desc* kv, int32_t ctx_len, float softmax_scale, int32_t num_splits, void* out, float* lse_out,
                      const hippo_mass_desc* mass, void* workspace, size_t workspace_bytes, void* stream) {
  if (kv == nullptr || mass == nullptr || mass->out == nullptr) return HIPPO_ERR_NULL_ARG;
  if ((k_new == nullptr) != (v_new == nullptr)) return HIPPO_ERR_NULL_ARG;
  const int rc = check_kv(kv);
  if (rc != HIPPO_OK) return rc;
  if (mass->in != nullptr && (mass->in_stride_b < 0 || mass->in_stride_h < 0)) return HIPPO_ERR_BAD_SHAPE;
  // every (batch element, KV head) writes a row of its own
  if (rows_meet({kv->batch, mass->out_stride_b}, {kv->n_kv_heads, mass->out_stride_h}, {1, 0}, (long long)ctx_len + q_len))
    return HIPPO_ERR_BAD_SHAPE;
  // in place: where it stood
  if (mass->in == mass->out && ((kv->n_kv_heads > 1 && mass->in_stride_h != mass->out_stride_h) ||
                                (kv->batch > 1 && mass->in_stride_b != mass->out_stride_b)))
    return HIPPO_ERR_BAD_SHAPE;
  if ((reinterpret_cast<uintptr_t>(mass->in) & 3u) || (reinterpret_cast<uintptr_t>(mass->out) & 3u)) return HIPPO_ERR_BAD_ALIGN;
  AttnExtra ex;
  ex.append = k_new != nullptr; ex.k_new = k_new; ex.v_new = v_new;
  ex.mass = true; ex.mass_in = mass->in; ex.mass_out = mass->out;
  ex.mass_isb = mass->in_stride_b; ex.mass_ish = mass->in_stride_h;
  ex.mass_osb = mass->out_stride_b; ex.mass_osh = mass->out_stride_h;
  return attention_entry(call, q, q_len, k_cache, v_cache, kv, ctx_len, softmax_scale, num_splits, out, lse_out, workspace,
                         workspace_bytes, stream, ex);
}

size_t hippo_attention_mass_workspace_bytes(const hippo_kv_desc* kv, int32_t q_len, int32_t seq_len, int32_t num_splits) {
  MassPlan pl;
  if (check_kv(kv) != HIPPO_OK || plan_mass(HIPPO_CALL_VERIFY_ATTENTION, kv, q_len, seq_len, num_splits, &pl) != HIPPO_OK) return 0;
  return pl.bytes;
}

int hippo_verify_attention_mass(const void* q, int32_t q_len, const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                                const hippo_kv_desc* kv, int32_t ctx_len, float softmax_scale, int32_t num_splits, void* out,
                                float* lse_out, const hippo_mass_desc* mass, void* workspace, size_t workspace_bytes,
                                void* stream) {
  return mass_entry(HIPPO_CALL_VERIFY_ATTENTION, q, q_len, k_new, v_new, k_cache, v_cache, kv, ctx_len, softmax_scale, num_splits,
                    out, lse_out, mass, workspace, workspace_bytes, stream);
}

int hippo_draft_attention_mass(const void* q, int32_t q_len, const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                               const hippo_kv_desc* kv, int32_t ctx_len, float softmax_scale, int32_t num_splits, void* out,
                               float* lse_out, const hippo_mass_desc* mass, void* workspace, size_t workspace_bytes,
                               void* stream) {
  return mass_entry(HIPPO_CALL_DRAFT_ATTENTION, q, q_len, k_new, v_new, k_cache, v_cache, kv, ctx_len, softmax_scale, num_splits,
                    out, lse_out, mass, workspace, workspace_bytes, stream);
}

// paged caches: translate the pool descriptor into the per-row strides the kernels use
static int paged_entry(int call, const void* q, int32_t q_len, const void* k_pool, const void* v_pool,
                       const int32_t* block_table, const hippo_paged_kv_desc* pd, int32_t ctx_len,
                       float softmax_scale, int32_t num_splits, void* out, float* lse_out, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (pd == nullptr || block_table == nullptr) return HIPPO_ERR_NULL_ARG;
  if (pd->page_size < 16 || pd->page_size > 256 || (pd->page_size & (pd->page_size - 1))) return HIPPO_ERR_BAD_SHAPE;
  if (pd->n_pool_pages < 1 || pd->max_pages < 1 || ctx_len < 0 || q_len < 1) return HIPPO_ERR_BAD_SHAPE;
  if (((long long)ctx_len + q_len + pd->page_size - 1) / pd->page_size > pd->max_pages) return HIPPO_ERR_BAD_SHAPE;
  if (pd->n_kv_heads < 1 || pd->head_dim < 1 || pd->stride_n < pd->head_dim || pd->stride_h < 0)
    return HIPPO_ERR_BAD_SHAPE;
  // every element of a page lies inside the page's stride, so a clamped page number keeps every
  // access inside the pool
  if ((long long)(pd->page_size - 1) * pd->stride_n + (long long)(pd->n_kv_heads - 1) * pd->stride_h + pd->head_dim >
      pd->stride_page)
    return HIPPO_ERR_BAD_SHAPE;
  if (reinterpret_cast<uintptr_t>(block_table) & 3u) return HIPPO_ERR_BAD_ALIGN;
  hippo_kv_desc kv;
  kv.batch = pd->batch; kv.n_q_heads = pd->n_q_heads; kv.n_kv_heads = pd->n_kv_heads;
  kv.head_dim = pd->head_dim; kv.dtype = pd->dtype;
  kv.stride_b = 0; kv.stride_h = pd->stride_h; kv.stride_n = pd->stride_n;
  const int per16 = 16 / (pd->dtype == HIPPO_DTYPE_BF16 ? 2 : 4);
  if (pd->stride_page % per16) return HIPPO_ERR_BAD_ALIGN;
  AttnExtra ex;
  ex.block_table = block_table; ex.page_size = pd->page_size; ex.max_pages = pd->max_pages;
  ex.n_pool_pages = pd->n_pool_pages; ex.page_stride = pd->stride_page;
  return attention_entry(call, q, q_len, k_pool, v_pool, &kv, ctx_len, softmax_scale, num_splits, out, lse_out,
                         workspace, workspace_bytes, stream, ex);
}

int hippo_verify_attention_paged(const void* q, int32_t q_len, const void* k_pool, const void* v_pool,
                                 const int32_t* block_table, const hippo_paged_kv_desc* kv, int32_t ctx_len,
                                 float softmax_scale, int32_t num_splits, void* out, float* lse_out,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  return paged_entry(HIPPO_CALL_VERIFY_ATTENTION, q, q_len, k_pool, v_pool, block_table, kv, ctx_len,
                     softmax_scale, num_splits, out, lse_out, workspace, workspace_bytes, stream);
}

int hippo_draft_attention_paged(const void* q, int32_t q_len, const void* k_pool, const void* v_pool,
                                const int32_t* block_table, const hippo_paged_kv_desc* kv, int32_t ctx_len,
                                float softmax_scale, int32_t num_splits, void* out, float* lse_out,
                                void* workspace, size_t workspace_bytes, void* stream) {
  return paged_entry(HIPPO_CALL_DRAFT_ATTENTION, q, q_len, k_pool, v_pool, block_table, kv, ctx_len,
                     softmax_scale, num_splits, out, lse_out, workspace, workspace_bytes, stream);
}

int hippo_verify_attention_fp8kv(const void* q, int32_t q_len, const void* k_codes, const void* v_codes,
                                 const float* k_scale, const float* v_scale, const hippo_kv_desc* kv,
                                 int32_t ctx_len, float softmax_scale, int32_t num_splits, void* out,
                                 float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  AttnExtra ex;
  ex.fp8 = true; ex.k_scale = k_scale; ex.v_scale = v_scale;
  return attention_entry(HIPPO_CALL_VERIFY_ATTENTION, q, q_len, k_codes, v_codes, kv, ctx_len, softmax_scale,
                         num_splits, out, lse_out, workspace, workspace_bytes, stream, ex);
}

int hippo_draft_attention_fp8kv(const void* q, int32_t q_len, const void* k_codes, const void* v_codes,
                                const float* k_scale, const float* v_scale, const hippo_kv_desc* kv,
                                int32_t ctx_len, float softmax_scale, int32_t num_splits, void* out,
                                float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  AttnExtra ex;
  ex.fp8 = true; ex.k_scale = k_scale; ex.v_scale = v_scale;
  return attention_entry(HIPPO_CALL_DRAFT_ATTENTION, q, q_len, k_codes, v_codes, kv, ctx_len, softmax_scale,
                         num_splits, out, lse_out, workspace, workspace_bytes, stream, ex);
}

size_t hippo_quantize_kv_workspace_bytes(const hippo_kv_desc* src, int32_t n_rows) {
  if (check_kv(src) != HIPPO_OK || n_rows < 1) return 0;
  return align_up((size_t)src->batch * src->n_kv_heads * 2 * align_up(quant_slices(n_rows, src->head_dim), 4) * sizeof(float), 256);
}

// polls: see QuantParams.  Not in hippo.h: it lets the tests end every wait at once.
int hippo_quantize_kv_e4m3_polls(const void* k_src, const void* v_src, const hippo_kv_desc* src, int32_t n_rows,
                                 void* k_codes, void* v_codes, const hippo_kv_desc* dst, float* k_scale, float* v_scale,
                                 void* workspace, size_t workspace_bytes, void* stream, int32_t polls) {
  if (k_src == nullptr || v_src == nullptr || k_codes == nullptr || v_codes == nullptr || k_scale == nullptr ||
      v_scale == nullptr || workspace == nullptr)
    return HIPPO_ERR_NULL_ARG;
  int rc = check_kv(src);
  if (rc != HIPPO_OK) return rc;
  if ((rc = check_kv(dst, true)) != HIPPO_OK) return rc;
  if (dst->dtype != HIPPO_DTYPE_FP8_E4M3) return HIPPO_ERR_BAD_DTYPE;
  if (dst->batch != src->batch || dst->n_kv_heads != src->n_kv_heads || dst->head_dim != src->head_dim || n_rows < 1)
    return HIPPO_ERR_BAD_SHAPE;
  if (2 * (long long)src->n_kv_heads > 65535) return HIPPO_ERR_BAD_SHAPE;   // (KV head, K or V) is grid y
  if (!aligned16(k_src) || !aligned16(v_src) || !aligned16(k_codes) || !aligned16(v_codes) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u) || (reinterpret_cast<uintptr_t>(k_scale) & 3u) ||
      (reinterpret_cast<uintptr_t>(v_scale) & 3u))
    return HIPPO_ERR_BAD_ALIGN;
  if (workspace_bytes < hippo_quantize_kv_workspace_bytes(src, n_rows)) return HIPPO_ERR_WORKSPACE_TOO_SMALL;
  QuantParams p;
  p.k_src = k_src; p.v_src = v_src; p.k_dst = k_codes; p.v_dst = v_codes; p.k_scale = k_scale; p.v_scale = v_scale;
  p.partial = reinterpret_cast<float*>(workspace);
  p.B = src->batch; p.Hkv = src->n_kv_heads; p.D = src->head_dim; p.n_rows = n_rows;
  p.n_slices = quant_slices(n_rows, src->head_dim); p.src_dtype = src->dtype;
  p.ssb = src->stride_b; p.ssh = src->stride_h; p.ssn = src->stride_n;
  p.dsb = dst->stride_b; p.dsh = dst->stride_h; p.dsn = dst->stride_n;
  p.polls = polls;
  const hipError_t e = launch_quantize(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

int hippo_quantize_kv_e4m3(const void* k_src, const void* v_src, const hippo_kv_desc* src, int32_t n_rows,
                           void* k_codes, void* v_codes, const hippo_kv_desc* dst, float* k_scale, float* v_scale,
                           void* workspace, size_t workspace_bytes, void* stream) {
  return hippo_quantize_kv_e4m3_polls(k_src, v_src, src, n_rows, k_codes, v_codes, dst, k_scale, v_scale, workspace,
                                      workspace_bytes, stream, -1);
}

size_t hippo_prefill_workspace_bytes(const hippo_packed_desc* desc, int32_t total_q, int32_t total_k, int32_t n_seqs,
                                     int32_t paged, int32_t num_splits) {
  RowsPlan pl;
  if (check_packed(desc) != HIPPO_OK || plan_prefill(desc, paged != 0, total_q, total_k, n_seqs, num_splits, &pl) != HIPPO_OK) return 0;
  return pl.bytes;
}

// pd null: packed K and V
static int prefill_entry(const void* q, int32_t total_q, const void* k, const void* v, int32_t total_k, const hippo_packed_desc* desc,
                         const hippo_paged_kv_desc* pd, const int32_t* block_table, const int32_t* cu_q, const int32_t* cu_k,
                         int32_t n_seqs, float softmax_scale, int32_t num_splits, void* out, float* lse_out, void* workspace,
                         size_t workspace_bytes, void* stream) {
  int rc = check_packed(desc);
  if (rc != HIPPO_OK) return rc;
  RowsPlan pl;
  rc = plan_prefill(desc, pd != nullptr, total_q, total_k, n_seqs, num_splits, &pl);
  if (rc != HIPPO_OK) return rc;
  if (total_q == 0) return HIPPO_OK;                          // no rows
  if (q == nullptr || cu_q == nullptr || cu_k == nullptr || out == nullptr || workspace == nullptr) return HIPPO_ERR_NULL_ARG;
  if ((k == nullptr || v == nullptr) && total_k > 0) return HIPPO_ERR_NULL_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || (reinterpret_cast<uintptr_t>(workspace) & 255u) ||
      !aligned4(cu_q) || !aligned4(cu_k) || !aligned4(lse_out) || !aligned4(block_table))
    return HIPPO_ERR_BAD_ALIGN;
  if (workspace_bytes < pl.bytes) return HIPPO_ERR_WORKSPACE_TOO_SMALL;
  RowsParams p{};
  p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse_out;
  p.q_sn = desc->q_stride_n; p.q_sh = desc->q_stride_h; p.k_sn = desc->kv_stride_n; p.k_sh = desc->kv_stride_h;
  p.n_seq = n_seqs; p.H = desc->n_q_heads; p.Hkv = desc->n_kv_heads; p.G = p.H / p.Hkv;
  p.total_q = total_q; p.total_k = total_k; p.cu_q = cu_q;
  if (pd == nullptr) {
    p.cu_k = cu_k;
  } else {
    p.kv_lens = cu_k;
    p.block_table = block_table; p.max_pages = pd->max_pages; p.n_pool_pages = pd->n_pool_pages; p.page_stride = pd->stride_page;
    while ((1 << p.page_shift) < pd->page_size) ++p.page_shift;
  }
  p.scale_log2 = scale_or_default(softmax_scale, desc->head_dim);
  carve_rows(&p, pl, workspace);
  const hipError_t e = launch_prefill(p, pl, desc->dtype, desc->head_dim, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

int hippo_prefill_attention(const void* q, int32_t total_q, const void* k, const void* v, int32_t total_k,
                            const hippo_packed_desc* desc, const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs,
                            float softmax_scale, int32_t num_splits, void* out, float* lse_out, void* workspace,
                            size_t workspace_bytes, void* stream) {
  return prefill_entry(q, total_q, k, v, total_k, desc, nullptr, nullptr, cu_q, cu_k, n_seqs, softmax_scale, num_splits, out, lse_out,
                       workspace, workspace_bytes, stream);
}

int hippo_prefill_attention_paged(const void* q, int32_t total_q, int64_t q_stride_n, int64_t q_stride_h, const void* k_pool,
                                  const void* v_pool, const int32_t* block_table, const hippo_paged_kv_desc* kv, const int32_t* cu_q,
                                  const int32_t* kv_lens, float softmax_scale, int32_t num_splits, void* out, float* lse_out,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_pool(kv);
  if (rc != HIPPO_OK) return rc;
  if (block_table == nullptr || k_pool == nullptr || v_pool == nullptr) return HIPPO_ERR_NULL_ARG;
  if (kv->max_pages < 1 || (long long)kv->max_pages * kv->page_size > 0x7fffff00ll) return HIPPO_ERR_BAD_SHAPE;
  const hippo_packed_desc d = {kv->n_q_heads, kv->n_kv_heads, kv->head_dim, kv->dtype, q_stride_n, q_stride_h, kv->stride_n, kv->stride_h};
  return prefill_entry(q, total_q, k_pool, v_pool, kv->max_pages * kv->page_size, &d, kv, block_table, cu_q, kv_lens, kv->batch,
                       softmax_scale, num_splits, out, lse_out, workspace, workspace_bytes, stream);
}

size_t hippo_tree_workspace_bytes(const hippo_kv_desc* kv, int32_t n_nodes, int32_t seq_len, int32_t num_splits) {
  RowsPlan pl;
  if (check_heads(kv, false) != HIPPO_OK || plan_tree(kv, n_nodes, seq_len, true, num_splits, &pl) != HIPPO_OK) return 0;
  return pl.bytes;
}

static int tree_entry(const void* q, int32_t n_nodes, const void* k, const void* v, const hippo_kv_desc* kv,
                      const hippo_paged_kv_desc* pd, const int32_t* block_table, int32_t seq_len, const int32_t* parents,
                      int64_t parents_stride_b, const int32_t* ctx_lens, int32_t ctx_len, float softmax_scale, int32_t num_splits,
                      void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (q == nullptr || k == nullptr || v == nullptr || parents == nullptr || out == nullptr || workspace == nullptr)
    return HIPPO_ERR_NULL_ARG;
  int rc = check_kv(kv);
  if (rc != HIPPO_OK) return rc;
  RowsPlan pl;
  rc = plan_tree(kv, n_nodes, seq_len, ctx_lens != nullptr, num_splits, &pl);
  if (rc != HIPPO_OK) return rc;
  if (parents_stride_b < 0) return HIPPO_ERR_BAD_SHAPE;
  if (ctx_lens == nullptr && (ctx_len < 0 || ctx_len > seq_len - n_nodes)) return HIPPO_ERR_BAD_SHAPE;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || (reinterpret_cast<uintptr_t>(workspace) & 255u) ||
      !aligned4(parents) || !aligned4(ctx_lens) || !aligned4(lse_out) || !aligned4(block_table))
    return HIPPO_ERR_BAD_ALIGN;
  if (workspace_bytes < pl.bytes) return HIPPO_ERR_WORKSPACE_TOO_SMALL;
  RowsParams p{};
  p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse_out;
  p.n_seq = kv->batch; p.H = kv->n_q_heads; p.Hkv = kv->n_kv_heads; p.G = p.H / p.Hkv;
  p.q_sn = (int64_t)p.H * kv->head_dim; p.q_sh = kv->head_dim;
  p.k_sb = kv->stride_b; p.k_sn = kv->stride_n; p.k_sh = kv->stride_h;
  p.total_q = kv->batch * n_nodes; p.total_k = seq_len;
  p.kv_lens = ctx_lens; p.ctx_len = ctx_len;
  p.parents = parents; p.parents_sb = parents_stride_b; p.nodes = n_nodes;
  if (pd != nullptr) {
    p.block_table = block_table; p.max_pages = pd->max_pages; p.n_pool_pages = pd->n_pool_pages; p.page_stride = pd->stride_page;
    while ((1 << p.page_shift) < pd->page_size) ++p.page_shift;
  }
  p.scale_log2 = scale_or_default(softmax_scale, kv->head_dim);
  carve_rows(&p, pl, workspace);
  const hipError_t e = launch_tree(p, pl, kv->dtype, kv->head_dim, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

int hippo_tree_attention(const void* q, int32_t n_nodes, const void* k_cache, const void* v_cache, const hippo_kv_desc* kv,
                         int32_t seq_len, const int32_t* parents, int64_t parents_stride_b, const int32_t* ctx_lens, int32_t ctx_len,
                         float softmax_scale, int32_t num_splits, void* out, float* lse_out, void* workspace, size_t workspace_bytes,
                         void* stream) {
  return tree_entry(q, n_nodes, k_cache, v_cache, kv, nullptr, nullptr, seq_len, parents, parents_stride_b, ctx_lens, ctx_len,
                    softmax_scale, num_splits, out, lse_out, workspace, workspace_bytes, stream);
}

int hippo_tree_attention_paged(const void* q, int32_t n_nodes, const void* k_pool, const void* v_pool, const int32_t* block_table,
                               const hippo_paged_kv_desc* kv, const int32_t* parents, int64_t parents_stride_b,
                               const int32_t* ctx_lens, int32_t ctx_len, float softmax_scale, int32_t num_splits, void* out,
                               float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_pool(kv);
  if (rc != HIPPO_OK) return rc;
  if (block_table == nullptr) return HIPPO_ERR_NULL_ARG;
  if (kv->max_pages < 1 || (long long)kv->max_pages * kv->page_size > 0x7fffff00ll) return HIPPO_ERR_BAD_SHAPE;
  const hippo_kv_desc flat = {kv->batch, kv->n_q_heads, kv->n_kv_heads, kv->head_dim, kv->dtype, 0, kv->stride_h, kv->stride_n};
  return tree_entry(q, n_nodes, k_pool, v_pool, &flat, kv, block_table, kv->max_pages * kv->page_size, parents, parents_stride_b,
                    ctx_lens, ctx_len, softmax_scale, num_splits, out, lse_out, workspace, workspace_bytes, stream);
}

int hippo_plan_pages(const int32_t* ctx_lens, const int32_t* new_lens, int32_t batch, int32_t* block_table, int32_t max_pages,
                     int32_t* free_pages, int32_t n_pool_pages, const int32_t* n_free, int32_t page_size, int32_t max_tokens,
                     int32_t* slots_out, int32_t* positions_out, int32_t* cu_q_out, int32_t* kv_lens_out, int32_t* n_free_out,
                     void* stream) {
  if (ctx_lens == nullptr || new_lens == nullptr || block_table == nullptr || free_pages == nullptr || n_free == nullptr ||
      cu_q_out == nullptr || kv_lens_out == nullptr || n_free_out == nullptr)
    return HIPPO_ERR_NULL_ARG;
  if (max_tokens > 0 && (slots_out == nullptr || positions_out == nullptr)) return HIPPO_ERR_NULL_ARG;
  if (batch < 1 || batch > kPlanMaxBatch || max_pages < 1 || (long long)batch * max_pages > (1 << 30) || max_pages > kPlanMost ||
      n_pool_pages < 1 || n_pool_pages > kPlanMost || max_tokens < 0 || max_tokens > kPlanMost)
    return HIPPO_ERR_BAD_SHAPE;
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1))) return HIPPO_ERR_BAD_SHAPE;
  const void* all[] = {ctx_lens, new_lens, block_table, free_pages, n_free, slots_out, positions_out, cu_q_out, kv_lens_out, n_free_out};
  for (const void* x : all)
    if (!aligned4(x)) return HIPPO_ERR_BAD_ALIGN;
  // Every block reads the lengths and the stack's height, some of them again for each item, while others write: an input that reached into
  // what is written would change under them, and with it the places that they look up in the table.
  struct Span {
    const void* first;
    long long n;
  };
  for (const Span& in : {Span{ctx_lens, batch}, Span{new_lens, batch}, Span{n_free, 1}})
    for (const Span& o : {Span{block_table, (long long)batch * max_pages}, Span{free_pages, n_pool_pages}, Span{slots_out, max_tokens},
                          Span{positions_out, max_tokens}, Span{cu_q_out, batch + 1}, Span{kv_lens_out, batch}, Span{n_free_out, 1}}) {
      const uintptr_t a = reinterpret_cast<uintptr_t>(in.first), b = reinterpret_cast<uintptr_t>(o.first);
      if (a < b + o.n * sizeof(int32_t) && b < a + in.n * sizeof(int32_t) && o.n > 0) return HIPPO_ERR_BAD_SHAPE;
    }
  PlanParams p;
  p.ctx_lens = ctx_lens; p.new_lens = new_lens; p.block_table = block_table; p.free_pages = free_pages; p.n_free = n_free;
  p.n_free_out = n_free_out; p.slots = slots_out; p.positions = positions_out; p.cu_q = cu_q_out; p.kv_lens = kv_lens_out;
  p.B = batch; p.max_pages = max_pages; p.n_pool = n_pool_pages; p.max_tokens = max_tokens;
  p.page_shift = 0;
  while ((1 << p.page_shift) < page_size) ++p.page_shift;
  const hipError_t e = launch_plan_pages(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

int hippo_write_kv_paged(const void* k_new, const void* v_new, int32_t n_rows, int64_t stride_n, int64_t stride_h,
                         const int32_t* slots, const int32_t* rows, int32_t n_tokens, void* k_pool, void* v_pool,
                         const hippo_paged_kv_desc* kv, void* stream) {
  const int rc = check_pool(kv);
  if (rc != HIPPO_OK) return rc;
  if (n_tokens < 0 || n_rows < 0 || stride_n < 0 || stride_h < 0) return HIPPO_ERR_BAD_SHAPE;
  // heads and rows of a page must not meet
  if (rows_meet({kv->n_pool_pages, kv->stride_page}, {kv->n_kv_heads, kv->stride_h}, {kv->page_size, kv->stride_n}, kv->head_dim))
    return HIPPO_ERR_BAD_SHAPE;
  const int es = elem_bytes(kv->dtype);
  if (stride_n % (16 / es) || stride_h % (16 / es)) return HIPPO_ERR_BAD_ALIGN;
  const int pieces = kv->head_dim * es / 16;
  if ((long long)n_tokens * kv->n_kv_heads * pieces > (1ll << 31) || (long long)kv->n_kv_heads * pieces > (1 << 20))
    return HIPPO_ERR_BAD_SHAPE;
  if (n_tokens == 0 || n_rows == 0) return HIPPO_OK;          // nothing to write
  if (k_new == nullptr || v_new == nullptr || slots == nullptr || k_pool == nullptr || v_pool == nullptr) return HIPPO_ERR_NULL_ARG;
  if (k_pool == v_pool) return HIPPO_ERR_BAD_SHAPE;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned4(slots) || !aligned4(rows))
    return HIPPO_ERR_BAD_ALIGN;
  WriteParams p;
  p.k = k_new; p.v = v_new; p.slots = slots; p.rows = rows; p.k_pool = k_pool; p.v_pool = v_pool;
  p.n_tokens = n_tokens; p.n_rows = n_rows; p.Hkv = kv->n_kv_heads; p.pieces = pieces;
  p.page_shift = 0;
  while ((1 << p.page_shift) < kv->page_size) ++p.page_shift;
  p.by_token = divisor(p.Hkv * pieces); p.by_head = divisor(pieces);
  p.n_slots = (long long)kv->n_pool_pages * kv->page_size;
  p.sn = stride_n * es; p.sh = stride_h * es;
  p.page_stride = kv->stride_page * es; p.pool_sn = kv->stride_n * es; p.pool_sh = kv->stride_h * es;
  const hipError_t e = launch_write_kv(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? HIPPO_OK : HIPPO_ERR_HIP;
}

}  // extern "C"
