// Attention of many query rows: the prompt calls (prefill.hip) and the draft-tree calls (tree.hip).
//
// The calls of attention.hip have a few query rows a KV head and are bound by the cache's bytes.  Here a KV head has tens to
// thousands of them (row r = i * G + g: row i of the sequence, query head g of the group, so that the heads of a group share every
// K and V row that reaches the LDS), and what counts is how much of a K or V row's trip from the LDS to the matrix unit is used: a wave
// owns 32 query rows (v_mfma_f32_32x32x16_bf16, in fp32 32x32x2), half the LDS bytes per product of 16-row tiles.
//
//   S^T = K Q^T      A = 32 tokens of K, B = 32 query rows: lane (j = lane % 32, h = lane / 32) gets query row j's logits of tokens
//                    8 (e / 4) + 4 h + e % 4 of the block, e = 0..15
//   O^T = V^T P^T    B = those same registers (the order of the tokens in a contraction is free), A = V^T by transposing LDS reads
//   softmax          one pass, with a running maximum and sum per row (the online softmax of Milakov and Gimelshein, 2018; its lazy form, in which
//                    the reference follows only a rise beyond a threshold, is published, too); a row's tokens lie in lanes j and j + 32,
//                    so one exchange of the wave's halves completes a maximum
//
// A block has RB x TG waves: wave (rb, tg) owns rows 32 rb .. 32 rb + 31 of the block's tile and of every stage tokens
// tg TW .. tg TW + TW - 1; the TG states of a row block meet in the LDS at the end.  K and V reach the LDS without registers in between,
// NST stages deep.  A sequence's stages may be dealt to S blocks (few rows over many tokens): their states go to a merge.
//
// What bounds it: long prompts and wide trees the matrix unit, at the clock that its power leaves (16640 rows x 28 heads x 128: 1716 to 1749 us,
// 1.15 PFLOP/s, where a library product of 16384^3 reaches 1.35); few rows over a long cache a block's start, its stages one behind the
// other and the merge's launch (16 nodes x 28 heads over 16640 rows: 128 blocks of eight or nine stages, 18 us for 34 MB, of which the bytes alone
// would be 5); short prompts a chain of trips to memory of some 4 us, beside which other blocks should run.
#pragma once

#include <type_traits>

#include "common.h"

namespace hippo {

struct RowsParams {
  const void* q;
  const void* k;
  const void* v;
  void* out;                    // [tokens, H, D]
  float* lse;                   // may be null: [H, total_q] of prompts, [B, H, nodes] of trees
  long long q_sn, q_sh;         // element strides of q's tokens and heads
  long long k_sb, k_sn, k_sh;   // of K and V: batch elements (contiguous caches), rows, KV heads
  int n_seq, H, Hkv, G;
  int total_q, total_k;         // rows of q; rows of packed K and V, or the most that a sequence's part of the cache holds
  const int32_t* cu_q;          // prompts: [n_seq + 1]
  const int32_t* cu_k;          // packed prompts: [n_seq + 1]
  const int32_t* kv_lens;       // paged prompts: rows of each sequence; trees: rows before the tree, null: ctx_len
  int ctx_len;
  const int32_t* parents;       // trees: [B, nodes]
  long long parents_sb;
  int nodes;
  const int32_t* block_table;   // [n_seq, max_pages]
  int page_shift, max_pages, n_pool_pages;
  long long page_stride;
  float scale_log2;
  Divisor by_heads, by_group, by_tiles;   // by Hkv, G, tiles_per_seq
  int tiles_per_seq;            // of trees
  int S;                        // blocks that share a tile's stages (parts in the workspace)
  int deal;                     // trees of 2 to 64 sequences: that many such blocks over all of them, by length; 0: S each
  int n_tiles;                  // row tiles of the launch
  float* part_o;                // [S, tokens * H, D] outputs before the division
  float* part_m;                // [S, tokens * H] maxima (log2), -inf: nothing seen
  float* part_l;
};

// how a call is cut: rows of a block (RB x 32), two such blocks on a compute unit, blocks that share a tile, see RowsParams
struct RowsPlan {
  int rb;
  bool pair;
  int S, n_tiles, deal;
  size_t off_m, off_l, bytes;
};

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short rows_s16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 rows_bf16x2;
typedef __attribute__((ext_vector_type(2))) float rows_f32x2;

// LDS geometry of a K or V tile: rows as in memory, the 16-byte pieces of a row exchanged so that neither the K reads (16 lanes, 16
// consecutive rows, the same piece) nor the V reads (bf16: 32 lanes, four rows, four neighbouring pieces; fp32: 64 lanes, two rows four
// apart, eight pieces each) meet in a bank: of 256 bytes, the K reads' rows differ in all four bits, the V reads' in those above.
template <typename T, int D>
struct RowsTile {
  static constexpr int kRowBytes = D * (int)sizeof(T);
  static constexpr int kPieces = kRowBytes / 16;
  static constexpr int kRowsPerXfer = 1024 / kRowBytes;
  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (sizeof(T) == 4) return (((r >> 2) & 1) << 3) | (((r >> 3) & 1) << 2) | (r & 3);
    else if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
};

template <typename T, int D, int RB, int TG, int TW, int NST>
struct RowsSmem {
  static constexpr int kTileBytes = TG * TW * RowsTile<T, D>::kRowBytes;   // of a stage's K (or V)
  static constexpr int kStage = 2 * kTileBytes;
  static constexpr int kMerge = TG == 1 ? 0 : TG * RB * (D / 2) * 256;     // the waves' accumulators
  static constexpr int kRing = NST * kStage > kMerge ? NST * kStage : kMerge;
  static constexpr int total() { return kRing + 2 * TG * RB * 32 * 4 + 16; }
};

struct RowsTileAt {
  int seq, tile;         // the sequence, its row tile
  int tok0, len_q;       // its first row of q, their number
  int row0_k, len_k;     // its first row of packed K and V, their number
};

// The block's (sequence, row tile).  Prompts: tiles in descending order of the tokens that they see, so that the longest start first:
// tile k of a sequence has the level (rows before it) / (rows of a tile) + k, and block t takes the t-th tile from the highest level
// down.  (A lane looks after a sequence; the level is found by bisection.  More than 64 sequences go in their own order, each
// from its last tile.)  False: no such tile.
template <int ROWS, bool PAGED>
__device__ __forceinline__ bool rows_find_tile(const RowsParams& p, int t, RowsTileAt* at) {
  const int lane = threadIdx.x & 63;
  auto look = [&](int b, int* base) {                       // a sequence's numbers, into *at; its tiles
    at->tok0 = min(max(p.cu_q[b], 0), p.total_q);
    at->len_q = min(max(p.cu_q[b + 1], at->tok0), p.total_q) - at->tok0;
    if constexpr (PAGED) {
      at->row0_k = 0;
      at->len_k = min(max(p.kv_lens[b], 0), p.total_k);
    } else {
      at->row0_k = min(max(p.cu_k[b], 0), p.total_k);
      at->len_k = min(max(p.cu_k[b + 1], at->row0_k), p.total_k) - at->row0_k;
    }
    *base = (int)min((long long)max(at->len_k - at->len_q, 0) * p.G / ROWS, (long long)(1 << 29));
    return (at->len_q * p.G + ROWS - 1) / ROWS;             // (rows: below 2^30)
  };
  auto take = [&](int from) {                               // the numbers of the lane that looked after the sequence
    at->tok0 = __builtin_amdgcn_readlane(at->tok0, from);
    at->len_q = __builtin_amdgcn_readlane(at->len_q, from);
    at->row0_k = __builtin_amdgcn_readlane(at->row0_k, from);
    at->len_k = __builtin_amdgcn_readlane(at->len_k, from);
  };
  auto add = [](int a, int b) { return a + b; };
  int base;
  if (p.n_seq == 1) {
    const int n = look(0, &base);
    at->seq = 0;
    at->tile = n - 1 - t;
    return t < n;
  }
  if (p.n_seq <= 64) {
    int n = look(min(lane, p.n_seq - 1), &base);
    if (lane >= p.n_seq) n = base = 0;
    if (t >= wave_reduce_i32(n, add)) return false;
    // the largest level that more than t tiles reach
    int lo = 0, hi = wave_reduce_i32(base + n, [](int a, int b) { return max(a, b); });
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (wave_reduce_i32(min(max(base + n - mid, 0), n), add) > t) lo = mid;
      else hi = mid;
    }
    const int above = wave_reduce_i32(min(max(base + n - lo - 1, 0), n), add);
    unsigned long long here = __ballot(base <= lo && lo < base + n);
    for (int i = t - above; i > 0; --i) here &= here - 1;
    const int b = __ffsll((long long)here) - 1;
    at->seq = b;
    at->tile = lo - __builtin_amdgcn_readlane(base, b);
    take(b);
    return true;
  }
  int before = 0;
  for (int b0 = 0; b0 < p.n_seq; b0 += 64) {
    int n = look(min(b0 + lane, p.n_seq - 1), &base);
    if (b0 + lane >= p.n_seq) n = 0;
    const int incl = (int)wave_scan_incl((unsigned)n) + before;
    const unsigned long long past = __ballot(incl > t);
    if (past != 0) {
      const int l = __ffsll((long long)past) - 1;
      at->seq = b0 + l;
      at->tile = __builtin_amdgcn_readlane(incl, l) - 1 - t;     // the last one first
      take(l);
      return true;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// Which nodes a node sees: lane i gets node i's, itself among them; 0: the node is none (its parent is below -1 or not before it, or
// an ancestor is none).  After round r the bits of 2^r ancestors are there.
// `up`: the lane's parent, -2 behind the last node.
__device__ __forceinline__ unsigned long long tree_masks(int up) {
  const int lane = threadIdx.x & 63;
  int none = up < -1 || up >= lane;
  unsigned lo = none ? 0u : lane < 32 ? 1u << lane : 0u, hi = none ? 0u : lane >= 32 ? 1u << (lane - 32) : 0u;
  if (none) up = -1;
#pragma unroll
  for (int r = 0; r < 6; ++r) {
    const int from = up < 0 ? lane : up;
    const unsigned alo = __shfl(lo, from), ahi = __shfl(hi, from);
    const int anone = __shfl(none, from), aup = __shfl(up, from);
    lo |= alo; hi |= ahi; none |= anone;
    up = up < 0 ? -1 : aup;
  }
  return none ? 0ull : (unsigned long long)hi << 32 | lo;
}

// N runs of 1 KB: 16 bytes a lane from `base` (uniform) + off[i] (of the lane) straight into LDS at lds_addr + 1024 i + lane * 16, see
// dma16
template <int N>
__device__ __forceinline__ void dma16_runs(const void* base, const unsigned* off, unsigned lds_addr) {
  if constexpr (N > 4) {
    dma16_runs<4>(base, off, lds_addr);
    dma16_runs<N - 4>(base, off + 4, lds_addr + 4096);
  } else {
    static_assert(N == 2 || N == 4, "");
    const unsigned uniform_addr = __builtin_amdgcn_readfirstlane(lds_addr);
    unsigned saved_m0;
    if constexpr (N == 2)
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
                   "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                   : "=&s"(saved_m0)
                   : "v"(off[0]), "v"(off[1]), "s"(base), "s"(uniform_addr)
                   : "memory", "scc");
    else
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\t"
                   "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %5\n\t"
                   "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %5\n\t"
                   "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %5\n\ts_mov_b32 m0, %0"
                   : "=&s"(saved_m0)
                   : "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base), "s"(uniform_addr)
                   : "memory", "scc");
  }
}
// The kernel's parts are lambdas over its registers: one that stayed a function would keep them in memory.
#define ROWS_INLINE __attribute__((always_inline))

// The compiler cannot always tell that a value is the same in all lanes.
__device__ __forceinline__ long long uniform64(long long x) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x), hi = __builtin_amdgcn_readfirstlane((unsigned)((unsigned long long)x >> 32));
  return (long long)((unsigned long long)hi << 32 | lo);
}

// Stages of a tree's sequence: what its blocks share out (counted alike by the merge).
__device__ __forceinline__ int tree_rows(const RowsParams& p, int seq) {
  const int ctx = p.kv_lens != nullptr ? p.kv_lens[seq] : p.ctx_len;
  return min(max(ctx, 0), p.total_k - p.nodes) + p.nodes;
}
// Trees of sequences of different lengths: p.deal blocks over all of them, each sequence so many that none of its blocks has more rows
// than c, the smallest of 64 lengths from (all rows) / deal up to three times that with which the blocks suffice (there is one: deal is
// at least twice the sequences).  Lane b gets sequence b's, 0 behind the last.  37120, 16640, 33280 and 29001 rows, 64 nodes, 64 x 8
// heads: 275 us with four blocks each, 261 like this.
__device__ __forceinline__ int tree_deal(const RowsParams& p) {
  const int lane = threadIdx.x & 63;
  const float len = lane < p.n_seq ? (float)tree_rows(p, lane) : 0.f;
  const float least = wave_sum(len) / (float)p.deal, mine = 1.f / (least * (1.f + (float)lane * (1.f / 32.f)));
  float blocks = 0.f;
  for (int b = 0; b < p.n_seq; ++b) blocks += ceilf(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(len), b)) * mine);
  const unsigned long long enough = __ballot(blocks <= (float)p.deal) | 1ull << 63;
  const float c = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), __ffsll((long long)enough) - 1));
  return lane < p.n_seq ? min(max((int)ceilf(len * c), 1), p.S) : 0;
}

template <typename T, int D, int RB, int TG, int TW, int NST, bool PAGED, bool TREE>
__global__ __launch_bounds__(RB * TG * 64, D * sizeof(T) <= 256 && (RB == 4 && TG == 1 || RB == 2 && TG == 2) ? (D * sizeof(T) == 128 ? 3 : 2) : RB * TG / 4) void attn_rows(RowsParams p) {
  using Tile = RowsTile<T, D>;
  using SM = RowsSmem<T, D, RB, TG, TW, NST>;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int ES = sizeof(T), ROWB = Tile::kRowBytes, RPT = Tile::kRowsPerXfer, CPR = Tile::kPieces;
  constexpr int WAVES = RB * TG, ROWS = RB * 32, ST = TG * TW, TB = TW / 32, DB = D / 32;
  constexpr int NLD = ST / RPT, PER = 2 * NLD / WAVES;      // transfers of a stage's K (or V); of a wave a stage
  constexpr int NPG = PER * RPT > 16 ? PER * RPT / 16 : 1;  // runs of 16 rows (of a page each) in a wave's transfers
  constexpr int TR = PER / NPG;                             // transfers of a run
  constexpr int QN = CPR / 2;                               // 16-byte pieces of a query row in a lane
  constexpr int SN = TB * 16;                               // logits of a wave's stage in a lane
  constexpr bool PIPE = !F32 && NST >= 4, LATE = PIPE && WAVES == 8;
  static_assert(2 * NLD % WAVES == 0 && NLD % PER == 0 && PER * NST <= 63 && NST >= 2, "transfer split");

  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* ring = smem;
  float* stat_m = (float*)(smem + SM::kRing);               // [TG][ROWS]
  float* stat_l = stat_m + TG * ROWS;
  int* odd_stage = (int*)(stat_l + TG * ROWS);              // the last edge stage whose V has infinities or NaN, from 1
  if (threadIdx.x == 0) *odd_stage = 0;                     // (before the barriers of the stages)
  wait_lds();
  const unsigned ring_addr = (unsigned)(uintptr_t)ring;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rb = wave % RB, tg = wave / RB;
  const int j = lane & 31, h = lane >> 5;
  const int tile_no = __builtin_amdgcn_readfirstlane(p.by_heads(blockIdx.x));
  const int hk = blockIdx.x - tile_no * p.Hkv;
  int split = blockIdx.y, n_split = p.S;

  // ---- the block's rows and the tokens that they may see ----
  int seq, tile, len_q, len_k, tok0;
  long long row0_k = 0;
  if constexpr (TREE) {
    if (p.deal > 0) {                                       // blocks of y: sequence after sequence
      const int mine = tree_deal(p), incl = (int)wave_scan_incl((unsigned)mine);
      const unsigned long long past = __ballot(incl > split);
      if (past == 0) return;
      seq = __builtin_amdgcn_readfirstlane(__ffsll((long long)past) - 1);
      n_split = __builtin_amdgcn_readlane(mine, seq);
      split -= __builtin_amdgcn_readlane(incl, seq) - n_split;
      tile = tile_no;
    } else {
      seq = __builtin_amdgcn_readfirstlane(p.by_tiles(tile_no));
      tile = tile_no - seq * p.tiles_per_seq;
    }
    len_q = p.nodes;
    tok0 = seq * p.nodes;
    len_k = __builtin_amdgcn_readfirstlane(tree_rows(p, seq));
  } else {
    RowsTileAt at;
    if (!rows_find_tile<ROWS, PAGED>(p, tile_no, &at)) return;
    seq = __builtin_amdgcn_readfirstlane(at.seq);
    tile = __builtin_amdgcn_readfirstlane(at.tile);
    tok0 = __builtin_amdgcn_readfirstlane(at.tok0);
    len_q = __builtin_amdgcn_readfirstlane(at.len_q);
    len_k = __builtin_amdgcn_readfirstlane(at.len_k);
    if constexpr (!PAGED) row0_k = __builtin_amdgcn_readfirstlane(at.row0_k);
  }
  const int off = len_k - len_q;                            // trees: the context's length
  const int R = len_q * p.G;
  const int last = __builtin_amdgcn_readfirstlane(p.by_group(min(tile * ROWS + ROWS, R) - 1));   // of the tile's rows
  const int ext = TREE ? len_k : min(max(off + last + 1, 0), len_k);
  const int all_stages = (ext + ST - 1) / ST;
  int s_lo = 0, n_stage = all_stages;
  if (n_split > 1) {                                        // as evenly as possible, the first blocks taking one more
    const int each = all_stages / n_split, more = all_stages - each * n_split;
    s_lo = split * each + min(split, more);
    n_stage = each + (split < more ? 1 : 0);
  }
  // the first token that some row of the block does not see: the stages before it need no mask
  const int block_edge = TREE ? off : __builtin_amdgcn_readfirstlane(off + p.by_group(tile * ROWS)) + 1;
  const int n_plain = min(max(block_edge / ST - s_lo, 0), n_stage);

  int parent = -2;                                          // of node `lane`: on its way before the transfers, which it would wait for
  if constexpr (TREE)
    if (lane < p.nodes) parent = p.parents[seq * p.parents_sb + lane];
  asm volatile("" : "+v"(parent));

  // ---- transfers: the first half of the waves fetches K, the other half V ----
  const bool fetch_v = wave >= WAVES / 2;
  const char* base = (const char*)(fetch_v ? p.v : p.k) +
                     ((PAGED ? 0ll : TREE ? (long long)seq * p.k_sb : row0_k * p.k_sn) + (long long)hk * p.k_sh) * ES;
  const int ld_row = lane / CPR, ld_pc = lane % CPR;
  const int cap = ext - 1, first_row = wave % (WAVES / 2) * PER * RPT;       // of the stage's rows, the wave's first
  const unsigned row_bytes = (unsigned)(p.k_sn * ES);       // (the host keeps a row's stride below 2^24 elements)
  unsigned lane_off[TR];                                    // of a run's transfers, from its first row on
#pragma unroll
  for (int u = 0; u < TR; ++u)
    lane_off[u] = (u * RPT + ld_row) * row_bytes + ((ld_pc ^ Tile::swizzle(first_row + u * RPT + ld_row)) * 16);
  const int page_mask = PAGED ? (1 << p.page_shift) - 1 : 0;
  // (in the constant address space: read through the scalar cache whatever assembly stands between.  As vector loads they wait for every
  // transfer that is under way: pieces over 37K pages 1747 us instead of 1487.)
  typedef const int32_t __attribute__((address_space(4))) * ScalarTable;
  const ScalarTable table = PAGED ? (ScalarTable)(uintptr_t)(p.block_table + (long long)seq * p.max_pages) : nullptr;
  // pages of the next stage to be fetched: asked for a stage ahead, through the scalar cache.  Rows of a run of 16 share a page, as
  // a page's size is a multiple of 16.
  int page[NPG];
  auto ask_pages = [&](int si) ROWS_INLINE {
    if constexpr (PAGED) {
#pragma unroll
      for (int i = 0; i < NPG; ++i) {
        const int row = min((s_lo + si) * ST + first_row + i * 16, cap);
        page[i] = table[max(row, 0) >> p.page_shift];
      }
    }
  };
  const long long stage_bytes = (long long)ST * p.k_sn * ES;
  const char* next = (const char*)uniform64((long long)(base + (long long)(s_lo * ST + first_row) * p.k_sn * ES));   // (of the next stage)
  auto issue = [&](int si) ROWS_INLINE {
    const unsigned dst = ring_addr + (si % NST) * SM::kStage + (fetch_v ? SM::kTileBytes : 0) + first_row * ROWB;
    const int n0 = (s_lo + si) * ST + first_row;
    auto page_at = [&](int i, int row0) ROWS_INLINE {       // where a run of rows starts
      return (const char*)uniform64((long long)(base + ((long long)min(max(page[i], 0), p.n_pool_pages - 1) * p.page_stride +
                                                        (long long)(row0 & page_mask) * p.k_sn) * ES));
    };
    if (n0 + PER * RPT <= ext) {
#pragma unroll
      for (int i = 0; i < NPG; ++i) {
        const char* from = next + (long long)i * TR * RPT * row_bytes;
        if constexpr (PAGED) from = page_at(i, n0 + i * TR * RPT);
        dma16_runs<TR>(from, lane_off, dst + i * TR * 1024);
      }
    } else {                                                // the sequence's last stage: rows behind its end repeat the last one
#pragma unroll
      for (int i = 0; i < NPG; ++i) {
        const int row0 = min(n0 + i * TR * RPT, cap);
        const char* from = (const char*)uniform64((long long)(base + (long long)row0 * p.k_sn * ES));
        if constexpr (PAGED) from = page_at(i, row0);
        unsigned last_off[TR];
#pragma unroll
        for (int u = 0; u < TR; ++u)
          last_off[u] = (min(n0 + (i * TR + u) * RPT + ld_row, cap) - row0) * row_bytes +
                        ((ld_pc ^ Tile::swizzle(first_row + u * RPT + ld_row)) * 16);
        dma16_runs<TR>(from, last_off, dst + i * TR * 1024);
      }
    }
    next += stage_bytes;
  };
  int issued = 0;
  auto issue_next = [&]() ROWS_INLINE {
    if (issued >= n_stage) return;
    issue(issued++);
    if (issued < n_stage) ask_pages(issued);
  };
  if (n_stage > 0) ask_pages(0);
  // Everyone is past stage `past`'s products: the places up to that one's are filled again.
  auto refill = [&](int past) ROWS_INLINE {
    if (issued < n_stage && issued <= past + NST) issue_next();
  };
#pragma unroll 1
  for (int i = 0; i < NST; ++i) refill(-1);

  // ---- the wave's query rows ----
  const int row = tile * ROWS + rb * 32 + j;
  const int qi = p.by_group(min(row, R - 1)), head = hk * p.G + min(row, R - 1) - qi * p.G;
  using QPiece = typename std::conditional<F32, f32x4, bf16x8>::type;
  QPiece qop[QN];
  {
    const T* src = (const T*)p.q + (long long)(tok0 + qi) * p.q_sn + (long long)head * p.q_sh;
#pragma unroll
    for (int c = 0; c < QN; ++c) qop[c] = *(const QPiece*)(src + (2 * c + h) * (16 / ES));
  }
  unsigned long long sees = 0;                              // trees: the nodes that the lane's row sees
  if constexpr (TREE) {
    const unsigned long long m = tree_masks(parent);
    sees = (unsigned long long)(unsigned)__shfl((int)(m >> 32), qi) << 32 | (unsigned)__shfl((int)(unsigned)m, qi);
  }
  const int lim = off + qi;                                 // prompts: the last token that the row sees

  float m_run = -INFINITY, l_run = 0.f;
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;

  // LDS offsets of the lane's operands in a tile: K piece c of row j at k_off ^ 32 c, V piece of d block db at v_off ^ 64 db (a tile's
  // rows are powers of two apart, and the swizzle is an exclusive or).  The reads' addresses are formed stage by stage: kept in
  // registers they are more than there are.
  const unsigned k_off = j * ROWB + ((h ^ Tile::swizzle(j)) * 16);
  const int v_row = 4 * h + ((lane & 15) >> 2);
  const unsigned v_off = v_row * ROWB + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ Tile::swizzle(v_row)) * 16) + (lane & 1) * 8;

  // LDS addresses of a stage's tiles (numbers: constants that are added to them become the reads' immediate offsets)
  auto k_tile = [&](int si) ROWS_INLINE { return ring_addr + (si % NST) * SM::kStage + tg * TW * ROWB; };
  auto v_tile = [&](int si) ROWS_INLINE { return ring_addr + (si % NST) * SM::kStage + SM::kTileBytes + tg * TW * ROWB; };
#define ROWS_LDS(type, address) ((__attribute__((address_space(3))) type*)(uintptr_t)(address))

  // S^T = K Q^T.  (Operands are read several products ahead, here and below, and held to that order: the compiler reads one right before
  // its product, and a wave that has a SIMD to itself waits for each.)
  auto k_piece = [&](unsigned Kt, int i) ROWS_INLINE {      // product i: piece i / TB of token block i % TB
    return *(ROWS_LDS(const u32x4, (Kt + k_off) ^ (32 * (i / TB))) + i % TB * 32 * ROWB / 16);
  };
  auto logits = [&](unsigned Kt, f32x16 (&s)[TB]) ROWS_INLINE {
    constexpr int N = TB * QN, AH = F32 ? 4 : 8;
    u32x4 ahead[AH];
#pragma unroll
    for (int i = 0; i < AH && i < N; ++i) ahead[i] = k_piece(Kt, i);
#pragma unroll
    for (int tb = 0; tb < TB; ++tb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[tb][e] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const QPiece kop = __builtin_bit_cast(QPiece, ahead[i % AH]);
      if constexpr (F32) {
#pragma unroll
        for (int x = 0; x < 4; ++x) s[i % TB] = __builtin_amdgcn_mfma_f32_32x32x2f32(kop[x], qop[i / TB][x], s[i % TB], 0, 0, 0);
      } else {
        s[i % TB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop, qop[i / TB], s[i % TB], 0, 0, 0);
      }
      if (i + AH < N) ahead[i % AH] = k_piece(Kt, i + AH < N ? i + AH : 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // The rows' reference moves only when a maximum exceeds it by 2^8: weights stay below that, and rescaling is rare.  mx: of the tokens
  // in this half of the wave, unscaled
  auto refer_to = [&](float mx, auto at_last) ROWS_INLINE {
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = max_nan(__uint_as_float(x[0]), __uint_as_float(x[1])) * p.scale_log2;
    const bool up = mx > m_run + 8.f;                       // also true of the first finite maximum
    const bool any = __any(up);
    at_last();
    if (any) {
      const float a = up ? fast_exp2(m_run - mx) : 1.f;
      if (up) m_run = mx;
      l_run *= a;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[db][e] *= a;
    }
  };
  auto refer = [&](const f32x16 (&s)[TB]) ROWS_INLINE {
    float sv[SN];
#pragma unroll
    for (int e = 0; e < SN; ++e) sv[e] = s[e / 16][e % 16];
    refer_to(max_nan_of(sv), []() ROWS_INLINE {});
  };
  // Logits become weights: fp32 in place, for bf16 pairs in pk.  For the matrix unit P is rounded to bf16, and the denominator sums the
  // same rounded values: a token that has nearly all the weight keeps its row of V.
  auto weights = [&](f32x16 (&s)[TB], unsigned (&pk)[SN / 2]) ROWS_INLINE {
    const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < SN; ++e) {
        s[e / 16][e % 16] = fast_exp2(fmaf(s[e / 16][e % 16], p.scale_log2, neg_m));
        l_run += s[e / 16][e % 16];
      }
    } else {
      const rows_bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
      for (int i = 0; i < SN / 2; ++i) {
        const rows_f32x2 x = {fast_exp2(fmaf(s[i / 8][(2 * i) % 16], p.scale_log2, neg_m)),
                              fast_exp2(fmaf(s[i / 8][(2 * i + 1) % 16], p.scale_log2, neg_m))};
        const rows_bf16x2 r = __builtin_convertvector(x, rows_bf16x2);
        pk[i] = __builtin_bit_cast(unsigned, r);
        l_run = __builtin_amdgcn_fdot2_f32_bf16(r, ones, l_run, false);
      }
    }
  };
  // V^T's operand of d block db: bf16 16 tokens (two transposing reads, eight rows apart: the rows' swizzle differs in one bit), fp32
  // channel j and the token that register e holds in this half
  auto v_bf16 = [&](unsigned Vt, int db, int ks) ROWS_INLINE {
    const rows_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(ROWS_LDS(rows_s16x4, (Vt + v_off) ^ (64 * db)) + 16 * ks * ROWB / 8);
    const rows_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(ROWS_LDS(rows_s16x4, (Vt + v_off) ^ (64 * db + 32)) + (16 * ks + 8) * ROWB / 8);
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto bit_of = [](int e) ROWS_INLINE { return e % 16 / 4 * 8 + e % 4; };         // token of logit e: e / 16 * 32 + bit_of(e) + 4 h
  const unsigned v32_off = 4 * h * ROWB + (((j >> 2) ^ (h << 3)) * 16) + (j & 3) * 4;
  auto v_f32 = [&](unsigned Vt, int db, int e) ROWS_INLINE {            // (the swizzle of the token's row, apart from its part in v32_off, and 8 db pieces)
    const unsigned flip = 128 * db + ((e % 16 / 4 & 1) << 6 | (e & 3) << 4);
    return *(ROWS_LDS(const float, (Vt + v32_off) ^ flip) + (e / 16 * 32 + e % 16 / 4 * 8 + e % 4) * ROWB / 4);
  };
  // O^T += V^T P^T
  auto values = [&](unsigned Vt, const f32x16 (&s)[TB], const unsigned (&pk)[SN / 2]) ROWS_INLINE {
    constexpr int N = DB * (F32 ? SN : SN / 8), AH = F32 ? 16 : 8;
    typename std::conditional<F32, float, u32x4>::type ahead[AH];
    auto read = [&](int i) ROWS_INLINE {                    // product i: d block i % DB
      if constexpr (F32) return v_f32(Vt, i % DB, i / DB);
      else return v_bf16(Vt, i % DB, i / DB);
    };
#pragma unroll
    for (int i = 0; i < AH && i < N; ++i) ahead[i] = read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (F32) {
        acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x2f32(ahead[i % AH], s[i / DB / 16][i / DB % 16], acc[i % DB], 0, 0, 0);
      } else {
        const int ks = i / DB;
        const u32x4 pr = {pk[4 * ks], pk[4 * ks + 1], pk[4 * ks + 2], pk[4 * ks + 3]};
        acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ahead[i % AH]), __builtin_bit_cast(bf16x8, pr),
                                                              acc[i % DB], 0, 0, 0);
      }
      if (i + AH < N) ahead[i % AH] = read(i + AH < N ? i + AH : 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // The same where some rows do not see some tokens and V holds infinities or NaN: 0 times one of them would reach the rows that do not
  // see it.  Such entries go as zeros, and each kind is counted for each row among the tokens that it sees.  Rare: written to be short.
  auto values_odd = [&](unsigned Vt, const f32x16 (&s)[TB], const unsigned (&pk)[SN / 2], const unsigned (&vis)[TB]) ROWS_INLINE {
#pragma unroll 1
    for (int db = 0; db < DB; ++db) {
      f32x16 sum;
#pragma unroll 1
      for (int kind = 0; kind < 4; ++kind) {                // the finite entries, inf, -inf, NaN
        f32x16 n;
#pragma unroll
        for (int e = 0; e < 16; ++e) n[e] = 0.f;
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < SN; ++e) {
            const float x = v_f32(Vt, db, e);
            const float a = kind == 0 ? (fabsf(x) < INFINITY ? x : 0.f)
                                      : (kind == 1 ? x == INFINITY : kind == 2 ? x == -INFINITY : x != x) ? 1.f : 0.f;
            n = __builtin_amdgcn_mfma_f32_32x32x2f32(a, kind == 0 ? s[e / 16][e % 16] : vis[e / 16] & 1u << bit_of(e) ? 1.f : 0.f, n, 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int ks = 0; ks < SN / 8; ++ks) {
            const u32x4 x = v_bf16(Vt, db, ks);
            u32x4 a, w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              a[i] = 0;
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const unsigned v = (x[i] >> (16 * y)) & 0xffffu, one = 0x3f80u;
                const bool finite = (v & 0x7f80u) != 0x7f80u;
                const bool hit = kind == 1 ? v == 0x7f80u : kind == 2 ? v == 0xff80u : (v & 0x7fffu) > 0x7f80u;
                a[i] |= (kind == 0 ? (finite ? v : 0u) : hit ? one : 0u) << (16 * y);
              }
              const int e = 8 * ks + 2 * i;
              const unsigned seen = (vis[e / 16] & 1u << bit_of(e) ? 0x3f80u : 0u) | (vis[e / 16] & 2u << bit_of(e) ? 0x3f800000u : 0u);
              w[i] = kind == 0 ? pk[4 * ks + i] : seen;
            }
            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, w), n, 0, 0, 0);
          }
        }
        const float add = kind == 1 ? INFINITY : kind == 2 ? -INFINITY : NAN;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = kind == 0 ? n[e] : n[e] > 0.f ? sum[e] + add : sum[e];
      }
#pragma unroll
      for (int k = 0; k < DB; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[k][e] = k == db ? acc[k][e] + sum[e] : acc[k][e];
    }
  };
  // Whether stage si's V has infinities or NaN, for the whole block: every thread looks at its share, and says so before the barrier
  // behind which everyone asks.
  auto look_for_odd = [&](int si) ROWS_INLINE {
    constexpr int SHARE = SM::kTileBytes / 16 / (WAVES * 64);
    bool odd = false;
#pragma unroll
    for (int i = 0; i < SHARE; ++i) {
      const u32x4 x = *ROWS_LDS(const u32x4, ring_addr + (si % NST) * SM::kStage + SM::kTileBytes + (i * WAVES * 64 + tid) * 16);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        odd |= F32 ? (x[w] & 0x7f800000u) == 0x7f800000u : (x[w] & 0x7f80u) == 0x7f80u || (x[w] & 0x7f800000u) == 0x7f800000u;
    }
    if (odd) *odd_stage = si + 1;                           // (any number of threads, the same value)
  };
  // Stage si is in the LDS.
  auto arrive = [&](int si) ROWS_INLINE {
    const int behind = issued - 1 - si;                     // stages asked for behind it
    if (LATE && behind == 1) wait_vmcnt<PER>();
    else WaitLadder<NST - 1>::template run<PER>(max(behind, 0));
    __syncthreads();
  };

  // One step of the loop below, bf16: the next stage's logits (t), this stage's weights (from s) and their products with V, and the
  // next stage's maxima, in this order of instructions.  LDS reads go out AHEAD products before their use, the first ones of the step
  // behind it among them (`ops` on the way in and out; that stage has landed); the vector unit's work lies evenly between the products,
  // where a step's weights need it.  (Left to itself the compiler reads an operand right before its product and forms the weights between
  // the two runs of products: 16640 x 28 heads x 128 2071 us, like this 1771.)
  constexpr int AHEAD = 4;
  u32x4 ops[AHEAD];
  auto step_bf16 = [&](unsigned Kt, unsigned Vt, unsigned Kt_behind, const f32x16 (&s)[TB], f32x16 (&t)[TB], auto fetch, auto between) ROWS_INLINE {
    constexpr int NK = TB * QN, NV = DB * SN / 8, NP = SN / 2, SPAN = NK + (SN / 8 - 1) * DB, MAX = SN / NV;
    unsigned pk[NP];
    const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
    const rows_bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int tb = 0; tb < TB; ++tb)
#pragma unroll
      for (int e = 0; e < 16; ++e) t[tb][e] = 0.f;
    auto pairs = [&](int slot) ROWS_INLINE {                            // the weights that belong into this slot
#pragma unroll
      for (int x = 0; x < NP; ++x)
        if (x * SPAN / NP == slot) {
          const rows_f32x2 w = {fast_exp2(fmaf(s[x / 8][(2 * x) % 16], p.scale_log2, neg_m)),
                                fast_exp2(fmaf(s[x / 8][(2 * x + 1) % 16], p.scale_log2, neg_m))};
          const rows_bf16x2 r = __builtin_convertvector(w, rows_bf16x2);
          pk[x] = __builtin_bit_cast(unsigned, r);
          l_run = __builtin_amdgcn_fdot2_f32_bf16(r, ones, l_run, false);
          asm volatile("" : "+v"(pk[x]), "+v"(l_run));      // here, and not where the weight is used
        }
    };
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      t[i % TB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ops[i % AHEAD]), qop[i / TB], t[i % TB], 0, 0, 0);
      const int next = i + AHEAD;
      ops[i % AHEAD] = next < NK ? k_piece(Kt, next < NK ? next : 0) : v_bf16(Vt, (next - NK) % DB, (next - NK) / DB);
      pairs(i);
      __builtin_amdgcn_sched_barrier(0);
      if (!LATE && i == 0) fetch();
    }
    between();
    float mx = t[0][0];
    auto product = [&](int i) ROWS_INLINE {
      const int ks = i / DB;
      const u32x4 pr = {pk[4 * ks], pk[4 * ks + 1], pk[4 * ks + 2], pk[4 * ks + 3]};
      acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ops[(NK + i) % AHEAD]), __builtin_bit_cast(bf16x8, pr),
                                                            acc[i % DB], 0, 0, 0);
      const int next = i + AHEAD;
      ops[(NK + i) % AHEAD] = next < NV ? v_bf16(Vt, next % DB, next / DB) : k_piece(Kt_behind, next - NV);
      pairs(NK + i);
      if (LATE && i == 0) fetch();
      if (i >= 1 && i <= NV / 2) {
#pragma unroll
        for (int x = (i - 1) * MAX; x < i * MAX; ++x)
          mx = max_nan(max_nan(mx, t[x / 8][(2 * x) % 16]), t[x / 8][(2 * x) % 16 + 1]);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int i = 0; i <= NV / 2; ++i) product(i);
    refer_to(mx, [&]() ROWS_INLINE {
#pragma unroll
      for (int i = NV / 2 + 1; i < NV; ++i) product(i);
    });
  };

  // ---- the stages that every row sees whole ----
  int si = 0;
  if constexpr (PIPE) {
    // A stage's logits are formed while the one before becomes weights: independent streams for the matrix and the vector unit.
    // Eight waves, two on a SIMD: those with V to fetch are half a step late, so that one of a SIMD's waves is at its logits
    // (much for the vector unit) while the other is at its products with V (little).  Step i: logits of stage i + 1, barrier, products of
    // stage i, barrier.  With the lateness K of stage i is free when the early waves begin step i and V of stage i - 1 when the late
    // ones do; each asks for what goes there beside its products, and waits ahead of the barrier in the step's middle for the K of stage
    // i + 2 (of which the step's end reads the first operands) or the V of stage i + 1.  (In step with each other the waves waited 950 of a
    // step's 3600 cycles for one another.)
    const bool late = LATE && fetch_v;
    if (n_plain > 0) {
      f32x16 s[TB];
      arrive(late ? 0 : 1);
      logits(k_tile(0), s);
      refer(s);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) ops[i] = k_piece(k_tile(1), i);     // (of a stage that may not exist: then not used)
      if (late) __syncthreads();
      auto step = [&](f32x16 (&from)[TB], f32x16 (&to)[TB]) ROWS_INLINE {
        if constexpr (LATE) {
          step_bf16(k_tile(si + 1), v_tile(si), k_tile(si + 2), from, to, [&]() ROWS_INLINE { refill(late ? si - 1 : si); },
                    [&]() ROWS_INLINE { arrive(late ? si + 1 : si + 2); });
          __syncthreads();
        } else {
          arrive(si + 2);
          step_bf16(k_tile(si + 1), v_tile(si), k_tile(si + 2), from, to, [&]() ROWS_INLINE { refill(si - 1); }, []() ROWS_INLINE {});
        }
        ++si;
      };
      while (si + 2 < n_plain) {                            // two at a time: which registers hold which stage is fixed
        f32x16 t[TB];
        step(s, t);
        step(t, s);
      }
      if (si + 1 < n_plain) {
        f32x16 t[TB];
        step(s, t);
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) s[tb] = t[tb];
      }
      if (LATE && !late) __syncthreads();
      unsigned pk[SN / 2];
      weights(s, pk);
      values(v_tile(si), s, pk);
      ++si;
    }
  } else {
    for (; si < n_plain; ++si) {
      arrive(si);
      refill(si - 1);
      f32x16 s[TB];
      unsigned pk[SN / 2];
      logits(k_tile(si), s);
      refer(s);
      weights(s, pk);
      values(v_tile(si), s, pk);
    }
  }
  // ---- the others ----
  for (; si < n_stage; ++si) {
    arrive(si);
    refill(si - 1);
    f32x16 s[TB];
    unsigned pk[SN / 2];
    logits(k_tile(si), s);
    look_for_odd(si);
    // which of the lane's tokens its row sees: bit bit_of(e) of token block e / 16.  (A question for each token by itself became branches:
    // 2.3 us a stage of a tree.)
    unsigned vis[TB];
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) {
      const int n0 = (s_lo + si) * ST + tg * TW + tb * 32 + 4 * h;
      if constexpr (TREE) {
        const int node = n0 - off, before = min(max(-node, 0), 31);     // rows of the context among the block's tokens
        unsigned w = (unsigned)(sees >> min(max(node, 0), 63));
        if (node >= 64) w = 0;
        vis[tb] = w << before | (sees != 0 ? (1u << before) - 1 : 0u);
      } else {
        const int more = lim - n0;                          // (only bits up to 27 are asked for)
        vis[tb] = more < 0 ? 0u : (2u << min(more, 30)) - 1;
      }
    }
#pragma unroll
    for (int e = 0; e < SN; ++e) s[e / 16][e % 16] = vis[e / 16] & 1u << bit_of(e) ? s[e / 16][e % 16] : -INFINITY;
    refer(s);
    weights(s, pk);
    wait_lds();
    __syncthreads();
    if (__builtin_expect(*(volatile int*)odd_stage == si + 1, 0)) values_odd(v_tile(si), s, pk, vis);
    else values(v_tile(si), s, pk);
  }
  wait_vmcnt<0>();                                          // no transfer may still be writing LDS past this point

  // ---- the row's sums, the token groups' states ----
  {
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
    l_run = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  // A wave writes out NI of the row's DB * 4 groups of four channels: of several token groups each takes its part of every row
  constexpr int NI = DB * 4 / TG;
  f32x4 o[NI];
  const int i0 = tg * NI;
  if constexpr (TG > 1) {
    if (h == 0) {
      stat_m[tg * ROWS + rb * 32 + j] = m_run;
      stat_l[tg * ROWS + rb * 32 + j] = l_run;
    }
    __syncthreads();                                        // everyone is done reading the ring
    f32x4* xbuf = (f32x4*)ring;                             // [TG][RB][DB * 4][64]
#pragma unroll
    for (int i = 0; i < DB * 4; ++i)
      xbuf[((tg * RB + rb) * DB * 4 + i) * 64 + lane] =
          (f32x4){acc[i / 4][4 * (i % 4)], acc[i / 4][4 * (i % 4) + 1], acc[i / 4][4 * (i % 4) + 2], acc[i / 4][4 * (i % 4) + 3]};
    __syncthreads();
    float f[TG], mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < TG; ++w) {
      f[w] = stat_m[w * ROWS + rb * 32 + j];
      mm = max_nan(mm, f[w]);
    }
    l_run = 0.f;
#pragma unroll
    for (int w = 0; w < TG; ++w) {
      f[w] = f[w] == -INFINITY ? 0.f : fast_exp2(f[w] - mm);
      l_run = fmaf(f[w], stat_l[w * ROWS + rb * 32 + j], l_run);
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < TG; ++w) o[i] += f[w] * xbuf[((w * RB + rb) * DB * 4 + i0 + i) * 64 + lane];
    }
    m_run = mm;
  } else {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      o[i] = (f32x4){acc[i / 4][4 * (i % 4)], acc[i / 4][4 * (i % 4) + 1], acc[i / 4][4 * (i % 4) + 2], acc[i / 4][4 * (i % 4) + 3]};
  }
  if (row >= R) return;
  const bool nothing = TREE ? sees == 0 : lim < 0;
  if (nothing) {
    m_run = -INFINITY;
    l_run = 0.f;
  }
  const long long at = (long long)(tok0 + qi) * p.H + head;
  if (p.S > 1) {
    const long long slot = (long long)split * p.total_q * p.H + at;
    if (h == 0 && tg == 0) {
      p.part_m[slot] = m_run;
      p.part_l[slot] = l_run;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      f32x4 x = o[i];
      if (nothing) x = (f32x4){0.f, 0.f, 0.f, 0.f};
      *(f32x4*)(p.part_o + slot * D + (i0 + i) * 8 + 4 * h) = x;
    }
    return;
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  T* out = (T*)p.out + at * D + 4 * h;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    f32x4 x = o[i] * inv;
    if (l_run == 0.f) x = (f32x4){0.f, 0.f, 0.f, 0.f};
    if constexpr (F32) {
      *(f32x4*)(out + (i0 + i) * 8) = x;
    } else {
      const rows_f32x2 a = {x[0], x[1]}, b = {x[2], x[3]};
      uint2 w;
      w.x = __builtin_bit_cast(unsigned, __builtin_convertvector(a, rows_bf16x2));
      w.y = __builtin_bit_cast(unsigned, __builtin_convertvector(b, rows_bf16x2));
      *(uint2*)(out + (i0 + i) * 8) = w;
    }
  }
  if (p.lse != nullptr && h == 0 && tg == 0) {
    const long long to = TREE ? ((long long)seq * p.H + head) * p.nodes + qi : (long long)head * p.total_q + tok0 + qi;
    p.lse[to] = (m_run + __log2f(l_run)) * kLn2;
  }
}

// Merge of the S blocks that shared a tile: a wave takes one (token, query head), D / 4 lanes a split's 16-byte pieces, so that 256 / D
// splits are read at once, four of them in a row under way.  (Few rows: a block a row puts them on as many compute units.)  Bound by the
// parts' bytes (3 x 2091 rows x 64 heads x 128: 66 us for 240 MB), few rows by two trips to memory (32 x 16 x 28: 4.6 us).
template <typename T, int D, bool TREE>
__global__ __launch_bounds__(64) void rows_combine(RowsParams p) {
  constexpr int LPR = D / 4, GROUPS = 64 / LPR, PF = 4;
  const int lane = threadIdx.x, g = lane / LPR, vec = lane % LPR;
  const long long n = (long long)p.total_q * p.H, at = blockIdx.x;
  const int tok = (int)(at / p.H), head = (int)(at - (long long)tok * p.H);
  // rows of no sequence stay as they were
  if (!TREE && (tok < p.cu_q[0] || tok >= p.cu_q[p.n_seq])) return;
  float m = -INFINITY, l = 0.f;
  if (lane < p.S) {
    m = p.part_m[lane * n + at];
    l = p.part_l[lane * n + at];
  }
  int n_split = p.S;
  if (TREE && p.deal > 0) {
    n_split = __builtin_amdgcn_readlane(tree_deal(p), __builtin_amdgcn_readfirstlane(tok / p.nodes));
    if (lane >= n_split) {
      m = -INFINITY;
      l = 0.f;
    }
  }
  const float* src = p.part_o + at * D + vec * 4;
  auto piece = [&](int s) { return *(const f32x4*)(src + (long long)min(s, p.S - 1) * n * D); };
  f32x4 ahead[PF];
#pragma unroll
  for (int u = 0; u < PF; ++u) ahead[u] = piece(g + u * GROUPS);
  const float mm = wave_max(m);
  const float w = m == -INFINITY ? 0.f : fast_exp2(m - mm);
  const float den = wave_sum(w * l);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < n_split; s0 += PF * GROUPS) {
    f32x4 now[PF];
#pragma unroll
    for (int u = 0; u < PF; ++u) {
      now[u] = ahead[u];
      ahead[u] = piece(s0 + (PF + u) * GROUPS + g);
    }
#pragma unroll
    for (int u = 0; u < PF; ++u) {
      const float f = __shfl(w, s0 + u * GROUPS + g);
      // (a part of weight 0, too: as 0 times infinity its infinities are seen here as they are inside a block)
      if (s0 + u * GROUPS + g < n_split) o += f * now[u];
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (GROUPS == 4) {
      auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(o[e]), __float_as_uint(o[e]), false, false);
      o[e] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[e]), __float_as_uint(o[e]), false, false);
    o[e] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  if (g == 0) {
    const float inv = den == 0.f ? 0.f : 1.f / den;
    T* to = (T*)p.out + at * D + vec * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) Elem<T>::store(to + e, den == 0.f ? 0.f : o[e] * inv);
  }
  if (p.lse != nullptr && lane == 0) {
    const int i = TREE ? tok % p.nodes : tok;
    p.lse[TREE ? ((long long)(tok / p.nodes) * p.H + head) * p.nodes + i : (long long)head * p.total_q + tok] = (mm + __log2f(den)) * kLn2;
  }
}

// What a block of RB row blocks looks like: token groups, tokens of a wave in a stage, stages.  PAIR: one that leaves room for a second
// on its compute unit (bf16 x 64: two more), which works while the first starts, waits for its first rows or writes its last ones: for
// many blocks of few stages.  (200 prompts of 128 rows, 28 heads x 128: 177 us with 256 rows a block, 126 with 128 in pairs; of 14 x 64 61 and 36, in fp32
// 177 and 101; 16 of 2048, 28 x 128: 541 and 560.)
template <typename T, int D, int RB, bool PAIR>
struct RowsShape {
  static constexpr bool F32 = sizeof(T) == 4, WIDE = D * sizeof(T) > 256;      // WIDE: rows of 512 bytes
  static constexpr bool kThere = PAIR ? RB == 4 && !WIDE : RB == 8 ? !F32 || WIDE : RB > 1 || !WIDE;   // (as the host has them)
  static constexpr int TG = RB == 8 || PAIR ? 1 : RB == 4 || WIDE ? 2 : RB == 2 && D == 128 ? 2 : 4;
  static constexpr int TW = RB == 8 && !F32 ? 64 : 32;
  static constexpr int STAGE = 2 * TG * TW * D * (int)sizeof(T);
  // (bf16 x 128, 64 rows: two stages leave room for a second block, too.  A prompt of 1000 rows, 28 heads, 25.5 -> 22.2 us; 32 of 16 over 3000 66 -> 51)
  static constexpr int NST = RB == 2 && D == 128 || 4 * STAGE > 128 * 1024 ? 2 : 4;
};

template <typename T, int D, int RB, bool PAIR, bool PAGED, bool TREE>
static hipError_t launch_rows_rb(const RowsParams& p, hipStream_t st) {
  using Sh = RowsShape<T, D, RB, PAIR>;
  if constexpr (!Sh::kThere) {
    return hipErrorInvalidValue;
  } else {
    constexpr int smem = RowsSmem<T, D, RB, Sh::TG, Sh::TW, Sh::NST>::total();
    static_assert(!PAIR || 2 * smem <= 160 * 1024, "");
    constexpr auto kernel = attn_rows<T, D, RB, Sh::TG, Sh::TW, Sh::NST, PAGED, TREE>;
    const hipError_t e = allow_dynamic_lds<kernel>(smem);
    if (e != hipSuccess) return e;
    const dim3 grid = p.deal > 0 ? dim3((unsigned)p.tiles_per_seq * p.Hkv, p.deal) : dim3((unsigned)p.n_tiles * p.Hkv, p.S);
    hipLaunchKernelGGL(kernel, grid, dim3(RB * Sh::TG * 64), smem, st, p);
    return hipGetLastError();
  }
}

template <typename T, int D, bool PAGED, bool TREE>
static hipError_t launch_rows_d(const RowsParams& p, const RowsPlan& pl, hipStream_t st) {
  hipError_t e;
  switch (pl.rb) {
    case 8: e = launch_rows_rb<T, D, 8, false, PAGED, TREE>(p, st); break;
    case 4: e = pl.pair ? launch_rows_rb<T, D, 4, true, PAGED, TREE>(p, st) : launch_rows_rb<T, D, 4, false, PAGED, TREE>(p, st); break;
    case 2: e = launch_rows_rb<T, D, 2, false, PAGED, TREE>(p, st); break;
    case 1: e = launch_rows_rb<T, D, 1, false, PAGED, TREE>(p, st); break;
    default: return hipErrorInvalidValue;
  }
  if (e != hipSuccess || p.S == 1) return e;
  hipLaunchKernelGGL((rows_combine<T, D, TREE>), dim3((unsigned)((long long)p.total_q * p.H)), dim3(64), 0, st, p);
  return hipGetLastError();
}

template <bool TREE>
static hipError_t launch_rows(const RowsParams& p, const RowsPlan& pl, int dtype, int head_dim, hipStream_t st) {
  const bool paged = p.block_table != nullptr, bf16 = dtype == HIPPO_DTYPE_BF16;
  if (head_dim == 128) {
    if (bf16) return paged ? launch_rows_d<uint16_t, 128, true, TREE>(p, pl, st) : launch_rows_d<uint16_t, 128, false, TREE>(p, pl, st);
    return paged ? launch_rows_d<float, 128, true, TREE>(p, pl, st) : launch_rows_d<float, 128, false, TREE>(p, pl, st);
  }
  if (bf16) return paged ? launch_rows_d<uint16_t, 64, true, TREE>(p, pl, st) : launch_rows_d<uint16_t, 64, false, TREE>(p, pl, st);
  return paged ? launch_rows_d<float, 64, true, TREE>(p, pl, st) : launch_rows_d<float, 64, false, TREE>(p, pl, st);
}

hipError_t launch_prefill(const RowsParams& p, const RowsPlan& pl, int dtype, int head_dim, hipStream_t st);
hipError_t launch_tree(const RowsParams& p, const RowsPlan& pl, int dtype, int head_dim, hipStream_t st);

}  // namespace hippo
