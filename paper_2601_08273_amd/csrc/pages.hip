// Pages of a paged cache: what a step's new rows need, from the requests' lengths (hippo_plan_pages), and the copy of their K and V
// into the pages (hippo_write_kv_paged).
#include <algorithm>

#include "common.h"

namespace hippo {

// =================================================================================================
// plan
// =================================================================================================
// One launch.  Every block scans all the requests for itself (two rounds of prefix sums over at most 4096 of them: what is asked for
// and given back, then what of it is admitted), and then takes its share of one list: the tokens, the pages handed out, the pages
// given back.  An item finds its request by bisection of a prefix sum in the LDS; a thread has one item of a step of the usual size, as
// a second one is another trip to memory.  No block waits for another's writes: a page handed out is looked
// up on the stack of free pages or, where this call put it there, in the table that it came from; only entries that no block
// reads are written (a request either grows or gives back).  Two launches, the scans and then the lists, would cost a launch; the
// scans cost a block about 3 us, of which the loads of the lengths are most.  256 requests of a step, 48 prompts of
// up to 8192 tokens: 5.0 and 4.7 us.
constexpr int kPlanMany = 1 << 30;     // sums stop here: no stack of pages and no step is that large

struct PlanSums {                      // of the requests up to and with one
  int given, pages, tokens;
};

// Inclusive prefix sums over the block of three values of at most 2^22 each, behind `carry`, which moves on.
template <int THREADS>
__device__ __forceinline__ PlanSums plan_scan(PlanSums v, PlanSums* carry, int (*totals)[3]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int in[3] = {v.given, v.pages, v.tokens};
  int incl[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) incl[i] = (int)wave_scan_incl((unsigned)in[i]);
  __syncthreads();                     // the totals of the scan before are read
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < 3; ++i) totals[wave][i] = incl[i];
  __syncthreads();
  int before[3] = {carry->given, carry->pages, carry->tokens}, all[3] = {before[0], before[1], before[2]};
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (w == wave) before[i] = all[i];
      all[i] = min(all[i] + totals[w][i], kPlanMany);
    }
  *carry = {all[0], all[1], all[2]};
  return {min(before[0] + incl[0], kPlanMany), min(before[1] + incl[1], kPlanMany), min(before[2] + incl[2], kPlanMany)};
}

// the first of n ascending sums that exceeds x (there is one)
__device__ __forceinline__ int plan_find(const int* sums, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

struct PlanRequest {
  int ctx, held, want, after;          // rows and pages now, pages and rows then
  bool grows;
};
__device__ __forceinline__ PlanRequest plan_request(const PlanParams& p, int ctx, int add) {
  PlanRequest r;
  r.ctx = max(ctx, 0);
  const long long after = max((long long)r.ctx + add, 0ll), mask = (1 << p.page_shift) - 1;
  r.held = (int)(((long long)r.ctx + mask) >> p.page_shift);
  const long long want = (after + mask) >> p.page_shift;
  r.grows = add >= 0 && want <= p.max_pages;
  r.want = (int)min(want, (long long)kPlanMany);
  r.after = (int)min(after, (long long)0x7fffffff);
  return r;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void plan_pages(PlanParams p) {
  extern __shared__ int plan_lds[];
  __shared__ int totals[THREADS / 64][3];
  const int tid = threadIdx.x, B = p.B;
  int* tok_incl = plan_lds;                                 // tokens of the admitted requests up to and with each
  int* pg_incl = plan_lds + B;                              // pages
  int* given_incl = plan_lds + 2 * B;                       // pages given back
  int* ctx_of = plan_lds + 3 * B;
  const int n_free = min(max(*p.n_free, 0), p.n_pool);

  // ---- what is asked for and given back ----
  PlanSums carry = {0, 0, 0};
  for (int b0 = 0; b0 < B; b0 += THREADS) {
    const int b = b0 + tid;
    PlanSums v = {0, 0, 0};
    int ctx = 0;
    if (b < B) {
      const int add = p.new_lens[b];
      const PlanRequest r = plan_request(p, p.ctx_lens[b], add);
      ctx = r.ctx;
      if (add < 0) v.given = max(min(r.held, p.max_pages) - min(r.want, p.max_pages), 0);
      if (r.grows) {
        v.pages = max(r.want - r.held, 0);
        v.tokens = min(add, p.max_tokens + 1);              // (more than there are slots for is refused, however many)
      }
    }
    const PlanSums s = plan_scan<THREADS>(v, &carry, totals);
    if (b < B) {
      ctx_of[b] = ctx;
      given_incl[b] = s.given;
      pg_incl[b] = s.pages;
      tok_incl[b] = s.tokens;
    }
  }
  const int n_given = carry.given, available = min(n_free + n_given, p.n_pool);

  // ---- what of it is admitted: as long as pages and slots last, in the order of the requests ----
  carry = {0, 0, 0};
  for (int b0 = 0; b0 < B; b0 += THREADS) {
    const int b = b0 + tid;
    PlanSums v = {0, 0, 0};
    if (b < B) {
      const int add = p.new_lens[b];
      const PlanRequest r = plan_request(p, ctx_of[b], add);
      const int pages = r.grows ? max(r.want - r.held, 0) : 0;
      const bool admitted = r.grows && (pages == 0 || pg_incl[b] <= available) && (add == 0 || tok_incl[b] <= p.max_tokens);
      if (admitted) {
        v.pages = pages;
        v.tokens = add;
      }
      if (blockIdx.x == 0) p.kv_lens[b] = admitted || add < 0 ? r.after : r.ctx;
    }
    const PlanSums s = plan_scan<THREADS>(v, &carry, totals);
    if (b < B) {
      pg_incl[b] = s.pages;
      tok_incl[b] = s.tokens;
      if (blockIdx.x == 0) p.cu_q[b + 1] = s.tokens;
    }
  }
  const int n_pages = carry.pages, n_tokens = carry.tokens;
  if (blockIdx.x == 0 && tid == 0) {
    p.cu_q[0] = 0;
    *p.n_free_out = available - n_pages;
  }
  __syncthreads();

  // the page given back as number i of this call
  auto given_page = [&](int i) {
    const int b = plan_find(given_incl, B, i);
    const PlanRequest r = plan_request(p, ctx_of[b], p.new_lens[b]);
    return p.block_table[(long long)b * p.max_pages + r.want + i - (b > 0 ? given_incl[b - 1] : 0)];
  };
  // the page handed out as number g
  auto page_of = [&](int g) {
    const int at = available - 1 - g;
    return at >= n_free ? given_page(at - n_free) : p.free_pages[at];
  };
  const int pushed = available - n_free;                    // (more only where the stack holds pages twice)
  const int step = gridDim.x * THREADS;                     // (the three counts and a step stay below 2^31)
  for (int i = blockIdx.x * THREADS + tid; i < p.max_tokens + n_pages + pushed; i += step) {
    if (i < p.max_tokens) {
      int slot = -1, position = -1;
      if (i < n_tokens) {
        const int b = plan_find(tok_incl, B, i);
        const int held = (int)(((long long)ctx_of[b] + (1 << p.page_shift) - 1) >> p.page_shift);
        position = ctx_of[b] + i - (b > 0 ? tok_incl[b - 1] : 0);
        const int column = position >> p.page_shift;
        const int page = column < held ? p.block_table[(long long)b * p.max_pages + column]
                                       : page_of((b > 0 ? pg_incl[b - 1] : 0) + column - held);
        if (page >= 0 && page < p.n_pool) slot = (page << p.page_shift) + (position & ((1 << p.page_shift) - 1));
      }
      p.slots[i] = slot;
      p.positions[i] = position;
    } else if (i < p.max_tokens + n_pages) {
      const int g = i - p.max_tokens, b = plan_find(pg_incl, B, g);
      const int held = (int)(((long long)ctx_of[b] + (1 << p.page_shift) - 1) >> p.page_shift);
      p.block_table[(long long)b * p.max_pages + held + g - (b > 0 ? pg_incl[b - 1] : 0)] = page_of(g);
    } else {
      const int g = i - p.max_tokens - n_pages;
      p.free_pages[n_free + g] = given_page(g);
    }
  }
}

template <int THREADS>
static hipError_t launch_plan(const PlanParams& p, hipStream_t st) {
  const hipError_t e = allow_dynamic_lds<plan_pages<THREADS>>(4 * kPlanMaxBatch * (int)sizeof(int));
  if (e != hipSuccess) return e;
  // a thread for every token and two pages a request, while they are on the chip together
  const int blocks = std::min(1024 / (THREADS / 256), (p.max_tokens + 2 * p.B + THREADS - 1) / THREADS);
  hipLaunchKernelGGL(plan_pages<THREADS>, dim3(blocks), dim3(THREADS), 4 * p.B * (int)sizeof(int), st, p);
  return hipGetLastError();
}
hipError_t launch_plan_pages(const PlanParams& p, hipStream_t st) {
  return p.B <= 512 ? launch_plan<256>(p, st) : launch_plan<1024>(p, st);
}

// =================================================================================================
// write
// =================================================================================================
// Bit copies of 16-byte pieces: piece i of token t's K and V heads goes to row slots[t].  A thread takes the same piece of
// kWriteTokens tokens, so that their loads are under way together.  Bound by bytes (16640 tokens x 4 heads x 128: 11.8 us for 68 MB, found
// in the last-level cache), few tokens by a launch and two trips to memory (256: 3.8).
constexpr int kWriteTokens = 4;

__global__ __launch_bounds__(256) void write_kv(WriteParams p) {
  const int i = blockIdx.x * 256 + threadIdx.x, group = p.by_token(i);         // (the host keeps the threads below 2^31)
  const int piece = i - group * p.Hkv * p.pieces, hk = p.by_head(piece), c = piece - hk * p.pieces;
  const int t0 = group * kWriteTokens;
  u32x4 k[kWriteTokens], v[kWriteTokens];
  long long to[kWriteTokens];
#pragma unroll
  for (int u = 0; u < kWriteTokens; ++u) {
    to[u] = -1;
    if (t0 + u >= p.n_tokens) continue;
    const int slot = p.slots[t0 + u], row = p.rows != nullptr ? p.rows[t0 + u] : t0 + u;
    if (slot < 0 || slot >= p.n_slots || row < 0 || row >= p.n_rows) continue;
    to[u] = (long long)(slot >> p.page_shift) * p.page_stride + (long long)(slot & ((1 << p.page_shift) - 1)) * p.pool_sn +
            hk * p.pool_sh + c * 16;
    const long long from = row * p.sn + hk * p.sh + c * 16;
    k[u] = *(const u32x4*)((const char*)p.k + from);
    v[u] = *(const u32x4*)((const char*)p.v + from);
  }
#pragma unroll
  for (int u = 0; u < kWriteTokens; ++u)
    if (to[u] >= 0) {
      *(u32x4*)((char*)p.k_pool + to[u]) = k[u];
      *(u32x4*)((char*)p.v_pool + to[u]) = v[u];
    }
}

hipError_t launch_write_kv(const WriteParams& p, hipStream_t st) {
  const long long threads = (((long long)p.n_tokens + kWriteTokens - 1) / kWriteTokens) * p.Hkv * p.pieces;
  hipLaunchKernelGGL(write_kv, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace hippo
