// Log probabilities of given words under rows of logits, the rows' entropies and their most likely words.
//
// With y_v = x_v / T, M = max x and t_v = (x_v - M) / T <= 0:
//   Z = sum_v exp(t_v),  log p_v = t_v - log Z,  H = -sum_v p_v log p_v = log Z - (sum_v exp(t_v) t_v) / Z
// so one pass that keeps the running maximum, sum and weighted sum serves all three (sums in log2 units, rescaled when the
// maximum moves).  Neither term of H is negative, so nothing cancels.  The words that equal the maximum are counted and not
// summed, and log Z is log1p(count - 1 + rest): of a row whose best word has nearly all the weight, 1 + rest in 32 bits would keep
// few bits of the rest, which is all that the entropy and the best word's log probability consist of.
//
// Bound by HBM for many rows of fp32, about equally by the vector unit for bf16 (an exponential costs four issue slots of some
// eleven a word), by latency for few rows.  Grid: (row, range of the row); a block walks its range in chunks of 32 words a
// thread, the next chunk on its way while one is summed.  Where ranges are several, a second launch merges a row's.
#include <algorithm>

#include "common.h"

namespace hippo {

namespace {

constexpr int kWordBits = 20;                       // vocabularies of up to 2^20 words
constexpr int kWordMask = (1 << kWordBits) - 1;
static_assert(kLpMaxVocab <= 1 << kWordBits, "a word's number fits its bits");
constexpr int kListCap = 192;                       // a wave's candidates: three a lane
constexpr int kPerThread = 32;                      // words of a chunk in a thread's registers
constexpr float kNoWeight = -150.f;                 // 2^-150 is 0 in fp32, and times itself no NaN as -inf's would be

// (larger value, then lower word) as larger 52-bit integers, all above 0.  -0 is 0; a NaN ranks as -inf.
__device__ __forceinline__ unsigned long long candidate(float x, int word) {
  x = fmaxf(x, -INFINITY);
  unsigned u = __float_as_uint(x);
  if ((u << 1) == 0u) u = 0u;
  u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return ((unsigned long long)u << kWordBits) | (unsigned)(kWordMask - word);
}
__device__ __forceinline__ int candidate_word(unsigned long long c) { return kWordMask - (int)(c & kWordMask); }
__device__ __forceinline__ float candidate_value(unsigned long long c) {
  const unsigned u = (unsigned)(c >> kWordBits);
  return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u);
}
// the next larger float; of +inf a NaN, which no word exceeds
__device__ __forceinline__ float next_above(float x) {
  if (x == 0.f) return __uint_as_float(1u);
  const unsigned u = __float_as_uint(x);
  return __uint_as_float((u & 0x80000000u) ? u - 1u : u + 1u);
}

// what this wave's lanes wrote to LDS is there for its other lanes (a wave's LDS operations complete in order: this keeps the
// compiler from moving them)
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ int lanes_below(unsigned long long mask) {
  return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
}

// the k-th largest of the wave's PER values a lane (0: no value), k at most their number: its bits from the top down to LAST, zeros
// below them
template <int LAST, int PER>
__device__ __forceinline__ unsigned long long kth_largest(const unsigned long long (&v)[PER], int k) {
  unsigned long long at = 0;
#pragma unroll 1
  for (int bit = 32 + kWordBits - 1; bit >= LAST; --bit) {
    const unsigned long long want = at | (1ull << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += __popcll(__ballot(v[i] >= want));
    if (n >= k) at = want;
  }
  return at;
}

// A wave's candidates, in LDS.
struct Candidates {
  unsigned long long* list;      // [kListCap]
  int count = 0;
  float at_least = -INFINITY;    // words below it are not among the n best of this wave

  // keeps the n best of more than n; their least
  __device__ __forceinline__ unsigned long long keep(int n, int lane) {
    wave_lds_sync();
    unsigned long long v[kListCap / 64];
#pragma unroll
    for (int i = 0; i < kListCap / 64; ++i) v[i] = i * 64 + lane < count ? list[i * 64 + lane] : 0ull;
    const unsigned long long least = kth_largest<0>(v, n);
    wave_lds_sync();
    int at = 0;
#pragma unroll
    for (int i = 0; i < kListCap / 64; ++i) {
      const unsigned long long kept = __ballot(v[i] >= least);
      if (v[i] >= least) list[at + lanes_below(kept)] = v[i];
      at += __popcll(kept);
    }
    count = at;
    wave_lds_sync();
    return least;
  }

  // VEC words a lane, those of lane l from word0 + VEC l on: all of them behind the words that were added before
  template <int VEC>
  __device__ __forceinline__ void add(const float* x, int word0, int n_words, int n, int lane) {
    bool cut = false;
    float edge = at_least;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const int word = word0 + lane * VEC + e;
      const float v = fmaxf(x[e], -INFINITY);
      const bool in = v >= edge && word < n_words;
      const unsigned long long mask = __ballot(in);
      if (mask == 0ull) continue;
      if (count + 64 > kListCap) {
        // (a word equal to the least may still come, with a lower number)
        edge = fmaxf(edge, candidate_value(keep(n, lane)));
        cut = true;
      }
      if (in) list[count + lanes_below(mask)] = candidate(v, word);
      count += __popcll(mask);
    }
    if (cut) at_least = next_above(edge);        // of later words, which have higher numbers, only larger ones count
  }
};

// {maximum, sum of the others' weights, words at the maximum, weighted sum} relative to the maximum, and their union
struct Stat {
  float m, z, n, w;
};
__device__ __forceinline__ void move_reference(Stat& s, float m, float c) {     // m > s.m
  const float d = s.m == -INFINITY ? 0.f : fmaxf((s.m - m) * c, kNoWeight);
  const float a = s.m == -INFINITY ? 0.f : fast_exp2(d);
  const float all = s.z + s.n;
  s.w = a * fmaf(all, d, s.w);
  s.z = a * all;
  s.n = 0.f;
  s.m = m;
}
__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
  const float m = fmaxf(a.m, b.m);
  if (a.m < m) move_reference(a, m, c);
  if (b.m < m) move_reference(b, m, c);
  return Stat{m, a.z + b.z, a.n + b.n, a.w + b.w};
}

__device__ __forceinline__ float log_total(const Stat& s) { return log1pf((s.n - 1.f) + s.z); }
__device__ __forceinline__ float log_prob(float x, const Stat& s, float log_z, float inv_t) {
  if (s.m == -INFINITY || x == -INFINITY) return s.z != s.z ? s.z : -INFINITY;     // (a row of NaN and -inf)
  return (x - s.m) * inv_t - log_z;
}
__device__ __forceinline__ float entropy_of(const Stat& s, float log_z) {
  if (s.m == -INFINITY) return s.z != s.z ? s.z : 0.f;
  return log_z - s.w * kLn2 / (s.z + s.n);
}

// Ranks `total` candidates of LDS (0: none) by counting and leaves the n best in `best`, in order; by all threads of the block.
template <int THREADS>
__device__ __forceinline__ void rank_best(const unsigned long long* all, int total, int n, unsigned long long* best) {
  const int tid = threadIdx.x;
  if (tid < n) best[tid] = 0ull;
  __syncthreads();
  for (int i = tid; i < total; i += THREADS) {
    const unsigned long long mine = all[i];
    if (mine == 0ull) continue;
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < total; ++j) rank += all[j] > mine ? 1 : 0;
    if (rank < n) best[rank] = mine;
  }
  __syncthreads();
}

// the row's outputs from its statistics and best words
template <typename T>
__device__ __forceinline__ void write_row(const LogprobParams& p, int row, const Stat& s, const unsigned long long* best) {
  const int tid = threadIdx.x;
  const float log_z = log_total(s);
  if (tid == 0) {
    const int word = p.tokens[row];
    float lp = s.z != s.z ? s.z : -INFINITY;          // no word of the vocabulary has no probability
    if (word >= 0 && word < p.V) lp = log_prob(Elem<T>::load(static_cast<const T*>(p.logits) + row * p.stride + word), s, log_z, p.inv_t);
    p.logprob[row] = lp;
    p.entropy[row] = entropy_of(s, log_z);
  }
  if (tid < p.n_top) {
    p.top_ids[(long long)row * p.n_top + tid] = candidate_word(best[tid]);
    p.top_logprobs[(long long)row * p.n_top + tid] = log_prob(candidate_value(best[tid]), s, log_z, p.inv_t);
  }
}

template <typename T, int THREADS, bool TOP>
__global__ __launch_bounds__(THREADS) void lp_rows(LogprobParams p) {
  constexpr int VEC = Elem<T>::kPerVec, NV = kPerThread / VEC, WAVES = THREADS / 64;
  constexpr int CHUNK = THREADS * kPerThread;
  __shared__ Stat sh_stat[WAVES];
  __shared__ unsigned long long sh_list[TOP ? WAVES * kListCap : 1];
  __shared__ unsigned long long sh_all[TOP ? WAVES * kLpMaxTop : 1];
  __shared__ unsigned long long sh_best[kLpMaxTop];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x / p.n_range, range = blockIdx.x - row * p.n_range;
  const T* base = static_cast<const T*>(p.logits) + row * p.stride;
  const int v_lo = range * p.range_words, v_hi = min(v_lo + p.range_words, p.V);

  auto fetch = [&](int v0, u32x4 (&raw)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int word = v0 + (j * THREADS + tid) * VEC;
      if (word + VEC <= v_hi) {
        raw[j] = *reinterpret_cast<const u32x4*>(base + word);
      } else {                                          // the row's end, word by word; -inf behind it
        raw[j] = sizeof(T) == 2 ? (u32x4){0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}
                                : (u32x4){0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u};
        if (word < v_hi) {
          T at[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) at[e] = word + e < v_hi ? base[word + e] : T(0);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            if (word + e >= v_hi) continue;
            if constexpr (sizeof(T) == 2)
              raw[j][e / 2] = (raw[j][e / 2] & (e % 2 ? 0x0000ffffu : 0xffff0000u)) | ((unsigned)at[e] << (16 * (e % 2)));
            else
              raw[j][e] = __float_as_uint(at[e]);
          }
        }
      }
    }
  };

  Stat s{-INFINITY, 0.f, 0.f, 0.f};
  Candidates cand;
  cand.list = sh_list + (TOP ? wave * kListCap : 0);
  float lane_best = -INFINITY;                          // of all this lane's words so far
  u32x4 ahead[NV];
  fetch(v_lo, ahead);
  for (int v0 = v_lo; v0 < v_hi; v0 += CHUNK) {
    float x[kPerThread], top[NV], most = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j) Elem<T>::unpack(ahead[j], &x[j * VEC]);
    if (v0 + CHUNK < v_hi) fetch(v0 + CHUNK, ahead);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      top[j] = -INFINITY;                               // (fmaxf takes no NaN)
#pragma unroll
      for (int e = 0; e < VEC; ++e) top[j] = fmaxf(top[j], x[j * VEC + e]);
      most = fmaxf(most, top[j]);
    }
    // the reference is the wave's largest word so far
    if (__any(most > s.m)) move_reference(s, wave_max(fmaxf(most, s.m)), p.c);
    const float ref = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const bool at_top = __any(top[j] == s.m);         // few vectors hold a word at the maximum
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float v = x[j * VEC + e];
        const float t = max_nan((v - ref) * p.c, kNoWeight);
        const float weight = fast_exp2(t);
        s.w = fmaf(weight, t, s.w);
        if (at_top) {
          s.z += v == s.m ? 0.f : weight;
          s.n += v == s.m ? 1.f : 0.f;
        } else {
          s.z += weight;
        }
      }
    }
    if constexpr (TOP) {
      const unsigned long long promising = __ballot(most >= cand.at_least);
      if (promising != 0ull) {
        // n lanes' largest words are n words: none below the least of the n largest of them is among the n best
        lane_best = fmaxf(lane_best, most);
        if (__popcll(promising) >= 8) {
          // (to 16 bits, which all but tells bf16 words apart)
          const unsigned long long one[1] = {candidate(lane_best, kWordMask)};
          cand.at_least = fmaxf(cand.at_least, candidate_value(kth_largest<kWordBits + 16>(one, p.n_top)));
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (__any(top[j] >= cand.at_least))
            cand.template add<VEC>(&x[j * VEC], v0 + (j * THREADS + wave * 64) * VEC, v_hi, p.n_top, lane);
      }
    }
  }

  // the lanes' sums (they share the reference), then the waves'
  s.z = wave_sum(s.z);
  s.n = wave_sum(s.n);
  s.w = wave_sum(s.w);
  if (lane == 0) sh_stat[wave] = s;
  if constexpr (TOP) {
    if (cand.count > p.n_top) cand.keep(p.n_top, lane);
    wave_lds_sync();
    if (lane < p.n_top) sh_all[wave * p.n_top + lane] = lane < cand.count ? cand.list[lane] : 0ull;
  }
  __syncthreads();
  s = sh_stat[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) s = join(s, sh_stat[w], p.c);
  if constexpr (TOP) rank_best<THREADS>(sh_all, WAVES * p.n_top, p.n_top, sh_best);
  if (p.n_range == 1) {
    write_row<T>(p, row, s, sh_best);
  } else {
    if (tid == 0) reinterpret_cast<Stat*>(p.stats)[blockIdx.x] = s;
    if (TOP && tid < p.n_top) p.best[(long long)blockIdx.x * p.n_top + tid] = sh_best[tid];
  }
}

constexpr int kMergeThreads = 256;
static_assert(kLpMaxRanges <= kMergeThreads, "a thread a range");

// One block a row: the union of its ranges' statistics and of their best words.
template <typename T>
__global__ __launch_bounds__(kMergeThreads) void lp_merge(LogprobParams p) {
  __shared__ Stat sh_stat[kMergeThreads / 64];
  __shared__ unsigned long long sh_all[kLpMaxRanges * kLpMaxTop];
  __shared__ unsigned long long sh_best[kLpMaxTop], sh_edge;
  __shared__ int sh_count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x;
  Stat s{-INFINITY, 0.f, 0.f, 0.f};
  if (tid < p.n_range) s = reinterpret_cast<const Stat*>(p.stats)[(long long)row * p.n_range + tid];
  const unsigned long long* best = p.best + (long long)row * p.n_range * p.n_top;
  // Every range's words are in order: none below the largest of the ranges' last is among the row's best.
  unsigned long long last = 0;
  if (p.n_top > 0 && tid < p.n_range) last = best[(long long)tid * p.n_top + p.n_top - 1];
  if (tid == 0) { sh_edge = 0ull; sh_count = 0; }
  const float m = wave_max(s.m);
  if (s.m < m) move_reference(s, m, p.c);
  s.m = m;
  s.z = wave_sum(s.z);
  s.n = wave_sum(s.n);
  s.w = wave_sum(s.w);
  if (lane == 0) sh_stat[wave] = s;
  __syncthreads();
  s = sh_stat[0];
#pragma unroll
  for (int w = 1; w < kMergeThreads / 64; ++w) s = join(s, sh_stat[w], p.c);
  if (p.n_top > 0) {
    if (last != 0ull) atomicMax(&sh_edge, last);
    __syncthreads();
    const unsigned long long edge = sh_edge;
    for (int i = tid; i < p.n_range * p.n_top; i += kMergeThreads) {
      const unsigned long long c = best[i];
      if (c != 0ull && c >= edge) sh_all[atomicAdd(&sh_count, 1)] = c;       // (any order: they are ranked)
    }
    __syncthreads();
    rank_best<kMergeThreads>(sh_all, sh_count, p.n_top, sh_best);
  }
  write_row<T>(p, row, s, sh_best);
}

template <typename T>
hipError_t launch_typed(const LogprobParams& p, hipStream_t st) {
  const unsigned blocks = (unsigned)p.R * (unsigned)p.n_range;
  if (p.wide) {
    if (p.n_top > 0) lp_rows<T, kLpWide, true><<<blocks, kLpWide, 0, st>>>(p);
    else lp_rows<T, kLpWide, false><<<blocks, kLpWide, 0, st>>>(p);
  } else {
    if (p.n_top > 0) lp_rows<T, kLpThreads, true><<<blocks, kLpThreads, 0, st>>>(p);
    else lp_rows<T, kLpThreads, false><<<blocks, kLpThreads, 0, st>>>(p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_range == 1) return e;
  lp_merge<T><<<(unsigned)p.R, kMergeThreads, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

// How a row is cut: `wide` blocks of 1024 threads while one takes the row in a chunk and the rows leave compute units free, ...
void logprob_plan(int rows, int vocab, int* n_range, int* range_words, bool* wide) {
  *wide = vocab <= kLpWide * kPerThread && rows <= kNumCU;
  const int chunk = kLpThreads * kPerThread;
  const int chunks = (vocab + chunk - 1) / chunk;
  int n = 1;
  if (!*wide) n = std::max(1, std::min(chunks, (4 * kNumCU + rows - 1) / rows));
  const int per = (chunks + n - 1) / n;              // chunks of a range
  *n_range = *wide ? 1 : (chunks + per - 1) / per;
  *range_words = *wide ? vocab : per * chunk;
}

hipError_t launch_logprobs(const LogprobParams& p, int dtype, hipStream_t st) {
  return dtype == HIPPO_DTYPE_BF16 ? launch_typed<uint16_t>(p, st) : launch_typed<float>(p, st);
}

}  // namespace hippo
