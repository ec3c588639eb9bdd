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

// (larger value, then lower word) as larger integers, all above 0.  -0 is 0; words of -inf are no candidates (see write_row).  T's
// bits above kWordBits: 16 of bf16 tell its values apart.
template <typename T> constexpr int kValueBits = sizeof(T) == 2 ? 16 : 32;
template <typename T>
__device__ __forceinline__ unsigned value_key(float x) {
  unsigned u = __float_as_uint(x);
  if ((u << 1) == 0u) u = 0u;
  u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return u >> (32 - kValueBits<T>);
}
template <typename T>
__device__ __forceinline__ float key_value(unsigned key) {
  unsigned u = key << (32 - kValueBits<T>);
  if (!(u & 0x80000000u)) u = ~u & (0xffffffffu << (32 - kValueBits<T>));
  else u &= 0x7fffffffu;
  return __uint_as_float(u);
}
template <typename T>
__device__ __forceinline__ unsigned long long candidate(float x, int word) {
  return ((unsigned long long)value_key<T>(x) << kWordBits) | (unsigned)(kWordMask - word);
}
__device__ __forceinline__ int candidate_word(unsigned long long c) { return kWordMask - (int)(c & kWordMask); }
template <typename T>
__device__ __forceinline__ float candidate_value(unsigned long long c) { return key_value<T>((unsigned)(c >> kWordBits)); }
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

// the k-th largest of the wave's PER numbers a lane, k at most how many are above 0: its bits from FIRST down to LAST, zeros below
template <int FIRST, int LAST, typename I, int PER>
__device__ __forceinline__ I kth_largest(const I (&v)[PER], int k) {
  I at = 0;
#pragma unroll FIRST - LAST < 16 ? 16 : 4
  for (int bit = FIRST; bit >= LAST; --bit) {
    const I want = at | ((I)1 << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += __popcll(__ballot(v[i] >= want));
    at = n >= k ? want : at;
  }
  return at;
}

// x[i], another i in every lane: a tree of bitwise choices (of selects the compiler makes an array in memory)
__device__ __forceinline__ float pick(const float (&x)[kPerThread], int i) {
  unsigned v[kPerThread];
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) v[k] = __float_as_uint(x[k]);
#pragma unroll
  for (int bit = 0; kPerThread >> bit > 1; ++bit) {
    const unsigned odd = (unsigned)((i << (31 - bit)) >> 31);          // all bits of the bit
#pragma unroll
    for (int k = 0; k < kPerThread / 2 >> bit; ++k) v[k] = (v[2 * k + 1] & odd) | (v[2 * k] & ~odd);
  }
  return __uint_as_float(v[0]);
}

constexpr float kLowest = -3.402823466e38f;       // the least word above -inf

// A wave's candidates for the n best words, in LDS, in no order.
template <typename T>
struct Candidates {
  static constexpr int VEC = Elem<T>::kPerVec, NV = kPerThread / VEC;
  unsigned long long* list;      // [kListCap]
  int count = 0;
  float at_least = kLowest;      // words below it are not among the n best of this wave

  // Keeps the n best of more than n; returns the value of the least.
  __device__ __forceinline__ float keep(int n, int lane) {
    wave_lds_sync();
    unsigned long long v[kListCap / 64];
#pragma unroll
    for (int i = 0; i < kListCap / 64; ++i) v[i] = i * 64 + lane < count ? list[i * 64 + lane] : 0ull;
    const unsigned long long least = kth_largest<kWordBits + kValueBits<T> - 1, 0>(v, n);
    wave_lds_sync();
    count = 0;
#pragma unroll
    for (int i = 0; i < kListCap / 64; ++i) {
      const unsigned long long kept = __ballot(v[i] >= least);
      if (v[i] >= least) list[count + lanes_below(kept)] = v[i];
      count += __popcll(kept);
    }
    wave_lds_sync();
    return candidate_value<T>(least);
  }

  // A chunk's words, all of them behind the words of earlier chunks; word_of(i) is the number of x[i].  Every lane marks its words and
  // then gives up one at a time: few lanes have more than one or two, and a branch for each of the words took three times as long.
  template <typename WordOf>
  __device__ __forceinline__ void add(const float (&x)[kPerThread], int n, int lane, WordOf word_of) {
    static_assert(kPerThread == 32, "a mark a word");
    unsigned marks = 0;
#pragma unroll
    for (int i = kPerThread - 1; i >= 0; --i) marks = 2 * marks + (x[i] >= at_least ? 1u : 0u);
    float edge = -INFINITY;
    for (unsigned long long some = __ballot(marks != 0u); some != 0ull; some = __ballot(marks != 0u)) {
      const int i = __ffs(marks) - 1;
      const float v = pick(x, i);
      if (count + 64 > kListCap) edge = keep(n, lane);
      if (marks != 0u) list[count + lanes_below(some)] = candidate<T>(v, word_of(i));
      count += __popcll(some);
      marks &= marks - 1;
    }
    // (of later chunks, whose words have higher numbers, only larger ones than n that are in the list count)
    if (edge > -INFINITY) at_least = fmaxf(at_least, next_above(edge));
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
// the union of WAVES statistics in LDS (a power of two up to 16), in every lane
template <int WAVES>
__device__ __forceinline__ Stat join_waves(const Stat* all, int lane, float c) {
  Stat s = all[lane & (WAVES - 1)];
  float m = s.m;
#pragma unroll
  for (int x = 1; x < WAVES; x *= 2)
    m = fmaxf(m, x == 1 ? dpp_f32<kDppQuadXor1>(m) : x == 2 ? dpp_f32<kDppQuadXor2>(m) : x == 4 ? dpp_f32<kDppRowHalfMirror>(m)
                                                                                           : dpp_f32<kDppRowMirror>(m));
  if (s.m < m) move_reference(s, m, c);
#pragma unroll
  for (int x = 1; x < WAVES; x *= 2) {
    float* v[3] = {&s.z, &s.n, &s.w};
#pragma unroll
    for (int i = 0; i < 3; ++i)
      *v[i] += x == 1 ? dpp_f32<kDppQuadXor1>(*v[i]) : x == 2 ? dpp_f32<kDppQuadXor2>(*v[i]) : x == 4 ? dpp_f32<kDppRowHalfMirror>(*v[i])
                                                                                                      : dpp_f32<kDppRowMirror>(*v[i]);
  }
  s.m = m;
  return s;
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

// ---- sorting candidates: a bitonic network over a wave's lanes, its exchanges inside the vector ALU ----
template <int X>
__device__ __forceinline__ unsigned lane_xor(unsigned v, int lane) {
  if constexpr (X == 1) return dpp_u32<kDppQuadXor1>(v);
  else if constexpr (X == 2) return dpp_u32<kDppQuadXor2>(v);
  else if constexpr (X == 3) return dpp_u32<0x1B>(v);                    // quad_perm [3,2,1,0]
  else if constexpr (X == 4) return lane_xor<3>(lane_xor<7>(v, lane), lane);
  else if constexpr (X == 7) return dpp_u32<kDppRowHalfMirror>(v);
  else if constexpr (X == 8) return dpp_u32<0x128>(v);                   // row_ror:8
  else if constexpr (X == 15) return dpp_u32<kDppRowMirror>(v);
  else if constexpr (X == 16) {
    auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);       // (even rows' value, odd rows')
    return (lane & 16) ? s[0] : s[1];
  } else if constexpr (X == 31) return lane_xor<15>(lane_xor<16>(v, lane), lane);
  else {
    static_assert(X == 63, "an exchange that the network uses");
    auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return lane_xor<31>((lane & 32) ? s[0] : s[1], lane);
  }
}
// lanes l and l ^ X: the larger goes to the one in front
template <int X>
__device__ __forceinline__ void exchange(unsigned long long& v, int lane) {
  const unsigned lo = lane_xor<X>((unsigned)v, lane), hi = lane_xor<X>((unsigned)(v >> 32), lane);
  const unsigned long long other = ((unsigned long long)hi << 32) | lo;
  const bool front = (lane & ((X + 1) & X ? X : (X + 1) / 2)) == 0;
  v = (v > other) == front ? v : other;
}
// lanes 0..31 and 32..63 hold two lists, the largest first: the 32 largest of both into lanes 0..31, the largest first
__device__ __forceinline__ void join_lists(unsigned long long& v, int lane) {
  exchange<63>(v, lane);
  exchange<16>(v, lane); exchange<8>(v, lane); exchange<4>(v, lane); exchange<2>(v, lane); exchange<1>(v, lane);
}
// of `count` in any order, in the lanes in front (zeros behind them): few need few rounds of the network (1 row x 32000, 1 best word,
// 10.7 -> 9.8 us; x 1000, 5 words, 6.2 -> 5.7)
__device__ __forceinline__ void best_of_wave(unsigned long long& v, int count, int lane) {
  exchange<1>(v, lane);
  exchange<3>(v, lane); exchange<1>(v, lane);
  exchange<7>(v, lane); exchange<2>(v, lane); exchange<1>(v, lane);
  if (count <= 8) return;
  exchange<15>(v, lane); exchange<4>(v, lane); exchange<2>(v, lane); exchange<1>(v, lane);
  if (count <= 16) return;
  exchange<31>(v, lane); exchange<8>(v, lane); exchange<4>(v, lane); exchange<2>(v, lane); exchange<1>(v, lane);
  if (count > 32) join_lists(v, lane);
}
// every wave's list in its lanes 0..31 -> the block's 32 best, in order, in lists[0..31]; ends with a barrier
template <int WAVES>
__device__ __forceinline__ void best_of_block(unsigned long long v, unsigned long long* lists, int lane, int wave) {
  if (lane < 32) lists[wave * 32 + lane] = v;
  __syncthreads();
#pragma unroll
  for (int step = 1; step < WAVES; step *= 2) {
    if (wave % (2 * step) == 0) {
      v = lists[(lane < 32 ? wave : wave + step) * 32 + (lane & 31)];
      join_lists(v, lane);
      if (lane < 32) lists[wave * 32 + lane] = v;
    }
    __syncthreads();
  }
}

// the row's token's logit; -inf of a token outside the vocabulary.  Two trips to memory, one behind the other: asked for first.
template <typename T>
__device__ __forceinline__ float token_logit(const LogprobParams& p, int row) {
  const int word = p.tokens[row];
  if (word < 0 || word >= p.V) return -INFINITY;
  return Elem<T>::load(static_cast<const T*>(p.logits) + row * p.stride + word);
}
// the row's outputs from its statistics, the token's logit (of thread 0) and the best words
template <typename T>
__device__ __forceinline__ void write_row(const LogprobParams& p, int row, const Stat& s, float logit, const unsigned long long* best) {
  const int tid = threadIdx.x;
  if (tid >= max(1, p.n_top)) return;
  const float log_z = log_total(s);
  if (tid == 0) {
    p.logprob[row] = log_prob(logit, s, log_z, p.inv_t);
    p.entropy[row] = entropy_of(s, log_z);
  }
  if (tid < p.n_top) {
    int word = candidate_word(best[tid]);
    float x = candidate_value<T>(best[tid]);
    if (best[tid] == 0ull) {
      // Fewer words than n above -inf: all of those are in the list, and the others follow by their numbers, the k-th being the k-th
      // number that is not in the list.
      int found = 0;
      while (found < p.n_top && best[found] != 0ull) ++found;
      const int k = tid - found;
      word = k;
      for (int again = 1; again != 0;) {
        int below = 0;
        for (int i = 0; i < found; ++i) below += candidate_word(best[i]) <= word ? 1 : 0;
        again = k + below - word;
        word = k + below;
      }
      x = -INFINITY;
    }
    p.top_ids[(long long)row * p.n_top + tid] = word;
    p.top_logprobs[(long long)row * p.n_top + tid] = log_prob(x, s, log_z, p.inv_t);
  }
}

template <typename T, int THREADS, bool TOP>
__global__ __launch_bounds__(THREADS, sizeof(T) == 2 ? 5 : 4) void lp_rows(LogprobParams p) {
  constexpr int VEC = Elem<T>::kPerVec, NV = kPerThread / VEC, WAVES = THREADS / 64;
  constexpr int CHUNK = THREADS * kPerThread;
  __shared__ Stat sh_stat[WAVES];
  __shared__ unsigned long long sh_list[TOP ? WAVES * kListCap : 1];
  __shared__ unsigned long long sh_best[TOP ? WAVES * 32 : 1];
  __shared__ unsigned sh_edge;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x / p.n_range, range = blockIdx.x - row * p.n_range;
  const T* base = static_cast<const T*>(p.logits) + row * p.stride;
  const int v_lo = range * p.range_words, v_hi = min(v_lo + p.range_words, p.V);

  auto fetch = [&](int v0, u32x4 (&raw)[NV]) {
    if (v0 + CHUNK <= v_hi) {
#pragma unroll
      for (int j = 0; j < NV; ++j) raw[j] = *reinterpret_cast<const u32x4*>(base + v0 + (j * THREADS + tid) * VEC);
      return;
    }
    // The row's last chunk: -inf behind its end.  (The vector that the end cuts starts at v_hi rounded down and is fetched word by
    // word.)
    const int whole = v_hi / VEC * VEC;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int word = v0 + (j * THREADS + tid) * VEC;
      u32x4 r = {0u, 0u, 0u, 0u};
      if (word + VEC <= v_hi) r = *reinterpret_cast<const u32x4*>(base + word);
      const unsigned none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
      if (word + VEC > v_hi) r = (u32x4){none, none, none, none};
      if (word == whole && word < v_hi) {
#pragma unroll 1
        for (int e = 0; word + e < v_hi; ++e) {
          const unsigned bits = sizeof(T) == 2 ? (unsigned)reinterpret_cast<const uint16_t*>(base)[word + e]
                                               : reinterpret_cast<const unsigned*>(base)[word + e];
          const int at = sizeof(T) == 2 ? e / 2 : e;
          const unsigned keep = sizeof(T) == 4 ? 0u : e % 2 ? 0x0000ffffu : 0xffff0000u;
          const unsigned put = sizeof(T) == 4 ? bits : bits << (16 * (e % 2));
          r.x = at == 0 ? (r.x & keep) | put : r.x;
          r.y = at == 1 ? (r.y & keep) | put : r.y;
          r.z = at == 2 ? (r.z & keep) | put : r.z;
          r.w = at == 3 ? (r.w & keep) | put : r.w;
        }
      }
      raw[j] = r;
    }
  };

  u32x4 ahead[NV];
  fetch(v_lo, ahead);
  float logit = 0.f;
  if (p.n_range == 1 && tid == 0) logit = token_logit<T>(p, row);
  Stat s{-INFINITY, 0.f, 0.f, 0.f};
  Candidates<T> cand;
  cand.list = sh_list + (TOP ? wave * kListCap : 0);
  float lane_best = -INFINITY;                          // of all this lane's words so far
  // What one wave's n-th best word reaches, the block's does: the waves tell each other (a wave that looks too early only takes more
  // candidates).  As integers in their order; 0: nothing yet.
  if (TOP && tid == 0) sh_edge = 0u;
  if constexpr (TOP) __syncthreads();
  for (int v0 = v_lo; v0 < v_hi; v0 += CHUNK) {
    float x[kPerThread], most = -INFINITY;              // (fmaxf takes no NaN)
#pragma unroll
    for (int j = 0; j < NV; ++j) Elem<T>::unpack(ahead[j], &x[j * VEC]);
    if (v0 + CHUNK < v_hi) fetch(v0 + CHUNK, ahead);
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) most = fmaxf(most, x[i]);
    if constexpr (TOP) {
      const unsigned shared = __hip_atomic_load(&sh_edge, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      if (shared != 0u) cand.at_least = fmaxf(cand.at_least, key_value<T>(shared));
      const unsigned long long promising = __ballot(most >= cand.at_least);
      if (promising != 0ull) {
        // n lanes' largest words are n words: none below the least of the n largest of them is among the n best
        lane_best = fmaxf(lane_best, most);
        if (__popcll(promising) >= 8) {
          // (to 16 bits, which tell bf16 words apart)
          // (lanes of -inf alone stand below all others)
          const unsigned one[1] = {lane_best > -INFINITY ? value_key<T>(lane_best) : 0u};
          const unsigned nth = kth_largest<kValueBits<T> - 1, kValueBits<T> - 16>(one, p.n_top);
          if (nth > shared) {
            cand.at_least = fmaxf(cand.at_least, key_value<T>(nth));
            if (WAVES > 1 && lane == 0) atomicMax(&sh_edge, nth);
          }
        }
        cand.add(x, p.n_top, lane, [&](int i) { return v0 + (i / VEC * THREADS + tid) * VEC + i % VEC; });
      }
    }
    // the reference is the wave's largest word so far
    if (__any(most > s.m)) move_reference(s, wave_max(fmaxf(most, s.m)), p.c);
    const float ref = s.m == -INFINITY ? 0.f : s.m;
    if (__any(most == s.m)) {                           // few chunks hold a word at the maximum: counted, and out of the sums
      asm volatile("");                                 // (a branch: as selects this costs every word three instructions)
#pragma unroll
      for (int i = 0; i < kPerThread; ++i) {
        s.n += x[i] == s.m ? 1.f : 0.f;
        x[i] = x[i] == s.m ? -INFINITY : x[i];
      }
    }
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const float t = max_nan((x[i] - ref) * p.c, kNoWeight);
      const float weight = fast_exp2(t);
      s.w = fmaf(weight, t, s.w);
      s.z += weight;
    }
  }

  // the lanes' sums (they share the reference), then the waves'
  s.z = wave_sum(s.z);
  s.n = wave_sum(s.n);
  s.w = wave_sum(s.w);
  if (lane == 0) sh_stat[wave] = s;
  if constexpr (TOP) {
    if (cand.count > 64) cand.keep(p.n_top, lane);
    wave_lds_sync();
    unsigned long long v = lane < cand.count ? cand.list[lane] : 0ull;
    best_of_wave(v, cand.count, lane);
    best_of_block<WAVES>(v, sh_best, lane, wave);        // (and the statistics of all waves are in LDS)
  } else {
    __syncthreads();
  }
  s = join_waves<WAVES>(sh_stat, lane, p.c);
  if (p.n_range == 1) {
    write_row<T>(p, row, s, logit, sh_best);
  } else {
    if (tid == 0) reinterpret_cast<Stat*>(p.stats)[blockIdx.x] = s;
    if (TOP && tid < p.n_top) p.best[(long long)blockIdx.x * p.n_top + tid] = sh_best[tid];
  }
}

constexpr int kMergeThreads = 1024;
static_assert(kLpMaxTop <= 32, "a list fits half a wave");
static_assert(kLpMaxRanges <= kMergeThreads, "a thread a range");

// One block a row: the union of its ranges' statistics and of their best words.  One trip to memory (two for the token's logit).
template <typename T>
__global__ __launch_bounds__(kMergeThreads) void lp_merge(LogprobParams p) {
  constexpr int WAVES = kMergeThreads / 64;
  __shared__ Stat sh_stat[WAVES];
  __shared__ unsigned long long sh_best[WAVES * 32];
  const int tid = threadIdx.x, lane = tid & 63, row = blockIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float logit = 0.f;
  if (tid == 0) logit = token_logit<T>(p, row);
  // wave w takes ranges w, w + WAVES, ..: their lists, which are in order, two at a time
  unsigned long long v = 0ull;
  if (p.n_top > 0) {
    const unsigned long long* best = p.best + (long long)row * p.n_range * p.n_top;
    const int at = lane & 31;
    for (int r = wave; r < p.n_range; r += WAVES) {
      const unsigned long long next = at < p.n_top ? best[(long long)r * p.n_top + at] : 0ull;
      if (r == wave) { v = next; continue; }
      v = lane < 32 ? v : next;
      join_lists(v, lane);
    }
  }
  Stat s{-INFINITY, 0.f, 0.f, 0.f};
  if (tid < p.n_range) s = reinterpret_cast<const Stat*>(p.stats)[(long long)row * p.n_range + tid];
  const float m = wave_max(s.m);
  if (s.m < m) move_reference(s, m, p.c);
  s.m = m;
  s.z = wave_sum(s.z);
  s.n = wave_sum(s.n);
  s.w = wave_sum(s.w);
  if (lane == 0) sh_stat[wave] = s;
  best_of_block<WAVES>(v, sh_best, lane, wave);
  s = join_waves<WAVES>(sh_stat, lane, p.c);
  write_row<T>(p, row, s, logit, sh_best);
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

// How a row is cut, us a call from a graph:
//   Up to 32768 words, beyond a chunk of 256 threads, and up to a row a compute unit: one block of 1024 threads takes the row in a chunk,
//   and there is nothing to join (n_top 5: 200 rows of 32000 words 15.9 -> 12.0, one of 9000 10.2 -> 9.5; but one of 1000 5.9 -> 8.7).
//   Few rows: a chunk a block (6 rows of 152064 words in blocks of one chunk and a join 12; 40 rows in 5 ranges 15.9, in 19 14.4).
//   More, up to 640: six blocks a compute unit and at least three chunks a block (152064 words, n_top 20: 300 rows whole 45.8, in 2
//   ranges 41.6, 4 37.6, 7 37.0; 100 rows 35.1, in 5 and in 19 21.5; but 400 rows of 32000 words whole 16.3, in 2 ranges 21.5).
//   Others whole (n_top 5: 640 rows of 152064 words whole 59.5, in 3 ranges 60.1, 768 61.4 and 69.0, 1000 76 and 85).
void logprob_plan(int rows, int vocab, int* n_range, int* range_words, bool* wide) {
  const int chunk = kLpThreads * kPerThread;
  const int chunks = (vocab + chunk - 1) / chunk;
  *wide = chunks > 1 && vocab <= kLpWide * kPerThread && rows <= kNumCU;
  int n = 1;
  if (!*wide && 2 * rows < 5 * kNumCU) {
    n = std::min(chunks, (6 * kNumCU + rows - 1) / rows);
    if (rows >= kNumCU / 4) n = std::min(n, std::max(1, chunks / 3));
  }
  const int per = (chunks + n - 1) / n;              // chunks of a range
  *n_range = *wide ? 1 : (chunks + per - 1) / per;
  *range_words = *wide ? vocab : per * chunk;
}

hipError_t launch_logprobs(const LogprobParams& p, int dtype, hipStream_t st) {
  return dtype == HIPPO_DTYPE_BF16 ? launch_typed<uint16_t>(p, st) : launch_typed<float>(p, st);
}

}  // namespace hippo
