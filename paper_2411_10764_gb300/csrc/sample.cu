// Draws from rows of scores: temperature, top-k, top-p and min-p cuts, then the
// m largest of score + noise among the kept entries (with Gumbel noise, m draws
// without replacement from the kept entries' softmax).
//
// Entries are ordered by a 59-bit composite: the scaled score as an ordered integer, then the
// index, lower ones first.  No two are equal, and every cut keeps a prefix of this order, so
// the kept set is {composite >= edge}.  An edge is found without sorting the row: one
// pass counts entries (top-k) or adds their probability mass (top-p) in 2,048 bins, linear in
// the score from the row's best down; the bin where the sum reaches its target is
// collected (a few dozen entries as a rule, at most 4,096) and sorted, which settles
// ties by index too.  A bin with more entries (equal or nearly equal scores) is first
// narrowed down by digits of the composite.  The m draws are found the same way from
// composites of score + noise.  Linear bins matter: the leading bits of a float put most
// scores of a vocabulary in two dozen bins, and shared-memory atomics to one address
// take turns (64 rows x 50,021: 177 us with leading bits and 64-bit atomics).
// Masses are added as integers (fixed point), so neither atomics nor the split of a
// row over CTAs changes a result.
//
// Bound: the scores are read from HBM once and from L1 or L2 by the later passes;
// noise is read for kept entries only.  What is left beside the first read is latency: two
// to five passes over a CTA's share and a barrier for each.  Measured, whole calls: 64 rows x
// 50,021 with a rule each 44 us; 8 x 1,048,576, top-k 8,192 and 512 draws, 72 us; one row of
// 16,777,216 with min-p and 1,024 draws 53 to 66 us (its first pass 10.4 us, 6.4 TB/s).
//
// Two kernels:
//   k_sample_warp  rows of up to 512 entries and m <= 32: a warp per row, the row in
//                  registers, selection by ballots and warp sums, no barrier;
//   k_sample_row   longer rows: a team of CTAs per row.  Where there are fewer
//                  rows than SMs the team has several CTAs: a cluster, or where a few
//                  rows have more than 32 each CTAs that meet at a barrier in
//                  global memory (cooperative launch, so all are resident; the wait is
//                  bounded).
#include <atomic>
#include <cfloat>

#include "seq.cuh"

namespace mlt {
namespace {

constexpr int kWarpMaxN = 512;
constexpr int kWarpMaxM = 32;
constexpr int kBins = 2048;
constexpr int kList = 4096;  // composites that are sorted
constexpr int kIndexBits = 27;
constexpr unsigned kNoTies = 0xFFFFFFFFu;

// Order-preserving map of finite floats; -0 as +0.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ float clamp_finite(float v) { return fminf(fmaxf(v, -FLT_MAX), FLT_MAX); }

// Scaled score, finite; -infinity where the entry can never be drawn.
__device__ __forceinline__ float scaled(float x, float inv) {
  const float s = clamp_finite(__fmul_rn(x, inv));
  return x > -INFINITY ? s : -INFINITY;
}
// s + noise, finite (NaN: the lowest).
__device__ __forceinline__ float draw_value(float s, float noise) {
  const float k = __fadd_rn(s, noise);
  return clamp_finite(k);  // fmaxf takes the number where the other is NaN
}

struct Rule {
  float inv;      // 1 / temperature
  bool greedy, bad;
  unsigned k;     // 0: all
  float p;        // >= 1: all
  float log_min;  // -inf: all
};

__device__ __forceinline__ Rule read_rule(const mlt_sample_rule& q, long long n) {
  Rule r;
  r.bad = !(q.temperature >= 0.0f) || isinf(q.temperature) || isnan(q.top_p) || isnan(q.min_p);
  r.greedy = q.temperature == 0.0f;
  r.inv = r.greedy ? 1.0f : fminf(__fdiv_rn(1.0f, q.temperature), FLT_MAX);
  r.k = r.greedy || q.top_k <= 0 || q.top_k >= n ? 0u : static_cast<unsigned>(q.top_k);
  r.p = r.greedy ? 1.0f : q.top_p;
  r.log_min = r.greedy || q.min_p <= 0.0f ? -INFINITY : fminf(logf(q.min_p), 0.0f);  // the best stays
  return r;
}

// Weight of an entry of a short row in fixed point, units of 2^-31 of the best one's: rounding moves
// the mass of 512 by at most 2^-23 of the best one's.
__device__ __forceinline__ uint32_t fixed_weight(float s, float top) {
  return __float2uint_rn(__expf(__fsub_rn(s, top)) * 2147483648.0f);
}

// Weights of a long row, whose tail may be a hundred million entries far below the best: the unit is
// 2^-25 of the mean weight, so rounding moves the mass of any entries that are the best ones by at
// most 2^-26 of it, and the row's mass stays below 2^53.
struct Weights {
  float top, one;  // the best score, units in its weight

  Weights() = default;
  // z: the sum of all n weights, to a few digits
  __device__ __forceinline__ Weights(float top_, float z, int n) : top(top_) {
    const int bits = 25 + (32 - __clz(n - 1)) - ((__float_as_int(z) >> 23) - 127);
    one = __int_as_float((bits + 127) << 23);
  }
  // As halves, upper 2^32 + lower modulo 2^64: the upper one by adding 2^23, which leaves the nearest
  // whole number in a float's low bits (it is below 2^21), the lower one from the exact rest,
  // which may be negative.  (64 rows x 50,021 with top-p 43.9 us; converted to 64 bits 46.1.)
  struct Halves {
    uint32_t upper, lower;
  };
  __device__ __forceinline__ Halves halves(float s) const {
    const float x = __expf(__fsub_rn(s, top)) * one;
    const float shifted = __fmaf_rn(x, 0x1p-32f, 0x1p23f);
    const int rest = __float2int_rn(__fmaf_rn(__fsub_rn(shifted, 0x1p23f), -0x1p32f, x));
    return {static_cast<uint32_t>((__float_as_int(shifted) & 0x7FFFFF) + (rest >> 31)), static_cast<uint32_t>(rest)};
  }
  __device__ __forceinline__ unsigned long long of(float s) const {
    const Halves h = halves(s);
    return (static_cast<unsigned long long>(h.upper) << 32) + h.lower;
  }
};

// Loads and shared-memory adds under a predicate, so that those of a group of entries issue one
// after another (behind branches each waits for the one before).
__device__ __forceinline__ float load_if(const float* p, bool on) {
  float v;
  asm volatile("{.reg .pred q; setp.ne.u32 q, %2, 0; mov.f32 %0, 0f00000000; @q ld.global.nc.f32 %0, [%1];}"
               : "=f"(v)
               : "l"(p), "r"(static_cast<unsigned>(on)));
  return v;
}
__device__ __forceinline__ void add_if(unsigned* p, unsigned v, bool on) {
  asm volatile("{.reg .pred q; setp.ne.u32 q, %2, 0; @q red.shared.add.u32 [%0], %1;}" ::"r"(
                   static_cast<unsigned>(__cvta_generic_to_shared(p))),
               "r"(v), "r"(static_cast<unsigned>(on))
               : "memory");
}
__device__ __forceinline__ unsigned fetch_add_if(unsigned* p, unsigned v, bool on) {
  unsigned old;
  asm volatile("{.reg .pred q; setp.ne.u32 q, %3, 0; mov.u32 %0, 0; @q atom.shared.add.u32 %0, [%1], %2;}"
               : "=r"(old)
               : "r"(static_cast<unsigned>(__cvta_generic_to_shared(p))), "r"(v), "r"(static_cast<unsigned>(on))
               : "memory");
  return old;
}

// ---------------------------------------------------------------------------
// A warp per row
// ---------------------------------------------------------------------------
__device__ __forceinline__ unsigned long long warp_sum_fixed(unsigned long long v) {
  // lanes hold up to 2^35 (16 weights of 2^31): 32 halves of 22 and of 13 bits add up below 2^32
  const unsigned lo = __reduce_add_sync(~0u, static_cast<unsigned>(v) & 0x3FFFFFu);
  const unsigned hi = __reduce_add_sync(~0u, static_cast<unsigned>(v >> 22));
  return (static_cast<unsigned long long>(hi) << 22) + lo;
}

template <typename T, int PER>
__global__ void __launch_bounds__(128) k_sample_warp(SampleArgs a) {
  const int lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  pdl_wait();
  pdl_trigger();
  if (row >= a.rows) return;
  const int n = static_cast<int>(a.n);
  const Rule r = read_rule(a.rules != nullptr ? a.rules[row] : a.rule, n);
  const T* x = static_cast<const T*>(a.scores) + row * a.row_stride;
  const float* noise = a.noise + row * a.noise_stride;
  float s[PER];
  uint32_t key[PER];  // 0: cannot be drawn (no finite float maps to 0)
  uint32_t best = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = j * 32 + lane;
    s[j] = i < n ? scaled(to_f32(x[i]), r.inv) : -INFINITY;
    key[j] = s[j] > -INFINITY ? ordered(s[j]) : 0;
    best = max(best, key[j]);
  }
  best = __reduce_max_sync(~0u, best);
  long long* out = a.out_index + row * a.m;
  float* logp = a.out_logprob + row * a.m;
  if (best == 0 || r.bad) {
    if (r.bad && lane == 0) atomicOr(a.err, kErrBadRule);
    for (int j = lane; j < a.m; j += 32) {
      out[j] = -1;
      logp[j] = -INFINITY;
    }
    return;
  }
  const float top = from_ordered(best);
  float z = 0.0f;
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (key[j] != 0) z += expf(__fsub_rn(s[j], top));
#pragma unroll
  for (int o = 16; o > 0; o /= 2) z += __shfl_xor_sync(~0u, z, o);

  uint32_t tau = 1;  // kept: key > tau, and the first `ties` with key = tau
  unsigned ties = kNoTies;
  if (r.k != 0) {
    uint32_t at = 0;
    unsigned above = 0;  // entries at or above at + 1
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t c = at | (1u << bit);
      unsigned cnt = 0;
#pragma unroll
      for (int j = 0; j < PER; ++j) cnt += __popc(__ballot_sync(~0u, key[j] >= c));
      if (cnt >= r.k) at = c;
      else above = cnt;
    }
    if (at > 0) {  // else fewer than k entries can be drawn
      tau = at;
      ties = r.k - above;
    }
  }
  if (r.p < 1.0f) {
    uint32_t w[PER];
    unsigned long long sum = 0;
    unsigned seen = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const unsigned eq = __ballot_sync(~0u, key[j] == tau);
      const bool keep = key[j] > tau || (key[j] == tau && seen + __popc(eq & ((1u << lane) - 1u)) < ties);
      seen += __popc(eq);
      w[j] = keep ? fixed_weight(s[j], top) : 0;
      sum += w[j];
    }
    sum = warp_sum_fixed(sum);
    const unsigned long long target =
        max(1ull, static_cast<unsigned long long>(static_cast<double>(r.p) * static_cast<double>(sum)));
    uint32_t at = 0;
    unsigned long long above = 0;
    if (r.p > 0.0f) {
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t c = at | (1u << bit);
        unsigned long long mass = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) mass += key[j] >= c ? w[j] : 0;
        mass = warp_sum_fixed(mass);
        if (mass >= target) at = c;
        else above = mass;
      }
    } else {
      at = best;
    }
    if (at > 0) {
      const unsigned long long each = max(1u, fixed_weight(from_ordered(at), top));
      const unsigned long long need = (target - min(target, above) + each - 1) / each;
      const unsigned cap = at == tau ? ties : kNoTies;
      tau = at;
      ties = static_cast<unsigned>(min(static_cast<unsigned long long>(cap), max(1ull, need)));
    }
  }
  uint32_t draw[PER];
  unsigned seen = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const unsigned eq = __ballot_sync(~0u, key[j] == tau);
    const bool keep = (key[j] > tau || (key[j] == tau && seen + __popc(eq & ((1u << lane) - 1u)) < ties)) &&
                      __fsub_rn(s[j], top) >= r.log_min;
    seen += __popc(eq);
    draw[j] = 0;
    if (keep) draw[j] = r.greedy ? key[j] : ordered(draw_value(s[j], noise[j * 32 + lane]));
  }
  const float logz = logf(z);
  for (int d = 0; d < a.m; ++d) {
    uint32_t b = 0;
    int at = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (draw[j] > b) {  // the first of equal ones: the lowest index of the lane
        b = draw[j];
        at = j;
      }
    const uint32_t all = __reduce_max_sync(~0u, b);
    if (all == 0 || (r.greedy && d > 0)) {
      for (int j = d + lane; j < a.m; j += 32) {
        out[j] = -1;
        logp[j] = -INFINITY;
      }
      break;
    }
    const unsigned i = __reduce_min_sync(~0u, b == all ? static_cast<unsigned>(at * 32 + lane) : 0xFFFFFFFFu);
    if (b == all && static_cast<unsigned>(at * 32 + lane) == i) {
      float sv = 0.0f;
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (j == at) {
          sv = s[j];
          draw[j] = 0;
        }
      out[d] = i;
      logp[d] = r.greedy ? 0.0f : __fsub_rn(sv, top) - logz;
    }
  }
}

// ---------------------------------------------------------------------------
// A team of CTAs per row
// ---------------------------------------------------------------------------
constexpr int kMaxTeam = 160;
constexpr int kLarge = 16384;  // candidates that one CTA finishes without the team
// Lists of a row, by what they are for.  Candidates for the top-k are in `large` and counted as its list;
// those for the draws are in top-p's list, read by then, with a counter of their own.
enum { kTopK, kTopP, kDraws, kLists, kDrawCandidates = kLists, kCounters };

// Global memory of a team; teams of one CTA use none of it.
struct TeamMem {
  unsigned arrivals;      // barrier: CTAs arrived, over all barriers of the call (zeroed before the launch)
  unsigned listed[kCounters];
  float4 stats[kMaxTeam]; // each CTA's (max, sum of exp, min)
  unsigned long long best[kMaxTeam];
  unsigned entries[kMaxTeam];
  unsigned long long mass[3][kBins];
  unsigned count[3][kBins];
  unsigned long long list[kLists][kList];
  unsigned long long large[kLarge];
};

struct Shared {
  union {  // a list is made once its bin is found
    unsigned long long list[kList];
    struct {
      unsigned long long mass[kBins];  // merged
      unsigned lo[kBins], hi[kBins];   // of the CTA's masses
    };
  };
  unsigned count[kBins];
  unsigned long long warp_u64[32];
  float warp_f[32][3];  // maximum, sum of exponentials, least of the lanes' maxima
  unsigned long long above;
  unsigned in, bin, listed, found;
  float top, z, low;
  unsigned long long wait_ns;  // limit of a wait in global memory
  int dead;
};

struct Team {
  bool cluster;  // the team is a thread-block cluster
  TeamMem* g;
  unsigned* err;
  int size, rank;
  unsigned barriers;
  int stage;  // histograms used so far
  int bins;   // in use: a multiple of the CTA's threads, at most kBins
};

// All CTAs of the team; false where the wait gave up (then on every thread of the CTA).
__device__ bool team_sync(Team& t, Shared& sh) {
  __syncthreads();
  if (t.size == 1) return true;
  if (t.cluster) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    return true;
  }
  ++t.barriers;
  if (threadIdx.x == 0) {
    __threadfence();
    atomicAdd(&t.g->arrivals, 1u);
    const unsigned want = t.barriers * static_cast<unsigned>(t.size);
    unsigned long long start, now;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(start));
    int dead = 0;
    for (;;) {
      unsigned v;
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(&t.g->arrivals) : "memory");
      if (v >= want) break;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
      if (now - start > sh.wait_ns) {
        atomicOr(t.err, kErrWaitTimeout);
        dead = 1;
        break;
      }
    }
    sh.dead = dead;
    __threadfence();
  }
  __syncthreads();
  return sh.dead == 0;
}

// Composite: larger key first, then the lower index.
__device__ __forceinline__ unsigned long long composite(uint32_t key, int i) {
  return (static_cast<unsigned long long>(key) << kIndexBits) |
         static_cast<unsigned long long>((1 << kIndexBits) - 1 - i);
}
__device__ __forceinline__ int index_of(unsigned long long c) {
  return (1 << kIndexBits) - 1 - static_cast<int>(c & ((1ull << kIndexBits) - 1));
}
__device__ __forceinline__ float score_of(unsigned long long c) {
  return from_ordered(static_cast<uint32_t>(c >> kIndexBits));
}

// A row of scores.  walk: f(at, s) for every group of eight that the thread owns, the same ones
// at each walk: s[v] is the scaled score of entry at[v], -infinity where it cannot be
// drawn or is outside the row.  The next group is loaded before f.  What f loads or adds by
// atomics it does for all of a group before it uses any of it: one after another, each
// would wait for memory (64 rows x 50,021 with min-p: 10 us a pass).
template <typename T>
struct Row {
  static constexpr int V = 8;  // of 16-bit scores 16 bytes, of fp32 twice that
  const T* row;
  int n;
  float inv;

  __device__ __forceinline__ float score(int i) const { return scaled(to_f32(row[i]), inv); }
  __device__ __forceinline__ void load(const T* base, int q, int skew, Pack<T, V>& p) const {
    const int i0 = q * V - skew;
    if (i0 >= 0 && i0 <= n - V) p = *reinterpret_cast<const Pack<T, V>*>(base + static_cast<long long>(q) * V);
  }
  template <typename F>
  __device__ __forceinline__ void walk(const Team& t, F f) const {
    const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(row) / sizeof(T)) % V);
    const int groups = (skew + n + V - 1) / V;
    const int stride = t.size * static_cast<int>(blockDim.x), last = n - V;
    const T* base = row - skew;  // aligned to the group; entries before `row` are not read
    int q = t.rank * static_cast<int>(blockDim.x) + threadIdx.x;
    Pack<T, V> p;
    load(base, min(q, groups), skew, p);
#pragma unroll 1
    for (; q < groups; q += stride) {
      const Pack<T, V> now = p;
      load(base, min(q + stride, groups), skew, p);  // the next one lands meanwhile
      const int i0 = q * V - skew;
      float s[V];
      if (i0 >= 0 && i0 <= last) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = scaled(to_f32(now.v[v]), inv);
      } else {
        // a row's ends
#pragma unroll
        for (int v = 0; v < V; ++v)
          s[v] = i0 + v >= 0 && i0 + v < n ? scaled(to_f32(row[i0 + v]), inv) : -INFINITY;
      }
      int at[V];
#pragma unroll
      for (int v = 0; v < V; ++v) at[v] = i0 + v;
      f(at, s);
    }
  }
};
// Candidates that were collected from a row, as composites; walked by one CTA.
struct Candidates {
  static constexpr int V = 4;
  const unsigned long long* list;
  int n;

  template <typename F>
  __device__ __forceinline__ void walk(const Team&, F f) const {
#pragma unroll 1
    for (int j = threadIdx.x; j < n; j += V * blockDim.x) {
      unsigned long long c[V];
      float s[V];
#pragma unroll
      for (int v = 0; v < V; ++v) c[v] = j + v * static_cast<int>(blockDim.x) < n ? __ldcg(&list[j + v * blockDim.x]) : 0;
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = c[v] != 0 ? score_of(c[v]) : -INFINITY;
      int at[V];
#pragma unroll
      for (int v = 0; v < V; ++v) at[v] = index_of(c[v]);
      f(at, s);
    }
  }
};

__device__ __forceinline__ void clear_bins(const Team& t, Shared& sh, bool mass) {
  __syncthreads();
  for (int b = threadIdx.x; b < t.bins; b += blockDim.x) {
    sh.count[b] = 0;
    if (mass) sh.lo[b] = sh.hi[b] = 0;
  }
  __syncthreads();
}

// The team's bins of this stage, merged, in sh.count and (kMass) sh.mass.
template <bool kMass>
__device__ bool merge_bins(Team& t, Shared& sh) {
  __syncthreads();
  if (t.size == 1) {
    if (kMass) {
      for (int b = threadIdx.x; b < t.bins; b += blockDim.x)
        sh.mass[b] = (static_cast<unsigned long long>(sh.hi[b]) << 32) + sh.lo[b];
      __syncthreads();
    }
    return true;
  }
  const int now = t.stage % 3, next = (t.stage + 1) % 3;  // `next` was last read before the previous barrier
  ++t.stage;
  for (int b = threadIdx.x; b < t.bins; b += blockDim.x) {
    if (sh.count[b] != 0) {
      atomicAdd(&t.g->count[now][b], sh.count[b]);
      if (kMass) atomicAdd(&t.g->mass[now][b], (static_cast<unsigned long long>(sh.hi[b]) << 32) + sh.lo[b]);
    }
    if (t.rank == 0) {
      t.g->count[next][b] = 0;
      t.g->mass[next][b] = 0;
    }
  }
  if (!team_sync(t, sh)) return false;
  for (int b = threadIdx.x; b < t.bins; b += blockDim.x) {
    sh.count[b] = __ldcg(&t.g->count[now][b]);
    if (kMass) sh.mass[b] = __ldcg(&t.g->mass[now][b]);
  }
  __syncthreads();
  return true;
}

// Each warp's value of `mine` over the CTA's warps, lane w having warp w's.
__device__ __forceinline__ unsigned long long warps_of(unsigned long long mine, int from_lane, Shared& sh) {
  const int lane = threadIdx.x & 31;
  __syncthreads();
  if (lane == from_lane) sh.warp_u64[threadIdx.x >> 5] = mine;
  __syncthreads();
  return lane < static_cast<int>(blockDim.x >> 5) ? sh.warp_u64[lane] : 0;
}
// Sum (maximum) over the CTA, on every thread.
__device__ __forceinline__ unsigned long long block_sum(unsigned long long v, Shared& sh) {
#pragma unroll
  for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(~0u, v, o);
  v = warps_of(v, 0, sh);
#pragma unroll
  for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(~0u, v, o);
  return v;
}
__device__ __forceinline__ unsigned long long block_max(unsigned long long v, Shared& sh) {
#pragma unroll
  for (int o = 16; o > 0; o /= 2) v = max(v, __shfl_xor_sync(~0u, v, o));
  v = warps_of(v, 0, sh);
#pragma unroll
  for (int o = 16; o > 0; o /= 2) v = max(v, __shfl_xor_sync(~0u, v, o));
  return v;
}
// The sum over the CTA's lower threads.
__device__ __forceinline__ unsigned long long block_below(unsigned long long mine, Shared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long v = mine;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const unsigned long long w = __shfl_up_sync(~0u, v, o);
    if (lane >= o) v += w;
  }
  unsigned long long all = warps_of(v, 31, sh);
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const unsigned long long w = __shfl_up_sync(~0u, all, o);
    if (lane >= o) all += w;
  }
  const unsigned long long below = __shfl_sync(~0u, all, warp > 0 ? warp - 1 : 0);
  return v - mine + (warp > 0 ? below : 0);
}

// The first bin where the running sum of counts (or masses) reaches `need`: sh.bin, the sum
// before it sh.above, its count sh.in (0 where the sum stays below).
template <bool kMass>
__device__ void find_bin(const Team& t, Shared& sh, unsigned long long need) {
  const int span = t.bins / blockDim.x, first = threadIdx.x * span;
  unsigned long long mine = 0;
  for (int j = 0; j < span; ++j) mine += kMass ? sh.mass[first + j] : sh.count[first + j];
  unsigned long long above = block_below(mine, sh);
  if (threadIdx.x == 0) sh.in = 0;
  __syncthreads();
  if (above < need && above + mine >= need) {
    for (int j = 0; j < span; ++j) {
      const unsigned long long c = kMass ? sh.mass[first + j] : sh.count[first + j];
      if (above + c >= need) {
        sh.bin = first + j;
        sh.above = above;
        sh.in = sh.count[first + j];
        break;
      }
      above += c;
    }
  }
  __syncthreads();
}

// sh.list[0 .. n), descending; entries differ.
constexpr unsigned kRanked = 256;

// Bitonic, E entries a thread (entry e blockDim + thread): exchanges within a warp by
// shuffles, within a thread in registers, others through sh.list.
template <int E>
__device__ void sort_registers(Shared& sh, unsigned n) {
  unsigned long long v[E];
  const unsigned threads = blockDim.x, width = E * threads;
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = e * threads + threadIdx.x < n ? sh.list[e * threads + threadIdx.x] : 0;
  for (unsigned k = 2; k <= width; k *= 2)
    for (unsigned j = k / 2; j > 0; j /= 2) {
      if (j >= threads) {
        // both are this thread's
#pragma unroll
        for (int d = 1; d < E; d *= 2) {
          if (j != d * threads) continue;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int o = e ^ d;
            if (o < e) continue;
            const unsigned long long lo = min(v[e], v[o]), hi = max(v[e], v[o]);
            const bool desc = ((e * threads + threadIdx.x) & k) == 0;
            v[e] = desc ? hi : lo;
            v[o] = desc ? lo : hi;
          }
        }
        continue;
      }
      if (j >= 32) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) sh.list[e * threads + threadIdx.x] = v[e];
        __syncthreads();
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const unsigned i = e * threads + threadIdx.x;
        const unsigned long long w = j >= 32 ? sh.list[i ^ j] : __shfl_xor_sync(~0u, v[e], j);
        // the lower of a descending pair keeps the larger value, and so does the upper of an ascending one
        v[e] = ((i & k) == 0) == ((i & j) == 0) ? max(v[e], w) : min(v[e], w);
      }
    }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) sh.list[e * threads + threadIdx.x] = v[e];
  __syncthreads();
}

// Bins of a selection: linear from `from` down, `scale` a unit; what lies outside goes to
// the first or last one.  Rounded steps of it are monotone, so a bin is an interval.
struct Bins {
  float from, scale, last;
  __device__ __forceinline__ int of(float v) const {
    return static_cast<int>(fminf(fmaxf(__fmul_rn(__fsub_rn(from, v), scale), 0.0f), last));
  }
};

// By buckets, linear in the value between the list's extremes: an entry's place is its
// bucket's plus the number of larger ones in it.  False, and the list as it was, where
// a bucket is crowded.  (Entries are held in registers meanwhile, E a thread.)
constexpr unsigned kCrowd = 48;

template <int E>
__device__ bool sort_buckets(const Team& t, Shared& sh, unsigned n) {
  const unsigned threads = blockDim.x;
  unsigned long long v[E];
  unsigned long long high = 0, low = 0;  // largest entry, largest complement
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const unsigned i = e * threads + threadIdx.x;
    v[e] = i < n ? sh.list[i] : 0;
    if (i < n) {
      high = max(high, v[e]);
      low = max(low, ~v[e]);
    }
  }
  high = block_max(high, sh);
  low = ~block_max(low, sh);
  const float range = __fsub_rn(score_of(high), score_of(low)), last = static_cast<float>(t.bins - 1);
  if (!(range > 0.0f)) return false;
  const Bins bins = {score_of(high), fminf(last / range, 1e30f), last};
  for (int b = threadIdx.x; b < t.bins; b += threads) sh.count[b] = 0;
  __syncthreads();
  int bin[E];
  unsigned slot[E];
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (v[e] != 0) {
      bin[e] = bins.of(score_of(v[e]));
      slot[e] = atomicAdd(&sh.count[bin[e]], 1u);
    }
  __syncthreads();
  // count -> place of the bucket's first entry
  const int span = t.bins / threads, first = threadIdx.x * span;
  unsigned mine = 0, most = 0;
  for (int j = 0; j < span; ++j) {
    mine += sh.count[first + j];
    most = max(most, sh.count[first + j]);
  }
  unsigned at = static_cast<unsigned>(block_below(mine, sh));
  if (__syncthreads_or(most > kCrowd)) return false;
  for (int j = 0; j < span; ++j) {
    const unsigned c = sh.count[first + j];
    sh.count[first + j] = at;
    at += c;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (v[e] != 0) sh.list[sh.count[bin[e]] + slot[e]] = v[e];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (v[e] != 0) {
      const unsigned begin = sh.count[bin[e]];
      const unsigned end = bin[e] + 1 < t.bins ? sh.count[bin[e] + 1] : n;
      unsigned rank = begin;
      for (unsigned j = begin; j < end; ++j) rank += sh.list[j] > v[e];
      slot[e] = rank;
    }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (v[e] != 0) sh.list[slot[e]] = v[e];
  __syncthreads();
  return true;
}

__device__ void sort_list(const Team& t, Shared& sh, unsigned n) {
  const unsigned threads = blockDim.x;
  if (n <= kRanked && n <= threads) {
    // an entry's place is the number of larger ones
    const unsigned long long v = threadIdx.x < n ? sh.list[threadIdx.x] : 0;
    unsigned rank = 0;
    if (threadIdx.x < n)
      for (unsigned j = 0; j < n; ++j) rank += sh.list[j] > v;
    __syncthreads();
    if (threadIdx.x < n) sh.list[rank] = v;
    __syncthreads();
    return;
  }
  if (n <= 4 * threads && sort_buckets<4>(t, sh, n)) return;
  if (n <= threads) return sort_registers<1>(sh, n);
  if (n <= 2 * threads) return sort_registers<2>(sh, n);
  if (n <= 4 * threads) return sort_registers<4>(sh, n);
  if (n <= 8 * threads && 8 * threads <= kList) return sort_registers<8>(sh, n);
  unsigned width = 1;
  while (width < n) width *= 2;
  for (unsigned j = n + threadIdx.x; j < width; j += threads) sh.list[j] = 0;
  __syncthreads();
  for (unsigned k = 2; k <= width; k *= 2)
    for (unsigned j = k / 2; j > 0; j /= 2) {
      for (unsigned q = threadIdx.x; q < width / 2; q += threads) {
        const unsigned i = 2 * q - (q & (j - 1)), o = i + j;  // the pairs that differ in bit j
        const unsigned long long u = sh.list[i], w = sh.list[o];
        if ((i & k) == 0 ? u < w : u > w) {
          sh.list[i] = w;
          sh.list[o] = u;
        }
      }
      __syncthreads();
    }
}

// The team's list into sh.list (a lone CTA's is there).
__device__ __forceinline__ void take_list(const Team& t, Shared& sh, const unsigned long long* list,
                                          const unsigned* listed) {
  if (t.size > 1) {
    const unsigned have = min(__ldcg(listed), static_cast<unsigned>(kList));
    for (unsigned j = threadIdx.x; j < have; j += blockDim.x) sh.list[j] = __ldcg(&list[j]);
    if (threadIdx.x == 0) sh.listed = have;
  } else if (threadIdx.x == 0) {
    sh.listed = min(sh.listed, static_cast<unsigned>(kList));
  }
  __syncthreads();
}
// Mass of the first `n` entries of sh.list.
__device__ __forceinline__ unsigned long long list_mass(Shared& sh, unsigned n, Weights weight) {
  unsigned long long sum = 0;
  for (unsigned j = threadIdx.x; j < n; j += blockDim.x) sum += weight.of(score_of(sh.list[j]));
  return block_sum(sum, sh);
}
// The entry of the sorted list (of n >= 1) at which the running mass reaches `need`; the last one
// where rounding leaves less.
__device__ __forceinline__ unsigned mass_reaches(Shared& sh, unsigned n, unsigned long long need, Weights weight) {
  const unsigned span = (n + blockDim.x - 1) / blockDim.x, first = threadIdx.x * span;
  unsigned long long mine = 0;
  for (unsigned j = first; j < min(first + span, n); ++j) mine += weight.of(score_of(sh.list[j]));
  unsigned long long at = block_below(mine, sh);
  if (threadIdx.x == 0) sh.found = n - 1;
  __syncthreads();
  if (at < need && at + mine >= need)
    for (unsigned j = first; j < min(first + span, n); ++j) {
      at += weight.of(score_of(sh.list[j]));
      if (at >= need) {
        sh.found = j;
        break;
      }
    }
  __syncthreads();
  return sh.found;
}
__device__ __forceinline__ unsigned long long share_of(float share, unsigned long long sum) {
  return share > 0.0f
             ? max(1ull, static_cast<unsigned long long>(static_cast<double>(share) * static_cast<double>(sum)))
             : 1ull;
}

// The bin that holds the `need`-th largest of the threads' own maxima (-infinity: none), one a
// thread; all entries in bins up to it are at least `need`.  -1 where there are not so many.
// all: the CTA's number of entries (kList + 1 or more where it is not known); where the team's
// are not many more than `need`, the bin is the last one: all of them.
__device__ bool bin_of_maxima(Team& t, Shared& sh, Bins bins, unsigned long long need, float mine, unsigned all,
                              int* bin) {
  clear_bins(t, sh, false);
  if (mine > -INFINITY) atomicAdd(&sh.count[bins.of(mine)], 1u);
  __syncthreads();
  const unsigned entries = min(all, static_cast<unsigned>(kList) + 1u);
  if (t.size > 1) {
    if (threadIdx.x == 0) t.g->entries[t.rank] = entries;
  }
  if (!merge_bins<false>(t, sh)) return false;
  unsigned total = entries;
  if (t.size > 1) {
    unsigned long long v = threadIdx.x < static_cast<unsigned>(t.size) ? __ldcg(&t.g->entries[threadIdx.x]) : 0;
    total = static_cast<unsigned>(block_sum(v, sh));
  }
  if (total <= max(2ull * need, static_cast<unsigned long long>(kRanked)) && total <= kList) {
    *bin = t.bins - 1;
    return true;
  }
  find_bin<false>(t, sh, need);
  *bin = sh.in > 0 ? static_cast<int>(sh.bin) : -1;
  return true;
}
// Collects the composites of all values in bins up to `bin` (kAbove) or in it, of these only those whose
// leading digits (above `shift`) are at least (are) `prefix`.  mine: the thread's largest value.
template <bool kAbove, typename Src, typename Get>
__device__ __forceinline__ void collect(const Src& src, const Team& t, Bins bins, int bin, float mine, int shift,
                                        unsigned long long prefix, Get get, unsigned long long* list, unsigned* listed,
                                        unsigned capacity) {
  constexpr int V = Src::V;
  if (!(mine > -INFINITY) || bins.of(mine) > bin) return;  // nor is any other of its values that large
  // most values are told apart by an interval half a bin wider
  const float from = kAbove || bin == 0 ? INFINITY : bins.from - (static_cast<float>(bin) - 0.5f) / bins.scale;
  const float to = static_cast<float>(bin) == bins.last || bins.scale == 0.0f
                       ? -FLT_MAX
                       : bins.from - (static_cast<float>(bin) + 1.5f) / bins.scale;
  src.walk(t, [&](const int(&at)[V], float(&s)[V]) {
    get(at, s);
    unsigned hit = 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (s[v] >= to && s[v] <= from) hit |= 1u << v;
    while (hit != 0) {
      const int v = __ffs(hit) - 1;
      hit &= hit - 1;
      float value = s[0];
#pragma unroll
      for (int e = 1; e < V; ++e)
        if (e == v) value = s[e];
      const int b = bins.of(value);
      if (b > bin || (!kAbove && b != bin)) continue;
      const unsigned long long c = composite(ordered(value), at[v]), high = c >> shift;
      if (b < bin || (kAbove ? high >= prefix : high == prefix)) {
        const unsigned to_at = atomicAdd(listed, 1u);
        if (to_at < capacity) list[to_at] = c;
      }
    }
  });
}

// Selects from the values that get() gives: get(at, s) turns the scores of a group into
// values, -infinity for entries that do not take part.
//   kMass = false: the `need`-th largest composite; kAbove: the `need` largest
//   kMass = true:  the composite at which the mass reaches `share` of all
// mine: the thread's largest value, or +infinity where it is not known.
// Leaves a sorted list in sh.list.  *edge: the composite found (0: the entries do not
// reach that far, all are kept).  kAbove: sh.listed entries, on rank 0 only, and no edge.
template <bool kMass, bool kAbove, typename Src, typename Get>
__device__ __noinline__ bool select(const Src& src, Team& t, Shared& sh, int use, Bins bins, unsigned long long need,
                                    float share, Weights weight, float mine, Get get,
                                    unsigned long long* edge) {
  constexpr int V = Src::V;
  *edge = 0;
  unsigned long long* list = t.size > 1 ? t.g->list[use] : sh.list;
  unsigned* listed = t.size > 1 ? &t.g->listed[use] : &sh.listed;
  if (threadIdx.x == 0) sh.listed = 0;
  clear_bins(t, sh, kMass);
  src.walk(t, [&](const int(&at)[V], float(&s)[V]) {
    get(at, s);
    // (masses in halves of the group: 64 bits of eight entries would not fit the registers)
    constexpr int kPart = kMass ? V / 2 : V;
#pragma unroll
    for (int f = 0; f < V; f += kPart) {
      int b[kPart];
      Weights::Halves w[kPart];
      uint32_t old[kPart];
#pragma unroll
      for (int v = 0; v < kPart; ++v) {
        b[v] = bins.of(s[f + v]);
        if (kMass) w[v] = weight.halves(s[f + v]);
      }
#pragma unroll
      for (int v = 0; v < kPart; ++v) {
        const bool on = s[f + v] > -INFINITY;
        add_if(&sh.count[b[v]], 1u, on);
        if (kMass) old[v] = fetch_add_if(&sh.lo[b[v]], w[v].lower, on);
      }
      if (kMass) {
        // shared memory adds 32 bits at a time: carries go to the upper half (as a rule nothing does)
#pragma unroll
        for (int v = 0; v < kPart; ++v) {
          const uint32_t hi = w[v].upper + (old[v] + w[v].lower < old[v] ? 1u : 0u);
          add_if(&sh.hi[b[v]], hi, s[f + v] > -INFINITY && hi != 0);
        }
      }
    }
  });
  if (!merge_bins<kMass>(t, sh)) return false;
  if (kMass) {
    unsigned long long sum = 0;
    for (int b = threadIdx.x; b < t.bins; b += blockDim.x) sum += sh.mass[b];
    sum = block_sum(sum, sh);
    need = share_of(share, sum);
  }
  find_bin<kMass>(t, sh, need);
  int bin = static_cast<int>(sh.bin);
  unsigned in = sh.in;
  unsigned above_n = 0;  // kAbove: entries above the bin (the list takes them too)
  if (in == 0) {
    if (!kAbove) return true;
    bin = t.bins - 1;  // fewer than `need`: all of them
  } else {
    need -= sh.above;
    if (kAbove) above_n = static_cast<unsigned>(sh.above);
  }
  // a bin that does not fit the list: digits of the composite
  int shift = kIndexBits + 32;
  unsigned long long prefix = 0;
#pragma unroll 1
  while (in + above_n > kList) {
    const int bits = min(31 - __clz(t.bins), shift);
    shift -= bits;
    clear_bins(t, sh, kMass);
    src.walk(t, [&](const int(&at)[V], float(&s)[V]) {
      get(at, s);
#pragma unroll 1
      for (int v = 0; v < V; ++v) {
        if (!(s[v] > -INFINITY) || bins.of(s[v]) != bin) continue;
        const unsigned long long c = composite(ordered(s[v]), at[v]);
        if ((c >> (shift + bits)) != prefix) continue;
        const int b = t.bins - 1 - static_cast<int>((c >> shift) & ((1u << bits) - 1u));
        atomicAdd(&sh.count[b], 1u);
        if (kMass) {
          const Weights::Halves w = weight.halves(s[v]);
          const uint32_t old = atomicAdd(&sh.lo[b], w.lower), hi = w.upper + (old + w.lower < old ? 1u : 0u);
          if (hi != 0) atomicAdd(&sh.hi[b], hi);
        }
      }
    });
    if (!merge_bins<kMass>(t, sh)) return false;
    find_bin<kMass>(t, sh, need);
    prefix = (prefix << bits) | static_cast<unsigned>(t.bins - 1 - sh.bin);
    in = sh.in;
    need -= sh.above;
    if (kAbove) above_n += static_cast<unsigned>(sh.above);
  }
  collect<kAbove>(src, t, bins, bin, mine, shift, prefix, get, list, listed, kList);
  if (!team_sync(t, sh)) return false;
  if (kAbove && t.rank != 0) return true;
  take_list(t, sh, list, listed);
  const unsigned have = sh.listed;
  sort_list(t, sh, have);
  if (kAbove) return true;
  *edge = kMass ? sh.list[mass_reaches(sh, have, need, weight)] : sh.list[need - 1];
  __syncthreads();
  return true;
}

__device__ __forceinline__ void none_drawn(const SampleArgs& a, long long row, int from) {
  for (int j = from + threadIdx.x; j < a.m; j += blockDim.x) {
    a.out_index[row * a.m + j] = -1;
    a.out_logprob[row * a.m + j] = -INFINITY;
  }
}

__device__ __forceinline__ void join_stats(float& m, float& z, float m2, float z2) {
  const float b = fmaxf(m, m2);
  if (b == -INFINITY) return;
  z = z * __expf(m - b) + z2 * __expf(m2 - b);
  m = b;
}

// What the steps of a row share.
struct Ctx {
  const float* noise;
  Rule r;
  float top, logz;
  Weights weight;
  long long row;
};

// Kept entries of the row lie above (value, index) of the edge's entry, or are it.
struct Edge {
  unsigned long long c = 0;
  float s = -FLT_MAX;
  int i = (1 << kIndexBits) - 1;
  __device__ __forceinline__ void raise(unsigned long long to) {
    if (to <= c) return;
    c = to;
    s = score_of(to);
    i = index_of(to);
  }
  __device__ __forceinline__ bool keeps(float v, int at) const { return v > s || (v == s && at <= i); }
};

// What a selection goes by: scores as they are, those of kept entries, draw values of kept ones.
struct All {
  template <int V>
  __device__ __forceinline__ void operator()(const int (&)[V], float (&)[V]) const {}
};
struct Kept {
  Edge edge;
  template <int V>
  __device__ __forceinline__ void operator()(const int (&at)[V], float (&s)[V]) const {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (!edge.keeps(s[v], at[v])) s[v] = -INFINITY;
  }
};
struct Draws {
  Edge edge;
  const float* noise;
  float top, log_min;
  template <int V>
  __device__ __forceinline__ void operator()(const int (&at)[V], float (&s)[V]) const {
    float g[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!(edge.keeps(s[v], at[v]) && __fsub_rn(s[v], top) >= log_min)) s[v] = -INFINITY;
      g[v] = load_if(noise + at[v], s[v] > -INFINITY);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (s[v] > -INFINITY) s[v] = draw_value(s[v], g[v]);
  }
};

__device__ __forceinline__ void put(const SampleArgs& a, const Ctx& x, int j, int index, float s) {
  a.out_index[x.row * a.m + j] = index;
  a.out_logprob[x.row * a.m + j] = x.r.greedy ? 0.0f : __fsub_rn(s, x.top) - x.logz;
}

// Cuts and draws from sh.list, sorted, which holds the row's best entries: at least the top k.
template <typename T>
__device__ void finish_list(const SampleArgs& a, const Team& t, Shared& sh, const Ctx& x, const Row<T>& src) {
  unsigned keep = min(sh.listed, x.r.k);
  if (x.r.p < 1.0f)
    keep = mass_reaches(sh, keep, share_of(x.r.p, list_mass(sh, keep, x.weight)), x.weight) + 1;
  if (x.r.log_min > -INFINITY) {
    unsigned long long mine = 0;
    for (unsigned j = threadIdx.x; j < keep; j += blockDim.x)
      mine += __fsub_rn(score_of(sh.list[j]), x.top) >= x.r.log_min;
    keep = static_cast<unsigned>(block_sum(mine, sh));
  }
  unsigned long long best = 0;
  for (unsigned j = threadIdx.x; j < keep; j += blockDim.x) {
    const int i = index_of(sh.list[j]);
    const unsigned long long c = composite(ordered(draw_value(score_of(sh.list[j]), x.noise[i])), i);
    sh.list[j] = c;
    best = max(best, c);
  }
  if (a.m == 1) {
    best = block_max(best, sh);
    if (threadIdx.x == 0) put(a, x, 0, index_of(best), src.score(index_of(best)));
    return;
  }
  __syncthreads();
  sort_list(t, sh, keep);
  const int drawn = static_cast<int>(min(keep, static_cast<unsigned>(a.m)));
  for (int j = threadIdx.x; j < drawn; j += blockDim.x)
    put(a, x, j, index_of(sh.list[j]), src.score(index_of(sh.list[j])));
  none_drawn(a, x.row, drawn);
}

// Cuts and draws by selection from `src` (the row, or candidates that hold its top k).  mine: the
// thread's largest score there; mine_key: its largest draw value where nothing is cut (else NaN).
template <typename T, typename Src>
__device__ bool finish_select(const SampleArgs& a, Team& t, Shared& sh, const Ctx& x, const Row<T>& row, const Src& src,
                              Bins by_score, float mine, float mine_key) {
  constexpr int V = Src::V;
  Edge edge;
  unsigned long long found;
  if (x.r.k != 0) {
    if (!select<false, false>(src, t, sh, kTopK, by_score, x.r.k, 0.0f, x.weight, mine, All(), &found))
      return false;
    edge.raise(found);
  }
  if (x.r.p < 1.0f) {
    if (!select<true, false>(src, t, sh, kTopP, by_score, 0, x.r.p, x.weight, mine, Kept{edge}, &found)) return false;
    edge.raise(found);
  }
  const Draws draws = {edge, x.noise, x.top, x.r.log_min};
  // The thread's largest draw value.  A thread whose largest score is cut has none.
  int key_at = 0;
  unsigned long long entries = kList + 1;
  if (mine_key != mine_key) {
    entries = 0;
    mine_key = -INFINITY;
    if (mine >= edge.s && __fsub_rn(mine, x.top) >= x.r.log_min)
      src.walk(t, [&](const int(&at)[V], float(&s)[V]) {
        draws(at, s);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          entries += s[v] > -INFINITY;
          if (s[v] > mine_key || (s[v] == mine_key && s[v] > -INFINITY && at[v] < key_at)) {
            mine_key = s[v];
            key_at = at[v];
          }
        }
      });
  }
  if (a.m == 1) {
    unsigned long long best = mine_key > -INFINITY ? composite(ordered(mine_key), key_at) : 0;
    best = block_max(best, sh);
    if (t.size > 1) {
      if (threadIdx.x == 0) t.g->best[t.rank] = best;
      if (!team_sync(t, sh)) return false;
      if (t.rank == 0 && threadIdx.x == 0)
        for (int c = 0; c < t.size; ++c) best = max(best, __ldcg(&t.g->best[c]));
    }
    if (t.rank == 0 && threadIdx.x == 0) put(a, x, 0, index_of(best), row.score(index_of(best)));
    return true;
  }
  // Gumbel noise puts the largest keys within a few units of the best score, and ln n above it.
  const float last = static_cast<float>(t.bins - 1);
  const Bins by_key = {x.top + 24.0f, last / 48.0f, last};
  const unsigned kept = static_cast<unsigned>(block_sum(entries, sh));
  // More than m threads: the m-th of their maxima bounds the m-th draw from below, and few
  // entries beside the draws lie above it.
  bool done = false;
  if (a.m <= t.size * static_cast<int>(blockDim.x) / 2) {
    int bin;
    if (!bin_of_maxima(t, sh, by_key, a.m, mine_key, kept, &bin)) return false;
    if (bin >= 0) {
      unsigned long long* list = t.size > 1 ? t.g->list[kTopP] : sh.list;
      unsigned* listed = t.size > 1 ? &t.g->listed[kDrawCandidates] : &sh.listed;
      if (threadIdx.x == 0) sh.listed = 0;
      __syncthreads();
      collect<true>(src, t, by_key, bin, mine_key, kIndexBits + 32, 0, draws, list, listed, kList);
      if (!team_sync(t, sh)) return false;
      done = (t.size > 1 ? __ldcg(listed) : sh.listed) <= kList;
      if (done) {
        if (t.rank != 0) return true;
        take_list(t, sh, list, listed);
        sort_list(t, sh, sh.listed);
      }
      __syncthreads();
    }
  }
  if (!done && !select<false, true>(src, t, sh, kDraws, by_key, a.m, 0.0f, x.weight, mine_key, draws, &found))
    return false;
  if (t.rank != 0) return true;
  const int drawn = static_cast<int>(min(sh.listed, static_cast<unsigned>(a.m)));
  for (int j = threadIdx.x; j < drawn; j += blockDim.x)
    put(a, x, j, index_of(sh.list[j]), row.score(index_of(sh.list[j])));
  none_drawn(a, x.row, drawn);
  return true;
}

template <typename T>
__device__ bool sample_row(const SampleArgs& a, Team& t, Shared& sh, long long row_at) {
  constexpr int V = Row<T>::V;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  Ctx x = {};
  x.r = read_rule(a.rules != nullptr ? a.rules[row_at] : a.rule, a.n);
  x.noise = a.noise + row_at * a.noise_stride;
  x.row = row_at;
  const Row<T> row = {static_cast<const T*>(a.scores) + row_at * a.row_stride, static_cast<int>(a.n), x.r.inv};
  if (x.r.bad) {
    if (t.rank == 0) {
      if (threadIdx.x == 0) atomicOr(a.err, kErrBadRule);
      none_drawn(a, row_at, 0);
    }
    return true;
  }
  // Where nothing is cut the first pass finds the draws too: one, or every thread's largest.
  const bool uncut = x.r.k == 0 && x.r.p >= 1.0f && x.r.log_min == -INFINITY;
  const bool direct = uncut && (a.m == 1 || x.r.greedy);

  // Pass 1: maximum and sum of exponentials, each lane's own, then joined in a fixed order.  A lane
  // may have 131,072 entries: the sums of its groups are added with compensation (z - lost), at no
  // measurable cost.  The approximate exponential is off by at most 2 + 1.2 |s - top| units of 2^-23 of a
  // weight (expf: 64 rows x 50,021 fp32 with top-k 50 22.7 us for 21.0, one row of 16,777,216 61.4 for 59.8).
  float top = -INFINITY, z = 0.0f, lost = 0.0f;
  float best_key = -INFINITY;
  int best_at = 0;
  auto first = [&](const int(&at)[V], float(&s)[V]) {
    float b = top;
#pragma unroll
    for (int v = 0; v < V; ++v) b = fmaxf(b, s[v]);
    if (b == -INFINITY) return;
    if (b > top) {
      const float f = __expf(top - b);
      z *= f;
      lost *= f;
      top = b;
    }
    float w[V];
#pragma unroll
    for (int v = 0; v < V; ++v) w[v] = __expf(s[v] - top);
#pragma unroll
    for (int o = V / 2; o > 0; o /= 2)
#pragma unroll
      for (int v = 0; v < o; ++v) w[v] += w[v + o];
    const float y = __fsub_rn(w[0], lost), t1 = __fadd_rn(z, y);
    lost = __fsub_rn(__fsub_rn(t1, z), y);
    z = t1;
    if (uncut) {
      float g[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        g[v] = load_if(x.noise + at[v], s[v] > -INFINITY && !x.r.greedy);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!(s[v] > -INFINITY)) continue;
        const float k = x.r.greedy ? s[v] : draw_value(s[v], g[v]);
        if (k > best_key) {  // indices grow: the first of equal ones stays
          best_key = k;
          best_at = at[v];
        }
      }
    }
  };
  // (two copies, each compiled for its case: one for both took 45.5 us for 43.9 on 64 rows x 50,021 with
  // top-p, and 237 for 217 on 80 uncut ones of 1,048,576)
  if (uncut) row.walk(t, first);
  else row.walk(t, first);
  z = __fsub_rn(z, lost);
  const float mine = top;
  float low = mine > -INFINITY ? mine : INFINITY;  // least of the lanes' maxima
  unsigned long long best = best_key > -INFINITY ? composite(ordered(best_key), best_at) : 0;
  auto join_lanes = [&]() {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
      join_stats(top, z, __shfl_xor_sync(~0u, top, o), __shfl_xor_sync(~0u, z, o));
      low = fminf(low, __shfl_xor_sync(~0u, low, o));
    }
  };
  join_lanes();
  if (lane == 0) {
    sh.warp_f[warp][0] = top;
    sh.warp_f[warp][1] = z;
    sh.warp_f[warp][2] = low;
  }
  if (direct) best = block_max(best, sh);
  __syncthreads();
  if (warp == 0) {
    top = lane < warps ? sh.warp_f[lane][0] : -INFINITY;
    z = lane < warps ? sh.warp_f[lane][1] : 0.0f;
    low = lane < warps ? sh.warp_f[lane][2] : INFINITY;
    join_lanes();
    if (lane == 0) {
      sh.top = top;
      sh.z = z;
      sh.low = low;
      if (t.size > 1) {
        t.g->stats[t.rank] = make_float4(top, z, low, 0.0f);
        t.g->best[t.rank] = best;
      }
    }
  }
  if (t.size > 1) {
    if (t.rank == 0) {
      for (int b = threadIdx.x; b < t.bins; b += blockDim.x) {
        t.g->count[t.stage % 3][b] = 0;
        t.g->mass[t.stage % 3][b] = 0;
      }
      if (threadIdx.x < kCounters) t.g->listed[threadIdx.x] = 0;
    }
    if (!team_sync(t, sh)) return false;
    if (warp == 0) {
      top = -INFINITY;
      z = 0.0f;
      low = INFINITY;
      best = 0;
      for (int c = lane; c < t.size; c += 32) {
        const float4 q = __ldcg(&t.g->stats[c]);
        join_stats(top, z, q.x, q.y);
        low = fminf(low, q.z);
        best = max(best, __ldcg(&t.g->best[c]));
      }
      join_lanes();
#pragma unroll
      for (int o = 16; o > 0; o /= 2) best = max(best, __shfl_xor_sync(~0u, best, o));
      if (lane == 0) {
        sh.top = top;
        sh.z = z;
        sh.low = low;
      }
    }
  }
  __syncthreads();
  x.top = sh.top;
  if (x.top == -INFINITY) {
    if (t.rank == 0) none_drawn(a, row_at, 0);
    return true;
  }
  x.logz = logf(sh.z);
  x.weight = Weights(x.top, sh.z, static_cast<int>(a.n));
  if (direct) {
    if (t.rank == 0) {
      if (threadIdx.x == 0) put(a, x, 0, index_of(best), row.score(index_of(best)));
      none_drawn(a, row_at, 1);
    }
    return true;
  }
  // Bins reach four times as far down as the least of the threads' maxima, which covers a row of
  // any usual shape; what lies below shares the last bin.  Further than 40 there is no mass.
  const float range = fminf(4.0f * __fsub_rn(x.top, sh.low), 40.0f), last = static_cast<float>(t.bins - 1);
  const Bins by_score = {x.top, range > 0.0f ? fminf(last / range, 1e30f) : 0.0f, last};

  // A top-k of less than half as many entries as threads: the k-th of the threads' maxima bounds the
  // k-th entry from below.  Few entries beside the k lie above it; they are collected in one
  // more pass, which most threads skip, and one CTA does the rest from the list.
  const long long threads = static_cast<long long>(t.size) * blockDim.x;
  if (x.r.k != 0 && 2ll * x.r.k <= threads) {
    int bin;
    if (!bin_of_maxima(t, sh, by_score, x.r.k, mine, kList + 1, &bin)) return false;
    if (bin >= 0) {
      unsigned long long* list = t.size > 1 ? t.g->large : sh.list;
      unsigned* listed = t.size > 1 ? &t.g->listed[kTopK] : &sh.listed;
      const unsigned capacity = t.size > 1 ? kLarge : kList;
      if (threadIdx.x == 0) sh.listed = 0;
      __syncthreads();
      collect<true>(row, t, by_score, bin, mine, kIndexBits + 32, 0, All(), list, listed, capacity);
      if (!team_sync(t, sh)) return false;
      const unsigned have = t.size > 1 ? __ldcg(listed) : sh.listed;
      if (have <= capacity) {
        if (t.rank != 0) return true;
        if (have <= kList) {
          take_list(t, sh, list, listed);
          sort_list(t, sh, have);
          finish_list(a, t, sh, x, row);
          return true;
        }
        // more than can be sorted: the same selections, from the candidates and by this CTA alone
        const Candidates src = {list, static_cast<int>(have)};
        float own = -INFINITY;
        src.walk(t, [&](const int(&)[Candidates::V], float(&s)[Candidates::V]) {
#pragma unroll
          for (int v = 0; v < Candidates::V; ++v) own = fmaxf(own, s[v]);
        });
        Team alone = t;
        alone.size = 1;
        return finish_select(a, alone, sh, x, row, src, by_score, own, __int_as_float(0x7FFFFFFF));
      }
      if (t.size > 1) {
        // a crowded bin: the list's counter starts anew
        if (!team_sync(t, sh)) return false;
        if (t.rank == 0 && threadIdx.x == 0) t.g->listed[kTopK] = 0;
        if (!team_sync(t, sh)) return false;
      }
    }
  }
  return finish_select(a, t, sh, x, row, row, by_score, mine, uncut ? best_key : __int_as_float(0x7FFFFFFF));
}

template <typename T>
__global__ void __launch_bounds__(1024) k_sample_row(SampleArgs a, int team_size, int bins, int cluster) {
  extern __shared__ __align__(16) unsigned char smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  Team t;
  t.size = team_size;
  t.rank = blockIdx.x % team_size;
  t.g = team_size > 1 ? static_cast<TeamMem*>(a.ws) + blockIdx.x / team_size : nullptr;
  t.err = a.err;
  t.cluster = cluster != 0;
  t.barriers = 0;
  t.stage = 0;
  t.bins = bins;
  if (team_size > 1 && !t.cluster) {
    if (a.stall_us != 0 && t.rank == team_size - 1) return;
    // thread 0 alone reads it
    if (threadIdx.x == 0) sh.wait_ns = a.stall_us != 0 ? a.stall_us * 1000ull : kWaitLimitNs;
    // rank 0 writes the row's draws after its last wait; where a wait gives up this is what remains
    if (t.rank == 0) none_drawn(a, blockIdx.x / team_size, 0);
  }
  sample_row<T>(a, t, sh, blockIdx.x / team_size);
}

bool by_warp(long long n, int m) { return n <= kWarpMaxN && m <= kWarpMaxM; }

constexpr int kMaxCluster = 16;

size_t row_smem() { return sizeof(Shared); }

// Clusters of `size` CTAs that the device holds at once (0: none, or no device).
int resident_clusters(int size) {
  static std::atomic<int> known[kMaxCluster + 1];  // 0: not asked yet, else one more than the number
  int v = known[size].load(std::memory_order_relaxed);
  if (v == 0) {
    auto kernel = k_sample_row<float>;
    int n = 0;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = size;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(size);
    cfg.blockDim = dim3(1024);
    cfg.dynamicSmemBytes = row_smem();
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (allow_smem(reinterpret_cast<const void*>(kernel), row_smem()) != cudaSuccess ||
        cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeNonPortableClusterSizeAllowed, 1) !=
            cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
      cudaGetLastError();  // no device: nothing sticks
      n = 0;
    }
    v = n + 1;
    known[size].store(v, std::memory_order_relaxed);
  }
  return v - 1;
}

// CTAs of a team: all SMs divided over the rows, but no CTA with less than 4,096 entries (one row of
// 50,021 with top-p: 35 us by 13 CTAs, 55 by two).  Teams are clusters, whose barrier takes a
// tenth of one in global memory (0.3 us against 3), of the largest size of which the device
// holds one for every row; where these would use less than two thirds of the SMs that a
// barrier in global memory could, it is that.  (8 rows of 1,048,576 scores: eight clusters of 16
// are not resident at once and take two turns, 157 us with top-p against 81.)
struct TeamPlan {
  int size;
  bool cluster;
};
TeamPlan team_of(long long rows, long long n, int sms) {
  if (rows * 2 > sms) return {1, false};
  long long t = sms / rows;
  t = t < (n + 4095) / 4096 ? t : (n + 4095) / 4096;
  t = t < kMaxTeam ? t : kMaxTeam;
  if (t < 2) return {1, false};
  int c = t < kMaxCluster ? static_cast<int>(t) : kMaxCluster;
  while (c > 1 && resident_clusters(c) < rows) --c;
  if (c > 1 && 3 * c >= 2 * t) return {c, true};
  return {static_cast<int>(t), false};
}

}  // namespace

size_t sample_workspace(int, long long rows, long long n, int m, int sms) {
  if (rows == 0 || by_warp(n, m)) return 0;
  return team_of(rows, n, sms).size > 1 ? up256(sizeof(TeamMem) * static_cast<size_t>(rows)) : 0;
}

cudaError_t launch_sample(const SampleArgs& a, int sms, long long* launches, cudaStream_t st) {
  return with_dtype(a.dtype, [&](auto tag) -> cudaError_t {
    using T = decltype(tag);
    if (by_warp(a.n, a.m)) {
      ++*launches;
      const dim3 grid(static_cast<unsigned>((a.rows + 3) / 4));
      const int per = static_cast<int>((a.n + 31) / 32);
      if (per <= 1) return launch_pdl(k_sample_warp<T, 1>, grid, dim3(128), 0, st, a);
      if (per <= 2) return launch_pdl(k_sample_warp<T, 2>, grid, dim3(128), 0, st, a);
      if (per <= 4) return launch_pdl(k_sample_warp<T, 4>, grid, dim3(128), 0, st, a);
      if (per <= 8) return launch_pdl(k_sample_warp<T, 8>, grid, dim3(128), 0, st, a);
      return launch_pdl(k_sample_warp<T, 16>, grid, dim3(128), 0, st, a);
    }
    const TeamPlan plan = team_of(a.rows, a.n, sms);
    const int team = plan.size;
    const size_t smem = row_smem();
    cudaError_t e = allow_smem(reinterpret_cast<const void*>(k_sample_row<T>), smem);
    if (e != cudaSuccess) return e;
    // small CTAs for short rows: several share an SM, and barriers take fewer warps
    // (many draws want threads to sort them)
    int threads = a.n <= 4096 ? 128 : a.n <= 16384 ? 256 : a.n <= 32768 ? 512 : 1024;
    while (threads < 1024 && threads * 4 < a.m) threads *= 2;
    if (team > 1) threads = 1024;
    // a multiple of the threads; fewer are more crowded (64 x 50,021: 49 us with 1,024, 43 with 2,048)
    const int bins = threads <= 512 && a.n <= 16384 ? 512 : kBins;
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    if (team == 1) {
      cfg.gridDim = dim3(static_cast<unsigned>(a.rows));
      ++*launches;
      return cudaLaunchKernelEx(&cfg, k_sample_row<T>, a, 1, bins, 0);
    }
    cfg.gridDim = dim3(static_cast<unsigned>(team * a.rows));
    cudaLaunchAttribute attr[1];
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ++*launches;
    if (plan.cluster) {
      e = cudaFuncSetAttribute(reinterpret_cast<const void*>(k_sample_row<T>),
                               cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = team;
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      return cudaLaunchKernelEx(&cfg, k_sample_row<T>, a, team, bins, 1);
    }
    // the barriers' counters start from zero
    e = cudaMemset2DAsync(a.ws, sizeof(TeamMem), 0, 16, static_cast<size_t>(a.rows), st);
    if (e != cudaSuccess) return e;
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    return cudaLaunchKernelEx(&cfg, k_sample_row<T>, a, team, bins, 0);
  });
}

}  // namespace mlt
