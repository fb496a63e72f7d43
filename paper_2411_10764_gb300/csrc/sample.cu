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
// to five passes over a CTA's share and a barrier for each.
//
// Two kernels:
//   k_sample_warp  rows of up to 512 entries and m <= 32: a warp per row, the row in
//                  registers, selection by ballots and warp sums, no barrier;
//   k_sample_row   longer rows: a team of CTAs per row.  Where there are fewer
//                  rows than SMs the team has several CTAs, which meet at a
//                  barrier in global memory (cooperative launch, so all are
//                  resident; the wait is bounded).
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

// Order-preserving map of finite floats (no -0: the caller adds +0).
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ float clamp_finite(float v) { return fminf(fmaxf(v, -FLT_MAX), FLT_MAX); }

// Scaled score; false where the entry can never be drawn.
__device__ __forceinline__ bool scaled(float x, float inv, float* s) {
  const float v = __fmul_rn(x, inv);
  *s = clamp_finite(v) + 0.0f;
  return v == v && x != -INFINITY;
}
__device__ __forceinline__ uint32_t draw_key(float s, float noise) {
  const float k = __fadd_rn(s, noise);
  return ordered(k == k ? clamp_finite(k) + 0.0f : -FLT_MAX);
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
  r.inv = r.greedy ? 1.0f : __fdiv_rn(1.0f, q.temperature);
  r.k = r.greedy || q.top_k <= 0 || q.top_k >= n ? 0u : static_cast<unsigned>(q.top_k);
  r.p = r.greedy ? 1.0f : q.top_p;
  r.log_min = r.greedy || q.min_p <= 0.0f ? -INFINITY : fminf(logf(q.min_p), 0.0f);  // the best stays
  return r;
}

// Weight of an entry in fixed point: exp(s - top) * 2^shift.
__device__ __forceinline__ unsigned long long fixed_weight(float s, float top, float unit) {
  return __float2ull_rn(expf(__fsub_rn(s, top)) * unit);
}

// ---------------------------------------------------------------------------
// A warp per row
// ---------------------------------------------------------------------------
__device__ __forceinline__ unsigned long long warp_sum_fixed(unsigned long long v) {
  // lanes hold up to 2^48 (16 weights of 2^44): 32 halves of 22 and of 26 bits add up below 2^32
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
    s[j] = 0.0f;
    key[j] = 0;
    if (i < n && scaled(to_f32(x[i]), r.inv, &s[j])) key[j] = ordered(s[j]);
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
    const float unit = static_cast<float>(1ull << 44);
    unsigned long long w[PER];
    unsigned long long sum = 0;
    unsigned seen = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const unsigned eq = __ballot_sync(~0u, key[j] == tau);
      const bool keep = key[j] > tau || (key[j] == tau && seen + __popc(eq & ((1u << lane) - 1u)) < ties);
      seen += __popc(eq);
      w[j] = keep ? fixed_weight(s[j], top, unit) : 0;
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
      const unsigned long long each = max(1ull, fixed_weight(from_ordered(at), top, unit));
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
    if (keep) draw[j] = r.greedy ? key[j] : draw_key(s[j], noise[j * 32 + lane]);
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
constexpr int kUses = 3;  // selections of a row: top-k, top-p, draws

// Global memory of a team; teams of one CTA use none of it.
struct TeamMem {
  unsigned arrivals;      // barrier: CTAs arrived, over all barriers of the call (zeroed before the launch)
  unsigned listed[kUses]; // entries in list
  float4 stats[kMaxTeam]; // each CTA's (max, sum of exp, min)
  unsigned long long best[kMaxTeam];
  unsigned long long mass[3][kBins];
  unsigned count[3][kBins];
  unsigned long long list[kUses][kList];
};

struct Shared {
  unsigned long long list[kList];
  unsigned long long mass[kBins];  // merged
  unsigned count[kBins];
  unsigned lo[kBins], hi[kBins];   // of the CTA's masses
  unsigned long long warp_u64[32];
  float warp_f[32][3];
  unsigned long long above, edge;
  unsigned in, bin, listed;
  float top, z, low;
  int dead;
};

struct Team {
  TeamMem* g;
  unsigned* err;
  int size, rank;
  unsigned barriers;
  int stage;  // histograms used so far
};

// All CTAs of the team; false where the wait gave up (then on every thread of the CTA).
__device__ bool team_sync(Team& t, Shared& sh) {
  __syncthreads();
  if (t.size == 1) return true;
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
      if (now - start > kWaitLimitNs) {
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

// f(i0, x, valid) for every 16-byte group of the row that the thread owns: x[v] is entry
// i0 + v where bit v of valid is set.
template <typename T, typename F>
__device__ __forceinline__ void walk(const T* row, long long n, const Team& t, F f) {
  constexpr int V = 16 / sizeof(T);
  constexpr int U = sizeof(T) == 4 ? 4 : 2;
  const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(row) / sizeof(T)) % V);
  const int groups = static_cast<int>((skew + n + V - 1) / V);  // n <= 2^27
  const int stride = t.size * static_cast<int>(blockDim.x);
  const T* base = row - skew;  // 16-byte aligned; entries before `row` are not read
  for (int q0 = t.rank * static_cast<int>(blockDim.x) + threadIdx.x; q0 < groups; q0 += stride * U) {
    Pack<T, V> p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = q0 + u * stride, i0 = q * V - skew;
      if (q < groups && i0 >= 0 && i0 + V <= n)
        p[u] = *reinterpret_cast<const Pack<T, V>*>(base + static_cast<long long>(q) * V);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int q = q0 + u * stride, i0 = q * V - skew;
      if (q >= groups) break;
      float x[V];
      unsigned valid = (1u << V) - 1u;
      if (i0 >= 0 && i0 + V <= n) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = to_f32(p[u].v[v]);
      } else {
        // a row's ends
        valid = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          x[v] = -INFINITY;
          if (i0 + v >= 0 && i0 + v < n) {
            x[v] = to_f32(row[i0 + v]);
            valid |= 1u << v;
          }
        }
      }
      f(i0, x, valid);
    }
  }
}

__device__ __forceinline__ void clear_bins(Shared& sh, bool mass) {
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += blockDim.x) {
    sh.count[b] = 0;
    if (mass) sh.lo[b] = sh.hi[b] = 0;
  }
  __syncthreads();
}

__device__ __forceinline__ void add_mass(Shared& sh, int b, unsigned long long w) {
  // shared memory adds 32 bits at a time: the carry goes to the upper half
  const unsigned lo = static_cast<unsigned>(w);
  const unsigned old = atomicAdd(&sh.lo[b], lo);
  const unsigned hi = static_cast<unsigned>(w >> 32) + (old + lo < old ? 1u : 0u);
  if (hi != 0) atomicAdd(&sh.hi[b], hi);
}

// The team's bins of this stage, merged, in sh.count and (kMass) sh.mass.
template <bool kMass>
__device__ bool merge_bins(Team& t, Shared& sh) {
  __syncthreads();
  if (t.size == 1) {
    if (kMass) {
      for (int b = threadIdx.x; b < kBins; b += blockDim.x)
        sh.mass[b] = (static_cast<unsigned long long>(sh.hi[b]) << 32) + sh.lo[b];
      __syncthreads();
    }
    return true;
  }
  const int now = t.stage % 3, next = (t.stage + 1) % 3;  // `next` was last read before the previous barrier
  ++t.stage;
  for (int b = threadIdx.x; b < kBins; b += blockDim.x) {
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
  for (int b = threadIdx.x; b < kBins; b += blockDim.x) {
    sh.count[b] = __ldcg(&t.g->count[now][b]);
    if (kMass) sh.mass[b] = __ldcg(&t.g->mass[now][b]);
  }
  __syncthreads();
  return true;
}

// Sum over the CTA, on every thread.
__device__ __forceinline__ unsigned long long block_sum(unsigned long long v, Shared& sh) {
#pragma unroll
  for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(~0u, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.warp_u64[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) v += sh.warp_u64[w];
  return v;
}
__device__ __forceinline__ unsigned long long block_max(unsigned long long v, Shared& sh) {
#pragma unroll
  for (int o = 16; o > 0; o /= 2) v = max(v, __shfl_xor_sync(~0u, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.warp_u64[threadIdx.x >> 5] = v;
  __syncthreads();
  for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) v = max(v, sh.warp_u64[w]);
  return v;
}
// The CTA's sum over lower threads; *all: over every thread.
__device__ __forceinline__ unsigned long long block_below(unsigned long long mine, Shared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long v = mine;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const unsigned long long w = __shfl_up_sync(~0u, v, o);
    if (lane >= o) v += w;
  }
  __syncthreads();
  if (lane == 31) sh.warp_u64[warp] = v;
  __syncthreads();
  v -= mine;
  for (int w = 0; w < warp; ++w) v += sh.warp_u64[w];
  return v;
}

// The first bin where the running sum of counts (or masses) reaches `need`: sh.bin, the sum
// before it sh.above, its count sh.in (0 where the sum stays below).
template <bool kMass>
__device__ void find_bin(Shared& sh, unsigned long long need) {
  const int span = kBins / blockDim.x, first = threadIdx.x * span;
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

// sh.list[0 .. n), descending.
__device__ void sort_list(Shared& sh, unsigned n) {
  unsigned width = 1;
  while (width < n) width *= 2;
  for (unsigned j = n + threadIdx.x; j < width; j += blockDim.x) sh.list[j] = 0;
  __syncthreads();
  for (unsigned k = 2; k <= width; k *= 2)
    for (unsigned j = k / 2; j > 0; j /= 2) {
      for (unsigned q = threadIdx.x; q < width / 2; q += blockDim.x) {
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

// Bins of a selection: linear from `from` down, kBins / range a unit; what lies outside goes to
// the first or last one.  Rounded steps of it are monotone, so a bin is an interval.
struct Bins {
  float from, scale;
  __device__ __forceinline__ int of(float v) const {
    return static_cast<int>(fminf(fmaxf(__fmul_rn(__fsub_rn(from, v), scale), 0.0f), static_cast<float>(kBins - 1)));
  }
};

// Selects from the entries that get() gives: get(i0, x, valid, key) -> bits of the entries that
// take part, with their keys.
//   kMass = false: the `need`-th largest composite; kAbove: the `need` largest
//   kMass = true:  the composite at which the mass reaches `share` of all
// Leaves a sorted list in sh.list.  *edge: the composite found (0: the entries do not
// reach that far, all are kept).  kAbove: sh.listed entries, on rank 0 only, and no edge.
template <typename T, bool kMass, bool kAbove, typename Get>
__device__ bool select(const T* x, long long n, Team& t, Shared& sh, int use, Bins bins, unsigned long long need,
                       float share, float top, float unit, Get get, unsigned long long* edge) {
  constexpr int V = 16 / sizeof(T);
  *edge = 0;
  if (threadIdx.x == 0) sh.listed = 0;
  clear_bins(sh, kMass);
  walk(x, n, t, [&](int i0, const float(&xs)[V], unsigned valid) {
    uint32_t key[V];
    const unsigned in = get(i0, xs, valid, key);
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (in >> e & 1u) {
        const float v = from_ordered(key[e]);
        const int b = bins.of(v);
        atomicAdd(&sh.count[b], 1u);
        if (kMass) add_mass(sh, b, fixed_weight(v, top, unit));
      }
  });
  if (!merge_bins<kMass>(t, sh)) return false;
  if (kMass) {
    unsigned long long sum = 0;
    for (int b = threadIdx.x; b < kBins; b += blockDim.x) sum += sh.mass[b];
    sum = block_sum(sum, sh);
    need = share > 0.0f ? max(1ull, static_cast<unsigned long long>(static_cast<double>(share) *
                                                                    static_cast<double>(sum)))
                        : 1ull;
  }
  find_bin<kMass>(sh, need);
  int bin = static_cast<int>(sh.bin);
  unsigned in = sh.in;
  unsigned above_n = 0;  // kAbove: entries above the bin (the list takes them too)
  if (in == 0) {
    if (!kAbove) return true;
    bin = kBins - 1;  // fewer than `need`: all of them
  } else {
    need -= sh.above;
    if (kAbove) above_n = static_cast<unsigned>(sh.above);
  }
  // a bin that does not fit the list: digits of the composite
  int shift = kIndexBits + 32;
  unsigned long long prefix = 0;
#pragma unroll 1
  while (in + above_n > kList) {
    const int bits = min(11, shift);
    shift -= bits;
    clear_bins(sh, kMass);
    walk(x, n, t, [&](int i0, const float(&xs)[V], unsigned valid) {
      uint32_t key[V];
      const unsigned on = get(i0, xs, valid, key);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const unsigned long long c = composite(key[e], i0 + e);
        if ((on >> e & 1u) && bins.of(from_ordered(key[e])) == bin && (c >> (shift + bits)) == prefix) {
          const int b = kBins - 1 - static_cast<int>((c >> shift) & ((1u << bits) - 1u));
          atomicAdd(&sh.count[b], 1u);
          if (kMass) add_mass(sh, b, fixed_weight(from_ordered(key[e]), top, unit));
        }
      }
    });
    if (!merge_bins<kMass>(t, sh)) return false;
    find_bin<kMass>(sh, need);
    prefix = (prefix << bits) | static_cast<unsigned>(kBins - 1 - sh.bin);
    in = sh.in;
    need -= sh.above;
    if (kAbove) above_n += static_cast<unsigned>(sh.above);
  }
  unsigned long long* list = t.size > 1 ? t.g->list[use] : sh.list;
  unsigned* listed = t.size > 1 ? &t.g->listed[use] : &sh.listed;
  walk(x, n, t, [&](int i0, const float(&xs)[V], unsigned valid) {
    uint32_t key[V];
    const unsigned on = get(i0, xs, valid, key);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (!(on >> e & 1u)) continue;
      const int b = bins.of(from_ordered(key[e]));
      if (b > bin || (!kAbove && b != bin)) continue;
      const unsigned long long c = composite(key[e], i0 + e), high = c >> shift;
      if (b < bin || (kAbove ? high >= prefix : high == prefix)) {
        const unsigned at = atomicAdd(listed, 1u);
        if (at < kList) list[at] = c;
      }
    }
  });
  if (!team_sync(t, sh)) return false;
  if (kAbove && t.rank != 0) return true;
  if (t.size > 1) {
    const unsigned have = min(__ldcg(listed), static_cast<unsigned>(kList));
    for (unsigned j = threadIdx.x; j < have; j += blockDim.x) sh.list[j] = __ldcg(&list[j]);
    if (threadIdx.x == 0) sh.listed = have;
    __syncthreads();
  }
  const unsigned have = min(sh.listed, static_cast<unsigned>(kList));
  sort_list(sh, have);
  if (kAbove) return true;
  if (!kMass) {
    *edge = sh.list[need - 1];
  } else {
    // the entry at which the running mass reaches `need` (the last one if rounding leaves less)
    const unsigned span = (have + blockDim.x - 1) / blockDim.x, first = threadIdx.x * span;
    unsigned long long mine = 0;
    for (unsigned j = first; j < min(first + span, have); ++j) mine += fixed_weight(score_of(sh.list[j]), top, unit);
    unsigned long long at = block_below(mine, sh);
    if (threadIdx.x == 0) sh.edge = sh.list[have - 1];
    __syncthreads();
    if (at < need && at + mine >= need)
      for (unsigned j = first; j < min(first + span, have); ++j) {
        at += fixed_weight(score_of(sh.list[j]), top, unit);
        if (at >= need) {
          sh.edge = sh.list[j];
          break;
        }
      }
    __syncthreads();
    *edge = sh.edge;
  }
  __syncthreads();
  return true;
}

__device__ __forceinline__ void none_drawn(const SampleArgs& a, long long row, int from) {
  for (int j = from + threadIdx.x; j < a.m; j += blockDim.x) {
    a.out_index[row * a.m + j] = -1;
    a.out_logprob[row * a.m + j] = -INFINITY;
  }
}

template <int V>
__device__ __forceinline__ unsigned scale_group(const float (&x)[V], unsigned valid, float inv, float (&s)[V]) {
  unsigned alive = 0;
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (scaled(x[v], inv, &s[v])) alive |= 1u << v;
  return alive & valid;
}

__device__ __forceinline__ void join_stats(float& m, float& z, float m2, float z2) {
  const float b = fmaxf(m, m2);
  if (b == -INFINITY) return;
  z = z * __expf(m - b) + z2 * __expf(m2 - b);
  m = b;
}

template <typename T>
__device__ bool sample_row(const SampleArgs& a, Team& t, Shared& sh, long long row) {
  constexpr int V = 16 / sizeof(T);
  const long long n = a.n;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const Rule r = read_rule(a.rules != nullptr ? a.rules[row] : a.rule, n);
  const T* x = static_cast<const T*>(a.scores) + row * a.row_stride;
  const float* noise = a.noise + row * a.noise_stride;
  if (r.bad) {
    if (t.rank == 0) {
      if (threadIdx.x == 0) atomicOr(a.err, kErrBadRule);
      none_drawn(a, row, 0);
    }
    return true;
  }
  // One draw from an uncut row needs no edge: it is found in the first pass.
  const bool direct = (a.m == 1 || r.greedy) && r.k == 0 && r.p >= 1.0f && r.log_min == -INFINITY;

  // Pass 1: maximum, minimum and sum of exponentials, each lane's own, then joined in a fixed order.
  float top = -INFINITY, z = 0.0f, low = INFINITY;
  unsigned long long best = 0;
  walk(x, n, t, [&](int i0, const float(&xs)[V], unsigned valid) {
    float s[V];
    const unsigned alive = scale_group<V>(xs, valid, r.inv, s);
    float b = top;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (alive >> v & 1u) {
        b = fmaxf(b, s[v]);
        low = fminf(low, s[v]);
      }
    if (b > top) {
      z *= __expf(top - b);
      top = b;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (alive >> v & 1u) z += __expf(s[v] - top);
    if (direct) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (alive >> v & 1u)
          best = max(best, composite(r.greedy ? ordered(s[v]) : draw_key(s[v], noise[i0 + v]), i0 + v));
    }
  });
#pragma unroll
  for (int o = 16; o > 0; o /= 2) {
    join_stats(top, z, __shfl_xor_sync(~0u, top, o), __shfl_xor_sync(~0u, z, o));
    low = fminf(low, __shfl_xor_sync(~0u, low, o));
  }
  if (lane == 0) {
    sh.warp_f[warp][0] = top;
    sh.warp_f[warp][1] = z;
    sh.warp_f[warp][2] = low;
  }
  if (direct) best = block_max(best, sh);
  __syncthreads();
  if (warp == 0) {
    // one warp joins, by a tree too: its shape is fixed
    top = lane < warps ? sh.warp_f[lane][0] : -INFINITY;
    z = lane < warps ? sh.warp_f[lane][1] : 0.0f;
    low = lane < warps ? sh.warp_f[lane][2] : INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
      join_stats(top, z, __shfl_xor_sync(~0u, top, o), __shfl_xor_sync(~0u, z, o));
      low = fminf(low, __shfl_xor_sync(~0u, low, o));
    }
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
      for (int b = threadIdx.x; b < kBins; b += blockDim.x) {
        t.g->count[t.stage % 3][b] = 0;
        t.g->mass[t.stage % 3][b] = 0;
      }
      if (threadIdx.x < kUses) t.g->listed[threadIdx.x] = 0;
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
#pragma unroll
      for (int o = 16; o > 0; o /= 2) {
        join_stats(top, z, __shfl_xor_sync(~0u, top, o), __shfl_xor_sync(~0u, z, o));
        low = fminf(low, __shfl_xor_sync(~0u, low, o));
        best = max(best, __shfl_xor_sync(~0u, best, o));
      }
      if (lane == 0) {
        sh.top = top;
        sh.z = z;
        sh.low = low;
      }
    }
  }
  __syncthreads();
  top = sh.top;
  z = sh.z;
  if (direct || top == -INFINITY) {
    if (t.rank == 0) {
      if (threadIdx.x == 0 && top != -INFINITY) {
        const int i = index_of(best);
        float s;
        scaled(to_f32(x[i]), r.inv, &s);
        a.out_index[row * a.m] = i;
        a.out_logprob[row * a.m] = r.greedy ? 0.0f : __fsub_rn(s, top) - logf(z);
      }
      none_drawn(a, row, top != -INFINITY ? 1 : 0);
    }
    return true;
  }

  // The cuts.  Scores more than 40 below the best share the last bin: their mass is
  // nothing, and only a top-k of a very peaked row looks there.
  const float range = fminf(__fsub_rn(top, sh.low), 40.0f);
  const Bins by_score = {top, range > 0.0f ? fminf(static_cast<float>(kBins - 1) / range, 1e30f) : 0.0f};
  unsigned long long edge = 0;
  // an entry's composite is at or above the edge
  auto kept = [&](uint32_t key, int i) {
    const uint32_t ek = static_cast<uint32_t>(edge >> kIndexBits);
    return key > ek || (key == ek && i <= index_of(edge));
  };
  auto scores = [&](int i0, const float(&xs)[V], unsigned valid, uint32_t(&key)[V]) {
    float s[V];
    unsigned in = scale_group<V>(xs, valid, r.inv, s);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      key[v] = ordered(s[v]);
      if (!kept(key[v], i0 + v)) in &= ~(1u << v);
    }
    return in;
  };
  unsigned long long found;
  if (r.k != 0) {
    if (!select<T, false, false>(x, n, t, sh, 0, by_score, r.k, 0.0f, top, 0.0f, scores, &found)) return false;
    edge = found;
  }
  if (r.p < 1.0f) {
    int log_n = 0;
    while ((1ll << log_n) < n) ++log_n;
    const float unit = static_cast<float>(1ull << (62 - log_n));
    if (!select<T, true, false>(x, n, t, sh, 1, by_score, 0, r.p, top, unit, scores, &found)) return false;
    edge = max(edge, found);
  }

  // Bits of the group's kept entries and their draw keys.
  auto draws = [&](int i0, const float(&xs)[V], unsigned valid, uint32_t(&key)[V]) {
    float s[V];
    unsigned in = scale_group<V>(xs, valid, r.inv, s);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!kept(ordered(s[v]), i0 + v) || !(__fsub_rn(s[v], top) >= r.log_min)) in &= ~(1u << v);
      key[v] = in >> v & 1u ? draw_key(s[v], noise[i0 + v]) : 0;
    }
    return in;
  };
  const float logz = logf(z);
  if (a.m == 1) {
    best = 0;
    walk(x, n, t, [&](int i0, const float(&xs)[V], unsigned valid) {
      uint32_t key[V];
      const unsigned in = draws(i0, xs, valid, key);
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (in >> v & 1u) best = max(best, composite(key[v], i0 + v));
    });
    best = block_max(best, sh);
    if (t.size > 1) {
      if (threadIdx.x == 0) t.g->best[t.rank] = best;
      if (!team_sync(t, sh)) return false;
      if (t.rank == 0 && threadIdx.x == 0)
        for (int c = 0; c < t.size; ++c) best = max(best, __ldcg(&t.g->best[c]));
    }
    if (t.rank == 0 && threadIdx.x == 0) {
      const int i = index_of(best);  // no cut drops the best entry
      float s;
      scaled(to_f32(x[i]), r.inv, &s);
      a.out_index[row] = i;
      a.out_logprob[row] = __fsub_rn(s, top) - logz;
    }
    return true;
  }
  // Gumbel noise puts the largest keys within a few units of the best score, and ln n above it.
  const Bins by_key = {top + 24.0f, static_cast<float>(kBins) / 48.0f};
  if (!select<T, false, true>(x, n, t, sh, 2, by_key, a.m, 0.0f, top, 0.0f, draws, &found)) return false;
  if (t.rank != 0) return true;
  const int drawn = static_cast<int>(min(sh.listed, static_cast<unsigned>(a.m)));
  for (int j = threadIdx.x; j < drawn; j += blockDim.x) {
    const int i = index_of(sh.list[j]);
    float s;
    scaled(to_f32(x[i]), r.inv, &s);
    a.out_index[row * a.m + j] = i;
    a.out_logprob[row * a.m + j] = __fsub_rn(s, top) - logz;
  }
  none_drawn(a, row, drawn);
  __syncthreads();
  return true;
}

template <typename T>
__global__ void __launch_bounds__(1024) k_sample_row(SampleArgs a, int team_size) {
  extern __shared__ __align__(16) unsigned char smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  Team t;
  t.size = team_size;
  t.rank = blockIdx.x % team_size;
  t.g = team_size > 1 ? static_cast<TeamMem*>(a.ws) + blockIdx.x / team_size : nullptr;
  t.err = a.err;
  t.barriers = 0;
  t.stage = 0;
  sample_row<T>(a, t, sh, blockIdx.x / team_size);
}

bool by_warp(long long n, int m) { return n <= kWarpMaxN && m <= kWarpMaxM; }

// CTAs per row: all SMs divided over the rows, but no CTA with less than 4,096 entries
// (a barrier of a team costs about as much as a CTA's passes over that many).
int team_of(long long rows, long long n, int sms) {
  if (rows * 2 > sms) return 1;
  long long t = sms / rows;
  t = t < (n + 4095) / 4096 ? t : (n + 4095) / 4096;
  t = t < kMaxTeam ? t : kMaxTeam;
  return static_cast<int>(t < 1 ? 1 : t);
}

}  // namespace

size_t sample_workspace(int, long long rows, long long n, int m, int sms) {
  if (rows == 0 || by_warp(n, m)) return 0;
  return team_of(rows, n, sms) > 1 ? up256(sizeof(TeamMem) * static_cast<size_t>(rows)) : 0;
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
    const int team = team_of(a.rows, a.n, sms);
    const size_t smem = sizeof(Shared);
    cudaError_t e = allow_smem(reinterpret_cast<const void*>(k_sample_row<T>), smem);
    if (e != cudaSuccess) return e;
    const int threads = a.n <= 2048 ? 256 : a.n <= 8192 ? 512 : 1024;
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = dim3(team > 1 ? 1024 : threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    if (team == 1) {
      cfg.gridDim = dim3(static_cast<unsigned>(a.rows));
      ++*launches;
      return cudaLaunchKernelEx(&cfg, k_sample_row<T>, a, 1);
    }
    // the barriers' counters start from zero
    e = cudaMemset2DAsync(a.ws, sizeof(TeamMem), 0, 16, static_cast<size_t>(a.rows), st);
    if (e != cudaSuccess) return e;
    cfg.gridDim = dim3(static_cast<unsigned>(team * a.rows));
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ++*launches;
    return cudaLaunchKernelEx(&cfg, k_sample_row<T>, a, team);
  });
}

}  // namespace mlt
