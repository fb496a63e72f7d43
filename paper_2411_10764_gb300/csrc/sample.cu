// Draws from rows of scores: temperature, top-k, top-p and min-p cuts, then the
// m largest of score + noise among the kept entries (with Gumbel noise, m draws
// without replacement from the kept entries' softmax).
//
// Every cut keeps a prefix of the order (scaled score descending, index
// ascending), so the kept set is {key > tau} and the first `ties` entries with
// key = tau, where key is the scaled score as an ordered 32-bit integer.  tau is found by
// radix selection: histograms over 11, 11 and 10 bits of the key, of entry counts for
// top-k and of probability mass for top-p.  No row is sorted.  Masses are added
// as 64-bit integers (fixed point), so neither atomics nor the split of a row
// over CTAs changes a result.
//
// Bound: the scores are read from HBM once and from L1 or L2 by the later
// passes; noise is read for kept entries only.  What is left beside the first
// read is latency: a pass over a CTA's share and a barrier for each digit.
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
constexpr int kList = 4096;  // composite keys that the last step sorts
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
// Global memory of a team; teams of one CTA use none of it.
struct TeamMem {
  unsigned arrivals;  // barrier: CTAs arrived, over all barriers of the call (zeroed before the launch)
  unsigned listed;    // entries in list
  unsigned long long best;
  float2 stats[160];       // each CTA's (max, sum of exp)
  unsigned long long best_of[160];
  unsigned ties[160];
  unsigned long long hist[3][kBins];
  unsigned long long list[kList];
};
constexpr int kMaxTeam = 160;

struct Shared {
  unsigned long long hist[kBins];
  unsigned long long list[kList];
  unsigned long long warp_u64[32];
  float warp_f[32][2];
  unsigned warp_u32[32];
  unsigned long long found_above, found_in;
  unsigned found_bin;
  unsigned count;
  float top, z;
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

// f(i0, x, valid) for every 16-byte group of the row that the warp owns, in order of
// index: x[v] is entry i0 + v where bit v of valid is set.  Called by whole warps.
// A warp's groups are consecutive, so (CTA, warp, call, lane, v) is the order of indices.
template <typename T, typename F>
__device__ __forceinline__ void walk(const T* row, long long n, const Team& t, F f) {
  constexpr int V = 16 / sizeof(T);
  constexpr int U = 4;
  const int lane = threadIdx.x & 31;
  const int warps = blockDim.x >> 5;
  const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(row) / sizeof(T)) % V);
  const long long groups = (skew + n + V - 1) / V;
  const long long all = static_cast<long long>(t.size) * warps;
  const long long per = ((groups + all - 1) / all + 31) / 32 * 32;
  const long long begin = (static_cast<long long>(t.rank) * warps + (threadIdx.x >> 5)) * per;
  const long long end = min(begin + per, groups);
  const T* base = row - skew;  // 16-byte aligned; entries before `row` are not read
  for (long long q0 = begin; q0 < end; q0 += 32 * U) {
    Pack<T, V> p[U];
    unsigned valid[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long q = q0 + u * 32 + lane;
      const long long i0 = q * V - skew;
      valid[u] = 0;
      if (q < end) {
        if (i0 >= 0 && i0 + V <= n) {
          p[u] = *reinterpret_cast<const Pack<T, V>*>(base + q * V);
          valid[u] = (1u << V) - 1u;
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (i0 + v >= 0 && i0 + v < n) {
              p[u].v[v] = row[i0 + v];
              valid[u] |= 1u << v;
            }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (q0 + u * 32 >= end) break;
      float x[V];
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = (valid[u] >> v & 1u) ? to_f32(p[u].v[v]) : -INFINITY;
      f((q0 + u * 32 + lane) * V - skew, x, valid[u]);
    }
  }
}

// The team's histogram of this stage into sh.hist; then the bin from the top where the
// running sum first reaches `need` (found_bin, the sum above it and the bin's own).
// found_in = 0 where the whole histogram does not reach it.
__device__ bool team_find(Team& t, Shared& sh, unsigned long long need) {
  if (t.size > 1) {
    unsigned long long* h = t.g->hist[t.stage % 3];
    unsigned long long* next = t.g->hist[(t.stage + 1) % 3];  // last read before the previous barrier
    ++t.stage;
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += blockDim.x) {
      if (sh.hist[b] != 0) atomicAdd(&h[b], sh.hist[b]);
      if (t.rank == 0) next[b] = 0;
    }
    if (!team_sync(t, sh)) return false;
    for (int b = threadIdx.x; b < kBins; b += blockDim.x) sh.hist[b] = __ldcg(&h[b]);
  }
  if (threadIdx.x == 0) {
    sh.found_in = 0;
    sh.found_above = 0;
    sh.found_bin = 0;
  }
  __syncthreads();
  // thread j sums `span` bins from the top down
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int span = kBins / blockDim.x;
  unsigned long long mine = 0;
  for (int j = 0; j < span; ++j) mine += sh.hist[kBins - 1 - (threadIdx.x * span + j)];
  unsigned long long v = mine;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const unsigned long long w = __shfl_up_sync(~0u, v, o);
    if (lane >= o) v += w;
  }
  if (lane == 31) sh.warp_u64[warp] = v;
  __syncthreads();
  unsigned long long above = v - mine;
  for (int w = 0; w < warps; ++w)
    if (w < warp) above += sh.warp_u64[w];
  if (above < need && above + mine >= need) {
    for (int j = 0; j < span; ++j) {
      const int b = kBins - 1 - (threadIdx.x * span + j);
      const unsigned long long c = sh.hist[b];
      if (above + c >= need) {
        sh.found_bin = b;
        sh.found_above = above;
        sh.found_in = c;
        break;
      }
      above += c;
    }
  }
  __syncthreads();
  return true;
}

__device__ __forceinline__ void clear_hist(Shared& sh) {
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += blockDim.x) sh.hist[b] = 0;
  __syncthreads();
}

__device__ __forceinline__ void none_drawn(const SampleArgs& a, long long row, int from) {
  for (int j = from + threadIdx.x; j < a.m; j += blockDim.x) {
    a.out_index[row * a.m + j] = -1;
    a.out_logprob[row * a.m + j] = -INFINITY;
  }
}

// Row state after the cuts.
struct Cut {
  uint32_t tau;       // kept: key > tau, and the first `ties` with key = tau
  unsigned ties;
  bool ranked;        // more than `ties` entries have key = tau
  float top, log_min;
  unsigned rank0;     // entries with key = tau before the warp's first group
};

// Bits of the group's entries that are kept; `seen` counts the ties passed so far.
template <int V>
__device__ __forceinline__ unsigned kept_bits(const Cut& c, const float (&s)[V], unsigned alive, unsigned& seen) {
  unsigned keep = 0, eq = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t k = ordered(s[v]);
    if (k > c.tau) keep |= 1u << v;
    if (k == c.tau) eq |= 1u << v;
  }
  keep &= alive;
  eq &= alive;
  if (!c.ranked) {
    keep |= eq;
  } else if (__any_sync(~0u, eq != 0)) {
    const unsigned mine = __popc(eq);
    unsigned v = mine;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const unsigned w = __shfl_up_sync(~0u, v, o);
      if (lane >= o) v += w;
    }
    unsigned rank = seen + v - mine;
    seen += __shfl_sync(~0u, v, 31);
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (eq >> e & 1u) {
        if (rank < c.ties) keep |= 1u << e;
        ++rank;
      }
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (!(__fsub_rn(s[e], c.top) >= c.log_min)) keep &= ~(1u << e);
  return keep;
}

template <int V>
__device__ __forceinline__ unsigned scale_group(const float (&x)[V], unsigned valid, float inv, float (&s)[V]) {
  unsigned alive = 0;
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (scaled(x[v], inv, &s[v])) alive |= 1u << v;
  return alive & valid;
}

// Composite of a draw: larger key first, then the lower index.
__device__ __forceinline__ unsigned long long composite(uint32_t key, long long i) {
  return (static_cast<unsigned long long>(key) << kIndexBits) |
         static_cast<unsigned long long>((1ll << kIndexBits) - 1 - i);
}
__device__ __forceinline__ long long index_of(unsigned long long c) {
  return (1ll << kIndexBits) - 1 - static_cast<long long>(c & ((1ull << kIndexBits) - 1));
}

__device__ __forceinline__ unsigned long long block_max(unsigned long long v, Shared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) v = max(v, __shfl_xor_sync(~0u, v, o));
  __syncthreads();
  if (lane == 0) sh.warp_u64[warp] = v;
  __syncthreads();
  for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) v = max(v, sh.warp_u64[w]);
  return v;
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
  // One draw from an uncut row needs no threshold: it is found in the first pass.
  const bool direct = a.m == 1 && r.k == 0 && r.p >= 1.0f && r.log_min == -INFINITY;

  // Pass 1: maximum and sum of exponentials, each lane's own, then joined in a fixed order.
  float top = -INFINITY, z = 0.0f;
  unsigned long long best = 0;
  walk(x, n, t, [&](long long i0, const float(&xs)[V], unsigned valid) {
    float s[V];
    const unsigned alive = scale_group<V>(xs, valid, r.inv, s);
    float b = top;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (alive >> v & 1u) b = fmaxf(b, s[v]);
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
  for (int o = 16; o > 0; o /= 2) join_stats(top, z, __shfl_xor_sync(~0u, top, o), __shfl_xor_sync(~0u, z, o));
  if (lane == 0) {
    sh.warp_f[warp][0] = top;
    sh.warp_f[warp][1] = z;
  }
  if (direct) best = block_max(best, sh);
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < warps; ++w) join_stats(top, z, sh.warp_f[w][0], sh.warp_f[w][1]);
    sh.top = top;
    sh.z = z;
    if (t.size > 1) {
      t.g->stats[t.rank] = make_float2(top, z);
      t.g->best_of[t.rank] = best;
    }
  }
  if (t.size > 1) {
    if (t.rank == 0) {
      for (int b = threadIdx.x; b < kBins; b += blockDim.x) t.g->hist[t.stage % 3][b] = 0;
      if (threadIdx.x == 0) t.g->listed = 0;
    }
    if (!team_sync(t, sh)) return false;
    if (threadIdx.x == 0) {
      top = -INFINITY;
      z = 0.0f;
      best = 0;
      for (int c = 0; c < t.size; ++c) {
        const float2 q = __ldcg(&t.g->stats[c]);
        join_stats(top, z, q.x, q.y);
        best = max(best, __ldcg(&t.g->best_of[c]));
      }
      sh.top = top;
      sh.z = z;
    }
  }
  __syncthreads();
  top = sh.top;
  z = sh.z;
  if (direct || top == -INFINITY) {
    if (t.rank == 0) {
      if (threadIdx.x == 0 && top != -INFINITY) {
        const long long i = index_of(best);
        float s;
        scaled(to_f32(x[i]), r.inv, &s);
        a.out_index[row] = i;
        a.out_logprob[row] = r.greedy ? 0.0f : __fsub_rn(s, top) - logf(z);
      }
      if (top == -INFINITY) none_drawn(a, row, 0);
    }
    return true;
  }

  Cut cut;
  cut.tau = 0;
  cut.ties = kNoTies;
  cut.ranked = false;
  cut.top = top;
  cut.log_min = r.log_min;
  cut.rank0 = 0;

  // top-k: three digits of the key, counted.
  if (r.k != 0) {
    uint32_t prefix = 0;
    unsigned long long need = r.k;
    bool all = false;
#pragma unroll 1
    for (int level = 0; level < 3 && !all; ++level) {
      const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
      clear_hist(sh);
      walk(x, n, t, [&](long long, const float(&xs)[V], unsigned valid) {
        float s[V];
        const unsigned alive = scale_group<V>(xs, valid, r.inv, s);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const uint32_t k = ordered(s[v]);
          if ((alive >> v & 1u) && (level == 0 || (k >> (shift + bits)) == prefix))
            atomicAdd(reinterpret_cast<unsigned*>(&sh.hist[(k >> shift) & ((1u << bits) - 1u)]), 1u);
        }
      });
      if (!team_find(t, sh, need)) return false;
      if (sh.found_in == 0) {
        all = true;  // fewer than k entries can be drawn
      } else {
        prefix = (prefix << bits) | sh.found_bin;
        need -= sh.found_above;
        cut.ranked = sh.found_in > need;
      }
    }
    if (!all) {
      cut.tau = prefix;
      cut.ties = static_cast<unsigned>(need);
    } else {
      cut.ranked = false;
    }
  }

  // top-p: the same digits, weighed.  Of the ties at the top-k cut only the kept number counts.
  if (r.p < 1.0f) {
    int log_n = 0;
    while ((1ll << log_n) < n) ++log_n;
    const float unit = static_cast<float>(1ull << (62 - log_n));
    uint32_t prefix = 0;
    unsigned long long need = 0;
    bool all = false;
#pragma unroll 1
    for (int level = 0; level < 3 && !all; ++level) {
      const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
      clear_hist(sh);
      auto add = [&](uint32_t k, unsigned long long times) {
        if (level == 0 || (k >> (shift + bits)) == prefix)
          atomicAdd(&sh.hist[(k >> shift) & ((1u << bits) - 1u)], times * fixed_weight(from_ordered(k), top, unit));
      };
      walk(x, n, t, [&](long long, const float(&xs)[V], unsigned valid) {
        float s[V];
        const unsigned alive = scale_group<V>(xs, valid, r.inv, s);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const uint32_t k = ordered(s[v]);
          if ((alive >> v & 1u) && (k > cut.tau || (k == cut.tau && cut.ties == kNoTies))) add(k, 1);
        }
      });
      if (cut.ties != kNoTies && t.rank == 0 && threadIdx.x == 0) add(cut.tau, cut.ties);
      __syncthreads();
      if (level == 0) {
        // the target is a share of what the first histogram holds
        if (!team_find(t, sh, ~0ull)) return false;
        unsigned long long sum = 0;
        for (int b = threadIdx.x; b < kBins; b += blockDim.x) sum += sh.hist[b];
#pragma unroll
        for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
        if (lane == 0) sh.warp_u64[warp] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < warps; ++w) sum += sh.warp_u64[w];
        need = r.p > 0.0f ? max(1ull, static_cast<unsigned long long>(static_cast<double>(r.p) *
                                                                      static_cast<double>(sum)))
                          : 1ull;
        Team one = t;  // the histogram is whole by now
        one.size = 1;
        team_find(one, sh, need);
      } else if (!team_find(t, sh, need)) {
        return false;
      }
      if (sh.found_in == 0) {
        all = true;
      } else {
        prefix = (prefix << bits) | sh.found_bin;
        need -= sh.found_above;
      }
    }
    if (!all) {
      const unsigned long long each = max(1ull, fixed_weight(from_ordered(prefix), top, unit));
      const unsigned long long ties = (need + each - 1) / each, held = sh.found_in / each;
      if (prefix == cut.tau && cut.ties != kNoTies) {
        cut.ranked = cut.ranked || ties < cut.ties;
        cut.ties = static_cast<unsigned>(min(static_cast<unsigned long long>(cut.ties), ties));
      } else {
        cut.ranked = held > ties;
        cut.tau = prefix;
        cut.ties = static_cast<unsigned>(ties);
      }
    }
  }

  // Where not all ties are kept, each warp needs the number of ties before its groups.
  if (cut.ranked) {
    unsigned mine = 0;
    walk(x, n, t, [&](long long, const float(&xs)[V], unsigned valid) {
      float s[V];
      const unsigned alive = scale_group<V>(xs, valid, r.inv, s);
#pragma unroll
      for (int v = 0; v < V; ++v) mine += (alive >> v & 1u) && ordered(s[v]) == cut.tau;
    });
    mine = __reduce_add_sync(~0u, mine);
    __syncthreads();
    if (lane == 0) sh.warp_u32[warp] = mine;
    __syncthreads();
    unsigned before = 0, total = 0;
    for (int w = 0; w < warps; ++w) {
      if (w < warp) before += sh.warp_u32[w];
      total += sh.warp_u32[w];
    }
    if (t.size > 1) {
      if (threadIdx.x == 0) t.g->ties[t.rank] = total;
      if (!team_sync(t, sh)) return false;
      for (int c = 0; c < t.rank; ++c) before += __ldcg(&t.g->ties[c]);
    }
    cut.rank0 = before;
  }

  const float logz = logf(z);
  if (a.m == 1) {
    best = 0;
    unsigned seen = cut.rank0;
    walk(x, n, t, [&](long long i0, const float(&xs)[V], unsigned valid) {
      float s[V];
      const unsigned alive = scale_group<V>(xs, valid, r.inv, s);
      const unsigned keep = kept_bits<V>(cut, s, alive, seen);
      if (keep == 0) return;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (keep >> v & 1u) best = max(best, composite(draw_key(s[v], noise[i0 + v]), i0 + v));
    });
    best = block_max(best, sh);
    if (t.size > 1) {
      if (threadIdx.x == 0) t.g->best_of[t.rank] = best;
      if (!team_sync(t, sh)) return false;
      if (t.rank == 0 && threadIdx.x == 0)
        for (int c = 0; c < t.size; ++c) best = max(best, __ldcg(&t.g->best_of[c]));
    }
    if (t.rank == 0 && threadIdx.x == 0) {
      const long long i = index_of(best);  // the best entry is always kept
      float s;
      scaled(to_f32(x[i]), r.inv, &s);
      a.out_index[row] = i;
      a.out_logprob[row] = __fsub_rn(s, top) - logz;
    }
    return true;
  }

  // The m largest composites: histograms narrow them down until what lies at or above
  // the edge fits the list.  Composites differ, so the last digit leaves exactly m.
  unsigned long long edge = 0, need = a.m, above = 0;
  int shift = kIndexBits + 32;
  bool enough = false;
#pragma unroll 1
  while (!enough && shift > 0) {
    const int bits = min(11, shift);
    const unsigned long long high = edge >> shift;
    shift -= bits;
    clear_hist(sh);
    unsigned seen = cut.rank0;
    walk(x, n, t, [&](long long i0, const float(&xs)[V], unsigned valid) {
      float s[V];
      const unsigned alive = scale_group<V>(xs, valid, r.inv, s);
      const unsigned keep = r.greedy ? alive : kept_bits<V>(cut, s, alive, seen);
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (keep >> v & 1u) {
          const unsigned long long c =
              composite(r.greedy ? ordered(s[v]) : draw_key(s[v], noise[i0 + v]), i0 + v);
          if ((c >> (shift + bits)) == high)
            atomicAdd(reinterpret_cast<unsigned*>(&sh.hist[(c >> shift) & ((1u << bits) - 1u)]), 1u);
        }
    });
    if (!team_find(t, sh, need)) return false;
    if (sh.found_in == 0) {
      enough = true;  // fewer than m: all at or above the edge (only at the first digit)
    } else {
      edge |= static_cast<unsigned long long>(sh.found_bin) << shift;
      need -= sh.found_above;
      above += sh.found_above;
      enough = above + sh.found_in <= kList;
    }
  }
  if (threadIdx.x == 0) sh.count = 0;
  __syncthreads();
  unsigned seen = cut.rank0;
  unsigned long long* list = t.size > 1 ? t.g->list : sh.list;
  unsigned* count = t.size > 1 ? &t.g->listed : &sh.count;
  walk(x, n, t, [&](long long i0, const float(&xs)[V], unsigned valid) {
    float s[V];
    const unsigned alive = scale_group<V>(xs, valid, r.inv, s);
    const unsigned keep = r.greedy ? alive : kept_bits<V>(cut, s, alive, seen);
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (keep >> v & 1u) {
        const unsigned long long c = composite(r.greedy ? ordered(s[v]) : draw_key(s[v], noise[i0 + v]), i0 + v);
        if (c >= edge) {
          const unsigned at = atomicAdd(count, 1u);
          if (at < kList) list[at] = c;
        }
      }
  });
  if (!team_sync(t, sh)) return false;
  if (t.rank != 0) return true;
  unsigned total = t.size > 1 ? __ldcg(count) : sh.count;
  if (total > kList) total = kList;
  unsigned width = 1;
  while (width < total) width *= 2;
  for (unsigned j = threadIdx.x; j < width; j += blockDim.x) {
    if (j >= total) sh.list[j] = 0;
    else if (t.size > 1) sh.list[j] = __ldcg(&t.g->list[j]);
  }
  __syncthreads();
  for (unsigned k = 2; k <= width; k *= 2)
    for (unsigned j = k / 2; j > 0; j /= 2) {
      for (unsigned q = threadIdx.x; q < width; q += blockDim.x) {
        const unsigned o = q ^ j;
        if (o > q) {
          const unsigned long long u = sh.list[q], w = sh.list[o];
          const bool desc = (q & k) == 0;
          if (desc ? u < w : u > w) {
            sh.list[q] = w;
            sh.list[o] = u;
          }
        }
      }
      __syncthreads();
    }
  const int drawn = r.greedy ? 1 : static_cast<int>(min(total, static_cast<unsigned>(a.m)));
  for (int j = threadIdx.x; j < drawn; j += blockDim.x) {
    const long long i = index_of(sh.list[j]);
    float s;
    scaled(to_f32(x[i]), r.inv, &s);
    a.out_index[row * a.m + j] = i;
    a.out_logprob[row * a.m + j] = r.greedy ? 0.0f : __fsub_rn(s, top) - logz;
  }
  none_drawn(a, row, drawn);
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
  const long long teams = gridDim.x / team_size;
  for (long long row = blockIdx.x / team_size; row < a.rows; row += teams) {
    if (!sample_row<T>(a, t, sh, row)) return;
    // the next row's first writes to the team's memory come after all reads of this row's
    if (row + teams < a.rows && !team_sync(t, sh)) return;
  }
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
