// Beam search: the m best continuations of each item's beams, and the beams' states put in
// their new order.
//
// total = logp + (s - ln sum exp s) is the same shift for all of a beam's scores, so within a beam
// the raw scores decide, exactly; only totals of different beams are compared as numbers, and
// those are formed in 64 bits from a normaliser whose sum is kept in two fp32 numbers.  What it is off by are its terms:
// approximate powers, log2 e (below) and, in the pass over long rows, a pack's additions, up to eight terms in fp32
// (four roundings).  Over 4,800 rows of 700 to 262,144 normal scores 2^-24 to 2^-26 on average, 2^-22.6 at most.
// GB300 adds two fp64 numbers a cycle and SM, so only candidates that may win get that far.
//
//   k_beam_rows   long rows: one pass over the scores, CTAs of 256 threads, as many a row as fill
//                 the GPU.  Each thread keeps the running sum of exponentials, in units of a power of two, and
//                 the largest score of each of four slots of its packs.  The k-th largest of these
//                 maxima is at most the k-th largest score, so scores from it on are collected, from the few
//                 slots that reach it, and the k best of them are kept for the item.  Sums that are not
//                 finite (NaN, infinite or huge scores) are formed again score by score.
//   k_beam_few    up to 256 candidates an item: a thread each, which finds its beam's normaliser by itself;
//   k_beam_items  more: a CTA an item, the normalisers, then all candidates (the rows' lists, or all
//                 scores where there are at most 8,192).  Each candidate's total is bounded from both
//                 sides in fp32; m lower bounds reach some threshold, and those whose upper bound does
//                 are formed in 64 bits and sorted.
//
// Bound: memory for the scores, else the latency of two launches and some twenty barriers: 64 x 8 rows of 50,021
// bf16 scores 26 us (17 of them the pass, 51 MB), the same with all but 300 tokens masked 25 (by -infinity or
// a finite score), 4 rows of fp32 14, 256 beams of 8 options 16 on one SM.
#include <cfloat>
#include <cmath>
#include <type_traits>
#include <utility>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kSlots = 4;
constexpr int kRowQueue = 1024;  // packs that are looked at again
constexpr int kRowList = 2048;   // collected scores of a CTA's share of a row
constexpr int kMostCands = 8192;
constexpr int kItemThreads = 1024;
constexpr int kPerThread = kMostCands / kItemThreads;
constexpr int kCountSort = 128;  // up to so many are sorted by counting who is larger
constexpr unsigned kNone = 0x007FFFFFu;  // ordered(-infinity)

using u64 = unsigned long long;

__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned b = __float_as_uint(v + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(unsigned k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ u64 ordered(double v) {
  const u64 b = static_cast<u64>(__double_as_longlong(v + 0.0));
  return (b >> 63) ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ double double_from_ordered(u64 k) {
  return __longlong_as_double(static_cast<long long>((k >> 63) ? k & ~(1ull << 63) : ~k));
}

// A score as it counts: finite, or -infinity where it is no continuation.
__device__ __forceinline__ float clean(float x) { return x > -INFINITY ? fminf(fmaxf(x, -FLT_MAX), FLT_MAX) : -INFINITY; }

// exp(x) / 2^unit: the product by log2 e is exact inside the sum, so all there is are the sum's rounding and
// that of log2 e itself, 1.3e-8 of x, of which the distance from the largest score counts.
constexpr float kLog2E = 1.44269504f;
__device__ __forceinline__ float power(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float exp_in(float x, float unit) { return power(fmaf(x, kLog2E, -unit)); }
// Scores of 2^30 and more, whose neighbours are 64 and more apart: next to such a one only its equals count (2^22
// others are 2^-70 of it), and the unit is exp of it.  Below, the product by log2 e is off by at most 64 when it is rounded
// to a unit, so terms are at most 2^64 and sums finite; above 2^31 it is off by more than fp32's exponents hold.
__device__ __forceinline__ bool is_huge(float top) { return !(fabsf(top) < 0x1p30f); }
// The unit for terms up to exp(top); 0 where there are none.
__device__ __forceinline__ float unit_of(float top) { return is_huge(top) ? 0.0f : rintf(top * kLog2E); }
// exp(x) for x <= top, both finite or -infinity, in these units.
__device__ __forceinline__ float term(float x, float top, float unit) {
  if (is_huge(top)) return x == top ? 1.0f : 0.0f;
  return exp_in(x, unit);
}

// A sum in two numbers (Knuth's exact addition).
struct Two {
  float hi, lo;
  __device__ __forceinline__ void add(float v) {
    const float s = __fadd_rn(hi, v), b = __fsub_rn(s, hi);
    lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, b)), __fsub_rn(v, b)));
    hi = s;
  }
  __device__ __forceinline__ void add(const Two& o) {
    add(o.hi);
    lo = __fadd_rn(lo, o.lo);
  }
  // to another unit; an empty sum's may lie at any distance.  A NaN or infinite sum may not become a finite one:
  // it is what a row is looked at again for
  __device__ __forceinline__ void scale(float f) {
    const float g = hi > 0.0f ? f : 0.0f;
    hi *= g;
    lo *= g;
  }
  __device__ __forceinline__ Two shuffled(int o, int width = 32) const {
    return {__shfl_xor_sync(0xffffffffu, hi, o, width), __shfl_xor_sync(0xffffffffu, lo, o, width)};
  }
};

// ln(sum), by ln f = 2 atanh((f - 1) / (f + 1)) of its fraction f in [0.7, 1.42): the leading term in two
// numbers, the rest of the series (below 0.004) in fp32.  Off by some 2^-32.
__device__ __forceinline__ double log_sum(Two sum) {
  float hi = __fadd_rn(sum.hi, sum.lo);
  float lo = __fadd_rn(__fsub_rn(sum.hi, hi), sum.lo);
  int e = (__float_as_int(hi) >> 23) - 127;
  if ((__float_as_int(hi) & 0x7FFFFF) > 0x3504F3) ++e;
  const float down = __int_as_float((127 - e) << 23);
  hi *= down;
  lo *= down;
  const float num = __fsub_rn(hi, 1.0f);  // exact
  const float den = __fadd_rn(hi, 1.0f), den_lo = __fadd_rn(__fsub_rn(hi, __fsub_rn(den, 1.0f)), lo);
  const float s = __fdiv_rn(num, den);
  const float s_lo = __fdividef(__fmaf_rn(-s, den, num) + lo - s * den_lo, den);
  const float q = s * s;
  // 2 (s^3/3 + s^5/5 + ...), s^2 < 0.0295
  float r = fmaf(q, 2.0f / 13, 2.0f / 11);
  r = fmaf(q, r, 2.0f / 9);
  r = fmaf(q, r, 2.0f / 7);
  r = fmaf(q, r, 2.0f / 5);
  r = fmaf(q, r, 2.0f / 3);
  r = r * q * s + 2.0f * s_lo;
  return fma(static_cast<double>(e), 0.693147180559945309417, static_cast<double>(2.0f * s) + static_cast<double>(r));
}

// The normaliser: ln of a sum of terms up to exp(top), top finite, as top + ln(sum / its own term): what that
// term is off by falls out, and a row of one score has exactly that score as its normaliser.
__device__ __forceinline__ double normaliser(float top, Two sum) {
  const float one = term(top, top, unit_of(top));
  const float q = __fdiv_rn(sum.hi, one);
  return top + log_sum(Two{q, __fdividef(__fmaf_rn(-q, one, sum.hi) + sum.lo, one)});
}

// What a CTA found in its share of a row.
struct __align__(16) RowPart {
  float top;  // -infinity: no continuation
  int count;
  Two sum;    // in units of 2^unit_of(top)
};

// The normaliser of a row from its parts, NaN where it has no continuation.
__device__ __forceinline__ double join_parts(const RowPart* part, int parts, bool normalised) {
  float top = -INFINITY;
#pragma unroll 4
  for (int p = 0; p < parts; ++p) top = fmaxf(top, part[p].top);
  if (top == -INFINITY) return NAN;
  if (normalised) return 0.0;
  const float unit = unit_of(top);
  Two sum{0.0f, 0.0f};
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const RowPart q = part[p];
    // beside a huge top only its equals count, and a huge negative one counts beside its equals alone
    if (q.top == -INFINITY || ((is_huge(top) || is_huge(q.top)) && q.top != top)) continue;
    Two s = q.sum;
    s.scale(power(unit_of(q.top) - unit));
    sum.add(s);
  }
  return normaliser(top, sum);
}

// Whether beam `row` has continuations to be read.
__device__ __forceinline__ bool is_live(const mlt_beam_args& a, long long row) {
  return a.logp[row] > -INFINITY && (a.done == nullptr || a.done[row] == 0);
}

// Sorts `size` (a power of two) keys in shared memory, largest first.  `threads` a power of two.
template <typename K, typename Less>
__device__ void bitonic(K* key, int size, Less less) {
  for (int width = 2; width <= size; width *= 2)
    for (int hop = width / 2; hop > 0; hop /= 2) {
      for (int t = threadIdx.x; t < size / 2; t += blockDim.x) {
        const int i = 2 * t - (t & (hop - 1)), j = i + hop;
        const K a = key[i], b = key[j];
        if (less(a, b) == ((i & width) == 0)) {
          key[i] = b;
          key[j] = a;
        }
      }
      // a warp's pairs of the next stages lie among its own 64 keys
      if (hop > 32)
        __syncthreads();
      else if (hop == 1 && width >= 64)
        __syncthreads();
      else
        __syncwarp();
    }
  __syncthreads();
}

__device__ __forceinline__ int power_of_two(int n) { return n <= 1 ? 1 : 1 << (32 - __clz(n - 1)); }

// --- rows ------------------------------------------------------------------------------------

// A CTA's share of a row: packs [first, last), counted from the row's first entry wherever it lies, so that
// equal rows are summed in the same order and equal beams tie.  Packs that no aligned access
// fits are put together from the two aligned ones around them.
template <typename T>
struct Share {
  static constexpr int V = 16 / sizeof(T);
  const T* row;
  int n, skew, first, last;  // skew: entries from the last 16-byte boundary to the row's first

  __device__ __forceinline__ void load(int q, Pack<T, V>& p) const {
    const int i0 = q * V;
    if (skew == 0 && i0 + V <= n) {
      p = *reinterpret_cast<const Pack<T, V>*>(row + i0);
    } else if (skew != 0 && i0 >= skew && i0 + 2 * V - skew <= n) {
      const uint4* at = reinterpret_cast<const uint4*>(row + (i0 - skew));
      const uint4 x = at[0], y = at[1];
      const int words = static_cast<int>(skew * sizeof(T)) >> 2;
      const bool two = words & 2, one = words & 1;
      const unsigned a0 = two ? x.z : x.x, a1 = two ? x.w : x.y, a2 = two ? y.x : x.z, a3 = two ? y.y : x.w,
                     a4 = two ? y.z : y.x, a5 = two ? y.w : y.y;
      unsigned w[5] = {one ? a1 : a0, one ? a2 : a1, one ? a3 : a2, one ? a4 : a3, one ? a5 : a4};
      if (sizeof(T) == 2 && (skew & 1))
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], 16);
      *reinterpret_cast<uint4*>(&p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) p.v[e] = i0 + e < n ? row[i0 + e] : from_f32<T>(-INFINITY);
    }
  }
};

// Score first, then the lower token.
__device__ __forceinline__ u64 row_key(float s, int token) {
  return (static_cast<u64>(ordered(s)) << 32) | static_cast<unsigned>(~token);
}

// The largest of a pack's scores but NaN: -infinity or more.
template <typename T, int V>
__device__ __forceinline__ float pack_max(const Pack<T, V>& p) {
  if constexpr (sizeof(T) == 4) {
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < V; ++e) m = fmaxf(m, p.v[e]);
    return m;
  } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    const __nv_bfloat162* q = reinterpret_cast<const __nv_bfloat162*>(&p);
    const __nv_bfloat162 m = __hmax2(__hmax2(q[0], q[1]), __hmax2(q[2], q[3]));
    return fmaxf(fmaxf(__low2float(m), __high2float(m)), -INFINITY);
  } else {
    const __half2* q = reinterpret_cast<const __half2*>(&p);
    const __half2 m = __hmax2(__hmax2(q[0], q[1]), __hmax2(q[2], q[3]));
    return fmaxf(fmaxf(__low2float(m), __high2float(m)), -INFINITY);
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 4)
    k_beam_rows(const __grid_constant__ mlt_beam_args a, int parts, int k, RowPart* found, u64* lists) {
  __shared__ float warp_top[kRowWarps];
  __shared__ Two warp_sum[kRowWarps];
  __shared__ int total[2], listed, queued, queue[kRowQueue];
  __shared__ u64 list[kRowList];
  pdl_wait();
  pdl_trigger();
  constexpr int V = Share<T>::V;
  const long long r = blockIdx.x / parts;
  const int part = blockIdx.x % parts, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  RowPart& out = found[r * parts + part];
  if (!is_live(a, r)) return;  // the item's CTA looks at the same
  Share<T> sh;
  sh.row = static_cast<const T*>(a.scores) + (r / a.beams) * a.batch_stride + (r % a.beams) * a.beam_stride;
  sh.n = a.n;
  sh.skew = static_cast<int>((reinterpret_cast<uintptr_t>(sh.row) / sizeof(T)) % V);
  const int packs = (a.n + V - 1) / V;
  sh.first = static_cast<int>(static_cast<long long>(packs) * part / parts);
  sh.last = static_cast<int>(static_cast<long long>(packs) * (part + 1) / parts);

  float slot[kSlots], top = -INFINITY, unit = 0.0f;
  Two sum{0.0f, 0.0f};
#pragma unroll
  for (int u = 0; u < kSlots; ++u) slot[u] = -INFINITY;
#pragma unroll 1
  for (int q = sh.first + tid; q < sh.last; q += kSlots * kRowThreads) {
    Pack<T, V> p[kSlots];
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      if (q + u * kRowThreads < sh.last) {
        sh.load(q + u * kRowThreads, p[u]);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) p[u].v[e] = from_f32<T>(-INFINITY);
      }
    }
    float best = -INFINITY;
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      const float high = pack_max(p[u]);
      slot[u] = fmaxf(slot[u], high);
      best = fmaxf(best, high);
    }
    if (best > top) {
      top = best;
      const float now = unit_of(top);
      sum.scale(power(unit - now));
      unit = now;
    }
    if (a.normalised == 0) {
#pragma unroll
      for (int u = 0; u < kSlots; ++u) {
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < V; ++e) s[e & 1] += exp_in(to_f32(p[u].v[e]), unit);
        sum.add(s[0] + s[1]);
      }
    }
  }

  // the CTA's top, sum, and the least of the warps' tops
  auto cta_top = [&](float mine) {
    float high = mine;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
    __syncthreads();
    if (lane == 0) warp_top[warp] = high;
    if (tid == 0) listed = queued = total[0] = total[1] = 0;
    __syncthreads();
    high = -INFINITY;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) high = fmaxf(high, warp_top[w]);
    return high;
  };
  auto cta_sum = [&](float high) {
    const float now = unit_of(high);
    sum.scale(power(unit - now));
#pragma unroll
    for (int o = 16; o > 0; o /= 2) sum.add(sum.shuffled(o));
    if (lane == 0) warp_sum[warp] = sum;
    __syncthreads();
    Two all{0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) all.add(warp_sum[w]);
    return all;
  };
  float high = cta_top(top);
  Two all = cta_sum(high);
  // not finite: a NaN, an infinite or a huge score.  The same again, each score as it counts
  if (high > -INFINITY && (is_huge(high) || !(all.hi + all.lo < INFINITY))) {
    high = cta_top(clean(top));
    unit = unit_of(high);
    sum = Two{0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < kSlots; ++u) slot[u] = fminf(slot[u], FLT_MAX);
    if (a.normalised == 0)
      for (int q = sh.first + tid; q < sh.last; q += kRowThreads) {
        Pack<T, V> p;
        sh.load(q, p);
#pragma unroll
        for (int e = 0; e < V; ++e) sum.add(term(clean(to_f32(p.v[e])), high, unit));
      }
    all = cta_sum(high);
  }
  float mine = -INFINITY;
#pragma unroll
  for (int u = 0; u < kSlots; ++u) mine = fmaxf(mine, slot[u]);

  // the largest threshold found that at least k maxima reach
  const unsigned key = ordered(mine);
  unsigned low = kNone, up = ordered(high) + 1;  // `low` always reached by k of them, or it is -infinity
  const bool by_slot = k > kRowThreads / 4;
  const int enough = k + (k < 48 ? 24 : k / 2);
  int flip = 0;
  // with as many warps as wanted maxima the least of the warps' own is a good first try
  float least = INFINITY;
#pragma unroll
  for (int w = 0; w < kRowWarps; ++w) least = fminf(least, warp_top[w]);
  unsigned first = k <= kRowWarps ? ordered(fminf(least, high)) : 0u;
  while (up - low > 1) {
    const unsigned mid = first > low && first < up ? first : low + (up - low) / 2;
    first = 0;
    int c;
    if (!by_slot) {
      c = __syncthreads_count(key >= mid);
    } else {
      int have = 0;
#pragma unroll
      for (int u = 0; u < kSlots; ++u) have += ordered(slot[u]) >= mid;
      have = __reduce_add_sync(0xffffffffu, have);
      if (lane == 0 && have > 0) atomicAdd(&total[flip], have);
      __syncthreads();
      c = total[flip];
      if (tid == 0) total[flip ^ 1] = 0;
      __syncthreads();
      flip ^= 1;
    }
    if (c >= k)
      low = mid;
    else
      up = mid;
    if (c >= k && c <= enough) break;
  }
  // the scores that reach it
  const float from = from_ordered(low);
  auto keep = [&](float s, int i) {
    if (s > -INFINITY && s >= from) {
      const int at = atomicAdd(&listed, 1);
      if (at < kRowList) list[at] = row_key(s, i);
    }
  };
  // which packs these are, for all threads to share (each in its own slots: 64 x 8 rows of 50,021 12 us for 3)
#pragma unroll
  for (int u = 0; u < kSlots; ++u)
    if (slot[u] > -INFINITY && slot[u] >= from)
      for (int q = sh.first + tid + u * kRowThreads; q < sh.last; q += kSlots * kRowThreads) {
        const int at = atomicAdd(&queued, 1);
        if (at < kRowQueue) queue[at] = q;
      }
  __syncthreads();
  const bool few = queued <= kRowQueue;
  const int packs_again = few ? queued : sh.last - sh.first;
  for (int i = tid; i < packs_again; i += kRowThreads) {
    const int q = few ? queue[i] : sh.first + i;
    Pack<T, V> p;
    sh.load(q, p);
#pragma unroll
    for (int e = 0; e < V; ++e) keep(clean(to_f32(p.v[e])), q * V + e);
  }
  __syncthreads();
  int count = listed;
  if (count > kRowList) {
    // many equal scores: the k-th largest key by bisection, over the whole share each time
    u64 lo = static_cast<u64>(low) << 32, hi = (static_cast<u64>(ordered(high)) + 1) << 32;
    while (hi - lo > 1) {
      const u64 mid = lo + (hi - lo) / 2;
      __syncthreads();
      if (tid == 0) total[0] = 0;
      __syncthreads();
      int have = 0;
      for (int q = sh.first + tid; q < sh.last; q += kRowThreads) {
        Pack<T, V> p;
        sh.load(q, p);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float s = clean(to_f32(p.v[e]));
          have += s > -INFINITY && row_key(s, q * V + e) >= mid;
        }
      }
      have = __reduce_add_sync(0xffffffffu, have);
      if (lane == 0) atomicAdd(&total[0], have);
      __syncthreads();
      if (total[0] >= k)
        lo = mid;
      else
        hi = mid;
      if (total[0] == k) break;
    }
    __syncthreads();
    if (tid == 0) listed = 0;
    __syncthreads();
    for (int q = sh.first + tid; q < sh.last; q += kRowThreads) {
      Pack<T, V> p;
      sh.load(q, p);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float s = clean(to_f32(p.v[e]));
        const u64 one = row_key(s, q * V + e);
        if (s > -INFINITY && one >= lo) list[atomicAdd(&listed, 1) & (kRowList - 1)] = one;
      }
    }
    __syncthreads();
    count = min(listed, k);
  }
  u64* to = lists + (r * parts + part) * static_cast<long long>(k);
  if (count <= kCountSort) {
    if (tid < count) {
      const u64 v = list[tid];
      int rank = 0;
      for (int i = 0; i < count; ++i) rank += list[i] > v;
      if (rank < k) to[rank] = v;
    }
  } else {
    const int size = power_of_two(count);
    for (int i = count + tid; i < size; i += kRowThreads) list[i] = 0;
    __syncthreads();
    bitonic(list, size, [](u64 x, u64 y) { return x < y; });
    for (int i = tid; i < min(count, k); i += kRowThreads) to[i] = list[i];
  }
  if (tid == 0) out = RowPart{count > 0 ? high : -INFINITY, min(count, k), all};
}

// --- items -----------------------------------------------------------------------------------

struct Cand {
  u64 total, tie;
};
__device__ __forceinline__ bool less(const Cand& a, const Cand& b) {
  return a.total < b.total || (a.total == b.total && a.tie < b.tie);
}

// Sorts `size` (a power of two) candidates, largest first, bitonically: element i = thread + e * threads is held
// by its thread.  Partners in a warp are met by shuffles, others through `mem` (as many places).
// 512 of them in shared memory alone took 7.6 us.
template <int E>
__device__ void sort_held(Cand (&x)[E], Cand* mem, int size) {
  const int t = threadIdx.x, threads = blockDim.x;
  __syncthreads();
  for (int width = 2; width <= size; width *= 2)
    for (int hop = width / 2; hop > 0; hop /= 2) {
      if (hop >= 32 && hop < threads) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (t + e * threads < size) mem[t + e * threads] = x[e];
        __syncthreads();
      }
      Cand y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (hop >= threads) {
          y[e] = x[e];
#pragma unroll
          for (int f = 0; f < E; ++f)
            if (f == (e ^ (hop / threads))) y[e] = x[f];
        } else if (hop >= 32) {
          y[e] = t + e * threads < size ? mem[(t ^ hop) + e * threads] : x[e];
        } else {
          y[e].total = __shfl_xor_sync(0xffffffffu, x[e].total, hop);
          y[e].tie = __shfl_xor_sync(0xffffffffu, x[e].tie, hop);
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = t + e * threads;
        const bool larger = ((i & hop) == 0) == ((i & width) == 0);
        if (less(x[e], y[e]) == larger) x[e] = y[e];
      }
      if (hop >= 32 && hop < threads) __syncthreads();
    }
}

__device__ __forceinline__ Cand candidate_of(int w, float s, int token, double total) {
  return {ordered(total), (static_cast<u64>(1023 - w) << 54) | (static_cast<u64>(ordered(s)) << 22) |
                              static_cast<u64>((1 << 22) - 1 - token)};
}
__device__ __forceinline__ int beam_of(const Cand& c) { return 1023 - static_cast<int>(c.tie >> 54); }

__device__ __forceinline__ void write(const mlt_beam_args& a, int b, int at, const Cand& c, bool ended) {
  const long long o = static_cast<long long>(b) * a.m + at;
  const int token = (1 << 22) - 1 - static_cast<int>(c.tie & ((1 << 22) - 1));
  a.out_parent[o] = beam_of(c);
  a.out_token[o] = token;
  a.out_logp[o] = static_cast<float>(double_from_ordered(c.total));
  a.out_done[o] = ended || token == a.eos;
}
__device__ __forceinline__ void write_none(const mlt_beam_args& a, int b, int at) {
  const long long o = static_cast<long long>(b) * a.m + at;
  a.out_parent[o] = a.out_token[o] = -1;
  a.out_logp[o] = -INFINITY;
  a.out_done[o] = 0;
}

// Up to kFewMost candidates an item, out of the rows' lists: a thread forms one, several count together how many
// are larger.
constexpr int kFewMost = 256, kFewThreads = 512;
__global__ void __launch_bounds__(kFewThreads)
    k_beam_few(const __grid_constant__ mlt_beam_args a, int parts, int k, const RowPart* found, const u64* lists) {
  __shared__ Cand list[kFewMost];
  __shared__ int ranks[kFewMost];
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x, tid = threadIdx.x, each = parts * k, cands = a.beams * each;
  int wide = 32;
  while (wide < cands) wide *= 2;
  bool ended = false;
  if (tid < wide) {
    const int w = min(tid / each, a.beams - 1), at = tid - w * each;
    const long long r = static_cast<long long>(b) * a.beams + w, o = r * parts + min(at / k, parts - 1);
    const float lp = a.logp[r];
    const u64 key = tid < cands ? lists[o * k + at % k] : 0;
    ended = a.done != nullptr && a.done[r] != 0;
    Cand mine{0, 0};
    if (tid < cands && lp > -INFINITY) {
      if (ended) {
        if (at == 0) mine = candidate_of(w, 0.0f, static_cast<int>(a.eos), lp);
      } else if (at % k < found[o].count) {
        const double z = join_parts(found + r * parts, parts, a.normalised != 0);
        const float s = from_ordered(static_cast<unsigned>(key >> 32));
        mine = candidate_of(w, s, ~static_cast<int>(key), lp + (static_cast<double>(s) - z));
      }
    }
    list[tid] = mine;
    ranks[tid] = 0;
  }
  const int count = __syncthreads_count(tid < wide && list[tid].total != 0);
  const Cand mine = list[tid % wide];
  if (mine.total != 0) {
    int larger = 0;
#pragma unroll 4
    for (int j = tid / wide; j < cands; j += kFewThreads / wide) larger += less(mine, list[j]);
    if (larger > 0) atomicAdd(&ranks[tid % wide], larger);
  }
  __syncthreads();
  if (tid < wide && mine.total != 0 && ranks[tid] < a.m) write(a, b, ranks[tid], mine, ended);
  for (int i = count + tid; i < a.m; i += kFewThreads) write_none(a, b, i);
}

// T: the scores' type where candidates are all scores; else the rows' lists are read (FROM_ROWS).
template <typename T, bool FROM_ROWS>
__global__ void __launch_bounds__(kItemThreads, 1)
    k_beam_items(const __grid_constant__ mlt_beam_args a, int parts, int k, const RowPart* found, const u64* lists,
                 int cap) {
  extern __shared__ __align__(16) unsigned char mem[];
  Cand* list = reinterpret_cast<Cand*>(mem);                     // [cap]
  double* lse = reinterpret_cast<double*>(list + cap);           // [beams]
  float* logp = reinterpret_cast<float*>(lse + a.beams);         // [beams]; NaN: no continuations
  uint8_t* ended = reinterpret_cast<uint8_t*>(logp + a.beams);   // [beams]
  __shared__ int total[2], listed, all;
  __shared__ unsigned most, fewest;
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, threads = blockDim.x;
  const int each = FROM_ROWS ? parts * k : a.n, cands = a.beams * each;
  const T* scores = static_cast<const T*>(a.scores) + b * a.batch_stride;
  if (tid == 0) {
    listed = total[0] = total[1] = all = 0;
    most = 0;
    fewest = 0xFFFFFFFFu;
  }
  for (int w = tid; w < a.beams; w += threads) {
    const long long r = static_cast<long long>(b) * a.beams + w;
    const bool over = a.done != nullptr && a.done[r] != 0;
    float lp = a.logp[r];
    if (!(lp > -INFINITY)) lp = NAN;
    ended[w] = over;
    if (FROM_ROWS && !over && lp == lp) {
      const double z = join_parts(found + r * parts, parts, a.normalised != 0);
      if (z != z) lp = NAN;
      lse[w] = z;
    }
    logp[w] = lp;
  }
  __syncthreads();
  if (!FROM_ROWS) {
    // a power-of-two group of lanes a row, as few as let all rows go at once
    int lanes = 1;
    while (lanes < 32 && lanes < a.n && 2 * lanes * a.beams <= threads) lanes *= 2;
    const int j = tid & (lanes - 1), rows = threads / lanes;
    for (int w0 = 0; w0 < a.beams; w0 += rows) {
      const int w = w0 + tid / lanes;
      const bool on = w < a.beams && !ended[w] && logp[w] == logp[w];
      const T* row = scores + w * a.beam_stride;
      float top = -INFINITY;
      if (on)
#pragma unroll 8
        for (int i = j; i < a.n; i += lanes) top = fmaxf(top, clean(to_f32(row[i])));
      for (int o = lanes / 2; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      Two sum{0.0f, 0.0f};
      const float unit = unit_of(top);
      if (on && top > -INFINITY && a.normalised == 0)
#pragma unroll 8
        for (int i = j; i < a.n; i += lanes) sum.add(term(clean(to_f32(row[i])), top, unit));
      for (int o = lanes / 2; o > 0; o /= 2) sum.add(sum.shuffled(o));
      if (on && j == 0) {
        if (top == -INFINITY) logp[w] = NAN;
        lse[w] = top == -INFINITY || a.normalised != 0 ? 0.0 : normaliser(top, sum);
      }
    }
    __syncthreads();
  }

  // candidate i: whether there is one, its beam, score and token
  auto candidate = [&](int i, int& w, float& s, int& token) -> bool {
    w = i / each;
    const int at = i - w * each;
    if (!(logp[w] == logp[w])) return false;
    if (ended[w]) {
      s = 0.0f;
      token = static_cast<int>(a.eos);
      return at == 0;
    }
    if (FROM_ROWS) {
      const long long r = (static_cast<long long>(b) * a.beams + w) * parts + at / k;
      if (at % k >= found[r].count) return false;
      const u64 key = lists[r * k + at % k];
      s = from_ordered(static_cast<unsigned>(key >> 32));
      token = ~static_cast<int>(key);
      return true;
    }
    s = clean(to_f32(scores[w * a.beam_stride + at]));
    token = at;
    return s > -INFINITY;
  };
  // by whole warps: one addition to the list's length for each
  auto put = [&](bool on, int w, float s, int token) {
    const unsigned who = __ballot_sync(0xffffffffu, on);
    if (who == 0) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(&listed, __popc(who));
    at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1));
    if (!on) return;
    const double lp = logp[w];
    list[at] = candidate_of(w, s, token, ended[w] ? lp : lp + (static_cast<double>(s) - lse[w]));
  };

  if (cands <= kCountSort) {
    int w = 0, token = 0;
    float s = 0.0f;
    const bool on = tid < cands && candidate(tid, w, s, token);
    put(on, w, s, token);
  } else {
    unsigned lower[kPerThread], upper[kPerThread];
    unsigned best = 0, worst = 0xFFFFFFFFu;
    int valid = 0;
    const int per = (cands + threads - 1) / threads;
#pragma unroll
    for (int c = 0; c < kPerThread; ++c) {
      lower[c] = upper[c] = 0;
      const int i = c * threads + tid;
      int w, token;
      float s;
      if (c >= per || i >= cands || !candidate(i, w, s, token)) continue;
      const float z = ended[w] ? 0.0f : static_cast<float>(lse[w]), lp = logp[w];
      // three roundings, of the normaliser and two sums, each at most 2^-23 of these
      const float v = lp + (s - z), off = 0x1p-21f * (fabsf(lp) + fabsf(s) + fabsf(z));
      const float l = v - off, u = v + off;
      lower[c] = l == l ? ordered(l) : kNone;
      upper[c] = u == u ? ordered(u) : 0xFFFFFFFFu;
      best = max(best, lower[c]);
      worst = min(worst, lower[c]);
      ++valid;
    }
    best = __reduce_max_sync(0xffffffffu, best);
    worst = __reduce_min_sync(0xffffffffu, worst);
    valid = __reduce_add_sync(0xffffffffu, valid);
    if (lane == 0) {
      atomicMax(&most, best);
      atomicMin(&fewest, worst);
      atomicAdd(&all, valid);
    }
    __syncthreads();
    // the largest threshold found that m lower bounds reach: between two that are too low and too high, where
    // the counts' logarithms would put it if they fell evenly, or halfway, in turn
    unsigned low = 0, up = most + 1;
    const int enough = a.m + (a.m < 64 ? 64 : a.m / 4);
    int flip = 0;
    float at_low = static_cast<float>(all), at_up = 0.5f;
    if (all <= enough) up = 1;  // all of them
    unsigned from = fewest;
    for (int turn = 0; up - low > 1; ++turn) {
      unsigned mid = low + (up - low) / 2;
      if ((turn & 1) == 0) {
        const float f = __fdividef(__log2f(__fdividef(at_low, a.m + 0.5f * (enough - a.m))), __log2f(__fdividef(at_low, at_up)));
        const float lo = from_ordered(max(low, from)), v = lo + (from_ordered(up) - lo) * f;
        if (v == v && ordered(v) > low && ordered(v) < up) mid = ordered(v);
      }
      int have = 0;
#pragma unroll
      for (int c = 0; c < kPerThread; ++c)
        if (c < per) have += lower[c] >= mid;
      have = __reduce_add_sync(0xffffffffu, have);
      if (lane == 0 && have > 0) atomicAdd(&total[flip], have);
      __syncthreads();
      const int got = total[flip];
      if (tid == 0) total[flip ^ 1] = 0;
      __syncthreads();
      flip ^= 1;
      if (got >= a.m) {
        low = mid;
        at_low = static_cast<float>(got);
        if (got <= enough) break;
      } else {
        up = mid;
        at_up = fmaxf(static_cast<float>(got), 0.5f);
      }
    }
#pragma unroll
    for (int c = 0; c < kPerThread; ++c) {
      if (c >= per) continue;
      int w = 0, token = 0;
      float s = 0.0f;
      const bool on = upper[c] > 0 && upper[c] >= low && candidate(c * threads + tid, w, s, token);
      put(on, w, s, token);
    }
  }
  __syncthreads();
  const int count = listed;
  if (count <= kCountSort) {
    for (int i = tid; i < count; i += threads) {
      const Cand c = list[i];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < count; ++j) rank += less(c, list[j]);
      if (rank < a.m) write(a, b, rank, c, ended[beam_of(c)]);
    }
  } else {
    const int size = power_of_two(count);
    auto sorted = [&](auto each_thread) {
      constexpr int E = decltype(each_thread)::value;
      Cand x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = tid + e * threads < count ? list[tid + e * threads] : Cand{0, 0};
      sort_held(x, list, size);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = tid + e * threads;
        if (i < min(count, a.m)) write(a, b, i, x[e], ended[beam_of(x[e])]);
      }
    };
    if (size <= threads)
      sorted(std::integral_constant<int, 1>());
    else if (size <= 2 * threads)
      sorted(std::integral_constant<int, 2>());
    else {  // many equal totals: in shared memory alone
      for (int i = count + tid; i < size; i += threads) list[i] = Cand{0, 0};
      __syncthreads();
      bitonic(list, size, [](const Cand& x, const Cand& y) { return less(x, y); });
      for (int i = tid; i < min(count, a.m); i += threads) write(a, b, i, list[i], ended[beam_of(list[i])]);
    }
  }
  for (int i = count + tid; i < a.m; i += threads) write_none(a, b, i);
}

struct Plan {
  bool direct;
  int parts, k, threads, cap;
  size_t off_lists, bytes, smem;
};

Plan plan_of(const mlt_beam_args& a, int sms) {
  Plan p{};
  p.k = a.m < a.n ? a.m : a.n;
  const long long rows = static_cast<long long>(a.batch) * a.beams;
  p.direct = static_cast<long long>(a.beams) * a.n <= kMostCands;
  p.parts = 1;
  long long cands = static_cast<long long>(a.beams) * a.n;
  if (!p.direct) {
    // parts of a row until the GPU is full, none shorter than eight scores a thread
    const int least = kRowThreads * 8;
    while (p.parts < 64 && rows * p.parts < 2LL * sms && a.n / (2 * p.parts) >= least &&
           static_cast<long long>(a.beams) * p.k * p.parts * 2 <= kMostCands)
      p.parts *= 2;
    cands = static_cast<long long>(a.beams) * p.k * p.parts;
    p.off_lists = up256(sizeof(RowPart) * rows * p.parts);
    p.bytes = p.off_lists + up256(sizeof(u64) * rows * p.parts * p.k);
  }
  p.threads = 128;
  while (p.threads < kItemThreads && p.threads * 4 < cands) p.threads *= 2;
  p.cap = 128;
  while (p.cap < cands) p.cap *= 2;
  p.smem = sizeof(Cand) * p.cap + a.beams * (sizeof(double) + sizeof(float) + 1);
  return p;
}

template <typename T, bool FROM_ROWS>
cudaError_t launch_items(const mlt_beam_args& a, const Plan& p, const RowPart* found, const u64* lists, cudaStream_t st) {
  if (p.smem > 40 * 1024) {  // with the static part past what a kernel has unasked, 48 KB
    const cudaError_t e = allow_smem(reinterpret_cast<const void*>(k_beam_items<T, FROM_ROWS>), p.smem);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(k_beam_items<T, FROM_ROWS>, dim3(a.batch), dim3(p.threads), p.smem, st, a, p.parts, p.k, found, lists,
                    p.cap);
}

// --- states ----------------------------------------------------------------------------------

struct Move {
  unsigned char* data;
  long long row_bytes, row_stride;
  int unit;             // bytes of an access
  int slice;            // bytes of a row that a CTA takes
  unsigned first_cta;
};
constexpr int kMostMoves = 64;
constexpr int kHeldRows = 8;
struct Moves {
  Move t[kMostMoves];
  int count, beams;
  const int64_t* parent;
  unsigned* err;
};

// A CTA takes a slice of columns of all beams of an item: it reads what moves into shared memory before it
// writes any of it, so rows may change places freely.
template <typename U>
__device__ __forceinline__ void move_slice(const Move& t, unsigned char* base, long long from, int bytes, const int* to,
                                           const int* of, int count, unsigned char* mem) {
  const int units = bytes / static_cast<int>(sizeof(U)), all = units * count;
  if (count <= kHeldRows) {  // each thread its columns, in registers (64 x 8 rows of 143 KB 21 us through shared memory)
    for (int c = threadIdx.x; c < units; c += blockDim.x) {
      unsigned char* at = base + from + c * sizeof(U);
      U v[kHeldRows];
#pragma unroll
      for (int i = 0; i < kHeldRows; ++i)
        if (i < count) v[i] = *reinterpret_cast<const U*>(at + of[i] * t.row_stride);
#pragma unroll
      for (int i = 0; i < kHeldRows; ++i)
        if (i < count) *reinterpret_cast<U*>(at + to[i] * t.row_stride) = v[i];
    }
    return;
  }
  U* held = reinterpret_cast<U*>(mem);
#pragma unroll 4
  for (int i = threadIdx.x; i < all; i += blockDim.x) {
    const int row = i / units, c = i - row * units;
    held[i] = *reinterpret_cast<const U*>(base + of[row] * t.row_stride + from + c * sizeof(U));
  }
  __syncthreads();
#pragma unroll 4
  for (int i = threadIdx.x; i < all; i += blockDim.x) {
    const int row = i / units, c = i - row * units;
    *reinterpret_cast<U*>(base + to[row] * t.row_stride + from + c * sizeof(U)) = held[i];
  }
}

__global__ void __launch_bounds__(256) k_beam_reorder(const __grid_constant__ Moves q) {
  extern __shared__ __align__(16) unsigned char mem[];
  int* to = reinterpret_cast<int*>(mem);  // [beams]
  int* of = to + q.beams;
  unsigned char* held = mem + (2 * q.beams * sizeof(int) + 15) / 16 * 16;
  __shared__ int count;
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  const long long b = blockIdx.y;
  for (int w = threadIdx.x; w < q.beams; w += blockDim.x) {
    const long long p = q.parent[b * q.beams + w];
    if (p >= q.beams) atomicOr(q.err, kErrBadParent);
    if (p >= 0 && p < q.beams && p != w) {
      const int at = atomicAdd(&count, 1);
      to[at] = w;
      of[at] = static_cast<int>(p);
    }
  }
  __syncthreads();
  if (count == 0) return;
  int i = 0;
  while (i + 1 < q.count && q.t[i + 1].first_cta <= blockIdx.x) ++i;
  const Move& t = q.t[i];
  const long long from = static_cast<long long>(blockIdx.x - t.first_cta) * t.slice;
  const long long left = t.row_bytes - from;
  const int bytes = left < t.slice ? static_cast<int>(left) : t.slice;
  unsigned char* base = t.data + b * q.beams * t.row_stride;
  switch (t.unit) {
    case 16: move_slice<uint4>(t, base, from, bytes, to, of, count, held); break;
    case 8: move_slice<uint2>(t, base, from, bytes, to, of, count, held); break;
    case 4: move_slice<unsigned>(t, base, from, bytes, to, of, count, held); break;
    case 2: move_slice<unsigned short>(t, base, from, bytes, to, of, count, held); break;
    default: move_slice<unsigned char>(t, base, from, bytes, to, of, count, held);
  }
}

}  // namespace

size_t beam_workspace(const mlt_beam_args& a, int sms) { return a.batch == 0 ? 0 : plan_of(a, sms).bytes; }

cudaError_t launch_beam(const mlt_beam_args& a, void* ws, int sms, long long* launches, cudaStream_t st) {
  const Plan p = plan_of(a, sms);
  return with_dtype(a.dtype, [&](auto t) -> cudaError_t {
    using T = decltype(t);
    if (p.direct) {
      ++*launches;
      return launch_items<T, false>(a, p, nullptr, nullptr, st);
    }
    RowPart* found = static_cast<RowPart*>(ws);
    u64* lists = reinterpret_cast<u64*>(static_cast<unsigned char*>(ws) + p.off_lists);
    const long long rows = static_cast<long long>(a.batch) * a.beams;
    ++*launches;
    const cudaError_t e = launch_pdl(k_beam_rows<T>, dim3(static_cast<unsigned>(rows * p.parts)), dim3(kRowThreads), 0, st,
                                     a, p.parts, p.k, found, lists);
    if (e != cudaSuccess) return e;
    ++*launches;
    if (a.beams * p.parts * p.k <= kFewMost)
      return launch_pdl(k_beam_few, dim3(a.batch), dim3(kFewThreads), 0, st, a, p.parts, p.k,
                        static_cast<const RowPart*>(found), static_cast<const u64*>(lists));
    return launch_items<float, true>(a, p, found, lists, st);
  });
}

cudaError_t launch_reorder(const int64_t* parent, int batch, int beams, const mlt_beam_state* tensors, int count,
                           unsigned* err, long long* launches, cudaStream_t st) {
  Moves q{};
  q.beams = beams;
  q.parent = parent;
  q.err = err;
  // 48 KB for all beams' slices, at least 128 bytes of each
  int most = 48 * 1024 / beams / 16 * 16;
  if (most < 128) most = 128;
  if (most >= 4096) most = 4096;  // a 16-byte access for each of 256 threads
  unsigned long long ctas = 0;
  int widest = 0;
  for (int i = 0; i < count; ++i) {
    const mlt_beam_state& s = tensors[i];
    if (s.row_bytes == 0) continue;
    Move& t = q.t[q.count++];
    t.data = static_cast<unsigned char*>(s.data);
    t.row_bytes = s.row_bytes;
    t.row_stride = s.row_stride;
    t.unit = 16;
    const uintptr_t all = reinterpret_cast<uintptr_t>(s.data) | static_cast<uintptr_t>(s.row_bytes) |
                          (static_cast<long long>(batch) * beams > 1 ? static_cast<uintptr_t>(s.row_stride) : 0);
    while (all & (t.unit - 1)) t.unit /= 2;
    t.slice = s.row_bytes < most ? static_cast<int>(s.row_bytes) : most;
    t.first_cta = static_cast<unsigned>(ctas);
    ctas += (s.row_bytes + t.slice - 1) / t.slice;
    if (ctas > 0x7FFFFFFFull) return cudaErrorInvalidValue;
    widest = t.slice > widest ? t.slice : widest;
  }
  if (ctas == 0) return cudaSuccess;
  const size_t smem = (2 * beams * sizeof(int) + 15) / 16 * 16 + static_cast<size_t>(widest) * beams;
  if (smem > 40 * 1024) {  // with the static part past what a kernel has unasked, 48 KB
    const cudaError_t e = allow_smem(reinterpret_cast<const void*>(k_beam_reorder), smem);
    if (e != cudaSuccess) return e;
  }
  ++*launches;
  return launch_pdl(k_beam_reorder, dim3(static_cast<unsigned>(ctas), batch), dim3(256), smem, st, q);
}

}  // namespace mlt
