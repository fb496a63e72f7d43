// What the selective scan and its gradient share (not part of the C ABI).
//
// Four lanes share a channel (or two of them), each with S of its states (N <= 4 S); a CTA
// has CH channels of one group, so it reads one B and C row a position.
// Inputs are first turned into what the recurrence uses (step size, pushed input, gate) in
// shared memory, once per (position, channel): a thread does this for two adjacent
// channels and a run of consecutive positions, whose convolution windows overlap.
// Then each lane walks its states through the staged positions.
//
// Arithmetic on states goes through two-float instructions: they do not raise the rate of
// fp32 operations (128 a cycle and SM either way, measured) but take half the issue slots.
// They take no immediate operands, so formulas full of constants stay scalar.
#pragma once

#include <cfloat>
#include <cmath>
#include <type_traits>

#include "seq.cuh"

namespace mlt {
namespace scan {

constexpr int kGroups = 8;  // runs of positions staged side by side: 4 CH threads / (CH / 2) pairs

constexpr float kLog2E = 1.4426950408889634f;

struct Block {
  int b, c0, cn, g;  // sequence, first channel, channels, group
};

// Channel blocks are counted group by group (a block never spans two groups).
template <int CH>
__host__ __device__ inline int blocks_per_group(const mlt_scan_args& a) {
  return (a.dim / a.groups + CH - 1) / CH;
}

#ifdef __CUDACC__
template <int CH>
__device__ __forceinline__ Block block_of(const mlt_scan_args& a, int block, int b) {
  Block k;
  const int per = blocks_per_group<CH>(a), width = a.dim / a.groups;
  k.b = b;
  k.g = block / per;
  const int first = (block - k.g * per) * CH;
  k.c0 = k.g * width + first;
  k.cn = min(CH, width - first);
  return k;
}
__device__ __forceinline__ long long length_of(const mlt_scan_args& a, int b) {
  return a.lengths == nullptr ? a.length : min(max(static_cast<long long>(a.lengths[b]), 0ll),
                                               static_cast<long long>(a.length));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 1 / (1 + e^-x); e^-x may be infinite.
__device__ __forceinline__ float sigmoid(float x) { return rcp(1.0f + ex2(-kLog2E * x)); }

// ln(1 + e^x) = max(x, 0) + ln(1 + e), e = e^-|x| in (0, 1].  With s = e / (2 + e) <= 1/3,
// ln(1 + e) = 2 atanh s = 2 (s + s^3/3 + s^5/5 + ...): seven terms leave 2 s^15/15 < 1e-8, so
// the result keeps its relative precision where e is small (the usual step sizes are
// 0.001 .. 0.1), which log2 of 1 + e would lose.
__device__ __forceinline__ float softplus(float x) {
  const float e = ex2(-kLog2E * fabsf(x));
  const float s = e * rcp(2.0f + e);
  const float q = s * s;
  float p = 2.0f / 13.0f;
  p = fmaf(p, q, 2.0f / 11.0f);
  p = fmaf(p, q, 2.0f / 9.0f);
  p = fmaf(p, q, 2.0f / 7.0f);
  p = fmaf(p, q, 2.0f / 5.0f);
  p = fmaf(p, q, 2.0f / 3.0f);
  p = fmaf(p, q, 2.0f);
  return fmaxf(x, 0.0f) + p * s;
}

// Two floats through one issue slot (sm_100 and later).
struct F2 {
  unsigned long long v;
};
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void un2(F2 p, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v));
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 ex2_2(F2 a) {
  float x, y;
  un2(a, x, y);
  return f2(ex2(x), ex2(y));
}

// A log2 e, for powers of two.  Kept finite: the staged positions past a sequence's end have a step of
// 0, and 0 times an infinite rate would be NaN where the state is to stay as it is.  (NaN stays NaN.)
__device__ __forceinline__ float rate(float a) {
  const float r = a * kLog2E;
  return isinf(r) ? copysignf(FLT_MAX, r) : r;
}
__device__ __forceinline__ F2 rate2(F2 a) {
  float x, y;
  un2(a, x, y);
  return f2(rate(x), rate(y));
}

// exp(d A) of a position, log2 e within d or A.  ex2.approx takes its argument to a fixed-point number, rounded
// down: over 2^-8 .. 1 its results are 0.3 to 0.44 units of 2^-24 low on average, which over
// the hundred steps that a state remembers adds up to more than all else.  Adding 0.35 units
// to the argument, in the same instruction, leaves 0.2 either way (0.16 high below 2^-8); exp(0) stays 1.
__device__ __forceinline__ F2 decay2(F2 d, F2 A) {
  constexpr float kCentre = 0.35f / 16777216.0f;
  return ex2_2(fma2(d, A, f2(kCentre, kCentre)));
}

// States of a lane, as pairs (S = 1: the second half stays zero).
template <int S>
struct Lane {
  static constexpr int H = (S + 1) / 2;
  F2 v[H];
};
template <int S>
__device__ __forceinline__ Lane<S> lane_zero() {
  Lane<S> r;
#pragma unroll
  for (int h = 0; h < Lane<S>::H; ++h) r.v[h] = f2(0.0f, 0.0f);
  return r;
}
// p[j], j < S, zero where first + j >= n.
template <int S>
__device__ __forceinline__ Lane<S> lane_load(const float* p, int first, int n) {
  Lane<S> r;
#pragma unroll
  for (int h = 0; h < Lane<S>::H; ++h) {
    const float a = first + 2 * h < n ? p[2 * h] : 0.0f;
    const float b = 2 * h + 1 < S && first + 2 * h + 1 < n ? p[2 * h + 1] : 0.0f;
    r.v[h] = f2(a, b);
  }
  return r;
}
template <int S>
__device__ __forceinline__ void lane_store(float* p, int first, int n, const Lane<S>& r) {
#pragma unroll
  for (int h = 0; h < Lane<S>::H; ++h) {
    float a, b;
    un2(r.v[h], a, b);
    if (first + 2 * h < n) p[2 * h] = a;
    if (2 * h + 1 < S && first + 2 * h + 1 < n) p[2 * h + 1] = b;
  }
}
// S floats of shared memory, aligned to their size.
template <int S>
__device__ __forceinline__ Lane<S> lane_shared(const float* p) {
  Lane<S> r;
  if constexpr (S == 1) {
    r.v[0] = f2(p[0], 0.0f);
  } else if constexpr (S == 2) {
    const float2 q = *reinterpret_cast<const float2*>(p);
    r.v[0] = f2(q.x, q.y);
  } else {
#pragma unroll
    for (int k = 0; k < S / 4; ++k) {
      const float4 q = reinterpret_cast<const float4*>(p)[k];
      r.v[2 * k] = f2(q.x, q.y);
      r.v[2 * k + 1] = f2(q.z, q.w);
    }
  }
  return r;
}
template <int S>
__device__ __forceinline__ float lane_sum(const Lane<S>& r) {
  F2 s = r.v[0];
#pragma unroll
  for (int h = 1; h < Lane<S>::H; ++h) s = add2(s, r.v[h]);
  float a, b;
  un2(s, a, b);
  return a + b;
}

// Four values, one for each of four positions, of the four lanes of a channel: lane j gets the
// lanes' sum of value j (three shuffles instead of eight).
__device__ __forceinline__ float quad_sums(const float (&v)[4], int j) {
  const bool hi = j & 2, odd = j & 1;
  float a = hi ? v[2] : v[0], b = hi ? v[3] : v[1];
  a += __shfl_xor_sync(~0u, hi ? v[0] : v[2], 2);
  b += __shfl_xor_sync(~0u, hi ? v[1] : v[3], 2);
  float r = odd ? b : a;
  r += __shfl_xor_sync(~0u, odd ? a : b, 1);
  return r;
}

// ---------------------------------------------------------------------------
// Staging
// ---------------------------------------------------------------------------
__device__ __forceinline__ F2 dup2(float a) { return f2(a, a); }
__device__ __forceinline__ F2 rcp_2(F2 a) {
  float x, y;
  un2(a, x, y);
  return f2(rcp(x), rcp(y));
}
__device__ __forceinline__ F2 sigmoid2(F2 x) { return rcp_2(add2(ex2_2(mul2(x, dup2(-kLog2E))), dup2(1.0f))); }
__device__ __forceinline__ F2 softplus2(F2 x) {  // as softplus
  float a, b;
  un2(x, a, b);
  const F2 e = f2(ex2(-kLog2E * fabsf(a)), ex2(-kLog2E * fabsf(b)));
  const F2 s = mul2(e, rcp_2(add2(e, dup2(2.0f))));
  const F2 q = mul2(s, s);
  F2 p = dup2(2.0f / 13.0f);
  p = fma2(p, q, dup2(2.0f / 11.0f));
  p = fma2(p, q, dup2(2.0f / 9.0f));
  p = fma2(p, q, dup2(2.0f / 7.0f));
  p = fma2(p, q, dup2(2.0f / 5.0f));
  p = fma2(p, q, dup2(2.0f / 3.0f));
  p = fma2(p, q, dup2(2.0f));
  return fma2(p, s, f2(fmaxf(a, 0.0f), fmaxf(b, 0.0f)));
}

// Two adjacent channels of a row, as they are in memory: 16-bit types stay packed in one
// register until they are used.  (Held as two values they would be taken apart right
// after the load, which then waits for memory there.)
template <typename T>
struct Two {
  uint32_t w;
  __device__ __forceinline__ F2 f32() const {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      return f2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    } else {
      const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
      return f2(v.x, v.y);
    }
  }
};
template <>
struct Two<float> {
  F2 v;
  __device__ __forceinline__ F2 f32() const { return v; }
};
// kVec: one access (rows and addresses allow it), else element by element; `n` (1 or 2) of
// them belong to the block.
template <typename T, bool kVec>
__device__ __forceinline__ Two<T> load_two(const T* p, int n) {
  Two<T> r;
  if constexpr (sizeof(T) == 4) {
    if (kVec)
      r.v.v = *reinterpret_cast<const unsigned long long*>(p);
    else
      r.v = f2(p[0], n > 1 ? p[1] : 0.0f);
  } else {
    if (kVec) {
      r.w = *reinterpret_cast<const uint32_t*>(p);
    } else {
      const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
      r.w = h[0];
      if (n > 1) r.w |= static_cast<uint32_t>(h[1]) << 16;
    }
  }
  return r;
}
template <typename T>
__device__ __forceinline__ Two<T> two_zero() {
  Two<T> r;
  if constexpr (sizeof(T) == 4) r.v = f2(0.0f, 0.0f);
  else r.w = 0;
  return r;
}
template <typename T, bool kVec>
__device__ __forceinline__ void store_two(T* p, int n, F2 v) {
  float a, b;
  un2(v, a, b);
  Pack<T, 2> r;
  r.v[0] = from_f32<T>(a);
  r.v[1] = from_f32<T>(b);
  if (kVec) {
    *reinterpret_cast<Pack<T, 2>*>(p) = r;
  } else {
    p[0] = r.v[0];
    if (n > 1) p[1] = r.v[1];
  }
}
template <typename T>
__device__ __forceinline__ F2 two_f32(const Two<T>& p) {
  return p.f32();
}

// A thread's two channels and what staging needs of their parameters.
struct PairParams {
  int c, n;     // first channel within the block; how many of the two belong to it
  F2 w[kScanMaxTaps], conv_b, bias;  // w[0] meets x[t]
};
template <int CH>
__device__ __forceinline__ PairParams pair_params(const mlt_scan_args& a, const Block& k) {
  PairParams q;
  q.c = threadIdx.x % (CH / 2) * 2;
  q.n = max(0, min(2, k.cn - q.c));
  const int ch = k.c0 + q.c;
  auto two = [&](const float* p) {
    return p == nullptr ? dup2(0.0f) : f2(q.n > 0 ? p[ch] : 0.0f, q.n > 1 ? p[ch + 1] : 0.0f);
  };
  q.conv_b = two(a.taps > 0 ? a.conv_b : nullptr);
  q.bias = two(a.dt_bias);
#pragma unroll
  for (int j = 0; j < kScanMaxTaps; ++j) {
    const long long at = static_cast<long long>(ch) * a.taps + a.taps - 1 - j;
    const bool on = j < a.taps;
    q.w[j] = f2(on && q.n > 0 ? a.conv_w[at] : 0.0f, on && q.n > 1 ? a.conv_w[at + a.taps] : 0.0f);
  }
  return q;
}

// Inputs of a run of positions; x[kScanMaxTaps - 1 + i] belongs to position i.
template <typename T, int RUN>
struct RawRun {
  Two<T> x[RUN + kScanMaxTaps - 1], dt[RUN], z[RUN];
};

// Positions first .. first + RUN - 1 below `end`; what lies before the start comes from
// conv_state.
template <typename T, int RUN, bool kVec, bool kGate>
__device__ __forceinline__ void load_run(const mlt_scan_args& a, const Block& k, const PairParams& q, long long first,
                                         long long end, RawRun<T, RUN>& r) {
  if (q.n == 0 || first >= end) return;
  const int ch = k.c0 + q.c;
  const long long left = end - first;
  const T* x = static_cast<const T*>(a.x) + k.b * a.x_batch + first * a.x_step + ch;
  if (a.taps > 1) {
    if (first >= kScanMaxTaps - 1) {
      const T* p = x;
#pragma unroll
      for (int j = 1; j < kScanMaxTaps; ++j) {
        p -= a.x_step;
        if (j < a.taps) r.x[kScanMaxTaps - 1 - j] = load_two<T, kVec>(p, q.n);
      }
    } else {
#pragma unroll
      for (int j = 1; j < kScanMaxTaps; ++j) {
        if (j >= a.taps) break;
        const long long t = first - j;
        Two<T> v = two_zero<T>();
        if (t >= 0)
          v = load_two<T, kVec>(x - j * a.x_step, q.n);
        else if (a.conv_state != nullptr && t + a.taps - 1 >= 0)
          v = load_two<T, kVec>(static_cast<const T*>(a.conv_state) +
                                    (static_cast<long long>(k.b) * (a.taps - 1) + t + a.taps - 1) * a.dim + ch,
                                q.n);
        r.x[kScanMaxTaps - 1 - j] = v;
      }
    }
  }
  const T* d = static_cast<const T*>(a.dt) + k.b * a.dt_batch + first * a.dt_step + ch;
  const T* z = static_cast<const T*>(a.z) + k.b * a.z_batch + first * a.z_step + ch;
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    if (i < left) {
      r.x[kScanMaxTaps - 1 + i] = load_two<T, kVec>(x, q.n);
      r.dt[i] = load_two<T, kVec>(d, q.n);
      if (kGate && a.z != nullptr) r.z[i] = load_two<T, kVec>(z, q.n);
    }
    x += a.x_step;
    d += a.dt_step;
    z += a.z_step;
  }
}

// Convolution of position i of the run, before its activation (x itself without taps).
template <typename T, int RUN>
__device__ __forceinline__ F2 conv_run(const mlt_scan_args& a, const PairParams& q, const RawRun<T, RUN>& r, int i) {
  const F2 x0 = two_f32(r.x[kScanMaxTaps - 1 + i]);
  if (a.taps == 0) return x0;
  F2 v = fma2(q.w[0], x0, q.conv_b);
#pragma unroll
  for (int j = 1; j < kScanMaxTaps; ++j)
    if (j < a.taps) v = fma2(q.w[j], two_f32(r.x[kScanMaxTaps - 1 + i - j]), v);
  return v;
}

// Input at position t of the sequence (before the start: conv_state, or 0).
template <typename T>
__device__ __forceinline__ float input_at(const mlt_scan_args& a, int b, long long t, int ch) {
  if (t >= 0) return t < a.length ? to_f32(static_cast<const T*>(a.x)[b * a.x_batch + t * a.x_step + ch]) : 0.0f;
  if (a.conv_state == nullptr || t < -(a.taps - 1)) return 0.0f;
  return to_f32(static_cast<const T*>(a.conv_state)[(static_cast<long long>(b) * (a.taps - 1) + t + a.taps - 1) * a.dim +
                                                    ch]);
}
// Two adjacent elements of shared memory, aligned to both.
template <typename T>
__device__ __forceinline__ F2 shared_two(const T* p) {
  Two<T> r;
  if constexpr (sizeof(T) == 4) r.v.v = *reinterpret_cast<const unsigned long long*>(p);
  else r.w = *reinterpret_cast<const uint32_t*>(p);
  return r.f32();
}
template <typename T>
__device__ __forceinline__ void copy_two(T* to, const T* from) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<unsigned long long*>(to) = *reinterpret_cast<const unsigned long long*>(from);
  else *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
}
#endif

// Whether two adjacent channels are one aligned access in every row.
inline bool pairs_ok(const mlt_scan_args& a) {
  const size_t bytes = 2 * dtype_size(a.dtype);
  bool ok = a.dim / a.groups % 2 == 0 && aligned_to(a.conv_state, bytes);
  ok = ok && aligned_to(a.x, bytes) && a.x_step % 2 == 0 && a.x_batch % 2 == 0;
  ok = ok && aligned_to(a.dt, bytes) && a.dt_step % 2 == 0 && a.dt_batch % 2 == 0;
  return ok && (a.z == nullptr || (aligned_to(a.z, bytes) && a.z_step % 2 == 0 && a.z_batch % 2 == 0));
}
// Calls f with the number of states a lane takes.
template <typename F>
auto with_states(int n, F f) {
  if (n <= 4) return f(std::integral_constant<int, 1>());
  if (n <= 8) return f(std::integral_constant<int, 2>());
  if (n <= 16) return f(std::integral_constant<int, 4>());
  return f(std::integral_constant<int, 8>());
}
inline int states_padded(int n) { return n <= 4 ? 4 : n <= 8 ? 8 : n <= 16 ? 16 : 32; }

}  // namespace scan
}  // namespace mlt
