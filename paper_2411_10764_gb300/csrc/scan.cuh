// What the selective scan and its gradient share (not part of the C ABI).
//
// Four lanes share a channel, each with S of its states (N <= 4 S); a CTA has 64
// channels of one group, so it reads one B and C row a position.  Per tile of
// positions the CTA first turns the inputs into what the recurrence
// uses (step size, pushed input, gate) in shared memory, once per
// (position, channel), then each lane walks its states through the tile.
#pragma once

#include <cmath>
#include <type_traits>

#include "seq.cuh"

namespace mlt {
namespace scan {

constexpr int kChannels = 64;          // of a CTA
constexpr int kThreads = 4 * kChannels;
constexpr int kTile = 16;              // positions staged at a time
constexpr int kPackC = 4;              // channels a thread stages at once
static_assert(kTile * kChannels == kThreads * kPackC, "a thread stages one pack of a tile");

constexpr float kLog2E = 1.4426950408889634f;

struct Block {
  int b, c0, cn, g;  // sequence, first channel, channels, group
};

// blockIdx.x counts channel blocks, group by group (a block never spans two groups).
__host__ __device__ inline int blocks_per_group(const mlt_scan_args& a) {
  return (a.dim / a.groups + kChannels - 1) / kChannels;
}

#ifdef __CUDACC__
__device__ __forceinline__ Block block_of(const mlt_scan_args& a, int block, int b) {
  Block k;
  const int per = blocks_per_group(a), width = a.dim / a.groups;
  k.b = b;
  k.g = block / per;
  const int first = (block - k.g * per) * kChannels;
  k.c0 = k.g * width + first;
  k.cn = min(kChannels, width - first);
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
// ln(1 + e) = 2 atanh s = 2 (s + s^3/3 + s^5/5 + ...): nine terms leave 2 s^19/19 < 1e-10, so
// the result keeps its relative precision where e is small (the usual step sizes are
// 0.001 .. 0.1), which log2 of 1 + e would lose.
__device__ __forceinline__ float softplus(float x) {
  const float e = ex2(-kLog2E * fabsf(x));
  const float s = e * rcp(2.0f + e);
  const float q = s * s;
  float p = 2.0f / 17.0f;
  p = fmaf(p, q, 2.0f / 15.0f);
  p = fmaf(p, q, 2.0f / 13.0f);
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

// kPackC channels of a row: one access where the call's strides and addresses allow, else
// element by element; nothing past the block's channels is read or written.
template <typename T, bool kVec>
__device__ __forceinline__ Pack<T, kPackC> load_pack(const T* row, int c, int cn) {
  Pack<T, kPackC> p;
  if (kVec) {
    if (c < cn) p = *reinterpret_cast<const Pack<T, kPackC>*>(row + c);
  } else {
#pragma unroll
    for (int e = 0; e < kPackC; ++e)
      if (c + e < cn) p.v[e] = row[c + e];
  }
  return p;
}
template <typename T, bool kVec>
__device__ __forceinline__ void store_pack(T* row, int c, int cn, const Pack<T, kPackC>& p) {
  if (kVec) {
    if (c < cn) *reinterpret_cast<Pack<T, kPackC>*>(row + c) = p;
  } else {
#pragma unroll
    for (int e = 0; e < kPackC; ++e)
      if (c + e < cn) row[c + e] = p.v[e];
  }
}

// Input x at position t - back (before the start: conv_state, or zeros).
template <typename T, bool kVec>
__device__ __forceinline__ Pack<T, kPackC> load_x(const mlt_scan_args& a, const Block& k, long long t, int c) {
  if (t >= 0)
    return load_pack<T, kVec>(static_cast<const T*>(a.x) + k.b * a.x_batch + t * a.x_step + k.c0, c, k.cn);
  Pack<T, kPackC> p;
#pragma unroll
  for (int e = 0; e < kPackC; ++e) p.v[e] = from_f32<T>(0.0f);
  if (a.conv_state != nullptr)
    p = load_pack<T, kVec>(static_cast<const T*>(a.conv_state) +
                               (static_cast<long long>(k.b) * (a.taps - 1) + t + a.taps - 1) * a.dim + k.c0,
                           c, k.cn);
  return p;
}

// The convolution's weights of a thread's channels, last tap first: w[0] meets x[t].
struct Taps {
  float w[kScanMaxTaps][kPackC];
  float b[kPackC];
};
__device__ __forceinline__ Taps load_taps(const mlt_scan_args& a, const Block& k, int c) {
  Taps q;
#pragma unroll
  for (int e = 0; e < kPackC; ++e) {
    const int ch = k.c0 + c + e;
    const bool in = c + e < k.cn;
    q.b[e] = in && a.conv_b != nullptr && a.taps > 0 ? a.conv_b[ch] : 0.0f;
#pragma unroll
    for (int j = 0; j < kScanMaxTaps; ++j)
      q.w[j][e] = in && j < a.taps ? a.conv_w[static_cast<long long>(ch) * a.taps + a.taps - 1 - j] : 0.0f;
  }
  return q;
}
// The inputs that position t's convolution reads; [0] is x[t].
template <typename T>
struct Window {
  Pack<T, kPackC> x[kScanMaxTaps];
};
template <typename T, bool kVec>
__device__ __forceinline__ Window<T> load_window(const mlt_scan_args& a, const Block& k, long long t, int c) {
  Window<T> w;
  w.x[0] = load_x<T, kVec>(a, k, t, c);
#pragma unroll
  for (int j = 1; j < kScanMaxTaps; ++j)
    if (j < a.taps) w.x[j] = load_x<T, kVec>(a, k, t - j, c);
  return w;
}
// The convolution's output before its activation (x itself without taps).
template <typename T>
__device__ __forceinline__ float conv_at(const mlt_scan_args& a, const Taps& q, const Window<T>& w, int e) {
  if (a.taps == 0) return to_f32(w.x[0].v[e]);
  float v = fmaf(q.w[0][e], to_f32(w.x[0].v[e]), q.b[e]);
#pragma unroll
  for (int j = 1; j < kScanMaxTaps; ++j)
    if (j < a.taps) v = fmaf(q.w[j][e], to_f32(w.x[j].v[e]), v);
  return v;
}

// A tile's rows of B (or C) as floats, [kTile][4 S], zero past `live` positions and N states.
template <typename T, int S>
__device__ __forceinline__ void stage_rows(float* to, const T* rows, long long step, int n, int live) {
  for (int i = threadIdx.x; i < kTile * 4 * S; i += kThreads) {
    const int t = i / (4 * S), s = i - t * (4 * S);
    to[i] = t < live && s < n ? to_f32(rows[t * step + s]) : 0.0f;
  }
}
#endif

// Whether packs of kPackC channels are aligned in every row.
inline bool packs_ok(const mlt_scan_args& a) {
  const size_t e = dtype_size(a.dtype), bytes = e * kPackC;
  const int64_t w = kPackC;
  bool ok = a.dim / a.groups % w == 0 && aligned_to(a.conv_state, bytes) && aligned_to(a.conv_state_out, bytes);
  ok = ok && aligned_to(a.x, bytes) && a.x_step % w == 0 && a.x_batch % w == 0;
  ok = ok && aligned_to(a.dt, bytes) && a.dt_step % w == 0 && a.dt_batch % w == 0;
  ok = ok && (a.z == nullptr || (aligned_to(a.z, bytes) && a.z_step % w == 0 && a.z_batch % w == 0));
  return ok;
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

// Sequences are cut into `chunks` of `chunk` positions (a multiple of kTile).
struct Chunks {
  long long chunk;
  int chunks;
};

}  // namespace scan
}  // namespace mlt
