// One AdamW step over many tensors (Loshchilov and Hutter, decoupled weight decay), with
// moments in 32 bits or in 8 with one power-of-two scale for each 256 of them.
//
// The tensors' addresses travel in the launch's parameters (up to kMost of them, in
// two sizes of table), so nothing is copied to the device and a captured
// graph holds them by value.  Each CTA takes a span of 8 to 32 blocks of 256 elements; it finds its
// tensor by bisection over the table.  A warp takes a block at a time, each lane 2 x 4
// elements 128 apart, so every access of a warp is one contiguous run.
//
// Bound, for fp32 parameters with bf16 gradients and copies: 32 bits memory, 28 bytes an element (118 M of them
// 484 us, 6.8 TB/s); 8 bits 16 bytes, and 80 instructions (368 us, 5.2 TB/s at 77 % of the issue slots).
//
// 8 bits: scales are powers of two, so scaling is exact and a value that a code stands for
// stays where it is while the block's largest one keeps its octave.  Codes are cut from the bits of the value
// as an fp32 number, scaled so that the format's smallest normal is fp32's: subnormal
// codes come out as fp32's subnormals.  Adding a random number below one step to the bits before the cut
// rounds up with the probability of the value's place between two codes.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>
#include <vector>

#include <cuda_fp8.h>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kBlock = 256;
constexpr int kMostSpan = 32;  // blocks a CTA
constexpr int kMost = 500;

struct Tensor {
  void* param;
  const void* grad;
  void* copy;
  long long n;
  long long block;     // of the moments
  unsigned first_cta;  // of this launch
  float rate, keep;    // lr / (1 - beta1^step) and 1 - lr weight_decay; both of lr 1, the latter without
                       // the 1 -, where lr is on the device
  uint8_t dtype, grad_dtype, copy_dtype, wide;  // wide: four values at once are aligned everywhere
};
struct Common {
  float beta1, one_beta1, beta2, one_beta2, eps, root;  // root: 1 / sqrt(1 - beta2^step)
  float log_beta1, log_beta2;                           // for a step on the device
  const int64_t* step_device;
  const float* lr;
  const float* grad_scale;
  long long step;
  unsigned seed;
  int count, span;
  void *m, *v;
  float *m_scale, *v_scale;
};

template <int N>
struct Table {
  Common c;
  Tensor t[N];
};
static_assert(sizeof(Table<kMost>) <= 32764, "the table has to fit a launch's parameters");

// To two units in the last place; FAST takes subnormal numbers as 0.  p alone depends on them.
template <bool FAST>
__device__ __forceinline__ float root_of(float v) {
  float r;
  if constexpr (FAST)
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  else
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
template <bool FAST>
__device__ __forceinline__ float one_over(float v) {
  float r;
  if constexpr (FAST)
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  else
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

__device__ __forceinline__ unsigned mix(unsigned h) {
  h ^= h >> 16;
  h *= 0x9E3779B1u;
  h ^= h >> 15;
  h *= 0xB504F333u;
  return h ^ (h >> 16);
}

// Four values of any type as they lie in memory, loaded before any of them is looked at.
struct __align__(16) Four {
  unsigned r[4];
};
__device__ __forceinline__ Four wide4(const char* p) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  return {{w.x, w.y, w.z, w.w}};
}
__device__ __forceinline__ Four narrow4(const char* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return {{w.x, w.y, 0u, 0u}};
}
// As fp32, where addresses allow no packs or fewer than four are left.
__device__ __forceinline__ Four some4(const void* p, int dtype, long long i, int left) {
  Four q;
#pragma unroll
  for (int k = 0; k < 4; ++k) q.r[k] = k < left ? __float_as_uint(load_as_f32(p, dtype, i + k)) : 0u;
  return q;
}

__device__ __forceinline__ void values4(float (&v)[4], const Four& q, int dtype) {
  if (dtype == MLT_F32) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(q.r[k]);
  } else if (dtype == MLT_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(k & 1 ? q.r[k / 2] & 0xFFFF0000u : q.r[k / 2] << 16);
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&q.r[k]));
      v[2 * k] = f.x;
      v[2 * k + 1] = f.y;
    }
  }
}

__device__ __forceinline__ void store4(char* p, const float (&v)[4], int dtype) {
  if (dtype == MLT_F32) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else if (dtype == MLT_BF16) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
  } else {
    const __half2 a = __floats2half2_rn(v[0], v[1]), b = __floats2half2_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
  }
}

// Four codes of m (e4m3) or v (e5m2, the upper byte of a half) as numbers, times a factor.
__device__ __forceinline__ void decode_e4m3(float (&v)[4], unsigned word, float factor) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(word >> (16 * k)), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    v[2 * k] = __fmul_rn(f.x, factor);
    v[2 * k + 1] = __fmul_rn(f.y, factor);
  }
}
__device__ __forceinline__ void decode_e5m2(float (&v)[4], unsigned word, float factor) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const unsigned h = __byte_perm(word, 0, k == 0 ? 0x1404 : 0x3424);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    v[2 * k] = __fmul_rn(f.x, factor);
    v[2 * k + 1] = __fmul_rn(f.y, factor);
  }
}

// The words of four values' codes; e: the block's exponent (16 .. 255), r: the values' hashes.  A value is
// scaled so that its code is cut at a fixed bit (in two steps where one factor would be subnormal: SMALL
// tells that it is not), the code comes to lie in the upper byte of a word, the sign of m with it, and the four
// upper bytes are gathered.
__device__ __forceinline__ unsigned bytes_of(unsigned a, unsigned b, unsigned pick) {
  unsigned d;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(pick));
  return d;
}
__device__ __forceinline__ unsigned gather(const unsigned (&x)[4]) {
  return bytes_of(bytes_of(x[0], x[1], 0x0073), bytes_of(x[2], x[3], 0x0073), 0x5410);
}
template <bool SMALL>
__device__ __forceinline__ unsigned encode_e4m3(const float (&m)[4], unsigned e, const unsigned (&r)[4]) {
  const float up = __uint_as_float((127 + (SMALL ? 14 : 134) - e) << 23);
  unsigned x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float s = fabsf(m[k]) * up;
    if (!SMALL) s *= 0x1p-120f;
    // (the sum first: its terms scaled by 16 and added gave 0 from nvcc 13.0)
    const unsigned c = (__float_as_uint(s) + ((r[k] << 4) & 0xFFFF0u)) << 4;
    x[k] = (c & 0x7F000000u) | (__float_as_uint(m[k]) & ~0x7F000000u);
  }
  return e == 255 ? 0x7F7F7F7Fu : gather(x);
}
template <bool SMALL>
__device__ __forceinline__ unsigned encode_e5m2(const float (&v)[4], unsigned e, const unsigned (&r)[4]) {
  const float up = __uint_as_float((127 + (SMALL ? 29 : 141) - e) << 23);
  unsigned x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float s = v[k] * up;
    if (!SMALL) s *= 0x1p-112f;
    const unsigned c = (__float_as_uint(s) + ((r[k] >> 16) << 5)) << 3;
    x[k] = v[k] > 0.0f ? max(c, 1u << 24) : c;
  }
  return e == 255 ? 0x7F7F7F7Fu : gather(x);
}

// max(|a|, b), NaN where one is.
__device__ __forceinline__ float max_of(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(fabsf(a)), "f"(b));
  return d;
}

// What a lane of a block works on, as loaded.
template <int BITS>
struct Raw {
  Four p[2], g[2];
  Four m[BITS == 32 ? 2 : 1], v[BITS == 32 ? 2 : 1];  // 8 bits: words 0 and 1
  float ms, vs;
};

// A block a warp on its way, by thread.
struct Stage {
  Four p[2][256], g[2][256];
  unsigned m[2][256], v[2][256];
};
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  const unsigned at = static_cast<unsigned>(__cvta_generic_to_shared(to));
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}

// FAST: eps is large enough (1e-10) that roots and quotients of subnormal numbers are nothing beside it.
template <int N, int BITS, bool FAST>
__global__ void __launch_bounds__(256, 4) k_adamw(const __grid_constant__ Table<N> q) {
  pdl_wait();
  pdl_trigger();
  const Common& c = q.c;
  int lo = 0, hi = c.count - 1;  // the last tensor whose CTAs begin at or before this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (q.t[mid].first_cta <= blockIdx.x)
      lo = mid;
    else
      hi = mid - 1;
  }
  const Tensor& t = q.t[lo];
  float rate = t.rate, keep = t.keep, root = c.root;
  long long step = c.step;
  if (c.step_device != nullptr) {
    step = *c.step_device;
    const float s = static_cast<float>(step);
    rate /= -expm1f(s * c.log_beta1);
    root = 1.0f / sqrtf(-expm1f(s * c.log_beta2));
  }
  if (c.lr != nullptr) {
    const float lr = *c.lr;
    keep = 1.0f - lr * t.keep;
    rate *= lr;
  }
  const float scale = c.grad_scale != nullptr ? *c.grad_scale : 1.0f;
  const unsigned key = mix(mix(c.seed) + static_cast<unsigned>(step));
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long from = static_cast<long long>(blockIdx.x - t.first_cta) * c.span + warp;
  const long long blocks = (t.n + kBlock - 1) / kBlock;
  const int turns = static_cast<int>(min(static_cast<long long>(c.span) - warp, blocks - from) + 7) / 8;
  if (turns <= 0) return;
  const int dtype = t.dtype, grad_dtype = t.grad_dtype, copy_dtype = t.copy_dtype;
  const int ps = dtype == MLT_F32 ? 2 : 1, gs = grad_dtype == MLT_F32 ? 2 : 1, cs = copy_dtype == MLT_F32 ? 2 : 1;
  // a tensor's whole blocks with aligned addresses, then what is left
  const long long whole = t.wide ? t.n / kBlock : 0;
  // 8 bits: the next block's values are on their way to shared memory while this one's are worked on, each
  // thread's to places of its own (where they waited in registers, fewer warps fitted)
  __shared__ Stage staged[BITS == 8 ? 2 : 1];
  float next_ms = 0.0f, next_vs = 0.0f;
  auto fetch = [&](int k) {
    const long long at = from + 8 * k, i = at * kBlock + lane * 4, s0 = (t.block + at) * kBlock + lane * 4;
    Stage& to = staged[k & 1];
    if (at < whole) {
      const char *p = static_cast<const char*>(t.param) + (i << ps), *g = static_cast<const char*>(t.grad) + (i << gs);
      const char *m = static_cast<const char*>(c.m) + s0, *v = static_cast<const char*>(c.v) + s0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (dtype == MLT_F32)
          copy_async<16>(&to.p[h][threadIdx.x], p + 512 * h);
        else
          copy_async<8>(&to.p[h][threadIdx.x], p + 256 * h);
        if (grad_dtype == MLT_F32)
          copy_async<16>(&to.g[h][threadIdx.x], g + 512 * h);
        else
          copy_async<8>(&to.g[h][threadIdx.x], g + 256 * h);
        copy_async<4>(&to.m[h][threadIdx.x], m + 128 * h);
        copy_async<4>(&to.v[h][threadIdx.x], v + 128 * h);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    next_ms = c.m_scale[t.block + at];
    next_vs = c.v_scale[t.block + at];
  };
  if (BITS == 8) fetch(0);
#pragma unroll 1
  for (int k = 0; k < turns; ++k) {
    const long long at = from + 8 * k, i = at * kBlock + lane * 4;
    const long long s0 = (t.block + at) * kBlock + lane * 4;
    const unsigned b = static_cast<unsigned>(t.block + at);  // its low 32 bits, for the hash
    const bool full = at < whole;
    char* to_p = static_cast<char*>(t.param) + (i << ps);
    char *to_m = static_cast<char*>(c.m) + s0 * (BITS / 8), *to_v = static_cast<char*>(c.v) + s0 * (BITS / 8);
    Raw<BITS> now;
    int left[2] = {4, 4};
    if constexpr (BITS == 8) {
      now.ms = next_ms;
      now.vs = next_vs;
      if (k + 1 < turns) {
        fetch(k + 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      if (full) {
        const Stage& here = staged[k & 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          now.p[h] = here.p[h][threadIdx.x];
          now.g[h] = here.g[h][threadIdx.x];
          now.m[0].r[h] = here.m[h][threadIdx.x];
          now.v[0].r[h] = here.v[h][threadIdx.x];
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          now.m[0].r[h] = *reinterpret_cast<const unsigned*>(to_m + 128 * h);
          now.v[0].r[h] = *reinterpret_cast<const unsigned*>(to_v + 128 * h);
        }
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        now.m[h] = wide4(to_m + 512 * h);
        now.v[h] = wide4(to_v + 512 * h);
      }
      if (full) {
        const char* g = static_cast<const char*>(t.grad) + (i << gs);
        if (dtype == MLT_F32) {
          now.p[0] = wide4(to_p);
          now.p[1] = wide4(to_p + 512);
        } else {
          now.p[0] = narrow4(to_p);
          now.p[1] = narrow4(to_p + 256);
        }
        if (grad_dtype == MLT_F32) {
          now.g[0] = wide4(g);
          now.g[1] = wide4(g + 512);
        } else {
          now.g[0] = narrow4(g);
          now.g[1] = narrow4(g + 256);
        }
      }
    }
    if (!full) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const long long rest = t.n - (i + 128 * h);
        left[h] = rest < 0 ? 0 : rest > 4 ? 4 : static_cast<int>(rest);
        now.p[h] = some4(t.param, dtype, i + 128 * h, left[h]);
        now.g[h] = some4(t.grad, grad_dtype, i + 128 * h, left[h]);
      }
    }
    float m[2][4], v[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float p[4], g[4];
      values4(p, now.p[h], full ? dtype : MLT_F32);
      values4(g, now.g[h], full ? grad_dtype : MLT_F32);
      if constexpr (BITS == 32) {
        values4(m[h], now.m[h], MLT_F32);
        values4(v[h], now.v[h], MLT_F32);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m[h][e] = __fmul_rn(m[h][e], c.beta1);
          v[h][e] = __fmul_rn(v[h][e], c.beta2);
        }
      } else {
        // a moment, then beta times it; the scale is a power of two, so where nothing is subnormal one
        // product with both rounds alike
        const float fm = __fmul_rn(now.ms, c.beta1), fv = __fmul_rn(now.vs, c.beta2);
        if (fm >= 0x1p-100f && fv >= 0x1p-100f) {
          decode_e4m3(m[h], now.m[0].r[h], fm);
          decode_e5m2(v[h], now.v[0].r[h], fv);
        } else {
          decode_e4m3(m[h], now.m[0].r[h], now.ms);
          decode_e5m2(v[h], now.v[0].r[h], now.vs);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            m[h][e] = __fmul_rn(m[h][e], c.beta1);
            v[h][e] = __fmul_rn(v[h][e], c.beta2);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __fmul_rn(g[e], scale);
        m[h][e] = __fadd_rn(m[h][e], __fmul_rn(x, c.one_beta1));
        v[h][e] = __fadd_rn(v[h][e], __fmul_rn(__fmul_rn(x, x), c.one_beta2));
        const float d = m[h][e] * one_over<FAST>(fmaf(root_of<FAST>(v[h][e]), root, c.eps));
        p[e] = fmaf(-rate, d, __fmul_rn(p[e], keep));
      }
      if (full) {
        store4(to_p + ((128 * h) << ps), p, dtype);
        if (t.copy != nullptr) store4(static_cast<char*>(t.copy) + ((i + 128 * h) << cs), p, copy_dtype);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (e >= left[h]) continue;
          store_from_f32(t.param, dtype, i + 128 * h + e, p[e]);
          if (t.copy != nullptr) store_from_f32(t.copy, copy_dtype, i + 128 * h + e, p[e]);
        }
      }
    }
    if constexpr (BITS == 32) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (left[h] == 4) {
          *reinterpret_cast<float4*>(to_m + 512 * h) = make_float4(m[h][0], m[h][1], m[h][2], m[h][3]);
          *reinterpret_cast<float4*>(to_v + 512 * h) = make_float4(v[h][0], v[h][1], v[h][2], v[h][3]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < left[h]) {
              reinterpret_cast<float*>(to_m + 512 * h)[e] = m[h][e];
              reinterpret_cast<float*>(to_v + 512 * h)[e] = v[h][e];
            }
        }
      }
    } else {
      if (!full)  // what a tensor's last block has not
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e >= left[h]) m[h][e] = v[h][e] = 0.0f;
      float most_m = 0.0f, most_v = 0.0f;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          most_m = max_of(m[h][e], most_m);
          most_v = max_of(v[h][e], most_v);
        }
      const unsigned em = max(__reduce_max_sync(0xffffffffu, __float_as_uint(most_m)) >> 23, 16u);
      const unsigned ev = max(__reduce_max_sync(0xffffffffu, __float_as_uint(most_v)) >> 23, 16u);
      const unsigned kb = mix(b + key) + lane * 4 * 0x9E3779B9u;
      unsigned wm[2], wv[2];
      auto encode = [&](auto small) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          unsigned r[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) r[e] = mix(kb + (128u * h + e) * 0x9E3779B9u);
          wm[h] = encode_e4m3<decltype(small)::value>(m[h], em, r);
          wv[h] = encode_e5m2<decltype(small)::value>(v[h], ev, r);
        }
      };
      if (em <= 140 && ev <= 155)
        encode(std::true_type());
      else
        encode(std::false_type());
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (left[h] == 4) {
          *reinterpret_cast<unsigned*>(to_m + 128 * h) = wm[h];
          *reinterpret_cast<unsigned*>(to_v + 128 * h) = wv[h];
        } else {
          for (int e = 0; e < left[h]; ++e) {
            to_m[128 * h + e] = static_cast<char>(wm[h] >> (8 * e));
            to_v[128 * h + e] = static_cast<char>(wv[h] >> (8 * e));
          }
        }
      }
      if (lane == 0) {
        c.m_scale[t.block + at] = __uint_as_float((em - 7) << 23);
        c.v_scale[t.block + at] = __uint_as_float((ev - 14) << 23);
      }
    }
  }
}

template <int N>
cudaError_t launch_table(const Common& c, const std::vector<Tensor>& list, size_t from, int count, unsigned ctas, int bits,
                         cudaStream_t st) {
  static thread_local Table<N> q;  // 32 KB at most: not on the stack
  q.c = c;
  q.c.count = count;
  std::copy(list.begin() + from, list.begin() + from + count, q.t);
  const bool fast = c.eps >= 1e-10f;
  auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(ctas), dim3(256), 0, st, q); };
  if (bits == 8) return fast ? go(k_adamw<N, 8, true>) : go(k_adamw<N, 8, false>);
  return fast ? go(k_adamw<N, 32, true>) : go(k_adamw<N, 32, false>);
}

cudaError_t launch_part(const Common& c, const std::vector<Tensor>& list, size_t from, int count, unsigned ctas, int bits,
                        cudaStream_t st) {
  if (count <= 32) return launch_table<32>(c, list, from, count, ctas, bits, st);
  return launch_table<kMost>(c, list, from, count, ctas, bits, st);
}

}  // namespace

cudaError_t launch_adamw(const mlt_adamw_tensor* tensors, int count, const mlt_adamw_rule& r, void* m, void* v,
                         float* m_scale, float* v_scale, int sms, long long* launches, cudaStream_t st) {
  const bool on_device = r.step_device != nullptr;
  const double t = static_cast<double>(r.step);
  // 1 - beta^step without cancellation
  const double bias1 = on_device ? 1.0 : -std::expm1(t * std::log(r.beta1));
  const double bias2 = on_device ? 1.0 : -std::expm1(t * std::log(r.beta2));
  Common c{};
  c.beta1 = static_cast<float>(r.beta1);
  c.one_beta1 = static_cast<float>(1.0 - r.beta1);
  c.beta2 = static_cast<float>(r.beta2);
  c.one_beta2 = static_cast<float>(1.0 - r.beta2);
  c.eps = static_cast<float>(r.eps);
  c.root = static_cast<float>(1.0 / std::sqrt(bias2));
  c.log_beta1 = static_cast<float>(std::log(r.beta1));
  c.log_beta2 = static_cast<float>(std::log(r.beta2));
  c.step_device = r.step_device;
  c.lr = r.lr;
  c.grad_scale = r.grad_scale;
  c.step = r.step;
  c.seed = r.seed;
  c.m = m;
  c.v = v;
  c.m_scale = m_scale;
  c.v_scale = v_scale;
  // four blocks a warp where they fill the GPU several times over, else one
  long long all = 0;
  for (int i = 0; i < count; ++i) all += tensors[i].grad == nullptr ? 0 : (tensors[i].n + kBlock - 1) / kBlock;
  c.span = 8;
  while (c.span < kMostSpan && all > 16LL * sms * c.span) c.span *= 2;
  std::vector<Tensor> list;
  list.reserve(count);
  long long block = 0, ctas = 0;
  size_t from = 0;
  auto flush = [&]() -> cudaError_t {
    const int n = static_cast<int>(list.size() - from);
    if (n == 0) return cudaSuccess;
    ++*launches;
    const cudaError_t e = launch_part(c, list, from, n, static_cast<unsigned>(ctas), r.bits, st);
    from = list.size();
    ctas = 0;
    return e;
  };
  for (int i = 0; i < count; ++i) {
    const mlt_adamw_tensor& s = tensors[i];
    const long long blocks = (s.n + kBlock - 1) / kBlock;
    if (s.grad == nullptr) {
      block += blocks;
      continue;
    }
    // a launch has at most 2^31 - 1 CTAs: a longer tensor is taken in parts
    const long long most = 1LL << 30;
    for (long long at = 0; at < blocks; at += most * c.span) {
      const long long part = std::min(blocks - at, most * c.span), need = (part + c.span - 1) / c.span;
      if (list.size() - from == kMost || ctas + need > most) {
        const cudaError_t e = flush();
        if (e != cudaSuccess) return e;
      }
      auto moved = [&](const void* p, int dtype) {
        return p == nullptr ? nullptr
                            : const_cast<char*>(static_cast<const char*>(p)) + at * kBlock * static_cast<long long>(dtype_size(dtype));
      };
      Tensor d{};
      d.param = moved(s.param, s.dtype);
      d.grad = moved(s.grad, s.grad_dtype);
      d.copy = moved(s.copy, s.copy_dtype);
      d.n = std::min(static_cast<long long>(s.n) - at * kBlock, part * kBlock);
      d.block = block + at;
      d.first_cta = static_cast<unsigned>(ctas);
      d.dtype = static_cast<uint8_t>(s.dtype);
      d.grad_dtype = static_cast<uint8_t>(s.grad_dtype);
      d.copy_dtype = static_cast<uint8_t>(s.copy_dtype);
      const double decay = static_cast<double>(s.lr) * s.weight_decay;
      d.rate = static_cast<float>(s.lr / bias1);
      d.keep = static_cast<float>(r.lr != nullptr ? decay : 1.0 - decay);
      d.wide = aligned_to(d.param, 4 * dtype_size(s.dtype)) && aligned_to(d.grad, 4 * dtype_size(s.grad_dtype)) &&
               aligned_to(d.copy, 4 * dtype_size(s.copy_dtype));
      list.push_back(d);
      ctas += need;
    }
    block += blocks;
  }
  return flush();
}

}  // namespace mlt
