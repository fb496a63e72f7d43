// One AdamW step over many tensors (Loshchilov and Hutter, decoupled weight decay), with
// moments in 32 bits or in 8 with one power-of-two scale for each 256 of them.
//
// The tensors' addresses travel in the launch's parameters (up to kMost of them, in
// three sizes of table), so nothing is copied to the device and a captured
// graph holds them by value.  Each CTA takes a span of kSpan blocks of 256 elements; it finds its
// tensor by bisection over the table.  A warp takes a block at a time, each lane 2 x 4
// elements 128 apart, so every access of a warp is one contiguous run.
//
// Bound: memory.  32 bits: 28 bytes an element of fp32 parameters and gradients; 8 bits: 16, and some 70
// instructions.
//
// 8 bits: scales are powers of two, so scaling is exact and a value that a code stands for
// stays where it is while the block's largest one keeps its octave.  Codes are cut from the bits of the value
// as an fp32 number, scaled so that the format's smallest normal is fp32's: subnormal
// codes come out as fp32's subnormals.  Adding a random number below one step to the bits before the cut
// rounds up with the probability of the value's place between two codes.
#include <algorithm>
#include <cmath>
#include <utility>
#include <vector>

#include <cuda_fp8.h>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kBlock = 256;
constexpr int kSpan = 16;  // blocks a CTA: two for each of its eight warps
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
  uint8_t dtype, grad_dtype, copy_dtype, wide;
};
struct Common {
  float beta1, one_beta1, beta2, one_beta2, eps, root;  // root: 1 / sqrt(1 - beta2^step)
  float log_beta1, log_beta2;                           // for a step on the device
  const int64_t* step_device;
  const float* lr;
  const float* grad_scale;
  long long step;
  unsigned seed;
  int count;
  void *m, *v;
  float *m_scale, *v_scale;
};

template <int N>
struct Table {
  Common c;
  Tensor t[N];
};
static_assert(sizeof(Table<kMost>) <= 32764, "the table has to fit a launch's parameters");

// To two units in the last place, subnormal numbers too: p alone depends on it.
__device__ __forceinline__ float root_of(float v) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

__device__ __forceinline__ unsigned mix(unsigned h) {
  h ^= h >> 16;
  h *= 0x9E3779B1u;
  h ^= h >> 15;
  h *= 0xB504F333u;
  return h ^ (h >> 16);
}

// Four values of any type as they lie in memory, loaded before any of them is looked at.  Where the
// addresses allow no packs, or fewer than four are left, as fp32.
struct Four {
  unsigned r[4];
};

__device__ __forceinline__ Four load4(const void* p, int dtype, long long i, int left, bool wide) {
  Four q;
  if (wide && left == 4) {
    if (dtype == MLT_F32) {
      const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
      q = {{w.x, w.y, w.z, w.w}};
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
      q = {{w.x, w.y, 0u, 0u}};
    }
    return q;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) q.r[k] = k < left ? __float_as_uint(load_as_f32(p, dtype, i + k)) : 0u;
  return q;
}

__device__ __forceinline__ void values4(float (&v)[4], const Four& q, int dtype, int left, bool wide) {
  if (dtype == MLT_F32 || !wide || left < 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(q.r[k]);
  } else if (dtype == MLT_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(k & 1 ? q.r[k / 2] & 0xFFFF0000u : q.r[k / 2] << 16);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      v[k] = __half2float(__ushort_as_half(static_cast<unsigned short>(k & 1 ? q.r[k / 2] >> 16 : q.r[k / 2])));
  }
}

__device__ __forceinline__ void store4(const float (&v)[4], void* p, int dtype, long long i, int left, bool wide) {
  if (wide && left == 4) {
    if (dtype == MLT_F32) {
      *reinterpret_cast<Pack<float, 4>*>(static_cast<float*>(p) + i) = {{v[0], v[1], v[2], v[3]}};
    } else if (dtype == MLT_BF16) {
      Pack<__nv_bfloat16, 4> q;
#pragma unroll
      for (int k = 0; k < 4; ++k) q.v[k] = from_f32<__nv_bfloat16>(v[k]);
      *reinterpret_cast<Pack<__nv_bfloat16, 4>*>(static_cast<__nv_bfloat16*>(p) + i) = q;
    } else {
      Pack<__half, 4> q;
#pragma unroll
      for (int k = 0; k < 4; ++k) q.v[k] = from_f32<__half>(v[k]);
      *reinterpret_cast<Pack<__half, 4>*>(static_cast<__half*>(p) + i) = q;
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < left) store_from_f32(p, dtype, i + k, v[k]);
}

// Four codes of m (e4m3) or v (e5m2, the upper byte of a half) as numbers.
__device__ __forceinline__ void decode_e4m3(float (&v)[4], unsigned word, float scale) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(word >> (16 * k)), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    v[2 * k] = f.x * scale;
    v[2 * k + 1] = f.y * scale;
  }
}
__device__ __forceinline__ void decode_e5m2(float (&v)[4], unsigned word, float scale) {
#pragma unroll
  for (int k = 0; k < 4; ++k)
    v[k] = __half2float(__ushort_as_half(static_cast<unsigned short>((word >> (8 * k)) << 8))) * scale;
}

// The word of four values' codes; e: the block's exponent (16 .. 255), u: numbers below 2^16.
template <int MANTISSA>
__device__ __forceinline__ unsigned encode4(const float (&v)[4], unsigned e, const unsigned (&u)[4]) {
  constexpr int kBias = MANTISSA == 3 ? 134 : 141, kDrop = 23 - MANTISSA;
  const float up = __uint_as_float((127 + kBias - e) << 23);
  unsigned word = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float s = fabsf(v[k]) * up * (MANTISSA == 3 ? 0x1p-120f : 0x1p-112f);
    unsigned code = (__float_as_uint(s) + (u[k] << (kDrop - 16))) >> kDrop;
    if (MANTISSA == 3)
      code |= (__float_as_uint(v[k]) >> 24) & 0x80u;
    else if (v[k] > 0.0f && code == 0)
      code = 1;
    word |= code << (8 * k);
  }
  return e == 255 ? 0x7F7F7F7Fu : word;
}

template <int N, int BITS>
__global__ void __launch_bounds__(256) k_adamw(const __grid_constant__ Table<N> q) {
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
  const long long from = static_cast<long long>(blockIdx.x - t.first_cta) * kSpan;
  const long long blocks = (t.n + kBlock - 1) / kBlock;
#pragma unroll 1
  for (int k = warp; k < kSpan; k += 8) {
    if (from + k >= blocks) break;
    const long long i0 = (from + k) * kBlock + lane * 4, b = t.block + from + k, s0 = b * kBlock + lane * 4;
    float p[2][4], g[2][4], m[2][4], v[2][4];
    int left[2];
    Four rp[2], rg[2], rm[2], rv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const long long rest = t.n - (i0 + 128 * h);
      left[h] = rest < 0 ? 0 : rest > 4 ? 4 : static_cast<int>(rest);
      rp[h] = load4(t.param, t.dtype, i0 + 128 * h, left[h], t.wide);
      rg[h] = load4(t.grad, t.grad_dtype, i0 + 128 * h, left[h], t.wide);
      if (BITS == 32) {
        rm[h] = load4(c.m, MLT_F32, s0 + 128 * h, 4, true);
        rv[h] = load4(c.v, MLT_F32, s0 + 128 * h, 4, true);
      } else {
        rm[h].r[0] = *reinterpret_cast<const unsigned*>(static_cast<const uint8_t*>(c.m) + s0 + 128 * h);
        rv[h].r[0] = *reinterpret_cast<const unsigned*>(static_cast<const uint8_t*>(c.v) + s0 + 128 * h);
      }
    }
    const float ms = BITS == 8 ? c.m_scale[b] : 0.0f, vs = BITS == 8 ? c.v_scale[b] : 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      values4(p[h], rp[h], t.dtype, left[h], t.wide);
      values4(g[h], rg[h], t.grad_dtype, left[h], t.wide);
      if (BITS == 32) {
        values4(m[h], rm[h], MLT_F32, 4, true);
        values4(v[h], rv[h], MLT_F32, 4, true);
      } else {
        decode_e4m3(m[h], rm[h].r[0], ms);
        decode_e5m2(v[h], rv[h].r[0], vs);
      }
    }
    unsigned most_m = 0, most_v = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __fmul_rn(g[h][e], scale);
        m[h][e] = __fadd_rn(__fmul_rn(m[h][e], c.beta1), __fmul_rn(x, c.one_beta1));
        v[h][e] = __fadd_rn(__fmul_rn(v[h][e], c.beta2), __fmul_rn(__fmul_rn(x, x), c.one_beta2));
        if (e < left[h]) {
          most_m = max(most_m, __float_as_uint(m[h][e]) & 0x7FFFFFFFu);
          most_v = max(most_v, __float_as_uint(v[h][e]) & 0x7FFFFFFFu);
        }
        const float d = __fdividef(m[h][e], fmaf(root_of(v[h][e]), root, c.eps));
        p[h][e] = fmaf(-rate, d, __fmul_rn(p[h][e], keep));
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      store4(p[h], t.param, t.dtype, i0 + 128 * h, left[h], t.wide);
      if (t.copy != nullptr) store4(p[h], t.copy, t.copy_dtype, i0 + 128 * h, left[h], t.wide);
    }
    if (BITS == 32) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        store4(m[h], c.m, MLT_F32, s0 + 128 * h, left[h], true);
        store4(v[h], c.v, MLT_F32, s0 + 128 * h, left[h], true);
      }
    } else {
      const unsigned em = max(__reduce_max_sync(0xffffffffu, most_m) >> 23, 16u);
      const unsigned ev = max(__reduce_max_sync(0xffffffffu, most_v) >> 23, 16u);
      const unsigned kb = mix(static_cast<unsigned>(b) + key);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        unsigned um[4], uv[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned r = mix(kb + (lane * 4 + 128 * h + e) * 0x9E3779B9u);
          um[e] = r & 0xFFFFu;
          uv[e] = r >> 16;
        }
        const unsigned wm = encode4<3>(m[h], em, um), wv = encode4<2>(v[h], ev, uv);
        uint8_t* to_m = static_cast<uint8_t*>(c.m) + s0 + 128 * h;
        uint8_t* to_v = static_cast<uint8_t*>(c.v) + s0 + 128 * h;
        if (left[h] == 4) {
          *reinterpret_cast<unsigned*>(to_m) = wm;
          *reinterpret_cast<unsigned*>(to_v) = wv;
        } else {
          for (int e = 0; e < left[h]; ++e) {
            to_m[e] = static_cast<uint8_t>(wm >> (8 * e));
            to_v[e] = static_cast<uint8_t>(wv >> (8 * e));
          }
        }
      }
      if (lane == 0) {
        c.m_scale[b] = __uint_as_float((em - 7) << 23);
        c.v_scale[b] = __uint_as_float((ev - 14) << 23);
      }
    }
  }
}

template <int N, int BITS>
cudaError_t launch_table(const Common& c, const std::vector<Tensor>& list, size_t from, int count, unsigned ctas,
                         cudaStream_t st) {
  static thread_local Table<N> q;  // 32 KB at most: not on the stack
  q.c = c;
  q.c.count = count;
  std::copy(list.begin() + from, list.begin() + from + count, q.t);
  return launch_pdl(k_adamw<N, BITS>, dim3(ctas), dim3(256), 0, st, q);
}

template <int BITS>
cudaError_t launch_part(const Common& c, const std::vector<Tensor>& list, size_t from, int count, unsigned ctas,
                        cudaStream_t st) {
  if (count <= 32) return launch_table<32, BITS>(c, list, from, count, ctas, st);
  if (count <= 128) return launch_table<128, BITS>(c, list, from, count, ctas, st);
  return launch_table<kMost, BITS>(c, list, from, count, ctas, st);
}

}  // namespace

cudaError_t launch_adamw(const mlt_adamw_tensor* tensors, int count, const mlt_adamw_rule& r, void* m, void* v,
                         float* m_scale, float* v_scale, long long* launches, cudaStream_t st) {
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
  std::vector<Tensor> list;
  list.reserve(count);
  long long block = 0, ctas = 0;
  size_t from = 0;
  auto flush = [&]() -> cudaError_t {
    const int n = static_cast<int>(list.size() - from);
    if (n == 0) return cudaSuccess;
    ++*launches;
    const cudaError_t e = r.bits == 8 ? launch_part<8>(c, list, from, n, static_cast<unsigned>(ctas), st)
                                      : launch_part<32>(c, list, from, n, static_cast<unsigned>(ctas), st);
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
    for (long long at = 0; at < blocks; at += most * kSpan) {
      const long long part = std::min(blocks - at, most * kSpan), need = (part + kSpan - 1) / kSpan;
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
