// One AdamW step over many tensors (Loshchilov and Hutter, decoupled weight decay), with
// moments in 32 bits or in 8 with one power-of-two scale for each 256 of them.
//
// The tensors' addresses travel in the launch's parameters (up to kMost of them, in
// three sizes of table), so nothing is copied to the device and a captured
// graph holds them by value.  Each CTA takes a span of 8 to 32 blocks of 256 elements; it finds its
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

// Four values of any type as they lie in memory, loaded before any of them is looked at.
struct Four {
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

// A lane's eight values of a whole block.
__device__ __forceinline__ void store8(char* p, const float (&v)[2][4], int dtype) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (dtype == MLT_F32) {
      *reinterpret_cast<float4*>(p + 512 * h) = make_float4(v[h][0], v[h][1], v[h][2], v[h][3]);
    } else if (dtype == MLT_BF16) {
      const __nv_bfloat162 a = __floats2bfloat162_rn(v[h][0], v[h][1]), b = __floats2bfloat162_rn(v[h][2], v[h][3]);
      *reinterpret_cast<uint2*>(p + 256 * h) =
          make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
    } else {
      const __half2 a = __floats2half2_rn(v[h][0], v[h][1]), b = __floats2half2_rn(v[h][2], v[h][3]);
      *reinterpret_cast<uint2*>(p + 256 * h) =
          make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
    }
  }
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
  for (int k = 0; k < 2; ++k) {
    const unsigned h = __byte_perm(word, 0, k == 0 ? 0x1404 : 0x3424);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    v[2 * k] = f.x * scale;
    v[2 * k + 1] = f.y * scale;
  }
}

// The words of four values' codes; em, ev: the block's exponents (16 .. 255), r: the values' hashes.  A code
// is shifted into the upper byte of a word, the sign with it, and the four upper bytes are gathered.
__device__ __forceinline__ unsigned gather(const unsigned (&x)[4]) {
  return __byte_perm(__byte_perm(x[0], x[1], 0x0073), __byte_perm(x[2], x[3], 0x0073), 0x5410);
}
__device__ __forceinline__ unsigned encode_e4m3(const float (&m)[4], unsigned e, const unsigned (&r)[4]) {
  const float up = __uint_as_float((127 + 134 - e) << 23);
  unsigned x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float s = fabsf(m[k]) * up * 0x1p-120f;
    const unsigned c = (__float_as_uint(s) + ((r[k] << 4) & 0xFFFF0u)) << 4;
    x[k] = (c & 0x7F000000u) | (__float_as_uint(m[k]) & 0x80000000u);
  }
  return e == 255 ? 0x7F7F7F7Fu : gather(x);
}
__device__ __forceinline__ unsigned encode_e5m2(const float (&v)[4], unsigned e, const unsigned (&r)[4]) {
  const float up = __uint_as_float((127 + 141 - e) << 23);
  unsigned x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float s = v[k] * up * 0x1p-112f;
    const unsigned c = __float_as_uint(s) + ((r[k] >> 16) << 5);
    x[k] = (v[k] > 0.0f ? max(c, 1u << 21) : c) << 3;
  }
  return e == 255 ? 0x7F7F7F7Fu : gather(x);
}

template <int N, int BITS>
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
  const bool f32 = t.dtype == MLT_F32, g32 = t.grad_dtype == MLT_F32, c32 = t.copy_dtype == MLT_F32;
  // a tensor's whole blocks with aligned addresses, then what is left
  const long long whole = t.wide ? t.n / kBlock : 0;
#pragma unroll 1
  for (int k = 0; k < turns; ++k) {
    const long long at = from + 8 * k, b = t.block + at;
    const long long i0 = at * kBlock + lane * 4, s0 = b * kBlock + lane * 4;
    const bool full = at < whole;
    float p[2][4], g[2][4], m[2][4], v[2][4];
    int left[2] = {4, 4};
    Four rp[2], rg[2], rm[2], rv[2];
    if (full) {
      const char* pp = static_cast<const char*>(t.param) + (i0 << (f32 ? 2 : 1));
      const char* gg = static_cast<const char*>(t.grad) + (i0 << (g32 ? 2 : 1));
      if (f32) {
        rp[0] = wide4(pp);
        rp[1] = wide4(pp + 512);
      } else {
        rp[0] = narrow4(pp);
        rp[1] = narrow4(pp + 256);
      }
      if (g32) {
        rg[0] = wide4(gg);
        rg[1] = wide4(gg + 512);
      } else {
        rg[0] = narrow4(gg);
        rg[1] = narrow4(gg + 256);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const long long rest = t.n - (i0 + 128 * h);
        left[h] = rest < 0 ? 0 : rest > 4 ? 4 : static_cast<int>(rest);
        rp[h] = some4(t.param, t.dtype, i0 + 128 * h, left[h]);
        rg[h] = some4(t.grad, t.grad_dtype, i0 + 128 * h, left[h]);
      }
    }
    const char *mm = static_cast<const char*>(c.m) + s0 * (BITS / 8), *vv = static_cast<const char*>(c.v) + s0 * (BITS / 8);
    float ms = 0.0f, vs = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (BITS == 32) {
        rm[h] = wide4(mm + 512 * h);
        rv[h] = wide4(vv + 512 * h);
      } else {
        rm[h].r[0] = *reinterpret_cast<const unsigned*>(mm + 128 * h);
        rv[h].r[0] = *reinterpret_cast<const unsigned*>(vv + 128 * h);
      }
    }
    if (BITS == 8) {
      ms = c.m_scale[b];
      vs = c.v_scale[b];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      values4(p[h], rp[h], full ? t.dtype : MLT_F32);
      values4(g[h], rg[h], full ? t.grad_dtype : MLT_F32);
      if (BITS == 32) {
        values4(m[h], rm[h], MLT_F32);
        values4(v[h], rv[h], MLT_F32);
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
        const float d = __fdividef(m[h][e], fmaf(root_of(v[h][e]), root, c.eps));
        p[h][e] = fmaf(-rate, d, __fmul_rn(p[h][e], keep));
      }
    if (full) {
      char* pp = static_cast<char*>(t.param) + (i0 << (f32 ? 2 : 1));
      store8(pp, p, t.dtype);
      if (t.copy != nullptr) store8(static_cast<char*>(t.copy) + (i0 << (c32 ? 2 : 1)), p, t.copy_dtype);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (e >= left[h]) continue;
          store_from_f32(t.param, t.dtype, i0 + 128 * h + e, p[h][e]);
          if (t.copy != nullptr) store_from_f32(t.copy, t.copy_dtype, i0 + 128 * h + e, p[h][e]);
        }
    }
    if (BITS == 32) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        char *to_m = const_cast<char*>(mm) + 512 * h, *to_v = const_cast<char*>(vv) + 512 * h;
        if (left[h] == 4) {
          *reinterpret_cast<float4*>(to_m) = make_float4(m[h][0], m[h][1], m[h][2], m[h][3]);
          *reinterpret_cast<float4*>(to_v) = make_float4(v[h][0], v[h][1], v[h][2], v[h][3]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < left[h]) {
              reinterpret_cast<float*>(to_m)[e] = m[h][e];
              reinterpret_cast<float*>(to_v)[e] = v[h][e];
            }
        }
      }
      continue;
    }
    if (full) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          most_m = max(most_m, __float_as_uint(m[h][e]) & 0x7FFFFFFFu);
          most_v = max(most_v, __float_as_uint(v[h][e]) & 0x7FFFFFFFu);
        }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < left[h]) {
            most_m = max(most_m, __float_as_uint(m[h][e]) & 0x7FFFFFFFu);
            most_v = max(most_v, __float_as_uint(v[h][e]) & 0x7FFFFFFFu);
          }
    }
    const unsigned em = max(__reduce_max_sync(0xffffffffu, most_m) >> 23, 16u);
    const unsigned ev = max(__reduce_max_sync(0xffffffffu, most_v) >> 23, 16u);
    const unsigned kb = mix(static_cast<unsigned>(b) + key) + lane * 4 * 0x9E3779B9u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      unsigned r[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = mix(kb + (128u * h + e) * 0x9E3779B9u);
      const unsigned wm = encode_e4m3(m[h], em, r), wv = encode_e5m2(v[h], ev, r);
      uint8_t* to_m = reinterpret_cast<uint8_t*>(const_cast<char*>(mm)) + 128 * h;
      uint8_t* to_v = reinterpret_cast<uint8_t*>(const_cast<char*>(vv)) + 128 * h;
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
