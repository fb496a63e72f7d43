// Shared by layer norm's forward pass (norm.cu) and its gradients (norm_grad.cu):
// how rows are dealt to threads, sums over a row, launches.  Not part of the C ABI.
//
// A row is held in registers, E values a thread, so it is read once:
//   short rows      a power-of-two group of lanes a row, several rows a warp, sums by shuffles;
//   longer ones     a CTA a row, sums by shuffles and one barrier each;
//   the rest        a CTA a row that keeps it in shared memory or reads it again out of L2.  (Clusters of CTAs with
//                   a row in their registers wait for all their stores at each of two barriers a row:
//                   4,096 x 16,384 bf16 154 us by two CTAs a row, 216 by four.)
// What costs beside memory is the work for each row and thread (shuffles, barrier, addresses: some 200
// instructions), so threads take as many values as registers allow: 16,384 x 4,096 bf16 with eight a thread
// 136 us and 46 instructions a value, with sixteen 86 and, two-wide where they can be, 24.
//
// Threads take packs of 16 bytes wherever all tensors' rows lie alike towards 16-byte boundaries, as
// contiguous tensors of any dim do: packs are counted from the boundary before the row (`skew` values before
// its first), the two at its ends are read whole and written value by value.  A team takes
// rows whose skew is the same, so its columns stay its own.  Else packs are single values.
// Packs or not, and how many values a thread, follow from addresses, strides and dim alone.
#pragma once

#include <type_traits>

#include "seq.cuh"

namespace mlt {

constexpr int kNormMostWarps = 16;

// How the rows of some tensors lie towards 16-byte boundaries, in values: (skew + row * step) mod the values
// of a pack.
struct Skew {
  bool same = true;  // all alike so far
  int first = -1, step = 0;
  void add(const void* p, int64_t stride, size_t bytes, int pack) {
    if (p == nullptr) return;
    const int f = static_cast<int>((reinterpret_cast<uintptr_t>(p) / bytes) % pack), s = static_cast<int>(stride % pack);
    if (first < 0) {
      first = f;
      step = s;
    }
    same = same && f == first && s == step;
  }
  bool edges(int dim, int pack) const { return first != 0 || step != 0 || dim % pack != 0; }
  // rows after which it repeats
  int period(int pack) const {
    int n = 1;
    while (n * step % pack != 0) n *= 2;
    return n;
  }
};

// Calls f(input type, output type): the same, or a narrower one for fp32 inputs.
template <typename F>
auto with_norm_types(int in, int out, F f) {
  if (in == MLT_BF16) return f(__nv_bfloat16(), __nv_bfloat16());
  if (in == MLT_F16) return f(__half(), __half());
  if (out == MLT_BF16) return f(float(), __nv_bfloat16());
  if (out == MLT_F16) return f(float(), __half());
  return f(float(), float());
}

#ifdef __CUDACC__
__device__ __forceinline__ float load_as_f32(const void* p, int dtype, long long i) {
  if (dtype == MLT_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
  if (dtype == MLT_F16) return to_f32(static_cast<const __half*>(p)[i]);
  return static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_from_f32(void* p, int dtype, long long i, float v) {
  if (dtype == MLT_BF16)
    static_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(v);
  else if (dtype == MLT_F16)
    static_cast<__half*>(p)[i] = from_f32<__half>(v);
  else
    static_cast<float*>(p)[i] = v;
}

// Sums of N values over the threads of a row, the same in each of them.  Slots are used in turn, so one
// barrier a sum is enough: who writes a slot again has passed the barrier of the
// sum in between, which no thread reaches before it has read the slot.
template <int N>
struct RowSums {
  float4 warps[2][N][kNormMostWarps / 4];
  __device__ __forceinline__ void clear() {  // before the first sum, with a barrier in between
    float* w = reinterpret_cast<float*>(warps);
    for (int i = threadIdx.x; i < 2 * N * kNormMostWarps; i += blockDim.x) w[i] = 0.0f;
  }
};

template <int N>
__device__ __forceinline__ void group_sums(float (&v)[N], int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}
template <int N>
__device__ __forceinline__ void warp_sums(float (&v)[N]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], RowSums<N>& s, int& slot) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, fours = (blockDim.x + 127) / 128;
  warp_sums(v);
  if (blockDim.x > 32) {
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) reinterpret_cast<float*>(s.warps[slot][i])[warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.0f;
      for (int w = 0; w < fours; ++w) {
        const float4 q = s.warps[slot][i][w];
        v[i] += (q.x + q.y) + (q.z + q.w);
      }
    }
  }
  slot ^= 1;
}

// V values as they lie in memory, in whole registers: 16-bit ones kept as single values take a register
// each wherever a load is conditional (twice the registers of the row).
template <typename T, int V>
struct Vec {
  static constexpr int kWords = (V * static_cast<int>(sizeof(T)) + 3) / 4;
  unsigned w[kWords];

  __device__ __forceinline__ float get(int v) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[v]);
    const unsigned x = w[v / 2];
    if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(v & 1 ? x & 0xFFFF0000u : x << 16);
    return __half2float(__ushort_as_half(static_cast<unsigned short>(v & 1 ? x >> 16 : x & 0xFFFFu)));
  }
  __device__ __forceinline__ void put(const float (&f)[V]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int v = 0; v < V; ++v) w[v] = __float_as_uint(f[v]);
    } else {
#pragma unroll
      for (int v = 0; v < V; v += 2) {
        const float hi = v + 1 < V ? f[v + 1] : 0.0f;
        if constexpr (std::is_same<T, __nv_bfloat16>::value) {
          const __nv_bfloat162 q = __floats2bfloat162_rn(f[v], hi);
          w[v / 2] = *reinterpret_cast<const unsigned*>(&q);
        } else {
          const __half2 q = __floats2half2_rn(f[v], hi);
          w[v / 2] = *reinterpret_cast<const unsigned*>(&q);
        }
      }
    }
  }
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (V * sizeof(T) == 16) {
      const uint4 q = *reinterpret_cast<const uint4*>(p);
      w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    } else if constexpr (V * sizeof(T) == 8) {
      const uint2 q = *reinterpret_cast<const uint2*>(p);
      w[0] = q.x, w[1] = q.y;
    } else if constexpr (V * sizeof(T) == 4) {
      w[0] = *reinterpret_cast<const unsigned*>(p);
    } else {
      w[0] = *reinterpret_cast<const unsigned short*>(p);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (V * sizeof(T) == 16)
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (V * sizeof(T) == 8)
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (V * sizeof(T) == 4)
      *reinterpret_cast<unsigned*>(p) = w[0];
    else
      *reinterpret_cast<unsigned short*>(p) = static_cast<unsigned short>(w[0]);
  }
  // one value
  __device__ __forceinline__ void load_one(const T* p, int v) {
    if constexpr (sizeof(T) == 4) {
      w[v] = *reinterpret_cast<const unsigned*>(p);
    } else {
      const unsigned x = *reinterpret_cast<const unsigned short*>(p);
      w[v / 2] = v & 1 ? (w[v / 2] & 0xFFFFu) | (x << 16) : x;
    }
  }
  __device__ __forceinline__ void store_one(T* p, int v) const {
    if constexpr (sizeof(T) == 4)
      *reinterpret_cast<unsigned*>(p) = w[v];
    else
      *reinterpret_cast<unsigned short*>(p) = static_cast<unsigned short>(v & 1 ? w[v / 2] >> 16 : w[v / 2]);
  }
};

// Places i and i + 1 of packs, of numbers by pack, and one of numbers by two.
template <typename T, int V, int C>
__device__ __forceinline__ float2 two_of(const Vec<T, V> (&p)[C], int i) {
  return make_float2(p[i / V].get(i % V), p[(i + 1) / V].get((i + 1) % V));
}
template <int V, int C>
__device__ __forceinline__ float2 two_of(const float (&w)[C][V], int i) {
  return make_float2(w[i / V][i % V], w[(i + 1) / V][(i + 1) % V]);
}
template <int N>
__device__ __forceinline__ float& one_of(float2 (&x)[N], int i) {
  return i & 1 ? x[i / 2].y : x[i / 2].x;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 masked(float2 v, bool on0, bool on1) {
  return make_float2(on0 ? v.x : 0.0f, on1 ? v.y : 0.0f);
}

// The columns of a thread: C packs of V, `hop` values apart.
template <int V, int C, bool EDGE>
struct Columns {
  int first;     // column of the first pack's first value
  int hop;
  int mask[C];   // by value of a pack; not EDGE: 0 or all

  // pos: the thread's first place, counted from the boundary before the row
  __device__ __forceinline__ Columns(int pos, int hop_, int skew, int dim) : first(pos - skew), hop(hop_) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = first + c * hop;
      mask[c] = 0;
      if (!EDGE) {
        if (col < dim) mask[c] = (1 << V) - 1;
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (col + v >= 0 && col + v < dim) mask[c] |= 1 << v;
      }
    }
  }
  __device__ __forceinline__ bool on(int c, int v) const { return EDGE ? (mask[c] >> v) & 1 : mask[c] != 0; }
  __device__ __forceinline__ bool whole(int c) const { return mask[c] == (1 << V) - 1; }

  // begin, end: of the tensor's values.  A pack that reaches past its row is read whole all the same, its
  // other values belong to the rows beside it; only at the tensor's two ends they are read one by one.
  template <typename T>
  __device__ __forceinline__ void load(Vec<T, V> (&p)[C], const T* row, const T* begin, const T* end) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const T* at = row + first + c * hop;
      if (mask[c] == 0) continue;
      if (!EDGE || whole(c) || (at >= begin && at + V <= end)) {
        p[c].load(at);
      } else {
#pragma unroll
        for (int i = 0; i < Vec<T, V>::kWords; ++i) p[c].w[i] = 0;
#pragma unroll 1
        for (int v = 0; v < V; ++v)
          if (on(c, v)) {
            Vec<T, V> one;
#pragma unroll
            for (int i = 0; i < Vec<T, V>::kWords; ++i) one.w[i] = 0;
#pragma unroll
            for (int k = 0; k < V; ++k)
              if (k == v) one.load_one(at + k, k);
#pragma unroll
            for (int i = 0; i < Vec<T, V>::kWords; ++i) p[c].w[i] |= one.w[i];
          }
      }
    }
  }
  // f(i, whether the places i and i + 1 of the thread's C * V are values of the row) for each two places, which
  // go through two-wide operations together.  BRANCH: whole packs apart, where few have edges.
  template <bool BRANCH, typename F>
  __device__ __forceinline__ void pairs(F f) const {
    if constexpr (V == 1) {
#pragma unroll
      for (int c = 0; c < C; c += 2) f(c, mask[c] != 0, mask[c + 1] != 0);
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if ((BRANCH || !EDGE) && whole(c)) {
#pragma unroll
          for (int v = 0; v < V; v += 2) f(c * V + v, true, true);
        } else {
#pragma unroll
          for (int v = 0; v < V; v += 2) f(c * V + v, EDGE && on(c, v), EDGE && on(c, v + 1));
        }
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(const Vec<T, V>& p, T* row, int c) const {
    T* at = row + first + c * hop;
    if (whole(c)) {
      p.store(at);
    } else if (EDGE && mask[c] != 0) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (on(c, v)) p.store_one(at + v, v);
    }
  }
};

// Packs on their way to shared memory, each thread's to places of its own, so that a thread's own wait is all
// it takes.  kAhead rows of up to three tensors.
constexpr int kAhead = 3;
template <int V, int C>
struct Ring {
  static constexpr int kBytes = kAhead * (3 * C * 16 + 8);  // a thread
  unsigned char* at;  // of the CTA

  __device__ __forceinline__ unsigned char* pack(int stage, int tensor, int c) const {
    return at + ((((stage * 3 + tensor) * C + c) * static_cast<int>(blockDim.x)) + threadIdx.x) * 16;
  }
  __device__ __forceinline__ float2* pair(int stage) const {
    return reinterpret_cast<float2*>(at + kAhead * 3 * C * 16 * blockDim.x) + stage * blockDim.x + threadIdx.x;
  }
  template <int BYTES>
  static __device__ __forceinline__ void copy(void* to, const void* from) {
    const unsigned s = static_cast<unsigned>(__cvta_generic_to_shared(to));
    if constexpr (BYTES == 16)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(from) : "memory");
    else
      asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(s), "l"(from), "n"(BYTES) : "memory");
  }
  // begin, end: as for Columns::load
  template <typename T, bool EDGE>
  __device__ __forceinline__ void fetch(const Columns<V, C, EDGE>& cols, int stage, int tensor, const T* row,
                                        const T* begin, const T* end) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const T* from = row + cols.first + c * cols.hop;
      if (cols.mask[c] == 0) continue;
      if (!EDGE || cols.whole(c) || (from >= begin && from + V <= end))
        copy<V * sizeof(T)>(pack(stage, tensor, c), from);
      else
#pragma unroll 1
        for (int v = 0; v < V; ++v)
          if (cols.on(c, v)) reinterpret_cast<T*>(pack(stage, tensor, c))[v] = from[v];
    }
  }
  template <typename T>
  __device__ __forceinline__ Vec<T, V> get(int stage, int tensor, int c) const {
    Vec<T, V> q;
    q.load(reinterpret_cast<const T*>(pack(stage, tensor, c)));
    return q;
  }
  static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  static __device__ __forceinline__ void wait_oldest() { asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory"); }
};

// One value per column of a thread as fp32; all loads under way at once.
template <int V, int C, bool EDGE>
__device__ __forceinline__ void load_columns(float (&w)[C][V], const Columns<V, C, EDGE>& cols, const void* p, int dtype,
                                             float none) {
  auto with = [&](auto t) {
    using T = decltype(t);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        w[c][v] = none;
        if (p != nullptr && cols.on(c, v)) w[c][v] = to_f32(static_cast<const T*>(p)[cols.first + c * cols.hop + v]);
      }
  };
  if (dtype == MLT_BF16)
    with(__nv_bfloat16());
  else if (dtype == MLT_F16)
    with(__half());
  else
    with(float());
}

// The same kept in shared memory by a CTA whose registers they would fill: places of four, so that a warp's
// accesses fall on all banks.  Each thread reads what it wrote.
template <int V, int C>
struct Kept {
  static constexpr int kPart = V < 4 ? V : 4;
  float* at;
  __device__ __forceinline__ float* place(int c, int k) const {
    return at + ((c * (V / kPart) + k) * static_cast<int>(blockDim.x) + threadIdx.x) * kPart;
  }
  __device__ __forceinline__ void put(const float (&w)[C][V]) const {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < V / kPart; ++k) {
        Pack<float, kPart> q;
#pragma unroll
        for (int v = 0; v < kPart; ++v) q.v[v] = w[c][k * kPart + v];
        *reinterpret_cast<Pack<float, kPart>*>(place(c, k)) = q;
      }
  }
  __device__ __forceinline__ void get(float (&w)[V], int c) const {
#pragma unroll
    for (int k = 0; k < V / kPart; ++k) {
      const Pack<float, kPart> q = *reinterpret_cast<const Pack<float, kPart>*>(place(c, k));
#pragma unroll
      for (int v = 0; v < kPart; ++v) w[k * kPart + v] = q.v[v];
    }
  }
};

// A pack at a column that may lie before the row or reach past its end: 0 there.
template <int V, typename T>
__device__ __forceinline__ void load_some(float (&f)[V], const T* row, int col, int dim) {
  if (col >= 0 && col + V <= dim) {
    Vec<T, V> q;
    q.load(row + col);
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = q.get(v);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = col + v >= 0 && col + v < dim ? to_f32(row[col + v]) : 0.0f;
  }
}
template <int V, typename T>
__device__ __forceinline__ void store_some(const float (&f)[V], T* row, int col, int dim) {
  if (col >= 0 && col + V <= dim) {
    Vec<T, V> q;
    q.put(f);
    q.store(row + col);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (col + v >= 0 && col + v < dim) row[col + v] = from_f32<T>(f[v]);
  }
}
template <int V>
__device__ __forceinline__ void load_weights(float (&w)[V], const void* p, int dtype, int col, int dim, float none) {
  if (p == nullptr) {
#pragma unroll
    for (int v = 0; v < V; ++v) w[v] = none;
    return;
  }
  auto with = [&](auto t) {
    using T = decltype(t);
    const T* from = static_cast<const T*>(p);
    if (col >= 0 && col + V <= dim && reinterpret_cast<uintptr_t>(from + col) % 16 == 0 && V * sizeof(T) % 16 == 0) {
      constexpr int P = 16 / sizeof(T) < V ? 16 / sizeof(T) : V;
#pragma unroll
      for (int k = 0; k < V / P; ++k) {
        Vec<T, P> q;
        q.load(from + col + k * P);
#pragma unroll
        for (int v = 0; v < P; ++v) w[k * P + v] = q.get(v);
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) w[v] = col + v >= 0 && col + v < dim ? to_f32(from[col + v]) : none;
    }
  };
  if (dtype == MLT_BF16)
    with(__nv_bfloat16());
  else if (dtype == MLT_F16)
    with(__half());
  else
    with(float());
}

// How many CTAs of `threads` threads and `smem` bytes an SM holds.
template <auto kernel>
int resident_ctas(int threads, size_t smem) {
  static const int regs = [&] {
    cudaFuncAttributes at{};
    return cudaFuncGetAttributes(&at, kernel) == cudaSuccess ? at.numRegs : 255;
  }();
  const int warps = threads / 32, a_warp = (regs * 32 + 255) / 256 * 256;
  int n = 65536 / (a_warp * warps);
  if (n > 64 / warps) n = 64 / warps;
  const int by_smem = static_cast<int>(228 * 1024 / (smem + 3 * 1024));  // 1 KB of each CTA is the system's
  if (n > by_smem) n = by_smem;
  return n < 1 ? 1 : n > 32 ? 32 : n;
}

// A launch that may begin while the kernel before it ends (pdl_wait in the kernel).
template <typename... K, typename... A>
cudaError_t launch_rows(void (*kernel)(K...), unsigned grid, unsigned block, size_t smem, cudaStream_t st, A&&... args) {
  if (smem > 40 * 1024) {  // with the static part past what a kernel has unasked, 48 KB
    const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(kernel, dim3(grid), dim3(block), smem, st, std::forward<A>(args)...);
}
#endif

}  // namespace mlt
