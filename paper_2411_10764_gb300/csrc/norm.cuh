// Shared by layer norm's forward pass (norm.cu) and its gradients (norm_grad.cu):
// how rows are dealt to threads, sums over a row, launches.  Not part of the C ABI.
//
// A row is held in registers, kEach values a thread, so it is read once:
//   dim <= 256      a power-of-two group of lanes a row, several rows a warp, sums by shuffles;
//   dim <= a CTA's  a CTA a row, sums by shuffles and one barrier each;
//   longer          a cluster of up to eight CTAs a row, which exchange their sums through
//                   distributed shared memory;
//   longer still    a CTA a row that reads it from memory once for each pass.
// Threads take packs of 16 bytes where all addresses, strides and dim allow it, else
// single values, neighbouring threads neighbouring ones either way.
#pragma once

#include "seq.cuh"

namespace mlt {

constexpr int kNormGroupDim = 256;   // rows that a group of lanes takes
constexpr int kNormMaxCluster = 8;

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

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned cluster_ranks() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}

// Sums of N values over the threads of a row, the same in each of them.  Slots are used in turn, so one
// barrier a sum is enough: who writes a slot again has passed the barrier of the
// sum in between, which no thread reaches before it has read the slot.
template <int N>
struct RowSums {
  float warps[2][N][32];
  float peers[2][N][kNormMaxCluster];
};

template <int N>
__device__ __forceinline__ void group_sums(float (&v)[N], int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], RowSums<N>& s, int& slot, int ranks, int rank) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  group_sums(v, 32);
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) s.warps[slot][i][warp] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lane < warps ? s.warps[slot][i][lane] : 0.0f;
  group_sums(v, 32);
  if (ranks > 1) {
    if (threadIdx.x < ranks) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned mine = static_cast<unsigned>(__cvta_generic_to_shared(&s.peers[slot][i][rank]));
        unsigned there;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(threadIdx.x));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v[i]) : "memory");
      }
    }
    cluster_barrier();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float all = 0.0f;
      for (int r = 0; r < ranks; ++r) all += s.peers[slot][i][r];
      v[i] = all;
    }
  }
  slot ^= 1;
}

// How many CTAs of `threads` threads an SM holds by registers and threads (shared memory is small).
template <auto kernel>
int resident_ctas(int threads) {
  static const int regs = [&] {
    cudaFuncAttributes at{};
    return cudaFuncGetAttributes(&at, kernel) == cudaSuccess ? at.numRegs : 255;
  }();
  const int warps = threads / 32, a_warp = (regs * 32 + 255) / 256 * 256;
  const int by_regs = 65536 / (a_warp * warps), by_threads = 64 / warps;
  const int n = by_regs < by_threads ? by_regs : by_threads;
  return n < 1 ? 1 : n > 32 ? 32 : n;
}

// A launch that may begin while the kernel before it ends (pdl_wait in the kernel), in clusters.
template <typename... K, typename... A>
cudaError_t launch_cluster(void (*kernel)(K...), unsigned grid, unsigned block, unsigned cluster, cudaStream_t st,
                           A&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}
#endif

}  // namespace mlt
