// Gradients of layer norm: of its input row by row, of weight and bias as sums over all rows.
//
// With h = (t - mean) rstd and gw = gy weight, two sums over the row (gw and gw h) give the
// input's gradient.  Each thread keeps its columns' sums of gy h and gy in registers over
// all rows of its team; the teams' sums go to the workspace and a second
// kernel adds them up in a fixed order.  Bound: memory (x and gy read, gx written, once).
// Where a thread adds more than kPlainRows rows its sums are compensated (Kahan 1965): of n
// equal terms in a plain sum the error grows with n.
#include <utility>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kEach = 8;  // values of a row a thread (16: 300 to 1,400 bytes of spills)
constexpr int kPlainRows = 64;
constexpr int kLongRows = 256;  // rows a partial sum of the columns of long rows

enum { kNoSums, kPlainSums, kCompensated };

template <int MODE>
__device__ __forceinline__ void add_to(float& s, float& c, float v) {
  if (MODE == kCompensated) {
    const float y = __fsub_rn(v, c), t = __fadd_rn(s, y);
    c = __fsub_rn(__fsub_rn(t, s), y);
    s = t;
  } else if (MODE == kPlainSums) {
    s += v;
  }
}

// As k_norm in norm.cu.  partial: [teams][2][dim].
template <typename TI, typename TO, int V, bool MULTI, int MODE>
__global__ void __launch_bounds__(MULTI ? 512 : 256)
    k_norm_grad(const __grid_constant__ mlt_norm_args a, const __grid_constant__ mlt_norm_grads g, float* partial,
                int lanes, int seg) {
  constexpr int C = kEach / V;
  __shared__ RowSums<2> sums;
  __shared__ float by_warp[MULTI ? 1 : 8][2][MULTI ? 1 : kNormGroupDim];
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  const int ranks = MULTI ? cluster_ranks() : 1, rank = MULTI ? cluster_rank() : 0;
  if (MULTI && ranks > 1) cluster_barrier();
  const int j = MULTI ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int first = rank * seg, cols = min(seg, a.dim - first);
  const long long at = first + static_cast<long long>(j) * V;
  const int hop = lanes * V;
  bool on[C];
#pragma unroll
  for (int c = 0; c < C; ++c) on[c] = j * V + c * hop < cols;
  float w[C][V], sw[C][V], cw[C][V], sb[C][V], cb[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      w[c][v] = a.weight != nullptr && on[c] ? load_as_f32(a.weight, a.w_dtype, at + c * hop + v) : 1.0f;
      sw[c][v] = cw[c][v] = sb[c][v] = cb[c][v] = 0.0f;
    }
  const int in_warp = MULTI ? 1 : 32 / lanes;
  const long long step = MULTI ? gridDim.x / ranks : static_cast<long long>(gridDim.x) * 8 * in_warp;
  long long base = MULTI ? blockIdx.x / ranks : (blockIdx.x * 8LL + (threadIdx.x >> 5)) * in_warp;
  const int sub = MULTI ? 0 : (threadIdx.x & 31) / lanes;
  const bool more = g.g_total != nullptr;
  Pack<TI, V> px[C], pt[C];
  Pack<TO, V> pg[C];
  float next_mean = 0.0f, next_rstd = 0.0f;
  auto fetch = [&](long long row) {
    const TI* x = static_cast<const TI*>(a.x) + row * a.x_stride + at;
    const TO* gy = static_cast<const TO*>(g.gy) + row * g.gy_stride + at;
    if (row >= a.rows) return;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (on[c]) {
        px[c] = *reinterpret_cast<const Pack<TI, V>*>(x + c * hop);
        pg[c] = *reinterpret_cast<const Pack<TO, V>*>(gy + c * hop);
      }
    const float2 s = *reinterpret_cast<const float2*>(a.stats + 2 * row);
    next_mean = s.x;
    next_rstd = s.y;
  };
  fetch(base + sub);
  for (; base < a.rows; base += step) {
    const long long row = base + sub;
    const bool live = row < a.rows;
    const float mean = next_mean, rstd = next_rstd;
    if (more && live) {
      const TI* gt = static_cast<const TI*>(g.g_total) + row * g.g_total_stride + at;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (on[c]) pt[c] = *reinterpret_cast<const Pack<TI, V>*>(gt + c * hop);
    }
    float h[C][V], gy[C][V], total[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        h[c][v] = gy[c][v] = 0.0f;
        if (on[c] && live) {
          h[c][v] = (to_f32(px[c].v[v]) - mean) * rstd;
          gy[c][v] = to_f32(pg[c].v[v]);
        }
        add_to<MODE>(sw[c][v], cw[c][v], gy[c][v] * h[c][v]);
        add_to<MODE>(sb[c][v], cb[c][v], gy[c][v]);
        gy[c][v] *= w[c][v];
        total[0] += gy[c][v];
        total[1] = fmaf(gy[c][v], h[c][v], total[1]);
      }
    if (base + step < a.rows) fetch(row + step);
    if (MULTI)
      row_sums(total, sums, slot, ranks, rank);
    else
      group_sums(total, lanes);
    if (g.gx == nullptr || !live) continue;
    const float m0 = total[0] / a.dim, m1 = total[1] / a.dim;
    TI* to = static_cast<TI*>(g.gx) + row * g.gx_stride + at;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!on[c]) continue;
      Pack<TI, V> q;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float d = fmaf(-h[c][v], m1, gy[c][v] - m0) * rstd;
        if (more) d += to_f32(pt[c].v[v]);
        q.v[v] = from_f32<TI>(d);
      }
      *reinterpret_cast<Pack<TI, V>*>(to + c * hop) = q;
    }
  }
  if (MODE == kNoSums) return;
  if (MULTI) {
    float* out = partial + static_cast<long long>(blockIdx.x / ranks) * 2 * a.dim;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (on[c]) {
          out[at + c * hop + v] = sw[c][v] - cw[c][v];
          out[a.dim + at + c * hop + v] = sb[c][v] - cb[c][v];
        }
    return;
  }
  // the rows of a warp, then the warps of the CTA
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float s = sw[c][v] - cw[c][v], b = sb[c][v] - cb[c][v];
      for (int o = lanes; o < 32; o *= 2) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
      }
      if (sub == 0 && on[c]) {
        by_warp[threadIdx.x >> 5][0][j * V + c * hop + v] = s;
        by_warp[threadIdx.x >> 5][1][j * V + c * hop + v] = b;
      }
    }
  __syncthreads();
  if (threadIdx.x < a.dim)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float s = 0.0f;
#pragma unroll
      for (int q = 0; q < 8; ++q) s += by_warp[q][k][threadIdx.x];
      partial[(blockIdx.x * 2LL + k) * a.dim + threadIdx.x] = s;
    }
}

// Rows that no cluster holds: the input's gradient, a CTA a row.
template <typename TI, typename TO>
__global__ void __launch_bounds__(1024)
    k_norm_grad_long(const __grid_constant__ mlt_norm_args a, const __grid_constant__ mlt_norm_grads g) {
  __shared__ RowSums<2> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TI* x = static_cast<const TI*>(a.x) + row * a.x_stride;
    const TO* gy = static_cast<const TO*>(g.gy) + row * g.gy_stride;
    const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
    auto weighted = [&](int i) {
      const float v = to_f32(gy[i]);
      return a.weight != nullptr ? v * load_as_f32(a.weight, a.w_dtype, i) : v;
    };
    float total[2] = {0.0f, 0.0f};
    for (int i = threadIdx.x; i < a.dim; i += 1024) {
      const float v = weighted(i);
      total[0] += v;
      total[1] = fmaf(v, (to_f32(x[i]) - mean) * rstd, total[1]);
    }
    row_sums(total, sums, slot, 1, 0);
    const float m0 = total[0] / a.dim, m1 = total[1] / a.dim;
    for (int i = threadIdx.x; i < a.dim; i += 1024) {
      const float h = (to_f32(x[i]) - mean) * rstd;
      float d = fmaf(-h, m1, weighted(i) - m0) * rstd;
      if (g.g_total != nullptr) d += to_f32(static_cast<const TI*>(g.g_total)[row * g.g_total_stride + i]);
      static_cast<TI*>(g.gx)[row * g.gx_stride + i] = from_f32<TI>(d);
    }
  }
}

// Their columns' sums: a thread a column, `per` rows.
template <typename TI, typename TO>
__global__ void __launch_bounds__(256)
    k_norm_cols_long(const __grid_constant__ mlt_norm_args a, const __grid_constant__ mlt_norm_grads g, float* partial,
                     long long per) {
  pdl_wait();
  pdl_trigger();
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= a.dim) return;
  const long long from = blockIdx.y * per, to = min(static_cast<long long>(a.rows), from + per);
  float sw = 0.0f, cw = 0.0f, sb = 0.0f, cb = 0.0f;
#pragma unroll 4
  for (long long row = from; row < to; ++row) {
    const float gy = to_f32(static_cast<const TO*>(g.gy)[row * g.gy_stride + col]);
    const float x = to_f32(static_cast<const TI*>(a.x)[row * a.x_stride + col]);
    add_to<kCompensated>(sw, cw, gy * ((x - a.stats[2 * row]) * a.stats[2 * row + 1]));
    add_to<kCompensated>(sb, cb, gy);
  }
  float* out = partial + blockIdx.y * 2LL * a.dim;
  out[col] = sw - cw;
  out[a.dim + col] = sb - cb;
}

// The teams' sums of 32 columns: 32 threads a column take every 32nd team, then a tree.
__global__ void __launch_bounds__(1024)
    k_norm_cols(const float* partial, int teams, int dim, void* gweight, void* gbias, int dtype) {
  __shared__ float s[32][33];
  pdl_wait();
  pdl_trigger();
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 32 + x;
  void* to = blockIdx.y == 0 ? gweight : gbias;
  if (to == nullptr) return;
  float sum = 0.0f, c = 0.0f;
  if (col < dim)
#pragma unroll 8
    for (int t = y; t < teams; t += 32) add_to<kCompensated>(sum, c, partial[(t * 2LL + blockIdx.y) * dim + col]);
  s[y][x] = sum - c;
  __syncthreads();
  float v[1] = {s[x][y]};
  group_sums(v, 32);
  if (x == 0 && blockIdx.x * 32 + y < dim) store_from_f32(to, dtype, blockIdx.x * 32 + y, v[0]);
}

struct Plan {
  bool group, far;  // groups of lanes; rows that no cluster holds
  int lanes, threads, ranks, seg;
  long long teams;  // of rows, and of partial sums
  bool compensated;
};

// 24 warps an SM; the number of teams sets the order of the sums and follows from sizes alone.
Plan plan_of(long long rows, int dim, int sms) {
  Plan p{};
  if (dim <= kNormGroupDim) {
    p.group = true;
    p.lanes = 1;
    while (p.lanes * kEach < dim) p.lanes *= 2;
    p.threads = 256;
    p.ranks = 1;
    p.seg = dim;
    const long long need = (rows + 8 * (32 / p.lanes) - 1) / (8 * (32 / p.lanes)), most = 3LL * sms;
    p.teams = need < most ? need : most;
    p.compensated = rows > p.teams * 8 * (32 / p.lanes) * kPlainRows;
    return p;
  }
  if (dim > kNormMaxCluster * 512 * kEach) {
    p.far = true;
    p.teams = (rows + kLongRows - 1) / kLongRows;
    if (p.teams > 256) p.teams = 256;
    return p;
  }
  p.ranks = (dim + 512 * kEach - 1) / (512 * kEach);
  p.seg = ((dim + p.ranks - 1) / p.ranks + kEach - 1) / kEach * kEach;
  p.ranks = (dim + p.seg - 1) / p.seg;
  p.threads = p.lanes = ((p.seg + kEach - 1) / kEach + 31) / 32 * 32;
  if (p.ranks == 1) p.seg = dim;
  long long most = static_cast<long long>(sms) * (768 / p.threads) / p.ranks;
  if (most < 1) most = 1;
  p.teams = rows < most ? rows : most;
  p.compensated = rows > p.teams * kPlainRows;
  return p;
}

template <typename TI, typename TO, int V, bool MULTI>
cudaError_t launch_rows(const mlt_norm_args& a, const mlt_norm_grads& g, const Plan& p, float* partial, bool sums,
                        cudaStream_t st) {
  const unsigned grid = static_cast<unsigned>(p.teams * p.ranks);
  auto go = [&](auto kernel) {
    return launch_cluster(kernel, grid, p.threads, p.ranks, st, a, g, partial, p.lanes, p.seg);
  };
  if (!sums) return go(k_norm_grad<TI, TO, V, MULTI, kNoSums>);
  return p.compensated ? go(k_norm_grad<TI, TO, V, MULTI, kCompensated>)
                       : go(k_norm_grad<TI, TO, V, MULTI, kPlainSums>);
}

template <typename TI, typename TO, int V>
cudaError_t launch_as(const mlt_norm_args& a, const mlt_norm_grads& g, const Plan& p, float* partial, bool sums,
                      cudaStream_t st) {
  return p.group ? launch_rows<TI, TO, V, false>(a, g, p, partial, sums, st)
                 : launch_rows<TI, TO, V, true>(a, g, p, partial, sums, st);
}

}  // namespace

size_t norm_grad_workspace(long long rows, int dim, int sms) {
  return rows == 0 ? 0 : up256(static_cast<size_t>(plan_of(rows, dim, sms).teams) * 2 * dim * sizeof(float));
}

cudaError_t launch_norm_grad(const mlt_norm_args& a, const mlt_norm_grads& g, void* ws, int sms, long long* launches,
                             cudaStream_t st) {
  const Plan p = a.rows > 0 ? plan_of(a.rows, a.dim, sms) : Plan{};
  float* partial = static_cast<float*>(ws);
  const bool sums = g.gweight != nullptr || g.gbias != nullptr;
  cudaError_t e = cudaSuccess;
  if (a.rows > 0)
    e = with_norm_types(a.dtype, a.y_dtype, [&](auto ti, auto to) -> cudaError_t {
      using TI = decltype(ti);
      using TO = decltype(to);
      if (p.far) {
        // the sums first: gx may be written over gy
        if (sums) {
          ++*launches;
          const cudaError_t r =
              launch_pdl(k_norm_cols_long<TI, TO>, dim3((a.dim + 255) / 256, static_cast<unsigned>(p.teams)), dim3(256),
                         0, st, a, g, partial, (a.rows + p.teams - 1) / p.teams);
          if (r != cudaSuccess) return r;
        }
        if (g.gx == nullptr) return cudaSuccess;
        const long long most = 2LL * sms;
        ++*launches;
        return launch_cluster(k_norm_grad_long<TI, TO>, static_cast<unsigned>(a.rows < most ? a.rows : most), 1024, 1,
                              st, a, g);
      }
      constexpr int V = 16 / sizeof(TI);
      auto fits = [&](const void* q, int64_t stride, size_t bytes) {
        return q == nullptr || (aligned_to(q, bytes * V) && stride % V == 0);
      };
      const bool wide = a.dim % V == 0 && fits(a.x, a.x_stride, sizeof(TI)) && fits(g.gy, g.gy_stride, sizeof(TO)) &&
                        fits(g.g_total, g.g_total_stride, sizeof(TI)) && fits(g.gx, g.gx_stride, sizeof(TI));
      ++*launches;
      return wide ? launch_as<TI, TO, V>(a, g, p, partial, sums, st) : launch_as<TI, TO, 1>(a, g, p, partial, sums, st);
    });
  if (e != cudaSuccess || !sums) return e;
  ++*launches;
  return launch_pdl(k_norm_cols, dim3((a.dim + 31) / 32, 2), dim3(1024), 0, st, static_cast<const float*>(partial),
                    a.rows > 0 ? static_cast<int>(p.teams) : 0, a.dim, g.gweight, g.gbias, a.w_dtype);
}

}  // namespace mlt
