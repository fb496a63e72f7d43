// Layer norm of rows with an optional residual addition before it.
//
// Mean and variance are two sums over the row's registers, the second over squares of
// differences from the mean, so nothing cancels.  Bound: memory (each value read and
// written once; some ten operations for each).  See norm.cuh for how rows are dealt out.
// CTAs stay and take row after row: weights are loaded once, and the next row's packs are
// under way while this one is summed.
#include <utility>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kEach = 8;  // values of a row a thread

// MULTI: the CTA (of `lanes` threads), or its cluster with `seg` columns a CTA, takes a row; else groups
// of `lanes` lanes do.
template <typename TI, typename TO, int V, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 1024 : 256) k_norm(const __grid_constant__ mlt_norm_args a, int lanes, int seg) {
  constexpr int C = kEach / V;
  __shared__ RowSums<1> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  const int ranks = MULTI ? cluster_ranks() : 1, rank = MULTI ? cluster_rank() : 0;
  if (MULTI && ranks > 1) cluster_barrier();  // every CTA runs before its memory is written to
  const int j = MULTI ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int first = rank * seg, cols = min(seg, a.dim - first);
  const long long at = first + static_cast<long long>(j) * V;
  const int hop = lanes * V;
  bool on[C];
#pragma unroll
  for (int c = 0; c < C; ++c) on[c] = j * V + c * hop < cols;
  float w[C][V], b[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      w[c][v] = a.weight != nullptr && on[c] ? load_as_f32(a.weight, a.w_dtype, at + c * hop + v) : 1.0f;
      b[c][v] = a.bias != nullptr && on[c] ? load_as_f32(a.bias, a.w_dtype, at + c * hop + v) : 0.0f;
    }
  const int in_warp = MULTI ? 1 : 32 / lanes;  // rows a warp
  const long long step = MULTI ? gridDim.x / ranks : static_cast<long long>(gridDim.x) * 8 * in_warp;
  long long base = MULTI ? blockIdx.x / ranks : (blockIdx.x * 8LL + (threadIdx.x >> 5)) * in_warp;
  const int sub = MULTI ? 0 : (threadIdx.x & 31) / lanes;
  const bool add = a.residual != nullptr;
  Pack<TI, V> px[C], pr[C];
  auto fetch = [&](long long row) {
    const TI* x = static_cast<const TI*>(a.x) + row * a.x_stride + at;
    const TI* r = static_cast<const TI*>(a.residual) + row * a.residual_stride + at;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (on[c] && row < a.rows) {
        px[c] = *reinterpret_cast<const Pack<TI, V>*>(x + c * hop);
        if (add) pr[c] = *reinterpret_cast<const Pack<TI, V>*>(r + c * hop);
      }
  };
  fetch(base + sub);
  for (; base < a.rows; base += step) {
    const long long row = base + sub;
    const bool live = row < a.rows;
    float t[C][V], total[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        t[c][v] = 0.0f;
        if (on[c] && live) {
          t[c][v] = to_f32(px[c].v[v]);
          if (add) {
            px[c].v[v] = from_f32<TI>(__fadd_rn(t[c][v], to_f32(pr[c].v[v])));
            t[c][v] = to_f32(px[c].v[v]);
          }
        }
        total[0] += t[c][v];
      }
    if (a.total != nullptr && live) {
      TI* to = static_cast<TI*>(a.total) + row * a.total_stride + at;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (on[c]) *reinterpret_cast<Pack<TI, V>*>(to + c * hop) = px[c];
    }
    if (base + step < a.rows) fetch(row + step);
    if (MULTI)
      row_sums(total, sums, slot, ranks, rank);
    else
      group_sums(total, lanes);
    const float mean = total[0] / a.dim;
    total[0] = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        t[c][v] = on[c] ? t[c][v] - mean : 0.0f;
        total[0] = fmaf(t[c][v], t[c][v], total[0]);
      }
    if (MULTI)
      row_sums(total, sums, slot, ranks, rank);
    else
      group_sums(total, lanes);
    const float rstd = 1.0f / sqrtf(total[0] / a.dim + a.eps);
    if (!live) continue;
    if (a.stats != nullptr && j == 0 && rank == 0) {
      a.stats[2 * row] = mean;
      a.stats[2 * row + 1] = rstd;
    }
    TO* to = static_cast<TO*>(a.y) + row * a.y_stride + at;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!on[c]) continue;
      Pack<TO, V> q;
#pragma unroll
      for (int v = 0; v < V; ++v) q.v[v] = from_f32<TO>(fmaf(t[c][v] * rstd, w[c][v], b[c][v]));
      *reinterpret_cast<Pack<TO, V>*>(to + c * hop) = q;
    }
  }
}

// Rows that no cluster holds: a CTA reads the row three times.
template <typename TI, typename TO>
__global__ void __launch_bounds__(1024) k_norm_long(const __grid_constant__ mlt_norm_args a) {
  __shared__ RowSums<1> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TI* x = static_cast<const TI*>(a.x) + row * a.x_stride;
    const TI* r = static_cast<const TI*>(a.residual) + row * a.residual_stride;
    TI* to = a.total == nullptr ? nullptr : static_cast<TI*>(a.total) + row * a.total_stride;
    TO* y = static_cast<TO*>(a.y) + row * a.y_stride;
    // the first pass may write total over x or residual: later ones read what it wrote, each thread its own
    const bool stored = to != nullptr;
    auto value = [&](int i, bool again) {
      if (again && stored) return to_f32(to[i]);
      float t = to_f32(x[i]);
      if (a.residual != nullptr) t = to_f32(from_f32<TI>(__fadd_rn(t, to_f32(r[i]))));
      return t;
    };
    float total[1] = {0.0f};
    for (int i = threadIdx.x; i < a.dim; i += 1024) {
      const float t = value(i, false);
      if (stored) to[i] = from_f32<TI>(t);
      total[0] += t;
    }
    row_sums(total, sums, slot, 1, 0);
    const float mean = total[0] / a.dim;
    total[0] = 0.0f;
    for (int i = threadIdx.x; i < a.dim; i += 1024) {
      const float t = value(i, true) - mean;
      total[0] = fmaf(t, t, total[0]);
    }
    row_sums(total, sums, slot, 1, 0);
    const float rstd = 1.0f / sqrtf(total[0] / a.dim + a.eps);
    if (a.stats != nullptr && threadIdx.x == 0) {
      a.stats[2 * row] = mean;
      a.stats[2 * row + 1] = rstd;
    }
    for (int i = threadIdx.x; i < a.dim; i += 1024) {
      const float w = a.weight != nullptr ? load_as_f32(a.weight, a.w_dtype, i) : 1.0f;
      const float b = a.bias != nullptr ? load_as_f32(a.bias, a.w_dtype, i) : 0.0f;
      y[i] = from_f32<TO>(fmaf((value(i, true) - mean) * rstd, w, b));
    }
  }
}

template <typename TI, typename TO, int V>
cudaError_t launch_as(const mlt_norm_args& a, int sms, cudaStream_t st) {
  if (a.dim <= kNormGroupDim) {
    int lanes = 1;
    while (lanes * kEach < a.dim) lanes *= 2;
    const long long need = (a.rows + 8 * (32 / lanes) - 1) / (8 * (32 / lanes));
    const long long most = static_cast<long long>(sms) * resident_ctas<k_norm<TI, TO, V, false>>(256);
    return launch_cluster(k_norm<TI, TO, V, false>, static_cast<unsigned>(need < most ? need : most), 256, 1, st, a,
                          lanes, a.dim);
  }
  int ranks = (a.dim + 1024 * kEach - 1) / (1024 * kEach);
  const int seg = ((a.dim + ranks - 1) / ranks + kEach - 1) / kEach * kEach;
  ranks = (a.dim + seg - 1) / seg;
  const int threads = ((seg + kEach - 1) / kEach + 31) / 32 * 32;
  const long long most =
      static_cast<long long>(sms) * resident_ctas<k_norm<TI, TO, V, true>>(threads) / ranks;
  const long long teams = a.rows < most ? a.rows : most < 1 ? 1 : most;
  return launch_cluster(k_norm<TI, TO, V, true>, static_cast<unsigned>(teams * ranks), threads, ranks, st, a, threads,
                        ranks > 1 ? seg : a.dim);
}

}  // namespace

cudaError_t launch_norm(const mlt_norm_args& a, int sms, long long* launches, cudaStream_t st) {
  *launches = 1;
  return with_norm_types(a.dtype, a.y_dtype, [&](auto ti, auto to) -> cudaError_t {
    using TI = decltype(ti);
    using TO = decltype(to);
    if (a.dim > kNormMaxCluster * 1024 * kEach) {
      const long long most = 2LL * sms;
      return launch_cluster(k_norm_long<TI, TO>, static_cast<unsigned>(a.rows < most ? a.rows : most), 1024, 1, st, a);
    }
    constexpr int V = 16 / sizeof(TI);
    auto fits = [&](const void* p, int64_t stride, size_t bytes) {
      return aligned_to(p, bytes * V) && stride % V == 0;
    };
    const bool wide = a.dim % V == 0 && fits(a.x, a.x_stride, sizeof(TI)) && fits(a.y, a.y_stride, sizeof(TO)) &&
                      (a.residual == nullptr || fits(a.residual, a.residual_stride, sizeof(TI))) &&
                      (a.total == nullptr || fits(a.total, a.total_stride, sizeof(TI)));
    return wide ? launch_as<TI, TO, V>(a, sms, st) : launch_as<TI, TO, 1>(a, sms, st);
  });
}

}  // namespace mlt
