// Layer norm of rows with an optional residual addition before it.
//
// Mean and variance are two sums over the row's registers, the second over squares of
// differences from the mean, so nothing cancels.  Bound: memory (each value read and
// written once).  See norm.cuh for how rows are dealt out.
// CTAs stay and take row after row: weights are fetched once, and the next row's packs are
// under way while this one is summed.
#include <utility>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kMostThreads = 512;

// The fewest without spills of consequence (edges in packs of 16-bit values: up to 84 bytes at eight less).
constexpr int registers(bool cta, bool edge) { return cta ? (edge ? 80 : 72) : (edge ? 104 : 96); }

// CTA: the CTA, or its cluster with `seg` places a CTA, takes a row; else groups of `lanes` lanes do.
template <typename TI, typename TO, int V, int C, bool CTA, bool EDGE>
__global__ void __maxnreg__(registers(CTA, EDGE))
    k_norm(const __grid_constant__ mlt_norm_args a, int lanes, int seg, int skew, int skew_step) {
  extern __shared__ __align__(16) float affine[];
  __shared__ RowSums<1> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  const int ranks = CTA ? cluster_ranks() : 1, rank = CTA ? cluster_rank() : 0;
  const int j = CTA ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int in_warp = CTA ? 1 : 32 / lanes;  // rows a warp
  const long long step = CTA ? gridDim.x / ranks : static_cast<long long>(gridDim.x) * 8 * in_warp;
  const int sub = CTA ? 0 : (threadIdx.x & 31) / lanes;
  long long base = CTA ? blockIdx.x / ranks : (blockIdx.x * 8LL + (threadIdx.x >> 5)) * in_warp;
  if (EDGE) skew = static_cast<int>((skew + (base + sub) % V * skew_step) % V);  // of all rows of this thread
  const Columns<V, C, EDGE> cols(rank * seg + j * V, lanes * V, (rank + 1) * seg, skew, a.dim);
  const bool scaled = a.weight != nullptr || a.bias != nullptr;
  const Kept<V, C> ws{affine}, bs{affine + blockDim.x * C * V};
  const bool add = a.residual != nullptr;
  const TI *x0 = static_cast<const TI*>(a.x), *r0 = static_cast<const TI*>(a.residual);
  const TI *x1 = x0 + (a.rows - 1) * a.x_stride + a.dim, *r1 = r0 + (a.rows - 1) * a.residual_stride + a.dim;
  Vec<TI, V> px[C], pr[C];
  auto fetch = [&](long long row) {
    if (row >= a.rows) return;
    cols.load(px, x0 + row * a.x_stride, x0, x1);
    if (add) cols.load(pr, r0 + row * a.residual_stride, r0, r1);
  };
  fetch(base + sub);
  float w[C][V], b[C][V];
  if (!CTA || scaled) {
    load_columns(w, cols, a.weight, a.w_dtype, 1.0f);
    load_columns(b, cols, a.bias, a.w_dtype, 0.0f);
    if (CTA) {
      ws.put(w);
      bs.put(b);
    }
  }
  if (CTA) {
    sums.clear();
    __syncthreads();
    if (ranks > 1) cluster_barrier();  // every CTA runs before its memory is written to
  }
  for (; base < a.rows; base += step) {
    const long long row = base + sub;
    const bool live = row < a.rows;
    float t[C][V], total[1] = {0.0f};
    if (add && live) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float f[V];
#pragma unroll
        for (int v = 0; v < V; ++v) f[v] = __fadd_rn(px[c].get(v), pr[c].get(v));
        px[c].put(f);
        if (a.total != nullptr) cols.store(px[c], static_cast<TI*>(a.total) + row * a.total_stride, c);
      }
    } else if (a.total != nullptr && live) {
#pragma unroll
      for (int c = 0; c < C; ++c) cols.store(px[c], static_cast<TI*>(a.total) + row * a.total_stride, c);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float s = 0.0f;
      cols.each(
          c,
          [&](int c, int v) {
            t[c][v] = live ? px[c].get(v) : 0.0f;
            s += t[c][v];
          },
          [&](int c, int v) { t[c][v] = 0.0f; });
      total[0] += s;
    }
    if (base + step < a.rows) fetch(row + step);
    if (CTA)
      row_sums(total, sums, slot, ranks, rank);
    else
      group_sums(total, lanes);
    const float mean = total[0] / a.dim;
    total[0] = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float s = 0.0f;
      cols.each(
          c,
          [&](int c, int v) {
            t[c][v] -= mean;
            s = fmaf(t[c][v], t[c][v], s);
          },
          [](int, int) {});
      total[0] += s;
    }
    if (CTA)
      row_sums(total, sums, slot, ranks, rank);
    else
      group_sums(total, lanes);
    const float rstd = 1.0f / sqrtf(total[0] / a.dim + a.eps);
    if (!live) continue;
    if (a.stats != nullptr && j == 0 && rank == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
    TO* to = static_cast<TO*>(a.y) + row * a.y_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (CTA && scaled) {
        ws.get(w[c], c);
        bs.get(b[c], c);
      }
      float f[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float h = t[c][v] * rstd;
        f[v] = !CTA || scaled ? fmaf(h, w[c][v], b[c][v]) : h;
      }
      Vec<TO, V> q;
      q.put(f);
      cols.store(q, to, c);
    }
  }
}

// Rows that no cluster holds: a CTA reads the row three times.
template <typename TI, typename TO>
__global__ void __launch_bounds__(kMostThreads) k_norm_long(const __grid_constant__ mlt_norm_args a) {
  __shared__ RowSums<1> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  sums.clear();
  __syncthreads();
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
    for (int i = threadIdx.x; i < a.dim; i += kMostThreads) {
      const float t = value(i, false);
      if (stored) to[i] = from_f32<TI>(t);
      total[0] += t;
    }
    row_sums(total, sums, slot, 1, 0);
    const float mean = total[0] / a.dim;
    total[0] = 0.0f;
    for (int i = threadIdx.x; i < a.dim; i += kMostThreads) {
      const float t = value(i, true) - mean;
      total[0] = fmaf(t, t, total[0]);
    }
    row_sums(total, sums, slot, 1, 0);
    const float rstd = 1.0f / sqrtf(total[0] / a.dim + a.eps);
    if (a.stats != nullptr && threadIdx.x == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
    for (int i = threadIdx.x; i < a.dim; i += kMostThreads) {
      const float w = a.weight != nullptr ? load_as_f32(a.weight, a.w_dtype, i) : 1.0f;
      const float b = a.bias != nullptr ? load_as_f32(a.bias, a.w_dtype, i) : 0.0f;
      y[i] = from_f32<TO>(fmaf((value(i, true) - mean) * rstd, w, b));
    }
  }
}

// E: values of a row a thread.
template <typename TI, typename TO, int V, int E, bool EDGE>
cudaError_t launch_as(const mlt_norm_args& a, const Skew& skew, int sms, cudaStream_t st) {
  const int places = (a.dim + (EDGE ? V - 1 : 0) + V - 1) / V * V;
  if (places <= 32 * E) {
    constexpr auto kernel = k_norm<TI, TO, V, E / V, false, EDGE>;
    int lanes = 1;
    while (lanes * E < places) lanes *= 2;
    const long long per = 8 * (32 / lanes), need = (a.rows + per - 1) / per;
    const long long most = static_cast<long long>(sms) * resident_ctas<kernel>(256, 0);
    return launch_cluster(kernel, static_cast<unsigned>(need < most ? need : most), 256, 1, 0, st, a, lanes, places,
                          skew.first, skew.step);
  }
  constexpr auto kernel = k_norm<TI, TO, V, E / V, true, EDGE>;
  // CTAs of 256 threads leave room for one another's barriers; longer rows take clusters, then larger CTAs
  int ranks = (places + kMostThreads * E - 1) / (kMostThreads * E);
  if (ranks > kNormMaxCluster) ranks = kNormMaxCluster;
  const int seg = ((places + ranks - 1) / ranks + V - 1) / V * V;
  ranks = (places + seg - 1) / seg;
  const int threads = ((seg + E - 1) / E + 31) / 32 * 32;
  const size_t smem = a.weight != nullptr || a.bias != nullptr ? 2 * sizeof(float) * threads * E : 0;
  long long most = static_cast<long long>(sms) * resident_ctas<kernel>(threads, smem) / ranks;
  const int period = skew.period(V);
  most = most < period ? period : most / period * period;
  const long long teams = a.rows < most ? a.rows : most;
  return launch_cluster(kernel, static_cast<unsigned>(teams * ranks), threads, ranks, smem, st, a, threads, seg, skew.first,
                        skew.step);
}

}  // namespace

cudaError_t launch_norm(const mlt_norm_args& a, int sms, long long* launches, cudaStream_t st) {
  *launches = 1;
  return with_norm_types(a.dtype, a.y_dtype, [&](auto ti, auto to) -> cudaError_t {
    using TI = decltype(ti);
    using TO = decltype(to);
    constexpr int V = 16 / sizeof(TI), E = 2 * V;
    Skew skew;
    skew.add(a.x, a.x_stride, sizeof(TI), V);
    skew.add(a.residual, a.residual_stride, sizeof(TI), V);
    skew.add(a.total, a.total_stride, sizeof(TI), V);
    skew.add(a.y, a.y_stride, sizeof(TO), V);
    if (a.dim + V > kNormMaxCluster * kMostThreads * (skew.same ? E : 8)) {
      const long long most = 4LL * sms;
      return launch_cluster(k_norm_long<TI, TO>, static_cast<unsigned>(a.rows < most ? a.rows : most), kMostThreads, 1, 0,
                            st, a);
    }
    if (!skew.same) return launch_as<TI, TO, 1, 8, false>(a, Skew{true, 0, 0}, sms, st);
    return skew.edges(a.dim, V) ? launch_as<TI, TO, V, E, true>(a, skew, sms, st)
                                : launch_as<TI, TO, V, E, false>(a, skew, sms, st);
  });
}

}  // namespace mlt
