// Layer norm of rows with an optional residual addition before it.
//
// Mean and variance are two sums over the row's registers, the second over squares of
// differences from the mean, so nothing cancels.  Bound: memory (each value read and
// written once): 16,384 x 4,096 bf16 with a residual 86 us, 6.2 TB/s; fp32 with one, 32,768 x 2,048 174 us and
// 1,048,573 x 64 174, 6.2 TB/s both.  64 rows of 1,024 take 3 us, a launch.
// See norm.cuh for how rows are dealt out.
// CTAs stay and take row after row: weights are fetched once, and the next row's packs are
// under way while this one is summed.
#include <utility>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kMostThreads = 512;

// What lets most warps stay without spills of consequence (groups of lanes at 80: up to 120 bytes, and
// 1,048,573 x 64 bf16 56 us for 61).
constexpr int registers(bool cta, bool edge) { return cta && !edge ? 72 : 80; }

// CTA: the CTA takes a row; else groups of `lanes` lanes do.
template <typename TI, typename TO, int V, int C, bool CTA, bool EDGE>
__global__ void __maxnreg__(registers(CTA, EDGE))
    k_norm(const __grid_constant__ mlt_norm_args a, int lanes, int skew, int skew_step) {
  extern __shared__ __align__(16) float affine[];
  __shared__ RowSums<1> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  const int j = CTA ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int in_warp = CTA ? 1 : 32 / lanes;  // rows a warp
  const long long step = CTA ? gridDim.x : static_cast<long long>(gridDim.x) * 8 * in_warp;
  const int sub = CTA ? 0 : (threadIdx.x & 31) / lanes;
  long long base = CTA ? blockIdx.x : (blockIdx.x * 8LL + (threadIdx.x >> 5)) * in_warp;
  if (EDGE) skew = static_cast<int>((skew + (base + sub) % V * skew_step) % V);  // of all rows of this thread
  const Columns<V, C, EDGE> cols(j * V, lanes * V, skew, a.dim);
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
  }
  for (; base < a.rows; base += step) {
    const long long row = base + sub;
    const bool live = row < a.rows;
    constexpr int E = C * V;
    float2 t[E / 2], s = both(0.0f);
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
    cols.template pairs<CTA>([&](int i, bool on0, bool on1) {
      const bool all = CTA || live;
      t[i / 2] = masked(two_of(px, i), on0 && all, on1 && all);
      s = __fadd2_rn(s, t[i / 2]);
    });
    float total[1] = {s.x + s.y};
    if (base + step < a.rows) fetch(row + step);
    if (CTA)
      row_sums(total, sums, slot);
    else
      group_sums(total, lanes);
    const float mean = total[0] / a.dim;
    s = both(0.0f);
    cols.template pairs<CTA>([&](int i, bool on0, bool on1) {
      t[i / 2] = masked(__fadd2_rn(t[i / 2], both(-mean)), on0, on1);
      s = __ffma2_rn(t[i / 2], t[i / 2], s);
    });
    total[0] = s.x + s.y;
    if (CTA)
      row_sums(total, sums, slot);
    else
      group_sums(total, lanes);
    const float rstd = 1.0f / sqrtf(total[0] / a.dim + a.eps);
    if (!live) continue;
    if (a.stats != nullptr && j == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
    TO* to = static_cast<TO*>(a.y) + row * a.y_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (CTA && scaled) {
        ws.get(w[c], c);
        bs.get(b[c], c);
      }
      float f[V];
      auto value = [&](int i) {
        const float2 h = __fmul2_rn(t[i / 2], both(rstd));
        return !CTA || scaled ? __ffma2_rn(h, two_of(w, i), two_of(b, i)) : h;
      };
      if constexpr (V == 1) {
        const float h = one_of(t, c) * rstd;
        f[0] = !CTA || scaled ? fmaf(h, w[c][0], b[c][0]) : h;
      } else {
#pragma unroll
        for (int v = 0; v < V; v += 2) {
          const float2 d = value(c * V + v);
          f[v] = d.x;
          f[v + 1] = d.y;
        }
      }
      Vec<TO, V> q;
      q.put(f);
      cols.store(q, to, c);
    }
  }
}

// Rows that a CTA's registers do not hold: in shared memory (`kept`), each thread's packs in places of its own, or
// where that does not hold them either, read again for each pass.
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(kMostThreads, 2)
    k_norm_long(const __grid_constant__ mlt_norm_args a, int kept, int skew0, int skew_step) {
  extern __shared__ __align__(16) float affine[];
  TI* held = reinterpret_cast<TI*>(affine);
  __shared__ RowSums<1> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  sums.clear();
  __syncthreads();
  const float inv_dim = 1.0f / a.dim;
  const bool add = a.residual != nullptr;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int skew = static_cast<int>((skew0 + row % V * skew_step) % V), first = static_cast<int>(threadIdx.x) * V - skew;
    const TI* x = static_cast<const TI*>(a.x) + row * a.x_stride;
    const TI* r = static_cast<const TI*>(a.residual) + row * a.residual_stride;
    TI* to = static_cast<TI*>(a.total) + row * a.total_stride;
    TO* y = static_cast<TO*>(a.y) + row * a.y_stride;
    // the first pass may write total over x or residual: later ones read what it wrote, each thread its own
    const bool stored = a.total != nullptr;
    auto values = [&](float (&t)[V], int col, bool again) {
      if (again && kept) {
        Vec<TI, V> q;
        q.load(held + (col + skew));
#pragma unroll
        for (int v = 0; v < V; ++v) t[v] = q.get(v);
        return;
      }
      if (again && stored) {
        load_some<V>(t, to, col, a.dim);
        return;
      }
      load_some<V>(t, x, col, a.dim);
      if (!add) return;
      float e[V];
      load_some<V>(e, r, col, a.dim);
#pragma unroll
      for (int v = 0; v < V; ++v) t[v] = to_f32(from_f32<TI>(__fadd_rn(t[v], e[v])));
    };
    float total[1] = {0.0f};
#pragma unroll 4
    for (int col = first; col < a.dim; col += kMostThreads * V) {
      float t[V], s = 0.0f;
      values(t, col, false);
      if (stored) store_some<V>(t, to, col, a.dim);
      if (kept) {
        Vec<TI, V> q;
        q.put(t);
        q.store(held + (col + skew));
      }
#pragma unroll
      for (int v = 0; v < V; ++v) s += t[v];
      total[0] += s;
    }
    row_sums(total, sums, slot);
    const float mean = total[0] * inv_dim;
    total[0] = 0.0f;
#pragma unroll 2
    for (int col = first; col < a.dim; col += kMostThreads * V) {
      float t[V], s = 0.0f;
      values(t, col, true);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float d = V == 1 || (col + v >= 0 && col + v < a.dim) ? t[v] - mean : 0.0f;
        s = fmaf(d, d, s);
      }
      total[0] += s;
    }
    row_sums(total, sums, slot);
    const float rstd = 1.0f / sqrtf(total[0] * inv_dim + a.eps);
    if (a.stats != nullptr && threadIdx.x == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
#pragma unroll 2
    for (int col = first; col < a.dim; col += kMostThreads * V) {
      float t[V], w[V], b[V];
      values(t, col, true);
      load_weights<V>(w, a.weight, a.w_dtype, col, a.dim, 1.0f);
      load_weights<V>(b, a.bias, a.w_dtype, col, a.dim, 0.0f);
#pragma unroll
      for (int v = 0; v < V; ++v) t[v] = fmaf((t[v] - mean) * rstd, w[v], b[v]);
      store_some<V>(t, y, col, a.dim);
    }
  }
}

template <typename TI, typename TO, int V>
cudaError_t launch_long(const mlt_norm_args& a, const Skew& skew, int sms, cudaStream_t st) {
  size_t smem = (static_cast<size_t>(a.dim) + 2 * V) / V * V * sizeof(TI);
  const bool kept = smem <= 224 * 1024;
  if (!kept) smem = 0;
  const int per_sm = 2 * (smem + 2048) <= 227 * 1024 ? 2 : 1;
  const long long most = static_cast<long long>(per_sm) * sms;
  return launch_rows(k_norm_long<TI, TO, V>, static_cast<unsigned>(a.rows < most ? a.rows : most), kMostThreads, smem, st, a,
                     kept ? 1 : 0, skew.first, skew.step);
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
    return launch_rows(kernel, static_cast<unsigned>(need < most ? need : most), 256, 0, st, a, lanes, skew.first,
                       skew.step);
  }
  constexpr auto kernel = k_norm<TI, TO, V, E / V, true, EDGE>;
  if (places > kMostThreads * E) return launch_long<TI, TO, V>(a, skew, sms, st);
  const int threads = ((places + E - 1) / E + 31) / 32 * 32;
  const size_t smem = a.weight != nullptr || a.bias != nullptr ? 2 * sizeof(float) * threads * E : 0;
  long long most = static_cast<long long>(sms) * resident_ctas<kernel>(threads, smem);
  const int period = skew.period(V);
  most = most < period ? period : most / period * period;
  return launch_rows(kernel, static_cast<unsigned>(a.rows < most ? a.rows : most), threads, smem, st, a, threads,
                     skew.first, skew.step);
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
    if (!skew.same) return launch_as<TI, TO, 1, 8, false>(a, Skew{true, 0, 0}, sms, st);
    return skew.edges(a.dim, V) ? launch_as<TI, TO, V, E, true>(a, skew, sms, st)
                                : launch_as<TI, TO, V, E, false>(a, skew, sms, st);
  });
}

}  // namespace mlt
