// Gradients of layer norm: of its input row by row, of weight and bias as sums over all rows.
//
// With h = (t - mean) rstd and gw = gy weight, two sums over the row (gw and gw h) give the
// input's gradient.  Each thread keeps its columns' sums of gy h and gy in registers over
// all rows of its team; the teams' sums go to the workspace and a second
// kernel adds them up in a fixed order.  Bound: memory (x and gy read, gx written, once).
// Of n equal terms in a plain sum the error grows with n: where a thread has more than kPlainRows rows, its
// sums move to pairs of numbers in shared memory every kFlushRows of them (Knuth's exact addition).
#include <utility>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kPlainRows = 48;
constexpr int kFlushRows = 16;
constexpr int kMostThreads = 512;
constexpr int kGroupThreads = 256;
constexpr int kLongRows = 256;  // rows a partial sum of the columns of long rows

// (s, c) + v, s + c being the sum
__device__ __forceinline__ void add_exactly(float& s, float& c, float v) {
  const float t = __fadd_rn(s, v), b = __fsub_rn(t, s);
  c = __fadd_rn(c, __fadd_rn(__fsub_rn(s, __fsub_rn(t, b)), __fsub_rn(v, b)));
  s = t;
}

constexpr int registers(bool cta, bool edge) { return cta ? 128 : 128; }

// As k_norm in norm.cu.  SUMS: weight and bias have gradients; partial: [teams][2][dim]; flush: rows between
// moves to shared memory, or 0.
template <typename TI, typename TO, int V, int C, bool CTA, bool EDGE, bool SUMS>
__global__ void __maxnreg__(registers(CTA, EDGE))
    k_norm_grad(const __grid_constant__ mlt_norm_args a, const __grid_constant__ mlt_norm_grads g, float* partial,
                int lanes, int seg, int skew0, int skew_step, int flush) {
  extern __shared__ __align__(16) float mem[];
  __shared__ RowSums<2> sums;
  constexpr int E = C * V;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  const int ranks = CTA ? cluster_ranks() : 1, rank = CTA ? cluster_rank() : 0;
  const int j = CTA ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int in_warp = CTA ? 1 : 32 / lanes;
  const long long step = CTA ? gridDim.x / ranks : static_cast<long long>(gridDim.x) * 8 * in_warp;
  const int sub = CTA ? 0 : (threadIdx.x & 31) / lanes;
  const long long base0 = CTA ? blockIdx.x / ranks : (blockIdx.x * 8LL + (threadIdx.x >> 5)) * in_warp;
  const int skew = EDGE ? static_cast<int>((skew0 + (base0 + sub) % V * skew_step) % V) : 0;
  const Columns<V, C, EDGE> cols(rank * seg + j * V, lanes * V, (rank + 1) * seg, skew, a.dim);
  const bool scaled = a.weight != nullptr;
  const Kept<V, C> ws{mem};
  float* moved = CTA && scaled ? mem + blockDim.x * E : mem;  // [2 sums][2][E][threads]
  float w[C][V], sw[C][V], sb[C][V];
  const bool more = g.g_total != nullptr;
  const TI *x0 = static_cast<const TI*>(a.x), *t0 = static_cast<const TI*>(g.g_total);
  const TO* g0 = static_cast<const TO*>(g.gy);
  const TI *x1 = x0 + (a.rows - 1) * a.x_stride + a.dim, *t1 = t0 + (a.rows - 1) * g.g_total_stride + a.dim;
  const TO* g1 = g0 + (a.rows - 1) * g.gy_stride + a.dim;
  Vec<TI, V> px[C], pt[C];
  Vec<TO, V> pg[C];
  float2 next = make_float2(0.0f, 0.0f);
  auto fetch = [&](long long row) {
    if (row >= a.rows) return;
    cols.load(px, x0 + row * a.x_stride, x0, x1);
    cols.load(pg, g0 + row * g.gy_stride, g0, g1);
    next = *reinterpret_cast<const float2*>(a.stats + 2 * row);
  };
  fetch(base0 + sub);
  if (!CTA || scaled) {
    load_columns(w, cols, a.weight, a.w_dtype, 1.0f);
    if (CTA) ws.put(w);
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int v = 0; v < V; ++v) sw[c][v] = sb[c][v] = 0.0f;
  if (SUMS && flush > 0)
    for (int i = threadIdx.x; i < 4 * E * static_cast<int>(blockDim.x); i += blockDim.x) moved[i] = 0.0f;
  if (CTA) sums.clear();
  __syncthreads();
  if (CTA && ranks > 1) cluster_barrier();
  auto move = [&]() {
    if (!SUMS) return;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float* at = moved + (c * V + v) * blockDim.x + threadIdx.x;
        const int hop = E * blockDim.x;
        add_exactly(at[0], at[hop], sw[c][v]);
        add_exactly(at[2 * hop], at[3 * hop], sb[c][v]);
        sw[c][v] = sb[c][v] = 0.0f;
      }
  };
  int since = 0;
  for (long long base = base0; base < a.rows; base += step) {
    const long long row = base + sub;
    const bool live = row < a.rows;
    const float mean = next.x, rstd = next.y;
    if (more && live) cols.load(pt, t0 + row * g.g_total_stride, t0, t1);
    float h[C][V], gw[C][V], total[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (CTA && scaled) ws.get(w[c], c);
      float s0 = 0.0f, s1 = 0.0f;
      cols.each(
          c,
          [&](int c, int v) {
            h[c][v] = live ? (px[c].get(v) - mean) * rstd : 0.0f;
            const float gy = live ? pg[c].get(v) : 0.0f;
            if (SUMS) {
              sw[c][v] = fmaf(gy, h[c][v], sw[c][v]);
              sb[c][v] += gy;
            }
            gw[c][v] = !CTA || scaled ? gy * w[c][v] : gy;
            s0 += gw[c][v];
            s1 = fmaf(gw[c][v], h[c][v], s1);
          },
          [&](int c, int v) { h[c][v] = gw[c][v] = 0.0f; });
      total[0] += s0;
      total[1] += s1;
    }
    if (base + step < a.rows) fetch(row + step);
    if (CTA)
      row_sums(total, sums, slot, ranks, rank);
    else
      group_sums(total, lanes);
    if (flush > 0 && ++since == flush) {
      move();
      since = 0;
    }
    if (g.gx == nullptr || !live) continue;
    const float m0 = total[0] / a.dim, m1 = total[1] / a.dim;
    TI* to = static_cast<TI*>(g.gx) + row * g.gx_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float f[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float d = fmaf(-h[c][v], m1, gw[c][v] - m0) * rstd;
        f[v] = more ? d + pt[c].get(v) : d;
      }
      Vec<TI, V> q;
      q.put(f);
      cols.store(q, to, c);
    }
  }
  if (!SUMS) return;
  if (flush > 0) {
    move();
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float* at = moved + (c * V + v) * blockDim.x + threadIdx.x;
        const int hop = E * blockDim.x;
        sw[c][v] = at[0] + at[hop];
        sb[c][v] = at[2 * hop] + at[3 * hop];
      }
  }
  if (CTA) {
    float* out = partial + static_cast<long long>(blockIdx.x / ranks) * 2 * a.dim;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (cols.on(c, v)) {
          const int col = cols.first + c * cols.hop + v;
          out[col] = sw[c][v];
          out[a.dim + col] = sb[c][v];
        }
    return;
  }
  // the CTA's groups: their sums by place, then some threads a column, each over every so many groups in turn
  const int places = lanes * E, groups = kGroupThreads / lanes, group = threadIdx.x / lanes;
  int wide = 1;
  while (wide < a.dim) wide *= 2;
  const int teams = wide < kGroupThreads ? kGroupThreads / wide : 1;
  for (int k = 0; k < 2; ++k) {
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) mem[group * places + c * cols.hop + j * V + v] = k == 0 ? sw[c][v] : sb[c][v];
    __syncthreads();
    float s = 0.0f, rest = 0.0f;
    for (int col = threadIdx.x % wide; col < a.dim; col += kGroupThreads) {
      s = rest = 0.0f;
      for (int q = threadIdx.x / wide; q < groups; q += teams) {
        int at = col;
        if (EDGE) at += static_cast<int>((skew0 + (blockIdx.x * static_cast<long long>(groups) + q) % V * skew_step) % V);
        add_exactly(s, rest, mem[q * places + at]);
      }
      if (teams == 1) partial[(blockIdx.x * 2LL + k) * a.dim + col] = s + rest;
    }
    if (teams > 1) {
      __syncthreads();
      mem[threadIdx.x] = s + rest;
      for (int half = teams / 2; half > 0; half /= 2) {
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < half * wide) mem[threadIdx.x] += mem[threadIdx.x + half * wide];
      }
      if (static_cast<int>(threadIdx.x) < a.dim) partial[(blockIdx.x * 2LL + k) * a.dim + threadIdx.x] = mem[threadIdx.x];
    }
  }
}

// Rows that no cluster holds: the input's gradient, a CTA a row.
template <typename TI, typename TO>
__global__ void __launch_bounds__(kMostThreads)
    k_norm_grad_long(const __grid_constant__ mlt_norm_args a, const __grid_constant__ mlt_norm_grads g) {
  __shared__ RowSums<2> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  sums.clear();
  __syncthreads();
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TI* x = static_cast<const TI*>(a.x) + row * a.x_stride;
    const TO* gy = static_cast<const TO*>(g.gy) + row * g.gy_stride;
    const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
    auto weighted = [&](int i) {
      const float v = to_f32(gy[i]);
      return a.weight != nullptr ? v * load_as_f32(a.weight, a.w_dtype, i) : v;
    };
    float total[2] = {0.0f, 0.0f};
    for (int i = threadIdx.x; i < a.dim; i += kMostThreads) {
      const float v = weighted(i);
      total[0] += v;
      total[1] = fmaf(v, (to_f32(x[i]) - mean) * rstd, total[1]);
    }
    row_sums(total, sums, slot, 1, 0);
    const float m0 = total[0] / a.dim, m1 = total[1] / a.dim;
    for (int i = threadIdx.x; i < a.dim; i += kMostThreads) {
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
    add_exactly(sw, cw, gy * ((x - a.stats[2 * row]) * a.stats[2 * row + 1]));
    add_exactly(sb, cb, gy);
  }
  float* out = partial + blockIdx.y * 2LL * a.dim;
  out[col] = sw + cw;
  out[a.dim + col] = sb + cb;
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
    for (int t = y; t < teams; t += 32) add_exactly(sum, c, partial[(t * 2LL + blockIdx.y) * dim + col]);
  s[y][x] = sum + c;
  __syncthreads();
  float v[1] = {s[x][y]};
  warp_sums(v);
  if (x == 0 && blockIdx.x * 32 + y < dim) store_from_f32(to, dtype, blockIdx.x * 32 + y, v[0]);
}

struct Plan {
  bool far;  // rows that no cluster holds
  bool group;
  int lanes, threads, ranks, seg, flush;
  long long teams;  // of rows, and of partial sums
  size_t smem;
};

// Values of a row a thread: two packs where rows are read in packs of eight 16-bit values, else eight.
constexpr int each_of(int pack) { return pack == 8 ? 16 : 8; }

// By sizes and how the rows lie; the number of teams sets the order of the sums.
Plan plan_of(long long rows, int dim, int pack, bool edges, int period, bool scaled, int sms) {
  Plan p{};
  const int each = each_of(pack), places = (dim + (edges ? pack - 1 : 0) + pack - 1) / pack * pack;
  long long in_turn = 0;  // rows of a thread
  if (dim + pack > kNormMaxCluster * kMostThreads * each) {
    p.far = true;
    p.teams = (rows + kLongRows - 1) / kLongRows;
    if (p.teams > 256) p.teams = 256;
    return p;
  }
  if (places <= 32 * each) {
    p.group = true;
    p.lanes = 1;
    while (p.lanes * each < places) p.lanes *= 2;
    p.threads = kGroupThreads;
    p.ranks = 1;
    p.seg = places;
    const long long per = kGroupThreads / p.lanes, need = (rows + per - 1) / per, most = 2LL * sms;
    p.teams = need < most ? need : most;
    in_turn = (need + p.teams - 1) / p.teams;
  } else {
    p.ranks = (places + kMostThreads * each - 1) / (kMostThreads * each);
    p.seg = ((places + p.ranks - 1) / p.ranks + pack - 1) / pack * pack;
    p.ranks = (places + p.seg - 1) / p.seg;
    p.threads = p.lanes = ((p.seg + each - 1) / each + 31) / 32 * 32;
    int per_sm = 512 / p.threads;  // by registers
    if (per_sm > 16) per_sm = 16;
    long long most = static_cast<long long>(sms) * per_sm / p.ranks;
    most = most < period ? period : most / period * period;
    p.teams = rows < most ? rows : most;
    in_turn = (rows + p.teams - 1) / p.teams;
  }
  p.flush = in_turn > kPlainRows ? kFlushRows : 0;
  const size_t own = sizeof(float) * p.threads * each;
  p.smem = (p.group || !scaled ? 0 : own) + (p.flush > 0 ? 4 * own : 0);
  if (p.group && p.smem < own) p.smem = own;
  return p;
}

template <typename TI, typename TO, int V, bool EDGE>
cudaError_t launch_as(const mlt_norm_args& a, const mlt_norm_grads& g, const Plan& p, const Skew& skew, float* partial,
                      bool sums, cudaStream_t st) {
  constexpr int C = each_of(V) / V;
  const unsigned grid = static_cast<unsigned>(p.teams * p.ranks);
  auto go = [&](auto kernel) {
    return launch_cluster(kernel, grid, p.threads, p.ranks, p.smem, st, a, g, partial, p.lanes, p.seg, skew.first,
                          skew.step, p.flush);
  };
  if (p.group)
    return sums ? go(k_norm_grad<TI, TO, V, C, false, EDGE, true>) : go(k_norm_grad<TI, TO, V, C, false, EDGE, false>);
  return sums ? go(k_norm_grad<TI, TO, V, C, true, EDGE, true>) : go(k_norm_grad<TI, TO, V, C, true, EDGE, false>);
}

}  // namespace

size_t norm_grad_workspace(long long rows, int dim, int sms) {
  if (rows == 0) return 0;
  // whichever way the rows will lie
  long long most = 0;
  for (int pack : {1, 4, 8})
    for (int edges = 0; edges < 2; ++edges)
      for (int period = 1; period <= pack; period *= 2) {
        const long long teams = plan_of(rows, dim, pack, edges != 0, period, true, sms).teams;
        if (teams > most) most = teams;
      }
  return up256(static_cast<size_t>(most) * 2 * dim * sizeof(float));
}

cudaError_t launch_norm_grad(const mlt_norm_args& a, const mlt_norm_grads& g, void* ws, int sms, long long* launches,
                             cudaStream_t st) {
  float* partial = static_cast<float*>(ws);
  const bool sums = g.gweight != nullptr || g.gbias != nullptr;
  cudaError_t e = cudaSuccess;
  long long teams = 0;
  if (a.rows > 0)
    e = with_norm_types(a.dtype, a.y_dtype, [&](auto ti, auto to) -> cudaError_t {
      using TI = decltype(ti);
      using TO = decltype(to);
      constexpr int V = 16 / sizeof(TI);
      Skew skew;
      skew.add(a.x, a.x_stride, sizeof(TI), V);
      skew.add(g.gy, g.gy_stride, sizeof(TO), V);
      skew.add(g.g_total, g.g_total_stride, sizeof(TI), V);
      skew.add(g.gx, g.gx_stride, sizeof(TI), V);
      const bool edges = skew.same && skew.edges(a.dim, V);
      const Plan p = plan_of(a.rows, a.dim, skew.same ? V : 1, edges, skew.same ? skew.period(V) : 1,
                             a.weight != nullptr, sms);
      teams = p.teams;
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
        const long long most = 4LL * sms;
        ++*launches;
        return launch_cluster(k_norm_grad_long<TI, TO>, static_cast<unsigned>(a.rows < most ? a.rows : most), kMostThreads,
                              1, 0, st, a, g);
      }
      ++*launches;
      if (!skew.same) return launch_as<TI, TO, 1, false>(a, g, p, Skew{true, 0, 0}, partial, sums, st);
      return edges ? launch_as<TI, TO, V, true>(a, g, p, skew, partial, sums, st)
                   : launch_as<TI, TO, V, false>(a, g, p, skew, partial, sums, st);
    });
  if (e != cudaSuccess || !sums) return e;
  ++*launches;
  return launch_pdl(k_norm_cols, dim3((a.dim + 31) / 32, 2), dim3(1024), 0, st, static_cast<const float*>(partial),
                    static_cast<int>(teams), a.dim, g.gweight, g.gbias, a.w_dtype);
}

}  // namespace mlt
