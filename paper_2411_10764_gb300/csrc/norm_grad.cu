// Gradients of layer norm: of its input row by row, of weight and bias as sums over all rows.
//
// With h = (t - mean) rstd and gw = gy weight, two sums over the row (gw and gw h) give the
// input's gradient.  Each thread keeps its columns' sums of gy h and gy in registers over
// all rows of its team; the teams' sums go to the workspace and a second
// kernel adds them up in a fixed order.  Bound: memory (x and gy read, gx written, once), and
// instructions and latency: 32,768 x 2,048 bf16 with g_total 97 us, 5.5 TB/s, at 52 % of the issue slots (27
// instructions a value, two-wide where they can be; the sums' 32 registers leave 15 warps an SM);
// 1,048,573 x 61 fp32 155 us, 4.9 TB/s.
// Of n equal terms in a plain sum the error grows with n: where a thread has more than kPlainRows rows, every
// so many its sums move on to pairs of numbers in the workspace (Knuth's exact addition), 32 bytes a
// column that stay in L2.  (In shared memory they halved the warps that fit.)
// Rows are on their way two ahead, in shared memory: in registers, one ahead, 32,768 x 2,048 took 145 us for 104.
#include <utility>

#include "norm.cuh"

namespace mlt {
namespace {

constexpr int kPlainRows = 48;
constexpr int kMostThreads = 512;
constexpr int kGroupThreads = 256;

// (s, c) + v, s + c being the sum
__device__ __forceinline__ void add_exactly(float& s, float& c, float v) {
  const float t = __fadd_rn(s, v), b = __fsub_rn(t, s);
  c = __fadd_rn(c, __fadd_rn(__fsub_rn(s, __fsub_rn(t, b)), __fsub_rn(v, b)));
  s = t;
}

// The fewest without spills of consequence.
constexpr int registers(bool cta, int pack) {
  if (!cta) return 128;
  return pack == 8 ? 128 : 96;
}

// As k_norm in norm.cu.  SUMS: weight and bias have gradients; partial: [teams][2][dim]; moved: for long sums
// [CTAs][4][E][threads], else null.
template <typename TI, typename TO, int V, int C, bool CTA, bool EDGE, bool SUMS>
__global__ void __maxnreg__(registers(CTA, V))
    k_norm_grad(const __grid_constant__ mlt_norm_args a, const __grid_constant__ mlt_norm_grads g, float* partial,
                float* moved, int lanes, int skew0, int skew_step) {
  extern __shared__ __align__(16) float mem[];
  __shared__ RowSums<2> sums;
  constexpr int E = C * V;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  const int j = CTA ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int in_warp = CTA ? 1 : 32 / lanes;
  const long long step = CTA ? gridDim.x : static_cast<long long>(gridDim.x) * 8 * in_warp;
  const int sub = CTA ? 0 : (threadIdx.x & 31) / lanes;
  const long long base0 = CTA ? blockIdx.x : (blockIdx.x * 8LL + (threadIdx.x >> 5)) * in_warp;
  const int skew = EDGE ? static_cast<int>((skew0 + (base0 + sub) % V * skew_step) % V) : 0;
  const Columns<V, C, EDGE> cols(j * V, lanes * V, skew, a.dim);
  const bool scaled = a.weight != nullptr;
  const Kept<V, C> ws{mem};
  float w[C][V];
  float2 sw[E / 2], sb[E / 2];
  const bool more = g.g_total != nullptr;
  const float inv_dim = 1.0f / a.dim;
  const TI *x0 = static_cast<const TI*>(a.x), *t0 = static_cast<const TI*>(g.g_total);
  const TO* g0 = static_cast<const TO*>(g.gy);
  const TI *x1 = x0 + (a.rows - 1) * a.x_stride + a.dim, *t1 = t0 + (a.rows - 1) * g.g_total_stride + a.dim;
  const TO* g1 = g0 + (a.rows - 1) * g.gy_stride + a.dim;
  // rows ahead: a CTA's packs in shared memory, two rows of them; else in registers, one (short rows of 61 fp32
  // values 149 us so, 173 through shared memory)
  constexpr bool kInRing = CTA && V > 1;
  const Ring<V, C> ring{reinterpret_cast<unsigned char*>(scaled ? mem + blockDim.x * E : mem)};
  Vec<TI, V> px[C], pt[C];
  Vec<TO, V> pg[C];
  float2 next = make_float2(0.0f, 0.0f);
  auto fetch = [&](long long row, int stage) {
    if constexpr (kInRing) {
      if (row < a.rows) {
        ring.fetch(cols, stage, 0, x0 + row * a.x_stride, x0, x1);
        ring.fetch(cols, stage, 1, g0 + row * g.gy_stride, g0, g1);
        if (more) ring.fetch(cols, stage, 2, t0 + row * g.g_total_stride, t0, t1);
        ring.template copy<8>(ring.pair(stage), a.stats + 2 * row);
      }
      ring.commit();
    } else if (row < a.rows) {
      cols.load(px, x0 + row * a.x_stride, x0, x1);
      cols.load(pg, g0 + row * g.gy_stride, g0, g1);
      next = *reinterpret_cast<const float2*>(a.stats + 2 * row);
    }
  };
  fetch(base0 + sub, 0);
  if (kInRing)
#pragma unroll
    for (int d = 1; d < kAhead - 1; ++d) fetch(base0 + sub + d * step, d);
  if (!CTA || scaled) {
    load_columns(w, cols, a.weight, a.w_dtype, 1.0f);
    if (CTA) ws.put(w);
  }
#pragma unroll
  for (int i = 0; i < E / 2; ++i) sw[i] = sb[i] = both(0.0f);
  if (CTA) sums.clear();
  __syncthreads();
  float* own = moved + blockIdx.x * 4LL * E * blockDim.x + threadIdx.x;
  const int hop = E * blockDim.x;
  bool first_move = true;
  auto move = [&]() {
    if constexpr (SUMS) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float* at = own + (c * V + v) * blockDim.x;
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (!first_move)
#pragma unroll
          for (int k = 0; k < 4; ++k) s[k] = at[k * hop];
        add_exactly(s[0], s[1], one_of(sw, c * V + v));
        add_exactly(s[2], s[3], one_of(sb, c * V + v));
#pragma unroll
        for (int k = 0; k < 4; ++k) at[k * hop] = s[k];
        one_of(sw, c * V + v) = one_of(sb, c * V + v) = 0.0f;
      }
    }
    first_move = false;
  };
  int since = 0, stage = 0;
  for (long long base = base0; base < a.rows; base += step) {
    const long long row = base + sub;
    const bool live = row < a.rows;
    if constexpr (kInRing) {
      fetch(row + (kAhead - 1) * step, stage == 0 ? kAhead - 1 : stage - 1);
      ring.wait_oldest();
      next = *ring.pair(stage);
    } else if (more && live) {
      cols.load(pt, t0 + row * g.g_total_stride, t0, t1);
    }
    const float mean = next.x, rstd = next.y;
    if constexpr (kInRing)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        px[c] = ring.template get<TI>(stage, 0, c);
        pg[c] = ring.template get<TO>(stage, 1, c);
      }
    if (CTA && scaled)
#pragma unroll
      for (int c = 0; c < C; ++c) ws.get(w[c], c);
    float2 h[E / 2], gw[E / 2], s0 = both(0.0f), s1 = both(0.0f);
    cols.template pairs<CTA>([&](int i, bool on0, bool on1) {
      const bool all = CTA || live;
      const float2 x = __fmul2_rn(__fadd2_rn(two_of(px, i), both(-mean)), both(rstd));
      h[i / 2] = masked(x, on0 && all, on1 && all);
      const float2 gy = masked(two_of(pg, i), on0 && all, on1 && all);
      if (SUMS) {
        sw[i / 2] = __ffma2_rn(gy, h[i / 2], sw[i / 2]);
        sb[i / 2] = __fadd2_rn(sb[i / 2], gy);
      }
      gw[i / 2] = !CTA || scaled ? __fmul2_rn(gy, two_of(w, i)) : gy;
      s0 = __fadd2_rn(s0, gw[i / 2]);
      s1 = __ffma2_rn(gw[i / 2], h[i / 2], s1);
    });
    float total[2] = {s0.x + s0.y, s1.x + s1.y};
    if (!kInRing && base + step < a.rows) fetch(row + step, 0);
    if (CTA)
      row_sums(total, sums, slot);
    else
      group_sums(total, lanes);
    if (SUMS && moved != nullptr && ++since == kPlainRows) {
      move();
      since = 0;
    }
    const int now = stage;
    stage = stage == kAhead - 1 ? 0 : stage + 1;
    if (g.gx == nullptr || !live) continue;
    const float m0 = total[0] * inv_dim, m1 = total[1] * inv_dim;
    TI* to = static_cast<TI*>(g.gx) + row * g.gx_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (kInRing) {
        if (more) pt[c] = ring.template get<TI>(now, 2, c);
      }
      float f[V];
      auto value = [&](int i) {
        const float2 d = __fmul2_rn(__ffma2_rn(h[i / 2], both(-m1), __fadd2_rn(gw[i / 2], both(-m0))), both(rstd));
        return more ? __fadd2_rn(d, two_of(pt, i)) : d;
      };
      if constexpr (V == 1) {
        const float2 d = value(c & ~1);
        f[0] = c & 1 ? d.y : d.x;
      } else {
#pragma unroll
        for (int v = 0; v < V; v += 2) {
          const float2 d = value(c * V + v);
          f[v] = d.x;
          f[v + 1] = d.y;
        }
      }
      Vec<TI, V> q;
      q.put(f);
      cols.store(q, to, c);
    }
  }
  if (!SUMS) return;
  if (moved != nullptr && !first_move) {
    move();
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float* at = own + (c * V + v) * blockDim.x;
        one_of(sw, c * V + v) = at[0] + at[hop];
        one_of(sb, c * V + v) = at[2 * hop] + at[3 * hop];
      }
  }
  if (CTA) {
    float* out = partial + blockIdx.x * 2LL * a.dim;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (cols.on(c, v)) {
          const int col = cols.first + c * cols.hop + v;
          out[col] = one_of(sw, c * V + v);
          out[a.dim + col] = one_of(sb, c * V + v);
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
      for (int v = 0; v < V; ++v) mem[group * places + c * cols.hop + j * V + v] = k == 0 ? one_of(sw, c * V + v) : one_of(sb, c * V + v);
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

// Rows that a CTA's registers do not hold: the input's gradient, a CTA a row, which it reads twice, the second time
// out of L2.
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(kMostThreads, 2)
    k_norm_grad_long(const __grid_constant__ mlt_norm_args a, const __grid_constant__ mlt_norm_grads g, int skew0,
                     int skew_step) {
  __shared__ RowSums<2> sums;
  int slot = 0;
  pdl_wait();
  pdl_trigger();
  sums.clear();
  __syncthreads();
  const TI *x0 = static_cast<const TI*>(a.x), *t0 = static_cast<const TI*>(g.g_total);
  const TO* g0 = static_cast<const TO*>(g.gy);
  const float inv_dim = 1.0f / a.dim;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int skew = static_cast<int>((skew0 + row % V * skew_step) % V);
    const TI *x = x0 + row * a.x_stride, *t = t0 + row * g.g_total_stride;
    const TO* gy = g0 + row * g.gy_stride;
    TI* to = static_cast<TI*>(g.gx) + row * g.gx_stride;
    const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
    const float mean = st.x, rstd = st.y;
    float total[2] = {0.0f, 0.0f};
#pragma unroll 4
    for (int col = static_cast<int>(threadIdx.x) * V - skew; col < a.dim; col += kMostThreads * V) {
      float h[V], gw[V], w[V];
      load_some<V>(h, x, col, a.dim);
      load_some<V>(gw, gy, col, a.dim);
      load_weights<V>(w, a.weight, a.w_dtype, col, a.dim, 1.0f);
      float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float p = gw[v] * w[v];
        s0 += p;
        s1 = fmaf(p, (h[v] - mean) * rstd, s1);
      }
      total[0] += s0;
      total[1] += s1;
    }
    row_sums(total, sums, slot);
    const float m0 = total[0] * inv_dim, m1 = total[1] * inv_dim;
#pragma unroll 2
    for (int col = static_cast<int>(threadIdx.x) * V - skew; col < a.dim; col += kMostThreads * V) {
      float h[V], gw[V], w[V], f[V];
      load_some<V>(h, x, col, a.dim);
      load_some<V>(gw, gy, col, a.dim);
      load_weights<V>(w, a.weight, a.w_dtype, col, a.dim, 1.0f);
      if (g.g_total != nullptr)
        load_some<V>(f, t, col, a.dim);
      else
#pragma unroll
        for (int v = 0; v < V; ++v) f[v] = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v)
        f[v] = fmaf(-(h[v] - mean) * rstd, m1, gw[v] * w[v] - m0) * rstd + f[v];
      store_some<V>(f, to, col, a.dim);
    }
  }
}

// Their columns' sums: a thread a pack of columns, `per` rows.
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256)
    k_norm_cols_long(const __grid_constant__ mlt_norm_args a, const __grid_constant__ mlt_norm_grads g, float* partial,
                     long long per) {
  pdl_wait();
  pdl_trigger();
  const int col = (blockIdx.x * 256 + threadIdx.x) * V;
  if (col >= a.dim) return;
  const long long from = blockIdx.y * per, to = min(static_cast<long long>(a.rows), from + per);
  float sw[V], cw[V], sb[V], cb[V];
#pragma unroll
  for (int v = 0; v < V; ++v) sw[v] = cw[v] = sb[v] = cb[v] = 0.0f;
#pragma unroll 4
  for (long long row = from; row < to; ++row) {
    float gy[V], x[V];
    load_some<V>(gy, static_cast<const TO*>(g.gy) + row * g.gy_stride, col, a.dim);
    load_some<V>(x, static_cast<const TI*>(a.x) + row * a.x_stride, col, a.dim);
    const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      add_exactly(sw[v], cw[v], gy[v] * ((x[v] - st.x) * st.y));
      add_exactly(sb[v], cb[v], gy[v]);
    }
  }
  float* out = partial + blockIdx.y * 2LL * a.dim;
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (col + v < a.dim) {
      out[col + v] = sw[v] + cw[v];
      out[a.dim + col + v] = sb[v] + cb[v];
    }
}

// The teams' sums of 16 columns: 64 threads a column take every 64th team, then a tree.
constexpr int kColumns = 16;
__global__ void __launch_bounds__(1024)
    k_norm_cols(const float* partial, int teams, int dim, void* gweight, void* gbias, int dtype) {
  __shared__ float s[64][kColumns + 1];
  pdl_wait();
  pdl_trigger();
  const int x = threadIdx.x % kColumns, y = threadIdx.x / kColumns, col = blockIdx.x * kColumns + x;
  void* to = blockIdx.y == 0 ? gweight : gbias;
  if (to == nullptr) return;
  float sum = 0.0f, c = 0.0f;
  if (col < dim)
#pragma unroll 8
    for (int t = y; t < teams; t += 64) add_exactly(sum, c, partial[(t * 2LL + blockIdx.y) * dim + col]);
  s[y][x] = sum + c;
  __syncthreads();
  const int lane = threadIdx.x & 31, of = threadIdx.x >> 5;
  if (of >= kColumns) return;
  float v[1] = {s[lane][of] + s[lane + 32][of]};
  warp_sums(v);
  if (lane == 0 && blockIdx.x * kColumns + of < dim) store_from_f32(to, dtype, blockIdx.x * kColumns + of, v[0]);
}

struct Plan {
  bool far;  // rows that registers do not hold
  bool group;
  int lanes, threads;
  long long teams;  // of rows, and of partial sums
  size_t smem, off_moved, bytes;
};

// Values of a row a thread: two packs, or eight single ones; of 16-bit rows that groups of lanes take one pack,
// beside whose sums and weights registers have no room for another.
constexpr int each_of(int pack, bool group) { return pack == 8 && !group ? 16 : 8; }

// By sizes and how the rows lie; the number of teams sets the order of the sums.
Plan plan_of(long long rows, int dim, int pack, bool edges, int period, bool scaled, int sms) {
  Plan p{};
  const int places = (dim + (edges ? pack - 1 : 0) + pack - 1) / pack * pack;
  auto finish = [&](long long moved_floats) {
    p.off_moved = up256(sizeof(float) * p.teams * 2 * dim);
    p.bytes = p.off_moved + up256(sizeof(float) * moved_floats);
    if (moved_floats == 0) p.off_moved = 0;
    return p;
  };
  const bool group = places <= 32 * each_of(pack, true);
  const int each = each_of(pack, group);
  if (places > kMostThreads * each) {
    p.far = true;
    // six CTAs an SM over the columns' sums
    const long long wide = (dim + 256 * pack - 1) / (256 * pack), fill = (6LL * sms + wide - 1) / wide;
    p.teams = rows < fill ? rows : fill;
    return finish(0);
  }
  if (group) {
    p.group = true;
    p.lanes = 1;
    while (p.lanes * each < places) p.lanes *= 2;
    p.threads = kGroupThreads;
  } else {
    p.threads = p.lanes = ((places + each - 1) / each + 31) / 32 * 32;
  }
  // weights and rows ahead; at the end of short rows the sums by place
  const size_t own = sizeof(float) * p.threads * each;
  p.smem = (p.group || !scaled ? 0 : own) + (p.group || pack == 1 ? 0 : p.threads * static_cast<size_t>(Ring<8, 2>::kBytes));
  if (p.group && p.smem < own) p.smem = own;
  int per_sm = 65536 / registers(!p.group, pack) / p.threads;
  const int by_smem = static_cast<int>(227 * 1024 / (p.smem + 2048));
  if (per_sm > by_smem) per_sm = by_smem;
  per_sm = per_sm < 1 ? 1 : per_sm > 16 ? 16 : per_sm;
  const long long most_ctas = static_cast<long long>(sms) * per_sm;
  const long long in_turn_rows = p.group ? kGroupThreads / p.lanes : 1, need = (rows + in_turn_rows - 1) / in_turn_rows;
  long long most = most_ctas;
  if (!p.group) most = most < period ? period : most / period * period;
  p.teams = need < most ? need : most;
  const bool move = (need + p.teams - 1) / p.teams > kPlainRows;
  return finish(move ? p.teams * 4LL * each * p.threads : 0);
}

template <typename TI, typename TO, int V, bool EDGE>
cudaError_t launch_as(const mlt_norm_args& a, const mlt_norm_grads& g, const Plan& p, const Skew& skew, float* partial,
                      bool sums, cudaStream_t st) {
  float* moved = sums && p.off_moved > 0 ? partial + p.off_moved / sizeof(float) : nullptr;
  constexpr int GC = each_of(V, true) / V, CC = each_of(V, false) / V;
  const unsigned grid = static_cast<unsigned>(p.teams);
  auto go = [&](auto kernel) {
    return launch_rows(kernel, grid, p.threads, p.smem, st, a, g, partial, moved, p.lanes, skew.first, skew.step);
  };
  if (p.group)
    return sums ? go(k_norm_grad<TI, TO, V, GC, false, EDGE, true>) : go(k_norm_grad<TI, TO, V, GC, false, EDGE, false>);
  return sums ? go(k_norm_grad<TI, TO, V, CC, true, EDGE, true>) : go(k_norm_grad<TI, TO, V, CC, true, EDGE, false>);
}

}  // namespace

size_t norm_grad_workspace(long long rows, int dim, int sms) {
  if (rows == 0) return 0;
  // whichever way the rows will lie
  size_t most = 0;
  for (int pack : {1, 4, 8})
    for (int edges = 0; edges < 2; ++edges)
      for (int period = 1; period <= pack; period *= 2)
        for (int scaled = 0; scaled < 2; ++scaled) {
          const size_t n = plan_of(rows, dim, pack, edges != 0, period, scaled != 0, sms).bytes;
          if (n > most) most = n;
        }
  return most;
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
        auto both = [&](auto pack, const Skew& k) -> cudaError_t {
          constexpr int P = decltype(pack)::value;
          // the sums first: gx may be written over gy
          if (sums) {
            ++*launches;
            // columns keep their places in packs only where rows begin at boundaries
            auto columns = [&](auto width) {
              constexpr int W = decltype(width)::value;
              return launch_pdl(k_norm_cols_long<TI, TO, W>,
                                dim3((a.dim + 256 * W - 1) / (256 * W), static_cast<unsigned>(p.teams)), dim3(256), 0, st, a,
                                g, partial, (a.rows + p.teams - 1) / p.teams);
            };
            const cudaError_t r = k.first == 0 && k.step == 0 ? columns(pack) : columns(std::integral_constant<int, 1>());
            if (r != cudaSuccess) return r;
          }
          if (g.gx == nullptr) return cudaSuccess;
          const long long most = 2LL * sms;
          ++*launches;
          return launch_rows(k_norm_grad_long<TI, TO, P>, static_cast<unsigned>(a.rows < most ? a.rows : most), kMostThreads,
                             0, st, a, g, k.first, k.step);
        };
        return skew.same ? both(std::integral_constant<int, V>(), skew)
                         : both(std::integral_constant<int, 1>(), Skew{true, 0, 0});
      }
      ++*launches;
      if (!skew.same) return launch_as<TI, TO, 1, false>(a, g, p, Skew{true, 0, 0}, partial, sums, st);
      return edges ? launch_as<TI, TO, V, true>(a, g, p, skew, partial, sums, st)
                   : launch_as<TI, TO, V, false>(a, g, p, skew, partial, sums, st);
    });
  if (e != cudaSuccess || !sums) return e;
  ++*launches;
  return launch_pdl(k_norm_cols, dim3((a.dim + kColumns - 1) / kColumns, 2), dim3(1024), 0, st, static_cast<const float*>(partial),
                    static_cast<int>(teams), a.dim, g.gweight, g.gbias, a.w_dtype);
}

}  // namespace mlt
