// Selective scan with its short causal convolution: prompts and single tokens.
//
//   h_t = exp(d_t A) h_(t-1) + d_t u_t B_t,   y_t = (C_t . h_t + skip u_t) silu(z_t)
//   u = silu(causal convolution of x), d = softplus(dt + dt_bias)
//
// Prompts.  The recurrence is sequential in t and independent over channels and
// states.  Where sequences x channels fill the GPU, one CTA walks a sequence's
// 64 channels from start to end: inputs are read once, states stay in registers.  Where
// they do not, sequences are cut into chunks: since A does not depend on t, a
// chunk acts on a state as h -> exp(A sum d) h + e, with e its end state from zero.
//   k_scan_local  e and sum d of every chunk but the last
//   k_scan_carry  the state before each chunk
//   k_scan_main   the outputs of each chunk from the state before it
// which evaluates the exponentials twice.
//
// Single tokens (length 1).  Bound by reading and writing the states: k_scan_step.
#include "scan.cuh"

namespace mlt {
namespace {

using namespace scan;

struct Plan {
  Chunks cut;
  size_t off_e, off_sum, bytes;
};

// ---------------------------------------------------------------------------
// Prompts
// ---------------------------------------------------------------------------
template <int S>
struct alignas(16) Tile {
  float2 push[kTile][kChannels];  // (d, d u)
  float2 out[kTile][kChannels];   // (skip u, gate)
  float y[kTile][kChannels + 4];
  float B[kTile * 4 * S];
  float C[kTile * 4 * S];
};

template <typename T>
struct Raw {
  Window<T> x;
  Pack<T, kPackC> dt, z;
};

template <typename T, bool kVec, bool kOut>
__device__ __forceinline__ void load_raw(const mlt_scan_args& a, const Block& k, long long t, long long end, int c,
                                         Raw<T>& r) {
  if (t >= end) return;
  r.x = load_window<T, kVec>(a, k, t, c);
  r.dt = load_pack<T, kVec>(static_cast<const T*>(a.dt) + k.b * a.dt_batch + t * a.dt_step + k.c0, c, k.cn);
  if (kOut && a.z != nullptr)
    r.z = load_pack<T, kVec>(static_cast<const T*>(a.z) + k.b * a.z_batch + t * a.z_step + k.c0, c, k.cn);
}

// One thread's pack of the tile: (d, d u) and, for the outputs, (skip u, gate).
template <typename T, int S, bool kOut>
__device__ __forceinline__ void stage(const mlt_scan_args& a, const Raw<T>& r, const Taps& taps, const float* bias,
                                      const float* skip, bool live, int t, int c, int cn, Tile<S>& tile) {
#pragma unroll
  for (int e = 0; e < kPackC; ++e) {
    float2 p = make_float2(0.0f, 0.0f), o = make_float2(0.0f, 0.0f);
    if (live && c + e < cn) {
      const float v = conv_at(a, taps, r.x, e);
      const float u = a.taps > 0 ? v * sigmoid(v) : v;
      const float d = softplus(to_f32(r.dt.v[e]) + bias[e]);
      p = make_float2(d, d * u);
      if (kOut) {
        o.x = skip[e] * u;
        o.y = 1.0f;
        if (a.z != nullptr) {
          const float z = to_f32(r.z.v[e]);
          o.y = z * sigmoid(z);
        }
      }
    }
    tile.push[t][c + e] = p;
    if (kOut) tile.out[t][c + e] = o;
  }
}

// kOut: writes y and the last state; otherwise a chunk's end state from zero and sum of steps.
template <typename T, int S, bool kVec, bool kOut>
__global__ void __launch_bounds__(kThreads) k_scan(mlt_scan_args a, Plan p, unsigned char* ws) {
  extern __shared__ __align__(16) unsigned char smem[];
  Tile<S>& tile = *reinterpret_cast<Tile<S>*>(smem);
  pdl_wait();
  pdl_trigger();
  const Block k = block_of(a, blockIdx.x, blockIdx.y);
  const int chunk = blockIdx.z;
  const long long len = length_of(a, k.b);
  const long long begin = chunk * p.cut.chunk, stop = min(begin + p.cut.chunk, static_cast<long long>(a.length));
  const long long end = min(stop, len);  // positions begin .. end - 1 count
  // a lane's channel and states
  const int lane = threadIdx.x & 3, ch = threadIdx.x >> 2;
  const bool in = ch < k.cn;
  const long long at = static_cast<long long>(k.c0 + ch) * a.states + lane * S;
  const long long of_seq = static_cast<long long>(a.dim) * a.states;
  // a thread's place in staging
  const int st = threadIdx.x / (kChannels / kPackC), sc = threadIdx.x % (kChannels / kPackC) * kPackC;
  const Taps taps = load_taps(a, k, sc);
  float bias[kPackC], skip[kPackC];
#pragma unroll
  for (int e = 0; e < kPackC; ++e) {
    const bool ok = sc + e < k.cn;
    bias[e] = ok && a.dt_bias != nullptr ? a.dt_bias[k.c0 + sc + e] : 0.0f;
    skip[e] = ok && a.skip != nullptr ? a.skip[k.c0 + sc + e] : 0.0f;
  }
  Lane<S> A = lane_zero<S>(), h = lane_zero<S>();
  if (in) {
    A = lane_load<S>(a.A + at, lane * S, a.states);
    const float* from = p.cut.chunks > 1 ? (kOut ? reinterpret_cast<const float*>(ws + p.off_e) +
                                                       (static_cast<long long>(k.b) * p.cut.chunks + chunk) * of_seq
                                                 : nullptr)
                                         : (a.state != nullptr ? a.state + k.b * of_seq : nullptr);
    if (from != nullptr) h = lane_load<S>(from + at, lane * S, a.states);
  }
#pragma unroll
  for (int q = 0; q < Lane<S>::H; ++q) A.v[q] = mul2(A.v[q], f2(kLog2E, kLog2E));
  const T* Bp = static_cast<const T*>(a.B) + k.b * a.B_batch + static_cast<long long>(k.g) * a.states;
  const T* Cp = static_cast<const T*>(a.C) + k.b * a.C_batch + static_cast<long long>(k.g) * a.states;
  float sum = 0.0f;
  Raw<T> raw;
  load_raw<T, kVec, kOut>(a, k, begin + st, end, sc, raw);
  for (long long t0 = begin; t0 < stop; t0 += kTile) {
    const int live = static_cast<int>(min(static_cast<long long>(kTile), max(0ll, end - t0)));
    T* yrow = kOut ? static_cast<T*>(a.y) + k.b * a.y_batch + (t0 + st) * a.y_step + k.c0 : nullptr;
    if (live == 0) {
      if (!kOut) break;
      Pack<T, kPackC> zero;
#pragma unroll
      for (int e = 0; e < kPackC; ++e) zero.v[e] = from_f32<T>(0.0f);
      if (t0 + st < stop) store_pack<T, kVec>(yrow, sc, k.cn, zero);
      continue;
    }
    stage<T, S, kOut>(a, raw, taps, bias, skip, st < live, st, sc, k.cn, tile);
    stage_rows<T, S>(tile.B, Bp + t0 * a.B_step, a.B_step, a.states, live);
    if (kOut) stage_rows<T, S>(tile.C, Cp + t0 * a.C_step, a.C_step, a.states, live);
    load_raw<T, kVec, kOut>(a, k, t0 + kTile + st, end, sc, raw);  // lands behind the walk
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTile; t += 4) {
      float y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 d = tile.push[t + q][ch];
        const Lane<S> B = lane_shared<S>(tile.B + ((t + q) * 4 + lane) * S);
        const F2 step = f2(d.x, d.x), push = f2(d.y, d.y);
#pragma unroll
        for (int s = 0; s < Lane<S>::H; ++s)
          h.v[s] = fma2(ex2_2(mul2(step, A.v[s])), h.v[s], mul2(push, B.v[s]));
        if (kOut) {
          const Lane<S> C = lane_shared<S>(tile.C + ((t + q) * 4 + lane) * S);
          Lane<S> o;
#pragma unroll
          for (int s = 0; s < Lane<S>::H; ++s) o.v[s] = mul2(C.v[s], h.v[s]);
          y[q] = lane_sum(o);
        } else {
          sum += d.x;
        }
      }
      if (kOut) tile.y[t + lane][ch] = quad_sums(y, lane);
    }
    __syncthreads();
    if (kOut && t0 + st < stop) {
      Pack<T, kPackC> o;
#pragma unroll
      for (int e = 0; e < kPackC; ++e) {
        const float2 q = tile.out[st][sc + e];
        o.v[e] = from_f32<T>((tile.y[st][sc + e] + q.x) * q.y);
      }
      store_pack<T, kVec>(yrow, sc, k.cn, o);
    }
  }
  if (!kOut) {
    if (in) {
      const long long seq = static_cast<long long>(k.b) * p.cut.chunks + chunk;
      lane_store<S>(reinterpret_cast<float*>(ws + p.off_e) + seq * of_seq + at, lane * S, a.states, h);
      if (lane == 0) reinterpret_cast<float*>(ws + p.off_sum)[seq * a.dim + k.c0 + ch] = sum;
    }
    return;
  }
  if (in && a.state_out != nullptr && chunk == p.cut.chunks - 1)
    lane_store<S>(a.state_out + k.b * of_seq + at, lane * S, a.states, h);
  // the inputs before the sequence's end (chunk 0 is the only reader of conv_state, and has read it)
  if (chunk == 0 && a.conv_state_out != nullptr) {
    __syncthreads();
    const int c = threadIdx.x;
    if (c < k.cn) {
      T* out = static_cast<T*>(a.conv_state_out) + static_cast<long long>(k.b) * (a.taps - 1) * a.dim + k.c0 + c;
      const T* old = static_cast<const T*>(a.conv_state) + static_cast<long long>(k.b) * (a.taps - 1) * a.dim + k.c0 + c;
      const T* x = static_cast<const T*>(a.x) + k.b * a.x_batch + k.c0 + c;
      for (int j = 0; j < a.taps - 1; ++j) {
        const long long i = len + j;  // counted from taps - 1 before the start
        T v = from_f32<T>(0.0f);
        if (i >= a.taps - 1) v = x[(i - (a.taps - 1)) * a.x_step];
        else if (a.conv_state != nullptr) v = old[i * a.dim];
        out[static_cast<long long>(j) * a.dim] = v;
      }
    }
  }
}

// The state before each chunk, in the place of the chunk's end state from zero.
__global__ void __launch_bounds__(256) k_scan_carry(mlt_scan_args a, Plan p, unsigned char* ws) {
  pdl_wait();
  pdl_trigger();
  const long long of_seq = static_cast<long long>(a.dim) * a.states;
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= of_seq) return;
  const int b = blockIdx.y;
  float* e = reinterpret_cast<float*>(ws + p.off_e) + static_cast<long long>(b) * p.cut.chunks * of_seq + i;
  const float* sum = reinterpret_cast<const float*>(ws + p.off_sum) + static_cast<long long>(b) * p.cut.chunks * a.dim +
                     i / a.states;
  const float A = a.A[i] * kLog2E;
  float h = a.state != nullptr ? a.state[b * of_seq + i] : 0.0f;
  const int last = p.cut.chunks - 1;
#pragma unroll 8
  for (int c = 0; c < last; ++c) {
    const float end = e[c * of_seq];
    const float decay = ex2(A * sum[static_cast<long long>(c) * a.dim]);
    e[c * of_seq] = h;
    h = fmaf(decay, h, end);
  }
  e[last * of_seq] = h;
}

// ---------------------------------------------------------------------------
// Single tokens
// ---------------------------------------------------------------------------
// A warp has 32 channels: as lanes first (convolution, step size, gate), then eight at a
// time with four lanes each for the states, whose loads are under way from the start.
template <typename T, int S, bool kWide>
__global__ void __launch_bounds__(256) k_scan_step(mlt_scan_args a) {
  const int lane = threadIdx.x & 31, sub = lane & 3, quad = lane >> 2;
  const int b = blockIdx.y;
  const int width = a.dim / a.groups, per = (width + 31) / 32;
  const int block = blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_wait();
  pdl_trigger();
  if (block >= per * a.groups) return;
  const int g = block / per, first = (block - g * per) * 32;
  const int c0 = g * width + first, cn = min(32, width - first);
  const bool live = length_of(a, b) > 0;
  const long long of_seq = static_cast<long long>(a.dim) * a.states;
  Lane<S> h[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int ch = k * 8 + quad;
    h[k] = lane_zero<S>();
    if (ch < cn && a.state != nullptr) {
      const float* p = a.state + b * of_seq + static_cast<long long>(c0 + ch) * a.states + sub * S;
      h[k] = kWide ? lane_shared<S>(p) : lane_load<S>(p, sub * S, a.states);
    }
  }
  const int c = c0 + lane;
  const bool in = lane < cn;
  float d = 0.0f, push = 0.0f, add = 0.0f, gate = 0.0f;
  if (in) {
    const T zero = from_f32<T>(0.0f);
    const T x = live ? static_cast<const T*>(a.x)[b * a.x_batch + c] : zero;
    T old[kScanMaxTaps - 1];
    const long long cs = static_cast<long long>(b) * (a.taps - 1) * a.dim + c;
#pragma unroll
    for (int j = 0; j < kScanMaxTaps - 1; ++j)
      old[j] = j < a.taps - 1 && a.conv_state != nullptr
                   ? static_cast<const T*>(a.conv_state)[cs + static_cast<long long>(j) * a.dim]
                   : zero;
    if (a.conv_state_out != nullptr) {
#pragma unroll
      for (int j = 0; j < kScanMaxTaps - 1; ++j)
        if (j < a.taps - 1) {
          T v = old[j];
          if (live) v = j + 1 < a.taps - 1 ? old[j + 1 < kScanMaxTaps - 1 ? j + 1 : j] : x;
          static_cast<T*>(a.conv_state_out)[cs + static_cast<long long>(j) * a.dim] = v;
        }
    }
    if (live) {
      float u = to_f32(x);
      if (a.taps > 0) {
        const float* w = a.conv_w + static_cast<long long>(c) * a.taps;
        float v = fmaf(w[a.taps - 1], u, a.conv_b != nullptr ? a.conv_b[c] : 0.0f);
#pragma unroll
        for (int j = 0; j < kScanMaxTaps - 1; ++j)
          if (j < a.taps - 1) v = fmaf(w[j], to_f32(old[j]), v);
        u = v * sigmoid(v);
      }
      d = softplus(to_f32(static_cast<const T*>(a.dt)[b * a.dt_batch + c]) +
                   (a.dt_bias != nullptr ? a.dt_bias[c] : 0.0f));
      push = d * u;
      add = a.skip != nullptr ? a.skip[c] * u : 0.0f;
      gate = 1.0f;
      if (a.z != nullptr) {
        const float z = to_f32(static_cast<const T*>(a.z)[b * a.z_batch + c]);
        gate = z * sigmoid(z);
      }
    }
  }
  float Bs[2 * Lane<S>::H], Cs[2 * Lane<S>::H];
  const T* Bp = static_cast<const T*>(a.B) + b * a.B_batch + static_cast<long long>(g) * a.states + sub * S;
  const T* Cp = static_cast<const T*>(a.C) + b * a.C_batch + static_cast<long long>(g) * a.states + sub * S;
#pragma unroll
  for (int s = 0; s < 2 * Lane<S>::H; ++s) {
    const bool ok = live && s < S && sub * S + s < a.states;
    Bs[s] = ok ? to_f32(Bp[s]) : 0.0f;
    Cs[s] = ok ? to_f32(Cp[s]) : 0.0f;
  }
  float y = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int ch = k * 8 + quad;
    const float dk = __shfl_sync(~0u, d, ch), pk = __shfl_sync(~0u, push, ch);
    Lane<S> A = lane_zero<S>();
    const long long at = static_cast<long long>(c0 + ch) * a.states + sub * S;
    if (ch < cn) A = kWide ? lane_shared<S>(a.A + at) : lane_load<S>(a.A + at, sub * S, a.states);
    float o = 0.0f;
    Lane<S> r;
#pragma unroll
    for (int s = 0; s < Lane<S>::H; ++s) {
      const F2 decay = ex2_2(mul2(f2(dk * kLog2E, dk * kLog2E), A.v[s]));
      h[k].v[s] = fma2(decay, h[k].v[s], mul2(f2(pk, pk), f2(Bs[2 * s], Bs[2 * s + 1])));
      r.v[s] = mul2(h[k].v[s], f2(Cs[2 * s], Cs[2 * s + 1]));
    }
    o = lane_sum(r);
    o += __shfl_xor_sync(~0u, o, 1);
    o += __shfl_xor_sync(~0u, o, 2);
    const float mine = __shfl_sync(~0u, o, (lane & 7) * 4);
    if ((lane >> 3) == k) y = mine;
    if (ch < cn && a.state_out != nullptr) {
      float* p = a.state_out + b * of_seq + at;
      if constexpr (kWide && S >= 4) {
#pragma unroll
        for (int q = 0; q < S / 4; ++q) {
          float4 f;
          un2(h[k].v[2 * q], f.x, f.y);
          un2(h[k].v[2 * q + 1], f.z, f.w);
          reinterpret_cast<float4*>(p)[q] = f;
        }
      } else {
        lane_store<S>(p, sub * S, a.states, h[k]);
      }
    }
  }
  if (in) static_cast<T*>(a.y)[b * a.y_batch + c] = from_f32<T>((y + add) * gate);
}

// Length 0: the states as they were.
__global__ void __launch_bounds__(256) k_scan_nothing(mlt_scan_args a, int elem) {
  pdl_wait();
  pdl_trigger();
  const long long n = static_cast<long long>(a.batch) * a.dim * a.states;
  const long long stride = static_cast<long long>(gridDim.x) * 256;
  const long long first = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  if (a.state_out != nullptr && a.state_out != a.state)
    for (long long i = first; i < n; i += stride) a.state_out[i] = a.state != nullptr ? a.state[i] : 0.0f;
  if (a.conv_state_out == nullptr || a.conv_state_out == a.conv_state) return;
  const long long m = static_cast<long long>(a.batch) * (a.taps - 1) * a.dim * (elem / 2);
  unsigned short* to = static_cast<unsigned short*>(a.conv_state_out);
  const unsigned short* from = static_cast<const unsigned short*>(a.conv_state);
  for (long long i = first; i < m; i += stride) to[i] = from != nullptr ? from[i] : 0;
}

// One chunk where sequences x channel blocks give every SM two CTAs or more; else chunks of
// at least 64 positions, for about six CTAs an SM.
Plan plan_of(const mlt_scan_args& a, int sms) {
  Plan p{};
  const long long ctas = static_cast<long long>(a.batch) * a.groups * blocks_per_group(a);
  long long chunks = 1;
  if (ctas < 2LL * sms) chunks = (6LL * sms + ctas - 1) / (ctas > 0 ? ctas : 1);
  const long long most = (a.length + 63) / 64;
  if (chunks > most) chunks = most;
  if (chunks > 4096) chunks = 4096;
  if (chunks < 1) chunks = 1;
  p.cut.chunk = ((a.length + chunks - 1) / chunks + kTile - 1) / kTile * kTile;
  if (p.cut.chunk < kTile) p.cut.chunk = kTile;
  p.cut.chunks = static_cast<int>((a.length + p.cut.chunk - 1) / p.cut.chunk);
  if (p.cut.chunks < 1) p.cut.chunks = 1;
  if (p.cut.chunks > 1) {
    const size_t seqs = static_cast<size_t>(a.batch) * p.cut.chunks;
    p.off_e = 0;
    p.off_sum = up256(seqs * a.dim * a.states * 4);
    p.bytes = p.off_sum + up256(seqs * a.dim * 4);
  }
  return p;
}

}  // namespace

size_t scan_workspace(const mlt_scan_args& a, int sms) { return a.length <= 1 ? 0 : plan_of(a, sms).bytes; }

cudaError_t launch_scan(const mlt_scan_args& a, void* ws, int sms, long long* launches, cudaStream_t st) {
  if (a.length == 0) {
    ++*launches;
    return launch_pdl(k_scan_nothing, dim3(2 * sms), dim3(256), 0, st, a, static_cast<int>(dtype_size(a.dtype)));
  }
  const bool vec = packs_ok(a) && aligned_to(a.y, kPackC * dtype_size(a.dtype)) && a.y_step % kPackC == 0 &&
                   a.y_batch % kPackC == 0;
  return with_dtype(a.dtype, [&](auto tag) {
    return with_states(a.states, [&](auto states) -> cudaError_t {
      using T = decltype(tag);
      constexpr int S = decltype(states)::value;
      if (a.length == 1) {
        const int blocks = a.groups * ((a.dim / a.groups + 31) / 32);
        const dim3 grid((blocks + 7) / 8, a.batch);
        const bool wide = a.states == 4 * S && aligned_to(a.state, 16) && aligned_to(a.state_out, 16) &&
                          aligned_to(a.A, 16);
        ++*launches;
        return wide ? launch_pdl(k_scan_step<T, S, true>, grid, dim3(256), 0, st, a)
                    : launch_pdl(k_scan_step<T, S, false>, grid, dim3(256), 0, st, a);
      }
      const Plan p = plan_of(a, sms);
      unsigned char* w = static_cast<unsigned char*>(ws);
      const unsigned blocks = static_cast<unsigned>(a.groups * blocks_per_group(a));
      constexpr size_t smem = sizeof(Tile<S>);
      auto go = [&](auto kernel, unsigned chunks) {
        ++*launches;
        const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kernel), smem);
        if (e != cudaSuccess) return e;
        return launch_pdl(kernel, dim3(blocks, a.batch, chunks), dim3(kThreads), smem, st, a, p, w);
      };
      if (p.cut.chunks > 1) {
        cudaError_t e = vec ? go(k_scan<T, S, true, false>, p.cut.chunks - 1)
                            : go(k_scan<T, S, false, false>, p.cut.chunks - 1);
        if (e != cudaSuccess) return e;
        ++*launches;
        const long long of_seq = static_cast<long long>(a.dim) * a.states;
        e = launch_pdl(k_scan_carry, dim3(static_cast<unsigned>((of_seq + 255) / 256), a.batch), dim3(256), 0, st, a, p,
                       w);
        if (e != cudaSuccess) return e;
      }
      return vec ? go(k_scan<T, S, true, true>, p.cut.chunks) : go(k_scan<T, S, false, true>, p.cut.chunks);
    });
  });
}

}  // namespace mlt
