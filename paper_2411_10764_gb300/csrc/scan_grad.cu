// Gradients of the selective scan (scan.cu has the forward formulas).
//
// With gc_t the gradient of C_t . h_t + skip u_t, g_t that of h_t from position t on, and
// a_t = exp(d_t A):
//   g_t = gc_t C_t + a_(t+1) g_(t+1)          e_t = g_t a_t h_(t-1)
//   dB_t = sum over the group's channels of g_t d_t u_t       dC_t likewise of gc_t h_t
//   d(d_t) = u_t (g_t . B_t) + e_t . A        d(u_t) = d_t (g_t . B_t) + gc_t skip
//   dA = sum of d_t e_t                       d(h_(-1)) = a_0 g_0
// then through softplus, the gates and the convolution.
//
// Sequences are cut into chunks, all at once in the first and third step:
//   k_grad_local   per chunk: end state from zero, sum of d, and the chunk's own gradient
//                  of the state before it (sum over t of gc_t C_t exp(A sum of d up to t))
//   k_grad_carry   the state before and the gradient after each chunk, chunk by chunk
//   k_grad_chunk   per chunk: states recomputed from the one before it, then backwards
//   k_grad_finish  sums over chunks, sequences and channel blocks, in a fixed order, and
//                  the inputs whose convolution reaches into the next chunk
// No state is kept from the forward pass and none but a chunk's first is written: inside
// a chunk every kSub-th state is kept in shared memory and the others, with their decays,
// in registers while their kSub positions are walked backwards.
//
// Bound: issue.  Eight channels' position costs a warp about 190 instructions with 16 states: 18 to
// find the kept states, 22 to recompute, 56 backwards, 40 for the sums over lanes and
// channels, the rest for the activations' slopes and stores; about half of the issue slots are
// used at the 16 warps an SM that the registers allow.  Halves of the chunk (24 warps at 80
// registers) took 143 us where this takes 128.  The whole gradient of 4 x 1,021 x 1,024 with ragged
// lengths takes 126 to 156 us by the lengths drawn; 256 sequences of 8 x 128 in fp32 52 us.
#include "scan.cuh"

namespace mlt {
namespace {

using namespace scan;

// Positions of a chunk and of the part that is walked backwards at a time, by states a lane:
// the states kept of a chunk take 32 KB (S = 4) or 64 KB (S = 8) of shared memory.
template <int S>
struct Shape {
  static constexpr int kChunk = S > 4 ? 32 : 64;
  static constexpr int kSub = S > 4 ? 4 : 8;
  static constexpr int kSubs = kChunk / kSub;
};
int chunk_of(int states) { return states > 16 ? 32 : 64; }

constexpr int kChannels = 64;   // of a CTA
constexpr int kThreads = 4 * kChannels;
constexpr int kPairs = kChannels / 2;
constexpr int kRing = 16;       // rows of dv kept for the convolution
constexpr int kVecs = kScanMaxTaps + 3;       // per channel: conv_w (4), conv_b, skip, dt_bias
constexpr int kHalo = kScanMaxTaps - 1;

struct GradPlan {
  int chunk;
  long long chunks;
  int blocks;  // channel blocks of a group
  size_t off_e, off_g, off_sum, off_A, off_vec, off_head, off_part, off_bc, bytes;
};

template <int S>
struct alignas(16) Staged {
  float2 du[Shape<S>::kChunk][kChannels];  // (d, u)
  float gc[Shape<S>::kChunk][kChannels];
  float B[Shape<S>::kChunk * 4 * S];
  float C[Shape<S>::kChunk * 4 * S];
};

template <int S>
struct alignas(16) Walk {
  Staged<S> in;
  float kept[Shape<S>::kSubs][kChannels * 4 * S];  // the state before each part
  float y[Shape<S>::kSub][kChannels + 4];          // C . h
  float gp[Shape<S>::kSub][kChannels + 4];         // g . B
  float ga[Shape<S>::kSub][kChannels + 4];         // e . A, times log2 e
  float bc[kThreads / 32][Shape<S>::kSub][2 * 4 * S];  // each warp's share of dB, dC
  float dv[kRing][kChannels];
  float params[kScanMaxTaps + 3][kChannels];  // convolution weights and bias, dt_bias, skip
};

// Two channels of gy at `count` positions from t on.
template <typename T, int RUN, bool kVec>
__device__ __forceinline__ void load_gy(const mlt_scan_grads& g, const Block& k, const PairParams& q, long long t,
                                        int count, Two<T> (&gy)[RUN]) {
  const T* p = static_cast<const T*>(g.gy) + k.b * g.gy_batch + t * g.gy_step + k.c0 + q.c;
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    if (q.n > 0 && i < count) gy[i] = load_two<T, kVec>(p, q.n);
    p += g.gy_step;
  }
}

// The chunk's (d, u), gc, B and C in shared memory; zero from `live` on.
template <typename T, int S, bool kVec>
__device__ __forceinline__ void stage_chunk(const mlt_scan_args& a, const mlt_scan_grads& g, const Block& k,
                                            const PairParams& q, long long begin, int live, Staged<S>& st) {
  constexpr int kRun = Shape<S>::kChunk / kGroups;
  const int run = threadIdx.x / kPairs * kRun;
  RawRun<T, kRun> raw;
  Two<T> gy[kRun];
  load_run<T, kRun, kVec, true>(a, k, q, begin + run, begin + live, raw);
  load_gy<T, kRun, kVec>(g, k, q, begin + run, live - run, gy);
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    F2 d = dup2(0.0f), u = d, gc = d;
    if (run + i < live && q.n > 0) {
      u = conv_run(a, q, raw, i);
      if (a.taps > 0) u = mul2(u, sigmoid2(u));
      d = softplus2(add2(two_f32(raw.dt[i]), q.bias));
      gc = two_f32(gy[i]);
      if (a.z != nullptr) {
        const F2 z = two_f32(raw.z[i]);
        gc = mul2(gc, mul2(z, sigmoid2(z)));
      }
    }
    float4 o;
    un2(d, o.x, o.z);
    un2(u, o.y, o.w);
    *reinterpret_cast<float4*>(&st.du[run + i][q.c]) = o;
    float2 c;
    un2(gc, c.x, c.y);
    *reinterpret_cast<float2*>(&st.gc[run + i][q.c]) = c;
  }
  const T* Bp = static_cast<const T*>(a.B) + k.b * a.B_batch + begin * a.B_step + static_cast<long long>(k.g) * a.states;
  const T* Cp = static_cast<const T*>(a.C) + k.b * a.C_batch + begin * a.C_step + static_cast<long long>(k.g) * a.states;
#pragma unroll 4
  for (int i = threadIdx.x; i < Shape<S>::kChunk * 4 * S; i += kThreads) {
    const int t = i / (4 * S), s = i - t * (4 * S);
    const bool ok = t < live && s < a.states;
    st.B[i] = ok ? to_f32(Bp[t * a.B_step + s]) : 0.0f;
    st.C[i] = ok ? to_f32(Cp[t * a.C_step + s]) : 0.0f;
  }
}

// blockIdx.x counts (chunk, channel block), blockIdx.y sequences.
struct Where {
  Block k;
  long long chunk, begin, len;
  int live;  // positions of the chunk before the sequence's end
};
__device__ __forceinline__ Where where(const mlt_scan_args& a, int chunk_positions) {
  Where w;
  const int blocks = a.groups * blocks_per_group<kChannels>(a);
  w.chunk = blockIdx.x / blocks;
  w.k = block_of<kChannels>(a, static_cast<int>(blockIdx.x - w.chunk * blocks), blockIdx.y);
  w.begin = w.chunk * chunk_positions;
  w.len = length_of(a, w.k.b);
  w.live = static_cast<int>(min(static_cast<long long>(chunk_positions), max(0ll, w.len - w.begin)));
  return w;
}

template <typename T, int S, bool kVec>
__global__ void __launch_bounds__(kThreads) k_grad_local(mlt_scan_args a, mlt_scan_grads g, GradPlan p,
                                                         unsigned char* ws) {
  extern __shared__ __align__(16) unsigned char smem[];
  Staged<S>& st = *reinterpret_cast<Staged<S>*>(smem);
  pdl_wait();
  pdl_trigger();
  const Where w = where(a, Shape<S>::kChunk);
  if (w.live == 0) return;  // k_grad_carry stops before it
  stage_chunk<T, S, kVec>(a, g, w.k, pair_params<kChannels>(a, w.k), w.begin, w.live, st);
  const int lane = threadIdx.x & 3, ch = threadIdx.x >> 2;
  const bool in = ch < w.k.cn;
  const long long at = static_cast<long long>(w.k.c0 + ch) * a.states + lane * S;
  Lane<S> A = lane_zero<S>(), h = A, acc = A, prod = A;
  if (in) A = lane_load<S>(a.A + at, lane * S, a.states);
#pragma unroll
  for (int s = 0; s < Lane<S>::H; ++s) {
    A.v[s] = mul2(A.v[s], f2(kLog2E, kLog2E));
    prod.v[s] = f2(1.0f, 1.0f);
  }
  float sum = 0.0f;
  __syncthreads();
#pragma unroll 4
  for (int t = 0; t < Shape<S>::kChunk; ++t) {
    const float2 du = st.du[t][ch];
    const float gc = st.gc[t][ch];
    const Lane<S> B = lane_shared<S>(st.B + (t * 4 + lane) * S), C = lane_shared<S>(st.C + (t * 4 + lane) * S);
    const F2 d = f2(du.x, du.x), push = f2(du.x * du.y, du.x * du.y), gg = f2(gc, gc);
#pragma unroll
    for (int s = 0; s < Lane<S>::H; ++s) {
      const F2 decay = decay2(d, A.v[s]);
      h.v[s] = fma2(decay, h.v[s], mul2(push, B.v[s]));
      prod.v[s] = mul2(prod.v[s], decay);
      acc.v[s] = fma2(prod.v[s], mul2(gg, C.v[s]), acc.v[s]);
    }
    sum += du.x;
  }
  if (!in) return;
  const long long seq = static_cast<long long>(w.k.b) * p.chunks + w.chunk;
  const long long of_seq = static_cast<long long>(a.dim) * a.states;
  lane_store<S>(reinterpret_cast<float*>(ws + p.off_e) + seq * of_seq + at, lane * S, a.states, h);
  lane_store<S>(reinterpret_cast<float*>(ws + p.off_g) + seq * of_seq + at, lane * S, a.states, acc);
  if (lane == 0) reinterpret_cast<float*>(ws + p.off_sum)[seq * a.dim + w.k.c0 + ch] = sum;
}

// In place: a chunk's end state becomes the state before it, its own gradient the one after it.
__global__ void __launch_bounds__(256) k_grad_carry(mlt_scan_args a, mlt_scan_grads g, GradPlan p, unsigned char* ws) {
  pdl_wait();
  pdl_trigger();
  const long long of_seq = static_cast<long long>(a.dim) * a.states;
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= of_seq) return;
  const int b = blockIdx.y;
  const long long chunks = (length_of(a, b) + p.chunk - 1) / p.chunk;
  float* e = reinterpret_cast<float*>(ws + p.off_e) + b * p.chunks * of_seq + i;
  float* q = reinterpret_cast<float*>(ws + p.off_g) + b * p.chunks * of_seq + i;
  const float* sum = reinterpret_cast<const float*>(ws + p.off_sum) + b * p.chunks * a.dim + i / a.states;
  const float A = a.A[i] * kLog2E;
  float h = a.state != nullptr ? a.state[b * of_seq + i] : 0.0f;
  // loads of eight chunks first: the stores go to the same memory
  for (long long c0 = 0; c0 < chunks; c0 += 8) {
    float end[8], d[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c0 + k < chunks) {
        end[k] = e[(c0 + k) * of_seq];
        d[k] = sum[(c0 + k) * a.dim];
      }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c0 + k < chunks) {
        e[(c0 + k) * of_seq] = h;
        h = fmaf(ex2(A * d[k]), h, end[k]);
      }
  }
  float r = g.g_state_out != nullptr ? g.g_state_out[b * of_seq + i] : 0.0f;
  for (long long c0 = chunks - 1; c0 >= 0; c0 -= 8) {
    float own[8], d[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c0 - k >= 0) {
        own[k] = q[(c0 - k) * of_seq];
        d[k] = sum[(c0 - k) * a.dim];
      }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c0 - k >= 0) {
        q[(c0 - k) * of_seq] = r;
        r = fmaf(ex2(A * d[k]), r, own[k]);
      }
  }
}

// Sums over the eight channels of a warp of each lane's M values: halves of the values are
// exchanged with the lane whose channel differs in one bit, so M / 8 (at least 1) remain in
// a lane: with M >= 8, the values from (lane >> 2) M / 8 on.
template <int M>
struct ChannelSums {
  static constexpr int kLeft = M > 8 ? M / 8 : 1;
};
template <int M>
__device__ __forceinline__ int channel_sums(float (&v)[M]) {
  const int lane = threadIdx.x & 31;
  int first = 0;
  int left = M;
#pragma unroll
  for (int bit = 16; bit >= 4; bit /= 2) {
    if (left > 1) {
      const int half = left / 2;
      const bool hi = lane & bit;
#pragma unroll
      for (int i = 0; i < M / 2; ++i)
        if (i < half) {
          const float mine = hi ? v[i + half] : v[i], other = hi ? v[i] : v[i + half];
          v[i] = mine + __shfl_xor_sync(~0u, other, bit);
        }
      if (hi) first += half;
      left = half;
    } else {
      v[0] += __shfl_xor_sync(~0u, v[0], bit);
    }
  }
  return first;
}

template <typename T, int S, bool kVec>
__global__ void __launch_bounds__(kThreads, 2) k_grad_chunk(mlt_scan_args a, mlt_scan_grads g, GradPlan p,
                                                            unsigned char* ws) {
  using Sh = Shape<S>;
  constexpr int kSub = Sh::kSub;
  extern __shared__ __align__(16) unsigned char smem[];
  Walk<S>& sm = *reinterpret_cast<Walk<S>*>(smem);
  pdl_wait();
  pdl_trigger();
  const Where w = where(a, Sh::kChunk);
  const Block& k = w.k;
  const long long of_seq = static_cast<long long>(a.dim) * a.states;
  const long long seq = static_cast<long long>(k.b) * p.chunks + w.chunk;
  const int positions = static_cast<int>(min(static_cast<long long>(Sh::kChunk), a.length - w.begin));
  // a lane's channel and states in the walk
  const int lane = threadIdx.x & 3, ch = threadIdx.x >> 2;
  const bool in = ch < k.cn;
  const long long at = static_cast<long long>(k.c0 + ch) * a.states + lane * S;
  // a thread's two channels and first position (then every kGroups-th) elsewhere
  const PairParams q = pair_params<kChannels>(a, k);
  const int tl = threadIdx.x / kPairs, cc = k.c0 + q.c;
  const bool cin = q.n > 0;
  T* gx = static_cast<T*>(g.x) + (static_cast<long long>(k.b) * a.length + w.begin) * a.dim + cc;
  T* gdt = static_cast<T*>(g.dt) + (static_cast<long long>(k.b) * a.length + w.begin) * a.dim + cc;
  T* gz = static_cast<T*>(g.z) + (static_cast<long long>(k.b) * a.length + w.begin) * a.dim + cc;
  auto clear = [&](long long o) {
    if (g.x != nullptr) store_two<T, kVec>(gx + o, q.n, dup2(0.0f));
    if (g.dt != nullptr) store_two<T, kVec>(gdt + o, q.n, dup2(0.0f));
    if (g.z != nullptr) store_two<T, kVec>(gz + o, q.n, dup2(0.0f));
  };
  if (w.live == 0) {
    // past the sequence's end
    if (cin)
      for (int t = tl; t < positions; t += kGroups) clear(static_cast<long long>(t) * a.dim);
    if (w.chunk == 0 && in && g.state != nullptr) {
      Lane<S> r = lane_zero<S>();
      if (g.g_state_out != nullptr) r = lane_load<S>(g.g_state_out + k.b * of_seq + at, lane * S, a.states);
      lane_store<S>(g.state + k.b * of_seq + at, lane * S, a.states, r);
    }
    return;
  }
  stage_chunk<T, S, kVec>(a, g, k, q, w.begin, w.live, sm.in);
  if (tl == 0) {
    auto keep = [&](int row, F2 v) {
      float2 f;
      un2(v, f.x, f.y);
      *reinterpret_cast<float2*>(&sm.params[row][q.c]) = f;
    };
#pragma unroll
    for (int j = 0; j < kScanMaxTaps; ++j) keep(j, q.w[j]);
    keep(kScanMaxTaps, q.conv_b);
    keep(kScanMaxTaps + 1, q.bias);
    F2 skip = dup2(0.0f);
    if (cin && a.skip != nullptr) skip = f2(a.skip[cc], q.n > 1 ? a.skip[cc + 1] : 0.0f);
    keep(kScanMaxTaps + 2, skip);
  }
  for (int i = threadIdx.x; i < kRing * kChannels; i += kThreads) sm.dv[i / kChannels][i % kChannels] = 0.0f;
  Lane<S> A = lane_zero<S>(), h = A, r = A, dA = A;
  if (in) {
    A = lane_load<S>(a.A + at, lane * S, a.states);
    const bool one = p.chunks == 1;
    const float* hp = one ? (a.state != nullptr ? a.state + k.b * of_seq : nullptr)
                          : reinterpret_cast<const float*>(ws + p.off_e) + seq * of_seq;
    const float* rp = one ? (g.g_state_out != nullptr ? g.g_state_out + k.b * of_seq : nullptr)
                          : reinterpret_cast<const float*>(ws + p.off_g) + seq * of_seq;
    if (hp != nullptr) h = lane_load<S>(hp + at, lane * S, a.states);
    if (rp != nullptr) r = lane_load<S>(rp + at, lane * S, a.states);
  }
#pragma unroll
  for (int s = 0; s < Lane<S>::H; ++s) A.v[s] = mul2(A.v[s], f2(kLog2E, kLog2E));
  __syncthreads();

  // forwards: the state before each part
  float* kept = sm.kept[0] + (ch * 4 + lane) * S;
  const int parts = (w.live + kSub - 1) / kSub;  // later ones hold no live position
#pragma unroll 1
  for (int part = 0; part < parts; ++part) {
    lane_store<S>(kept + part * (kChannels * 4 * S), 0, S, h);
    if (part + 1 == parts) break;
#pragma unroll
    for (int t = 0; t < kSub; ++t) {
      const float2 du = sm.in.du[part * kSub + t][ch];
      const Lane<S> B = lane_shared<S>(sm.in.B + ((part * kSub + t) * 4 + lane) * S);
      const F2 d = f2(du.x, du.x), push = f2(du.x * du.y, du.x * du.y);
#pragma unroll
      for (int s = 0; s < Lane<S>::H; ++s) h.v[s] = fma2(decay2(d, A.v[s]), h.v[s], mul2(push, B.v[s]));
    }
  }

  // the parameters come from shared memory after each walk, which needs the registers
  auto kept_params = [&](F2& skip) {
    auto two = [&](int row) {
      const volatile float* v = &sm.params[row][q.c];  // volatile: not kept in registers
      return f2(v[0], v[1]);
    };
    PairParams r;
    r.c = q.c;
    r.n = q.n;
#pragma unroll
    for (int j = 0; j < kScanMaxTaps; ++j) r.w[j] = two(j);
    r.conv_b = two(kScanMaxTaps);
    r.bias = two(kScanMaxTaps + 1);
    skip = two(kScanMaxTaps + 2);
    return r;
  };
  const bool next_live = w.begin + Sh::kChunk < w.len;  // its convolution reads this chunk's last inputs
  const int halo = a.taps > 1 ? a.taps - 1 : 0;
  F2 vec[kVecs];
#pragma unroll
  for (int v = 0; v < kVecs; ++v) vec[v] = dup2(0.0f);
  // parts past the sequence's end
  if (cin)
    for (int t = parts * kSub + tl; t < positions; t += kGroups) clear(static_cast<long long>(t) * a.dim);

#pragma unroll 1
  for (int part = parts - 1; part >= 0; --part) {
    const int t0 = part * kSub;
    // what the activations' slopes need lands behind the walk
    static_assert(kSub <= kGroups, "a thread has one position of a part");
    const int ct = t0 + tl;  // position in the chunk
    const bool mine = tl < kSub && cin;
    RawRun<T, 1> raw;
    Two<T> gy[1];
    if (mine && ct < w.live) {
      load_run<T, 1, kVec, true>(a, k, q, w.begin + ct, w.begin + w.live, raw);
      load_gy<T, 1, kVec>(g, k, q, w.begin + ct, 1, gy);
    }
    {
      Lane<S> hs[kSub + 1], decay[kSub];
      hs[0] = lane_shared<S>(kept + part * (kChannels * 4 * S));
      float y[kSub], gp[kSub], ga[kSub];
#pragma unroll
      for (int t = 0; t < kSub; ++t) {
        const float2 du = sm.in.du[t0 + t][ch];
        const Lane<S> B = lane_shared<S>(sm.in.B + ((t0 + t) * 4 + lane) * S);
        const Lane<S> C = lane_shared<S>(sm.in.C + ((t0 + t) * 4 + lane) * S);
        const F2 d = f2(du.x, du.x), push = f2(du.x * du.y, du.x * du.y);
        Lane<S> o;
#pragma unroll
        for (int s = 0; s < Lane<S>::H; ++s) {
          decay[t].v[s] = decay2(d, A.v[s]);
          hs[t + 1].v[s] = fma2(decay[t].v[s], hs[t].v[s], mul2(push, B.v[s]));
          o.v[s] = mul2(C.v[s], hs[t + 1].v[s]);
        }
        y[t] = lane_sum(o);
      }
#pragma unroll
      for (int t = kSub - 1; t >= 0; --t) {
        const float2 du = sm.in.du[t0 + t][ch];
        const float gc = sm.in.gc[t0 + t][ch];
        const Lane<S> B = lane_shared<S>(sm.in.B + ((t0 + t) * 4 + lane) * S);
        const Lane<S> C = lane_shared<S>(sm.in.C + ((t0 + t) * 4 + lane) * S);
        const F2 d = f2(du.x, du.x), push = f2(du.x * du.y, du.x * du.y), gg = f2(gc, gc);
        float bc[2 * S];
        Lane<S> ob, oa;
#pragma unroll
        for (int s = 0; s < Lane<S>::H; ++s) {
          r.v[s] = fma2(gg, C.v[s], r.v[s]);
          const F2 db = mul2(r.v[s], push), dc = mul2(gg, hs[t + 1].v[s]);
          float v0, v1;
          un2(db, v0, v1);
          bc[2 * s < S ? 2 * s : 0] = v0;
          if (2 * s + 1 < S) bc[2 * s + 1] = v1;
          un2(dc, v0, v1);
          bc[S + (2 * s < S ? 2 * s : 0)] = v0;
          if (2 * s + 1 < S) bc[S + 2 * s + 1] = v1;
          ob.v[s] = mul2(r.v[s], B.v[s]);
          r.v[s] = mul2(r.v[s], decay[t].v[s]);
          const F2 e = mul2(r.v[s], hs[t].v[s]);
          oa.v[s] = mul2(e, A.v[s]);
          dA.v[s] = fma2(e, d, dA.v[s]);
        }
        gp[t] = lane_sum(ob);
        ga[t] = lane_sum(oa);
        // dB and dC: sums over the warp's channels
        const int first = channel_sums(bc);
        constexpr int kLeft = ChannelSums<2 * S>::kLeft;
        if (2 * S >= 8 || (threadIdx.x & 31 & (S == 2 ? 4 : 12)) == 0) {
#pragma unroll
          for (int i = 0; i < kLeft; ++i) {
            const int v = first + i;  // < S: dB, else dC
            sm.bc[threadIdx.x >> 5][t][(v < S ? 0 : 4 * S) + lane * S + (v < S ? v : v - S)] = bc[i];
          }
        }
      }
#pragma unroll
      for (int t = 0; t < kSub; t += 4) {
        const float yy[4] = {y[t], y[t + 1], y[t + 2], y[t + 3]};
        const float pp[4] = {gp[t], gp[t + 1], gp[t + 2], gp[t + 3]};
        const float aa[4] = {ga[t], ga[t + 1], ga[t + 2], ga[t + 3]};
        sm.y[t + lane][ch] = quad_sums(yy, lane);
        sm.gp[t + lane][ch] = quad_sums(pp, lane);
        sm.ga[t + lane][ch] = quad_sums(aa, lane);
      }
    }
    __syncthreads();
    // the CTA's share of dB and dC
    if (g.B != nullptr || g.C != nullptr) {
      float* to = reinterpret_cast<float*>(ws + p.off_bc);
      const long long row = (static_cast<long long>(k.b) * a.groups * p.blocks +
                             (blockIdx.x - w.chunk * (a.groups * p.blocks))) * a.length + w.begin + t0;
      for (int i = threadIdx.x; i < kSub * 8 * S; i += kThreads) {
        const int t = i / (8 * S), v = i - t * (8 * S);
        const int s = v % (4 * S);
        if (t0 + t >= w.live || s >= a.states) continue;
        float sum = 0.0f;
#pragma unroll
        for (int q = 0; q < kThreads / 32; ++q) sum += sm.bc[q][t][v];
        to[((row + t) * 2 + v / (4 * S)) * a.states + s] = sum;
      }
    }
    // through the gate, softplus and the convolution's activation
    const long long o = static_cast<long long>(ct) * a.dim;
    F2 skip;
    const PairParams par = kept_params(skip);
    if (mine) {
      F2 dv = dup2(0.0f);
      if (ct < w.live) {
        const float4 in4 = *reinterpret_cast<const float4*>(&sm.in.du[ct][q.c]);
        const F2 d = f2(in4.x, in4.z), u = f2(in4.y, in4.w);
        auto two = [&](const float* p) {
          const float2 v = *reinterpret_cast<const float2*>(p);
          return f2(v.x, v.y);
        };
        const F2 gc = two(&sm.in.gc[ct][q.c]), gp = two(&sm.gp[tl][q.c]);
        if (g.z != nullptr) {
          const F2 z = two_f32(raw.z[0]), sz = sigmoid2(z);
          const F2 slope = mul2(sz, fma2(z, fma2(sz, dup2(-1.0f), dup2(1.0f)), dup2(1.0f)));
          store_two<T, kVec>(gz + o, q.n, mul2(mul2(two_f32(gy[0]), fma2(skip, u, two(&sm.y[tl][q.c]))), slope));
        }
        const F2 graw = mul2(fma2(gp, u, mul2(two(&sm.ga[tl][q.c]), dup2(1.0f / kLog2E))),
                             sigmoid2(add2(two_f32(raw.dt[0]), par.bias)));
        if (g.dt != nullptr) store_two<T, kVec>(gdt + o, q.n, graw);
        vec[kScanMaxTaps + 1] = fma2(gc, u, vec[kScanMaxTaps + 1]);
        vec[kScanMaxTaps + 2] = add2(graw, vec[kScanMaxTaps + 2]);
        dv = fma2(gp, d, mul2(gc, skip));
        if (a.taps > 0) {
          const F2 v = conv_run(a, par, raw, 0), sv = sigmoid2(v);
          dv = mul2(dv, mul2(sv, fma2(v, fma2(sv, dup2(-1.0f), dup2(1.0f)), dup2(1.0f))));
#pragma unroll
          for (int j = 0; j < kScanMaxTaps; ++j)
            if (j < a.taps) vec[j] = fma2(dv, two_f32(raw.x[kScanMaxTaps - 1 - j]), vec[j]);
          vec[kScanMaxTaps] = add2(dv, vec[kScanMaxTaps]);
        }
      } else if (ct < positions) {
        if (g.z != nullptr) store_two<T, kVec>(gz + o, q.n, dup2(0.0f));
        if (g.dt != nullptr) store_two<T, kVec>(gdt + o, q.n, dup2(0.0f));
      }
      float2 v;
      un2(dv, v.x, v.y);
      *reinterpret_cast<float2*>(&sm.dv[ct % kRing][q.c]) = v;
      if (halo > 0 && ct < kHalo) {
        float* head = reinterpret_cast<float*>(ws + p.off_head) + (seq * kHalo + ct) * a.dim + cc;
        head[0] = v.x;
        if (q.n > 1) head[1] = v.y;
      }
    }
    __syncthreads();
    // x[t] meets weight j in v[t + j]
    if (g.x != nullptr && mine && ct < positions) {
      auto dv = [&](int j) {
        const float2 v = *reinterpret_cast<const float2*>(&sm.dv[(ct + j) % kRing][q.c]);
        return f2(v.x, v.y);
      };
      F2 d = dv(0);
      if (a.taps > 0) {
        d = mul2(d, par.w[0]);
#pragma unroll
        for (int j = 1; j < kScanMaxTaps; ++j)
          if (j < a.taps && ct + j < Sh::kChunk) d = fma2(par.w[j], dv(j), d);
      }
      if (next_live && ct >= Sh::kChunk - halo) {
        float v0, v1;
        un2(d, v0, v1);
        float* part_x = reinterpret_cast<float*>(ws + p.off_part) + (seq * kHalo + ct - (Sh::kChunk - halo)) * a.dim + cc;
        part_x[0] = v0;
        if (q.n > 1) part_x[1] = v1;
      } else {
        store_two<T, kVec>(gx + o, q.n, ct < w.live ? d : dup2(0.0f));
      }
    }
  }
  if (in) {
    lane_store<S>(reinterpret_cast<float*>(ws + p.off_A) + seq * of_seq + at, lane * S, a.states, dA);
    if (w.chunk == 0 && g.state != nullptr) lane_store<S>(g.state + k.b * of_seq + at, lane * S, a.states, r);
  }
  // the channels' sums over the chunk: kGroups threads each, through the staging memory
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int v = 0; v < kVecs; ++v) {
    float2 f;
    un2(vec[v], f.x, f.y);
    *reinterpret_cast<float2*>(&red[(v * kGroups + tl) * kChannels + q.c]) = f;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kVecs * kChannels; i += kThreads) {
    const int v = i / kChannels, c = i % kChannels;
    if (c >= k.cn) continue;
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < kGroups; ++e) sum += red[(v * kGroups + e) * kChannels + c];
    reinterpret_cast<float*>(ws + p.off_vec)[(seq * kVecs + v) * a.dim + k.c0 + c] = sum;
  }
}

// ---------------------------------------------------------------------------
// Sums and chunk borders
// ---------------------------------------------------------------------------
struct Finish {
  long long bc_blocks, sum_blocks, edge_blocks;
};

// Sum over the sequences' live chunks of at[(b chunks + chunk) stride]: `part`'s share of them, every
// eighth (sequence, chunk) pair, so that sequences of one chunk each are shared too.  Loads of eight
// pairs come before their sum, which is compensated: there may be 65,535 sequences, and a
// plain sum of as many equal terms in 32 bits is off by a thousandth.
__device__ __forceinline__ float sum_chunks(const mlt_scan_args& a, const GradPlan& p, const float* at, long long stride,
                                            int part) {
  constexpr int kAhead = 8;
  float sum = 0.0f, lost = 0.0f;
  int b = 0;
  long long k = part;  // the next pair's chunk
  auto wrap = [&]() {
    if (p.chunks == 1) {
      b += static_cast<int>(k);
      k = 0;
    }
    for (; k >= p.chunks && b < a.batch; ++b) k -= p.chunks;
  };
  wrap();
  while (b < a.batch) {
    float v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      v[i] = 0.0f;
      if (b < a.batch && k * p.chunk < length_of(a, b)) v[i] = at[(b * p.chunks + k) * stride];
      k += 8;
      wrap();
    }
    const float now = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    const float y = __fsub_rn(now, lost), t = __fadd_rn(sum, y);
    lost = isfinite(t) ? __fsub_rn(__fsub_rn(t, sum), y) : 0.0f;  // an infinite sum stays one
    sum = t;
  }
  return __fsub_rn(sum, lost);
}

template <typename T>
__global__ void __launch_bounds__(256) k_grad_finish(mlt_scan_args a, mlt_scan_grads g, GradPlan p, Finish f,
                                                     const unsigned char* ws) {
  __shared__ float red[8][33];
  pdl_wait();
  pdl_trigger();
  long long block = blockIdx.x;
  if (block < f.bc_blocks) {
    // dB, dC over the group's channel blocks
    const long long n = a.states, i = block * 256 + threadIdx.x;
    const long long rows = static_cast<long long>(a.batch) * a.length;
    if (i >= rows * a.groups * n) return;
    const long long s = i % n, gr = i / n % a.groups, row = i / n / a.groups;
    const long long b = row / a.length, t = row - b * a.length;
    float sb = 0.0f, sc = 0.0f;
    if (t < length_of(a, static_cast<int>(b))) {
      const float* q = reinterpret_cast<const float*>(ws + p.off_bc);
#pragma unroll 4
      for (int k = 0; k < p.blocks; ++k) {
        const float* r = q + (((b * a.groups + gr) * p.blocks + k) * a.length + t) * 2 * n + s;
        sb += r[0];
        sc += r[n];
      }
    }
    if (g.B != nullptr) static_cast<T*>(g.B)[i] = from_f32<T>(sb);
    if (g.C != nullptr) static_cast<T*>(g.C)[i] = from_f32<T>(sc);
    return;
  }
  block -= f.bc_blocks;
  if (block < f.sum_blocks) {
    // dA and the channels' vectors: 32 columns, 8 threads each
    const int col = threadIdx.x & 31, part = threadIdx.x >> 5;
    const long long of_seq = static_cast<long long>(a.dim) * a.states;
    const long long i = block * 32 + col, all = of_seq + static_cast<long long>(kVecs) * a.dim;
    float sum = 0.0f;
    if (i < of_seq)
      sum = sum_chunks(a, p, reinterpret_cast<const float*>(ws + p.off_A) + i, of_seq, part);
    else if (i < all)
      sum = sum_chunks(a, p, reinterpret_cast<const float*>(ws + p.off_vec) + (i - of_seq),
                       static_cast<long long>(kVecs) * a.dim, part);
    red[part][col] = sum;
    __syncthreads();
    if (part != 0 || i >= all) return;
#pragma unroll
    for (int q = 1; q < 8; ++q) sum += red[q][col];
    if (i < of_seq) {
      if (g.A != nullptr) g.A[i] = sum;
      return;
    }
    const int v = static_cast<int>((i - of_seq) / a.dim), ch = static_cast<int>((i - of_seq) % a.dim);
    if (v < kScanMaxTaps) {
      if (v < a.taps && g.conv_w != nullptr) g.conv_w[static_cast<long long>(ch) * a.taps + a.taps - 1 - v] = sum;
    } else {
      float* to = v == kScanMaxTaps ? g.conv_b : v == kScanMaxTaps + 1 ? g.skip : g.dt_bias;
      if (to != nullptr) to[ch] = sum;
    }
    return;
  }
  block -= f.sum_blocks;
  // inputs that the next chunk's convolution reads too, and those before the start (chunk -1)
  const long long i = block * 256 + threadIdx.x;
  const int halo = a.taps - 1;
  const long long per_seq = p.chunks * halo * a.dim;
  if (i >= a.batch * per_seq) return;
  const int b = static_cast<int>(i / per_seq);
  const long long rest = i - b * per_seq;
  const int ch = static_cast<int>(rest % a.dim), row = static_cast<int>(rest / a.dim % halo);
  const long long chunk = rest / a.dim / halo - 1;  // the next one is chunk + 1
  const long long len = length_of(a, b);
  const bool next_live = (chunk + 1) * p.chunk < len;
  if (chunk >= 0 && (!next_live || g.x == nullptr)) return;  // k_grad_chunk wrote them
  if (chunk < 0 && g.conv_state == nullptr) return;
  const long long seq = b * p.chunks + chunk;
  float d = 0.0f;
  if (next_live) {
    if (chunk >= 0) d = reinterpret_cast<const float*>(ws + p.off_part)[(seq * kHalo + row) * a.dim + ch];
    const float* head = reinterpret_cast<const float*>(ws + p.off_head) + (seq + 1) * kHalo * a.dim + ch;
    // row is halo - row positions before the next chunk: weight j meets its position j - (halo - row)
    for (int j = halo - row; j < a.taps; ++j)
      d = fmaf(a.conv_w[static_cast<long long>(ch) * a.taps + a.taps - 1 - j],
               head[static_cast<long long>(j - (halo - row)) * a.dim], d);
  }
  if (chunk < 0)
    static_cast<T*>(g.conv_state)[(static_cast<long long>(b) * halo + row) * a.dim + ch] = from_f32<T>(d);
  else
    static_cast<T*>(g.x)[(b * a.length + (chunk + 1) * p.chunk - halo + row) * a.dim + ch] = from_f32<T>(d);
}

// No positions or no sequences: sums are zero, the state's gradient passes through.
__global__ void __launch_bounds__(256) k_grad_nothing(mlt_scan_args a, mlt_scan_grads g, int elem) {
  pdl_wait();
  pdl_trigger();
  const long long stride = static_cast<long long>(gridDim.x) * 256;
  const long long first = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  const long long of_seq = static_cast<long long>(a.dim) * a.states;
  auto clear = [&](float* p, long long n) {
    if (p == nullptr) return;
    for (long long i = first; i < n; i += stride) p[i] = 0.0f;
  };
  clear(g.A, of_seq);
  clear(g.skip, a.dim);
  clear(g.dt_bias, a.dim);
  clear(g.conv_b, a.dim);
  clear(g.conv_w, static_cast<long long>(a.dim) * a.taps);
  if (g.state != nullptr)
    for (long long i = first; i < a.batch * of_seq; i += stride)
      g.state[i] = g.g_state_out != nullptr ? g.g_state_out[i] : 0.0f;
  if (g.conv_state != nullptr)
    for (long long i = first; i < static_cast<long long>(a.batch) * (a.taps - 1) * a.dim * (elem / 2); i += stride)
      static_cast<unsigned short*>(g.conv_state)[i] = 0;
}

GradPlan grad_plan(const mlt_scan_args& a) {
  GradPlan p{};
  p.chunk = chunk_of(a.states);
  p.chunks = (a.length + p.chunk - 1) / p.chunk;
  p.blocks = blocks_per_group<kChannels>(a);
  const size_t seqs = static_cast<size_t>(a.batch) * static_cast<size_t>(p.chunks), dim = a.dim;
  size_t at = 0;
  auto take = [&](size_t floats) {
    const size_t o = at;
    at += up256(floats * 4);
    return o;
  };
  if (p.chunks > 1) {
    p.off_e = take(seqs * dim * a.states);
    p.off_g = take(seqs * dim * a.states);
    p.off_sum = take(seqs * dim);
  }
  p.off_A = take(seqs * dim * a.states);
  p.off_vec = take(seqs * dim * kVecs);
  p.off_head = take(seqs * dim * kHalo);
  p.off_part = take(seqs * dim * kHalo);
  p.off_bc = take(static_cast<size_t>(a.batch) * a.groups * p.blocks * a.length * 2 * a.states);
  p.bytes = at;
  return p;
}

}  // namespace

size_t scan_grad_workspace(const mlt_scan_args& a, int) {
  return a.length == 0 || a.batch == 0 ? 0 : grad_plan(a).bytes;
}

cudaError_t launch_scan_grad(const mlt_scan_args& a, const mlt_scan_grads& g, void* ws, int sms, long long* launches,
                             cudaStream_t st) {
  if (a.length == 0 || a.batch == 0) {
    ++*launches;
    return launch_pdl(k_grad_nothing, dim3(sms), dim3(256), 0, st, a, g, static_cast<int>(dtype_size(a.dtype)));
  }
  const GradPlan p = grad_plan(a);
  unsigned char* w = static_cast<unsigned char*>(ws);
  const long long of_seq = static_cast<long long>(a.dim) * a.states;
  const size_t two = 2 * dtype_size(a.dtype);
  const bool vec = pairs_ok(a) && aligned_to(g.gy, two) && g.gy_step % 2 == 0 && g.gy_batch % 2 == 0 &&
                   aligned_to(g.x, two) && aligned_to(g.dt, two) && aligned_to(g.z, two);
  return with_dtype(a.dtype, [&](auto tag) {
    return with_states(a.states, [&](auto states) -> cudaError_t {
      using T = decltype(tag);
      constexpr int S = decltype(states)::value;
      const dim3 grid(static_cast<unsigned>(p.chunks * a.groups * p.blocks), a.batch);
      auto go = [&](auto kernel, size_t smem) {
        ++*launches;
        const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kernel), smem);
        if (e != cudaSuccess) return e;
        return launch_pdl(kernel, grid, dim3(kThreads), smem, st, a, g, p, w);
      };
      cudaError_t e;
      if (p.chunks > 1) {
        e = vec ? go(k_grad_local<T, S, true>, sizeof(Staged<S>)) : go(k_grad_local<T, S, false>, sizeof(Staged<S>));
        if (e != cudaSuccess) return e;
        ++*launches;
        e = launch_pdl(k_grad_carry, dim3(static_cast<unsigned>((of_seq + 255) / 256), a.batch), dim3(256), 0, st, a, g,
                       p, w);
        if (e != cudaSuccess) return e;
      }
      e = vec ? go(k_grad_chunk<T, S, true>, sizeof(Walk<S>)) : go(k_grad_chunk<T, S, false>, sizeof(Walk<S>));
      if (e != cudaSuccess) return e;
      Finish f{};
      if (g.B != nullptr || g.C != nullptr)
        f.bc_blocks = (a.batch * a.length * a.groups * a.states + 255) / 256;
      f.sum_blocks = (of_seq + static_cast<long long>(kVecs) * a.dim + 31) / 32;
      if (a.taps > 1) f.edge_blocks = (a.batch * p.chunks * (a.taps - 1) * a.dim + 255) / 256;
      ++*launches;
      return launch_pdl(k_grad_finish<T>, dim3(static_cast<unsigned>(f.bc_blocks + f.sum_blocks + f.edge_blocks)),
                        dim3(256), 0, st, a, g, p, f, static_cast<const unsigned char*>(w));
    });
  });
}

}  // namespace mlt
