// Selective scan with its short causal convolution: prompts and single tokens.
//
//   h_t = exp(d_t A) h_(t-1) + d_t u_t B_t,   y_t = (C_t . h_t + skip u_t) silu(z_t)
//   u = silu(causal convolution of x), d = softplus(dt + dt_bias)
//
// Prompts.  The recurrence is sequential in t and independent over channels and
// states.  Where sequences x channels fill the GPU, one CTA walks a sequence's 32 channels from
// start to end: inputs are read once, states stay in registers.  Where
// they do not, sequences are cut into chunks: since A does not depend on t, a
// chunk acts on a state as h -> exp(A sum d) h + e, with e its end state from zero.
//   k_scan<.., kOut = false>  e and sum d of every chunk but the last
//   k_scan_carry              the state before each chunk
//   k_scan<.., kOut = true>   the outputs of each chunk from the state before it
// which evaluates the exponentials twice.
//
// Bound: issue and shared memory.  With 16 states, 16 channels' step costs two warps about 70
// instructions (half of them the activations) and 23 wavefronts of shared memory: a
// load returns 128 bytes a cycle whether lanes read the same address or not, so each lane
// walks two channels with one load of B and C.  16 exponentials a channel at 32 a cycle and SM
// would take a third of the time.  History: registers for inputs of the next
// tile, unpacked after the load, waited for memory (466 us on 8 x 2048 x 2048 ragged; packed
// until used 329); two lanes of eight states a channel 310; staging by warps of their
// own behind the walk 270; two channels a lane 232.  Now 216 to 237 us by the lengths drawn;
// one sequence of 16,381 x 1,024 in fp32 169 us in chunks, 40 % of it the chunks' end states.
//
// Single tokens (length 1).  Bound by reading and writing the states: k_scan_step, 512 x 2,048
// channels of 16 states in 39 us (4.0 TB/s).
#include "scan.cuh"

namespace mlt {
namespace {

using namespace scan;

constexpr int kCh = 32;            // channels of a CTA
constexpr int kLanes = 4;          // lanes that share two channels, each with S states of both
constexpr int kWalkers = kLanes * kCh / 2;
constexpr int kStagers = 64;
constexpr int kThreads = kWalkers + kStagers;
constexpr int kPairs = kCh / 2;
constexpr int kTile = 16;          // positions staged at a time
constexpr int kRun = kTile / (kStagers / kPairs);  // of these, a stager's
constexpr int kHalo = kScanMaxTaps - 1;
static_assert(kRun >= kHalo, "one stager has the rows that the next tile's convolution reads");

// Sequences are cut into `chunks` of `chunk` positions (a multiple of kTile).
struct Plan {
  long long chunk;
  int chunks;
  size_t off_e, off_sum, bytes;
};

// ---------------------------------------------------------------------------
// Prompts
// ---------------------------------------------------------------------------
// Inputs as they are in memory.
template <typename T, int S>
struct alignas(16) Raw {
  T x[kHalo + kTile][kCh];  // the rows before the tile first
  T dt[kTile][kCh];
  T z[kTile][kCh];
  T B[kTile][kLanes * S];
  T C[kTile][kLanes * S];
};
// What the walk reads, by channel pairs, and its C . h.
template <int S>
struct alignas(16) Staged {
  float4 push[kTile][kPairs];  // d, d u of the first channel, of the second
  float4 out[kTile][kPairs];   // skip u of both, gate of both
  float2 y[kTile][kPairs];
  float B[kTile][kLanes * S];
  float C[kTile][kLanes * S];
};
template <typename T, int S>
struct alignas(16) Tiles {
  Raw<T, S> raw[2];
  Staged<S> staged[2];
};

template <int W>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  const unsigned s = static_cast<unsigned>(__cvta_generic_to_shared(to));
  if constexpr (W == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(s), "l"(from) : "memory");
}
// W bytes; 2 bytes cannot be copied asynchronously.
template <typename T, int W>
__device__ __forceinline__ void copy(T* to, const T* from) {
  if constexpr (W >= 4) copy_async<W>(to, from);
  else *to = *from;
}

// A stager's share of a tile of x, dt or z: column and first row; W bytes an access.
template <typename T, int W>
struct Columns {
  static constexpr int kEach = W / sizeof(T), kPer = kCh / kEach, kStride = kStagers / kPer;
  static_assert(kStagers % kPer == 0 && kTile % kStride == 0, "a stager keeps its column");
  const T* p;
  long long tile, stride;  // elements to the next tile's row, to its next row of this tile

  __device__ __forceinline__ Columns(const void* base, long long first, long long step, int id)
      : p(static_cast<const T*>(base) + first + (id / kPer) * step + id % kPer * kEach),
        tile(kTile * step), stride(kStride * step) {}
  __device__ __forceinline__ void fetch(T (*to)[kCh], int id, int rows, int cn) {
    const int c = id % kPer * kEach, r0 = id / kPer;
    const T* q = p;
    p += tile;
    if (c >= cn) return;
#pragma unroll
    for (int i = 0; i < kTile / kStride; ++i) {
      if (r0 + i * kStride < rows) copy<T, W>(&to[r0 + i * kStride][c], q);
      q += stride;
    }
  }
};
// The same of B or C; kRows: 16 bytes an access.
template <typename T, int S, bool kRows>
struct States {
  static constexpr int N = kLanes * S;
  static constexpr bool kWide = kRows && N * sizeof(T) >= 16;
  static constexpr int kEach = kWide ? 16 / sizeof(T) : 1, kPer = N / kEach;
  const T* p;
  long long tile, step;

  __device__ __forceinline__ States(const void* base, long long first, long long step_, int id)
      : p(static_cast<const T*>(base) + first + (id / kPer) * step_ + id % kPer * kEach), tile(kTile * step_), step(step_) {}
  __device__ __forceinline__ void fetch(T (*to)[N], int id, int rows, int n) {
    static_assert(kStagers % kPer == 0, "a stager keeps its states");
    constexpr int kStride = kStagers / kPer;
    const int c = id % kPer * kEach, r0 = id / kPer;
    const T* q = p;
    p += tile;
#pragma unroll
    for (int i = 0; i < (kTile + kStride - 1) / kStride; ++i) {
      const int r = r0 + i * kStride;
      if (r < rows && r < kTile && c < n) copy<T, kWide ? 16 : sizeof(T)>(&to[r][c], q);
      q += kStride * step;
    }
  }
};

// Two warps walk a tile while two others write the one before and stage the one after it, whose
// inputs land meanwhile: one barrier a tile.
// kOut: writes y and the last state; otherwise a chunk's end state from zero and sum of steps.
// W: bytes of an access to x, dt and z; kRows: B and C are read by 16 bytes.
template <typename T, int S, int W, bool kRows, bool kOut>
__global__ void __launch_bounds__(kThreads, 5) k_scan(mlt_scan_args a, Plan p, unsigned char* ws) {
  extern __shared__ __align__(16) unsigned char smem[];
  Tiles<T, S>& sm = *reinterpret_cast<Tiles<T, S>*>(smem);
  pdl_wait();
  pdl_trigger();
  const Block k = block_of<kCh>(a, blockIdx.x, blockIdx.y);
  const int chunk = blockIdx.z;
  const long long len = length_of(a, k.b);
  const long long begin = chunk * p.chunk, stop = min(begin + p.chunk, static_cast<long long>(a.length));
  const long long end = min(stop, len);  // positions begin .. end - 1 count
  const int tiles = end > begin ? static_cast<int>((end - begin + kTile - 1) / kTile) : 0;
  const long long of_seq = static_cast<long long>(a.dim) * a.states;

  if (threadIdx.x < kWalkers) {
    const int lane = threadIdx.x % kLanes, pair = threadIdx.x / kLanes;
    const long long at = static_cast<long long>(k.c0 + 2 * pair) * a.states + lane * S;
    Lane<S> A[2], h[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      A[c] = h[c] = lane_zero<S>();
      if (2 * pair + c >= k.cn) continue;
      const long long o = at + c * a.states;
      A[c] = lane_load<S>(a.A + o, lane * S, a.states);
      const float* from = p.chunks > 1 ? (kOut ? reinterpret_cast<const float*>(ws + p.off_e) +
                                                     (static_cast<long long>(k.b) * p.chunks + chunk) * of_seq
                                               : nullptr)
                                       : (a.state != nullptr ? a.state + k.b * of_seq : nullptr);
      if (from != nullptr) h[c] = lane_load<S>(from + o, lane * S, a.states);
#pragma unroll
      for (int s = 0; s < Lane<S>::H; ++s) A[c].v[s] = rate2(A[c].v[s]);
    }
    float sum[2] = {0.0f, 0.0f};
#pragma unroll 1
    for (int i = 0; i < tiles; ++i) {
      __syncthreads();
      Staged<S>& st = sm.staged[i & 1];
#pragma unroll(S > 4 ? 1 : 2)
      for (int t = 0; t < kTile; t += 4) {
        float y[2][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 dd = st.push[t + e][pair];
          const float d[2] = {dd.x, dd.z}, du[2] = {dd.y, dd.w};
          const Lane<S> B = lane_shared<S>(&st.B[t + e][lane * S]);
          Lane<S> C;
          if (kOut) C = lane_shared<S>(&st.C[t + e][lane * S]);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            F2 o = dup2(0.0f);
#pragma unroll
            for (int s = 0; s < Lane<S>::H; ++s) {
              h[c].v[s] = fma2(decay2(dup2(d[c]), A[c].v[s]), h[c].v[s], mul2(dup2(du[c]), B.v[s]));
              if (kOut) o = s == 0 ? mul2(C.v[0], h[c].v[0]) : fma2(C.v[s], h[c].v[s], o);
            }
            if (kOut) {
              float o0, o1;
              un2(o, o0, o1);
              y[c][e] = o0 + o1;
            } else {
              sum[c] += d[c];
            }
          }
        }
        if (kOut) st.y[t + lane][pair] = make_float2(quad_sums(y[0], lane), quad_sums(y[1], lane));
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if (2 * pair + c >= k.cn) continue;
      const long long o = at + c * a.states;
      if (!kOut) {
        const long long seq = static_cast<long long>(k.b) * p.chunks + chunk;
        lane_store<S>(reinterpret_cast<float*>(ws + p.off_e) + seq * of_seq + o, lane * S, a.states, h[c]);
        if (lane == 0) reinterpret_cast<float*>(ws + p.off_sum)[seq * a.dim + k.c0 + 2 * pair + c] = sum[c];
      } else if (a.state_out != nullptr && chunk == p.chunks - 1) {
        lane_store<S>(a.state_out + k.b * of_seq + o, lane * S, a.states, h[c]);
      }
    }
    return;
  }

  const int id = threadIdx.x - kWalkers;
  const bool gated = kOut && a.z != nullptr;
  const long long g0 = static_cast<long long>(k.g) * a.states;
  Columns<T, W> fx(a.x, k.b * a.x_batch + begin * a.x_step + k.c0, a.x_step, id);
  Columns<T, W> fd(a.dt, k.b * a.dt_batch + begin * a.dt_step + k.c0, a.dt_step, id);
  Columns<T, W> fz(a.z, k.b * a.z_batch + begin * a.z_step + k.c0, a.z_step, id);
  States<T, S, kRows> fB(a.B, k.b * a.B_batch + begin * a.B_step + g0, a.B_step, id);
  States<T, S, kRows> fC(a.C, k.b * a.C_batch + begin * a.C_step + g0, a.C_step, id);
  const int positions = static_cast<int>(max(0ll, end - begin)), written = static_cast<int>(max(0ll, stop - begin));
  auto fetch = [&](int i) {
    if (i < tiles) {
      const int rows = positions - i * kTile;
      Raw<T, S>& raw = sm.raw[i & 1];
      fx.fetch(raw.x + kHalo, id, rows, k.cn);
      fd.fetch(raw.dt, id, rows, k.cn);
      if (gated) fz.fetch(raw.z, id, rows, k.cn);
      fB.fetch(raw.B, id, rows, a.states);
      if (kOut) fC.fetch(raw.C, id, rows, a.states);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  fetch(0);
  if (a.taps > 1 && tiles > 0)
    for (int i = id; i < kHalo * kCh; i += kStagers)
      if (i % kCh < k.cn)
        sm.raw[0].x[i / kCh][i % kCh] = from_f32<T>(input_at<T>(a, k.b, begin - kHalo + i / kCh, k.c0 + i % kCh));
  // a thread's two channels and kRun positions
  const int c = id % kPairs * 2, n = max(0, min(2, k.cn - c)), run = id / kPairs * kRun;
  float skip[2], w[kScanMaxTaps][2], conv_b[2], bias[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int ch = k.c0 + c + e;
    skip[e] = kOut && a.skip != nullptr && e < n ? a.skip[ch] : 0.0f;
    bias[e] = a.dt_bias != nullptr && e < n ? a.dt_bias[ch] : 0.0f;
    conv_b[e] = a.taps > 0 && a.conv_b != nullptr && e < n ? a.conv_b[ch] : 0.0f;
#pragma unroll
    for (int j = 0; j < kScanMaxTaps; ++j)
      w[j][e] = j < a.taps && e < n ? a.conv_w[static_cast<long long>(ch) * a.taps + a.taps - 1 - j] : 0.0f;
  }
  T* const y0 = kOut ? static_cast<T*>(a.y) + k.b * a.y_batch + begin * a.y_step + k.c0 + c : nullptr;
  T* yp = kOut ? y0 + run * a.y_step : nullptr;
  auto write = [&](int i) {
    const Staged<S>& st = sm.staged[i & 1];
    const int rows = n > 0 ? written - i * kTile - run : 0, live = positions - i * kTile - run;
    T* to = yp;
    yp += kTile * a.y_step;
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      const float4 o = st.out[run + j][c / 2];
      const float2 y = st.y[run + j][c / 2];
      // (past the sequence's end 0, whatever the state: a factor of 0 would leave NaN)
      const F2 v = j < live ? f2((y.x + o.x) * o.z, (y.y + o.y) * o.w) : dup2(0.0f);
      if (j < rows) store_two<T, (W >= 2 * sizeof(T))>(to, n, v);
      to += a.y_step;
    }
  };
  // kFull: every position and channel counts, there is a convolution and (for y) a gate
  auto stage = [&](int i, auto full) {
    constexpr bool kFull = decltype(full)::value;
    const Raw<T, S>& raw = sm.raw[i & 1];
    Staged<S>& st = sm.staged[i & 1];
    const int live = min(kTile, positions - i * kTile);
    float x[kScanMaxTaps][2];  // the window: x[0] is the position's own
#pragma unroll
    for (int j = 1; j < kScanMaxTaps; ++j) un2(shared_two(&raw.x[kHalo + run - j][c]), x[j][0], x[j][1]);
#pragma unroll
    for (int r = 0; r < kRun; ++r) {
      const int t = run + r;
      un2(shared_two(&raw.x[kHalo + t][c]), x[0][0], x[0][1]);
      float dt[2], z[2] = {0.0f, 0.0f}, d[2], du[2], add[2], gate[2];
      un2(shared_two(&raw.dt[t][c]), dt[0], dt[1]);
      if (kOut && (kFull || gated)) un2(shared_two(&raw.z[t][c]), z[0], z[1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float u = x[0][e];
        if (kFull || a.taps > 0) {
          u = fmaf(w[0][e], u, conv_b[e]);
#pragma unroll
          for (int j = 1; j < kScanMaxTaps; ++j)
            if (j < a.taps) u = fmaf(w[j][e], x[j][e], u);
          u *= sigmoid(u);
        }
        const bool ok = kFull || (t < live && e < n);
        d[e] = ok ? softplus(dt[e] + bias[e]) : 0.0f;
        u = ok ? u : 0.0f;
        du[e] = d[e] * u;
        if (kOut) {
          add[e] = skip[e] * u;
          gate[e] = !ok ? 0.0f : kFull || gated ? z[e] * sigmoid(z[e]) : 1.0f;
        }
      }
      st.push[t][c / 2] = make_float4(d[0], du[0], d[1], du[1]);
      if (kOut) st.out[t][c / 2] = make_float4(add[0], add[1], gate[0], gate[1]);
#pragma unroll
      for (int j = kScanMaxTaps - 1; j > 0; --j)
#pragma unroll
        for (int e = 0; e < 2; ++e) x[j][e] = x[j - 1][e];
      // the next tile's rows before it
      if (r >= kRun - kHalo && run + kRun == kTile)
        copy_two(&sm.raw[(i & 1) ^ 1].x[r - (kRun - kHalo)][c], &raw.x[kHalo + t][c]);
    }
    // B and C as floats, zero where nothing was read
    constexpr int N = kLanes * S;
    auto rows = [&](const T (*from)[N], float (*to)[N]) {
      if constexpr (kFull && kRows && N % 4 == 0 && (kTile * N / 4) % kStagers == 0) {
#pragma unroll
        for (int j = 0; j < kTile * N / 4 / kStagers; ++j) {
          const int e = (id + j * kStagers) * 4;
          float4 v;
          un2(shared_two(&from[0][0] + e), v.x, v.y);
          un2(shared_two(&from[0][0] + e + 2), v.z, v.w);
          *reinterpret_cast<float4*>(&to[0][0] + e) = v;
        }
      } else {
        for (int j = id; j < kTile * N / 2; j += kStagers) {
          const int t = j / (N / 2), s = j % (N / 2) * 2;
          float2 v;
          un2(shared_two(&from[t][s]), v.x, v.y);
          if (t >= live || s >= a.states) v.x = 0.0f;
          if (t >= live || s + 1 >= a.states) v.y = 0.0f;
          *reinterpret_cast<float2*>(&to[t][s]) = v;
        }
      }
    };
    rows(raw.B, st.B);
    if (kOut) rows(raw.C, st.C);
  };
  const bool plain = k.cn == kCh && a.taps > 0 && (!kOut || gated);
  // inputs of tile i are here; those of the next are sent for; tile i is staged
  auto prepare = [&](int i) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    asm volatile("bar.sync 1, 64;" ::: "memory");
    fetch(i + 1);
    if (plain && positions >= (i + 1) * kTile) stage(i, std::true_type());
    else stage(i, std::false_type());
  };
  static_assert(kStagers == 64, "the stagers' barrier counts them");
  if (tiles > 0) prepare(0);
#pragma unroll 1
  for (int i = 0; i < tiles; ++i) {
    __syncthreads();
    if (kOut && i > 0) write(i - 1);
    if (i + 1 < tiles) prepare(i + 1);
  }
  __syncthreads();
  if (!kOut) return;
  if (tiles > 0) write(tiles - 1);
  if (n > 0)  // tiles past the sequence's end
    for (int t = tiles * kTile + id / kPairs; t < written; t += kStagers / kPairs)
      store_two<T, (W >= 2 * sizeof(T))>(y0 + t * a.y_step, n, dup2(0.0f));
  // the inputs before the sequence's end (chunk 0 is the only reader of conv_state, and has read it)
  if (chunk == 0 && a.conv_state_out != nullptr && id < k.cn) {
    T* out = static_cast<T*>(a.conv_state_out) + static_cast<long long>(k.b) * (a.taps - 1) * a.dim + k.c0 + id;
    const T* old = static_cast<const T*>(a.conv_state) + static_cast<long long>(k.b) * (a.taps - 1) * a.dim + k.c0 + id;
    const T* x = static_cast<const T*>(a.x) + k.b * a.x_batch + k.c0 + id;
    for (int j = 0; j < a.taps - 1; ++j) {
      const long long i = len + j;  // counted from taps - 1 before the start
      T v = from_f32<T>(0.0f);
      if (i >= a.taps - 1) v = x[(i - (a.taps - 1)) * a.x_step];
      else if (a.conv_state != nullptr) v = old[i * a.dim];
      out[static_cast<long long>(j) * a.dim] = v;
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
  float* e = reinterpret_cast<float*>(ws + p.off_e) + static_cast<long long>(b) * p.chunks * of_seq + i;
  const float* sum = reinterpret_cast<const float*>(ws + p.off_sum) + static_cast<long long>(b) * p.chunks * a.dim +
                     i / a.states;
  const float A = rate(a.A[i]);
  float h = a.state != nullptr ? a.state[b * of_seq + i] : 0.0f;
  const int last = p.chunks - 1;
  const int live = static_cast<int>((length_of(a, b) + p.chunk - 1) / p.chunk);  // later chunks leave the state
  // loads of eight chunks first: the stores go to the same memory
  for (int c0 = 0; c0 < last; c0 += 8) {
    float end[8], d[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c0 + k < last) {
        end[k] = e[(c0 + k) * of_seq];
        d[k] = sum[static_cast<long long>(c0 + k) * a.dim];
      }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c0 + k < last) {
        e[(c0 + k) * of_seq] = h;
        if (c0 + k < live) h = fmaf(ex2(A * d[k]), h, end[k]);
      }
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
      const F2 decay = decay2(f2(dk * kLog2E, dk * kLog2E), A.v[s]);
      if (live) h[k].v[s] = fma2(decay, h[k].v[s], mul2(f2(pk, pk), f2(Bs[2 * s], Bs[2 * s + 1])));
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
  if (in) static_cast<T*>(a.y)[b * a.y_batch + c] = from_f32<T>(live ? (y + add) * gate : 0.0f);
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

// One chunk where sequences x channel blocks give every SM three CTAs or more; else chunks for about ten
// CTAs an SM, no more of them than lengths of 64 (two of 48 for 65 positions).
Plan plan_of(const mlt_scan_args& a, int sms) {
  Plan p{};
  const long long ctas = static_cast<long long>(a.batch) * a.groups * blocks_per_group<kCh>(a);
  long long chunks = 1;
  if (ctas > 0 && ctas < 3LL * sms) chunks = (10LL * sms + ctas - 1) / ctas;
  const long long most = (a.length + 63) / 64;
  if (chunks > most) chunks = most;
  if (chunks > 4096) chunks = 4096;
  if (chunks < 1) chunks = 1;
  p.chunk = ((a.length + chunks - 1) / chunks + kTile - 1) / kTile * kTile;
  if (p.chunk < kTile) p.chunk = kTile;
  p.chunks = static_cast<int>((a.length + p.chunk - 1) / p.chunk);
  if (p.chunks < 1) p.chunks = 1;
  if (p.chunks > 1) {
    const size_t seqs = static_cast<size_t>(a.batch) * p.chunks;
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
  // bytes of an access to x, dt, z and y that every row's address allows
  const int e = static_cast<int>(dtype_size(a.dtype));
  auto all = [&](int bytes) {
    const int64_t n = bytes / e;
    auto ok = [&](const void* q, int64_t step, int64_t batch) {
      return q == nullptr || (aligned_to(q, bytes) && step % n == 0 && batch % n == 0);
    };
    return a.dim / a.groups % n == 0 && ok(a.x, a.x_step, a.x_batch) && ok(a.dt, a.dt_step, a.dt_batch) &&
           ok(a.z, a.z_step, a.z_batch) && ok(a.y, a.y_step, a.y_batch);
  };
  const int width = all(16) ? 16 : e == 2 && all(4) ? 4 : e;
  const int64_t n16 = 16 / e;
  const bool rows = a.states == states_padded(a.states) && a.states % n16 == 0 && aligned_to(a.B, 16) &&
                    aligned_to(a.C, 16) && a.B_step % n16 == 0 && a.C_step % n16 == 0 && a.B_batch % n16 == 0 &&
                    a.C_batch % n16 == 0;
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
      const unsigned blocks = static_cast<unsigned>(a.groups * blocks_per_group<kCh>(a));
      auto go = [&](auto kernel, unsigned chunks) {
        ++*launches;
        constexpr size_t smem = sizeof(Tiles<T, S>);
        const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kernel), smem);
        if (e != cudaSuccess) return e;
        return launch_pdl(kernel, dim3(blocks, a.batch, chunks), dim3(kThreads), smem, st, a, p, w);
      };
      auto pass = [&](auto out, unsigned chunks) {
        constexpr bool kOut = decltype(out)::value;
        if (width == 16)
          return rows ? go(k_scan<T, S, 16, true, kOut>, chunks) : go(k_scan<T, S, 16, false, kOut>, chunks);
        if (width == 4 || sizeof(T) == 4) return go(k_scan<T, S, 4, false, kOut>, chunks);
        return go(k_scan<T, S, sizeof(T), false, kOut>, chunks);
      };
      if (p.chunks > 1) {
        cudaError_t e = pass(std::false_type(), p.chunks - 1);
        if (e != cudaSuccess) return e;
        ++*launches;
        const long long of_seq = static_cast<long long>(a.dim) * a.states;
        e = launch_pdl(k_scan_carry, dim3(static_cast<unsigned>((of_seq + 255) / 256), a.batch), dim3(256), 0, st, a, p,
                       w);
        if (e != cudaSuccess) return e;
      }
      return pass(std::true_type(), p.chunks);
    });
  });
}

}  // namespace mlt
