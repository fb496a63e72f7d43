// Embedding lookup and its gradient.
//
//   out[i][c]  = round(scale * table[id_i][c])              (one rounding)
//   grad[v][c] = round(scale * sum over i with id_i = v of g[i][c])
//
// A negative id is padding: its output row is zero and it adds to no
// gradient.  An id >= vocab does the same and sets the error word.
//
// Both are bound by memory: the lookup reads each distinct row and writes
// tokens x dim values, the gradient reads tokens x dim values once and writes
// vocab x dim.  The gradient sorts the token positions by id (stable radix
// sort, 8 bits a pass, so equal ids keep the order of their positions) and adds each
// run of equal ids in that order: no atomics on floating point, so the result
// does not change from call to call, and every gradient row is written once.
#include "seq.cuh"

namespace mlt {
namespace {

template <typename I>
__device__ __forceinline__ long long load_id(const void* ids, long long i) {
  return static_cast<long long>(static_cast<const I*>(ids)[i]);
}
__device__ __forceinline__ long long id_of(const void* ids, int ids_64, long long i) {
  return ids_64 ? load_id<long long>(ids, i) : load_id<int>(ids, i);
}

// ---------------------------------------------------------------------------
// Lookup: `lanes` lanes of a warp per row (a power of two), kUnroll packs of V
// elements a lane, so every lane has kUnroll independent loads in flight.
// 32,768 bf16 rows of 2,048: 27.6 us, 6.1 TB/s with the reads.
// ---------------------------------------------------------------------------
constexpr int kUnroll = 4;

template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256) k_embed(const TI* table, long long in_stride, const void* ids, int ids_64,
                                               long long tokens, long long vocab, int dim, float scale, TO* out,
                                               long long out_stride, int lanes, unsigned* err) {
  const int lane = threadIdx.x & (lanes - 1);
  const long long i = static_cast<long long>(blockIdx.x) * (256 / lanes) + threadIdx.x / lanes;
  pdl_wait();
  pdl_trigger();
  if (i >= tokens) return;
  const long long id = id_of(ids, ids_64, i);
  const bool live = id >= 0 && id < vocab;
  const int packs = dim / V;
  const int first = blockIdx.y * lanes * kUnroll + lane;
  if (id >= vocab && first == 0) atomicOr(err, kErrBadToken);
  const TI* row = table + (live ? id : 0) * in_stride;
  TO* dst = out + i * out_stride;
  Pack<TI, V> p[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int c = first + u * lanes;
    if (live && c < packs) p[u] = *reinterpret_cast<const Pack<TI, V>*>(row + static_cast<long long>(c) * V);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int c = first + u * lanes;
    if (c >= packs) break;
    Pack<TO, V> q;
#pragma unroll
    for (int e = 0; e < V; ++e) q.v[e] = from_f32<TO>(live ? __fmul_rn(to_f32(p[u].v[e]), scale) : 0.0f);
    *reinterpret_cast<Pack<TO, V>*>(dst + static_cast<long long>(c) * V) = q;
  }
}

// The same with `rows` whole rows a warp, one after the other: for rows of more than 64 narrow packs, where
// k_embed's warps are short and what each does before its first load counts.  200,000 rows: of 269
// 16-bit values (packs of one) 33 us for 101, 269 fp32 values 42 for 102, 402 16-bit values 33 for
// 69; with 35 packs 24 for 20, and with packs of 16 bytes no gain.
constexpr int kRowsUnroll = 8;

template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256) k_embed_rows(const TI* table, long long in_stride, const void* ids, int ids_64,
                                                    long long tokens, long long vocab, int dim, float scale, TO* out,
                                                    long long out_stride, int rows, unsigned* err) {
  const int lane = threadIdx.x & 31;
  const long long first = (static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5)) * rows;
  pdl_wait();
  pdl_trigger();
  if (first >= tokens) return;
  const int have = static_cast<int>(min(static_cast<long long>(rows), tokens - first)), packs = dim / V;
  int mine = -1;
  if (lane < have) {
    const long long id = id_of(ids, ids_64, first + lane);
    if (id >= vocab) atomicOr(err, kErrBadToken);
    if (id >= 0 && id < vocab) mine = static_cast<int>(id);
  }
  TO* dst = out + first * out_stride;
  for (int r = 0; r < have; ++r, dst += out_stride) {
    const int id = __shfl_sync(0xffffffffu, mine, r);
    const bool live = id >= 0;
    const TI* row = table + (live ? id : 0) * in_stride;
    for (int c0 = 0; c0 < packs; c0 += 32 * kRowsUnroll) {
      const int c1 = c0 + lane, left = packs - c1;
      const TI* from = row + static_cast<long long>(c1) * V;
      TO* to = dst + static_cast<long long>(c1) * V;
      Pack<TI, V> p[kRowsUnroll];
#pragma unroll
      for (int u = 0; u < kRowsUnroll; ++u)
        if (live && u * 32 < left) p[u] = *reinterpret_cast<const Pack<TI, V>*>(from + u * 32 * V);
#pragma unroll
      for (int u = 0; u < kRowsUnroll; ++u) {
        if (u * 32 >= left) break;
        Pack<TO, V> q;
#pragma unroll
        for (int e = 0; e < V; ++e) q.v[e] = from_f32<TO>(live ? __fmul_rn(to_f32(p[u].v[e]), scale) : 0.0f);
        *reinterpret_cast<Pack<TO, V>*>(to + u * 32 * V) = q;
      }
    }
  }
}

// Widest pack (elements) that divides the row length, both strides and both
// addresses; at most 16 bytes of the narrower type.
int pack_width(const EmbedArgs& a) {
  const size_t si = dtype_size(a.in_dtype), so = dtype_size(a.out_dtype);
  for (int v = si == 4 && so == 4 ? 4 : 8; v > 1; v /= 2) {
    const size_t bi = v * si > 16 ? 16 : v * si, bo = v * so > 16 ? 16 : v * so;
    if (a.dim % v == 0 && a.in_stride % v == 0 && a.out_stride % v == 0 && aligned_to(a.table, bi) &&
        aligned_to(a.out, bo))
      return v;
  }
  return 1;
}

template <typename F>
cudaError_t with_width(int v, F f) {
  switch (v) {
    case 8: return f(std::integral_constant<int, 8>());
    case 4: return f(std::integral_constant<int, 4>());
    case 2: return f(std::integral_constant<int, 2>());
    default: return f(std::integral_constant<int, 1>());
  }
}

// ---------------------------------------------------------------------------
// Stable radix sort of token positions by id
// ---------------------------------------------------------------------------
// The warp's lanes with the caller's digit, among those `in`: a ballot for each of eight bits.
// (__match_any_sync gives it in one instruction, but takes the SM 190 cycles a warp.)
__device__ __forceinline__ unsigned lanes_with(uint32_t digit, bool in) {
  unsigned peers = __ballot_sync(~0u, in);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const unsigned set = __ballot_sync(~0u, digit >> b & 1u);
    peers &= digit >> b & 1u ? set : ~set;
  }
  return peers;
}

constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigits = 256;
// Positions a lane takes: a tile of 4,096 a CTA, or of 1,024 where there are too few
// positions to give every SM a large one.
int sort_per_lane(long long tokens) { return tokens > (1 << 18) ? 8 : 2; }

struct SortPass {
  const void* ids;  // first pass: the ids themselves, else null
  int ids_64;
  const uint2* in;  // (key, position) records
  uint2* out;
  uint32_t* counts;  // [kDigits][tiles], then prefixes over the tiles
  uint32_t* totals;  // [kDigits]
  long long tokens, vocab;
  int tiles, shift;
  unsigned char* named;  // first pass: 1 for ids that occur, else 0
  unsigned* err;
};

// Ids outside [0, vocab) sort behind all others.
__device__ __forceinline__ uint2 sort_record(const SortPass& s, long long i) {
  if (s.ids == nullptr) return s.in[i];
  const long long id = id_of(s.ids, s.ids_64, i);
  return make_uint2(static_cast<uint32_t>(id < 0 || id >= s.vocab ? s.vocab : id), static_cast<uint32_t>(i));
}

template <int kPerLane>
__global__ void __launch_bounds__(kSortThreads) k_sort_count(SortPass s) {
  __shared__ uint32_t hist[kDigits];
  for (int d = threadIdx.x; d < kDigits; d += kSortThreads) hist[d] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  if (s.named != nullptr)
    for (long long v = (static_cast<long long>(blockIdx.x) * kSortThreads + threadIdx.x) * 16; v < s.vocab;
         v += static_cast<long long>(gridDim.x) * kSortThreads * 16)
      *reinterpret_cast<uint4*>(s.named + v) = make_uint4(0, 0, 0, 0);  // the array is padded
  const long long base = static_cast<long long>(blockIdx.x) * (kSortThreads * kPerLane);
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    const long long i = base + k * kSortThreads + threadIdx.x;
    if (i >= s.tokens) break;
    if (s.ids != nullptr && id_of(s.ids, s.ids_64, i) >= s.vocab) atomicOr(s.err, kErrBadToken);
    atomicAdd(&hist[(sort_record(s, i).x >> s.shift) & (kDigits - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < kDigits; d += kSortThreads)
    s.counts[static_cast<long long>(d) * s.tiles + blockIdx.x] = hist[d];
}

// One CTA per digit: exclusive prefix over its tiles.
__global__ void __launch_bounds__(256) k_sort_scan(uint32_t* counts, uint32_t* totals, int tiles) {
  __shared__ uint32_t part[8];
  pdl_wait();
  pdl_trigger();
  uint32_t* row = counts + static_cast<long long>(blockIdx.x) * tiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t carry = 0;
  for (int t0 = 0; t0 < tiles; t0 += 256) {
    const int t = t0 + threadIdx.x;
    const uint32_t c = t < tiles ? row[t] : 0;
    uint32_t v = c;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t w = __shfl_up_sync(~0u, v, o);
      if (lane >= o) v += w;
    }
    if (lane == 31) part[warp] = v;
    __syncthreads();
    uint32_t below = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      if (w < warp) below += part[w];
      all += part[w];
    }
    if (t < tiles) row[t] = carry + below + v - c;
    carry += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

template <int kPerLane>
__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(SortPass s) {
  __shared__ uint32_t cnt[kSortWarps][kDigits];
  __shared__ uint2 warp_sum[kDigits / 32];
  __shared__ uint32_t start[kDigits], local[kDigits];
  extern __shared__ __align__(16) unsigned char smem[];
  uint2* tile = reinterpret_cast<uint2*>(smem);  // the tile's records in the order of their digits
  static_assert(kSortThreads == 2 * kDigits, "two threads a digit");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int d = lane; d < kDigits; d += 32) cnt[warp][d] = 0;
  __syncwarp();
  pdl_wait();
  pdl_trigger();
  // a warp owns kPerLane * 32 consecutive positions; rank[k] counts the
  // equal digits before the lane's k-th one within the warp
  const long long base = static_cast<long long>(blockIdx.x) * (kSortThreads * kPerLane) + warp * (kPerLane * 32) + lane;
  uint2 rec[kPerLane];
  uint32_t rank[kPerLane];
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    const long long i = base + k * 32;
    rec[k] = i < s.tokens ? sort_record(s, i) : make_uint2(0, 0);
  }
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    const bool in = base + k * 32 < s.tokens;
    const uint32_t d = (rec[k].x >> s.shift) & (kDigits - 1);
    const unsigned peers = lanes_with(d, in);
    const unsigned before = peers & ((1u << lane) - 1u);
    uint32_t seen = 0;
    if (in) seen = cnt[warp][d];
    __syncwarp();
    rank[k] = seen + __popc(before);
    if (in && before == 0) cnt[warp][d] = seen + __popc(peers);
    __syncwarp();
  }
  __syncthreads();
  // counts of the warps before, two threads a digit
  {
    constexpr int kHalf = kSortWarps / 2;
    const int d = threadIdx.x / 2, first = (threadIdx.x & 1) * kHalf;
    uint32_t c[kHalf], sum = 0;
#pragma unroll
    for (int w = 0; w < kHalf; ++w) {
      c[w] = cnt[first + w][d];
      sum += c[w];
    }
    const uint32_t other = __shfl_xor_sync(~0u, sum, 1);
    if (first == 0) local[d] = sum + other;  // of the tile
    uint32_t at = first > 0 ? other : 0;
#pragma unroll
    for (int w = 0; w < kHalf; ++w) {
      cnt[first + w][d] = at;
      at += c[w];
    }
  }
  __syncthreads();
  // digit d's first place: digits below it, tiles before this one; and within the tile
  const int d = threadIdx.x;
  uint32_t total = 0, v = 0, mine = 0, u = 0;
  if (d < kDigits) {
    total = s.totals[d];
    mine = local[d];
    v = total;
    u = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t w = __shfl_up_sync(~0u, v, o), x = __shfl_up_sync(~0u, u, o);
      if (lane >= o) {
        v += w;
        u += x;
      }
    }
    if (lane == 31) warp_sum[warp] = make_uint2(v, u);
  }
  __syncthreads();
  if (d < kDigits) {
    uint32_t at = v - total + s.counts[static_cast<long long>(d) * s.tiles + blockIdx.x];
    uint32_t here = u - mine;
    for (int w = 0; w < warp; ++w) {
      at += warp_sum[w].x;
      here += warp_sum[w].y;
    }
    local[d] = here;
    start[d] = at - here;  // a record's place in the tile's order plus this is its place
  }
  __syncthreads();
  // through shared memory, so that neighbouring threads write a digit's run
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    if (base + k * 32 >= s.tokens) break;
    const uint32_t digit = (rec[k].x >> s.shift) & (kDigits - 1);
    tile[local[digit] + cnt[warp][digit] + rank[k]] = rec[k];
  }
  __syncthreads();
  const int have = static_cast<int>(
      min(static_cast<long long>(kSortThreads) * kPerLane,
          s.tokens - static_cast<long long>(blockIdx.x) * (kSortThreads * kPerLane)));
#pragma unroll 4
  for (int j = threadIdx.x; j < have; j += kSortThreads) {
    const uint2 r = tile[j];
    s.out[start[(r.x >> s.shift) & (kDigits - 1)] + j] = r;
    // (once a run of equal ids: a million stores to 64 flags took 37 us)
    if (s.named != nullptr && r.x < s.vocab && (j == 0 || tile[j - 1].x != r.x)) s.named[r.x] = 1;
  }
}

// The whole sort in one launch for up to kClusterTokens positions: a cluster of eight CTAs, a
// tile each, that exchange their digit counts through distributed shared memory.  On 32,768
// positions with two digits 22 us, against 31 for six launches; the other CTAs of the
// launch clear the gradient's rows meanwhile (131 MB: 31 us together).  Bound by shared memory and
// the barriers of eight SMs.
constexpr int kCluster = 8;
constexpr int kClusterThreads = 1024;
constexpr int kClusterPerLane = 8;
constexpr int kClusterTokens = kCluster * kClusterThreads * kClusterPerLane;

struct ClusterSort {
  const void* ids;
  int ids_64;
  uint2* rec[2];
  int tokens, passes, per_lane;
  long long vocab;
  unsigned char* named;  // null: the other CTAs of the grid clear the table
  unsigned* err;
  unsigned char* table;
  long long rows, row_bytes, stride_bytes;
};

// Rows of the table to zero by the CTAs after the cluster that sorts: W bytes an access.
template <int W>
__device__ __forceinline__ void clear_rows(const ClusterSort& s) {
  const long long threads = static_cast<long long>(gridDim.x - kCluster) * kClusterThreads;
  const long long per = s.row_bytes / W, all = s.rows * per;
  long long i = static_cast<long long>(blockIdx.x - kCluster) * kClusterThreads + threadIdx.x;
  long long row = i / per, at = i - row * per;
  const long long step_row = threads / per, step_at = threads - step_row * per;
  for (; i < all; i += threads) {
    unsigned char* p = s.table + row * s.stride_bytes + at * W;
    if constexpr (W == 16) *reinterpret_cast<uint4*>(p) = make_uint4(0, 0, 0, 0);
    else *reinterpret_cast<unsigned short*>(p) = 0;
    row += step_row;
    at += step_at;
    if (at >= per) {
      at -= per;
      ++row;
    }
  }
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Word `at` of shared memory in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t remote_word(const uint32_t* at, unsigned rank) {
  uint32_t addr = static_cast<uint32_t>(__cvta_generic_to_shared(at)), there, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(there) : "memory");
  return v;
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kClusterThreads) k_sort_cluster(ClusterSort s) {
  constexpr int kWarps = kClusterThreads / 32;
  __shared__ uint32_t cnt[kWarps][kDigits];
  __shared__ uint32_t total[kDigits];  // of the CTA, read by the others
  __shared__ uint32_t start[kDigits], local[kDigits];
  extern __shared__ __align__(16) unsigned char smem[];
  uint2* tile = reinterpret_cast<uint2*>(smem);
  static_assert(kClusterThreads == 4 * kDigits, "four threads a digit");
  __shared__ uint2 warp_sum[kDigits / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = blockIdx.x;
  pdl_wait();
  pdl_trigger();
  if (rank >= kCluster) {
    if (s.row_bytes % 16 == 0 && s.stride_bytes % 16 == 0 && reinterpret_cast<uintptr_t>(s.table) % 16 == 0)
      clear_rows<16>(s);
    else
      clear_rows<2>(s);
    return;
  }
  if (s.named != nullptr)
    for (long long v = (static_cast<long long>(rank) * kClusterThreads + threadIdx.x) * 16; v < s.vocab;
         v += static_cast<long long>(kCluster) * kClusterThreads * 16)
    *reinterpret_cast<uint4*>(s.named + v) = make_uint4(0, 0, 0, 0);  // the array is padded
  const int base = (rank * kClusterThreads + warp * 32) * s.per_lane + lane;
  uint2 rec[kClusterPerLane];
  uint32_t place[kClusterPerLane];
#pragma unroll
  for (int k = 0; k < kClusterPerLane; ++k) {
    const int i = base + k * 32;
    rec[k] = make_uint2(0, i);
    if (k < s.per_lane && i < s.tokens) {
      const long long id = id_of(s.ids, s.ids_64, i);
      if (id >= s.vocab) atomicOr(s.err, kErrBadToken);
      rec[k].x = static_cast<uint32_t>(id < 0 || id >= s.vocab ? s.vocab : id);
    }
  }
#pragma unroll 1
  for (int pass = 0; pass < s.passes; ++pass) {
    const int shift = 8 * pass;
    if (pass > 0) {
#pragma unroll
      for (int k = 0; k < kClusterPerLane; ++k) {
        const int i = base + k * 32;
        if (k < s.per_lane && i < s.tokens) rec[k] = __ldcg(&s.rec[(pass - 1) & 1][i]);
      }
    }
    for (int d = lane; d < kDigits; d += 32) cnt[warp][d] = 0;
    __syncwarp();
    // place[k]: equal digits before it within the warp
#pragma unroll
    for (int k = 0; k < kClusterPerLane; ++k) {
      if (k >= s.per_lane) break;
      const bool in = base + k * 32 < s.tokens;
      const uint32_t d = (rec[k].x >> shift) & (kDigits - 1);
      const unsigned peers = lanes_with(d, in);
      const unsigned before = peers & ((1u << lane) - 1u);
      const uint32_t seen = in ? cnt[warp][d] : 0;
      __syncwarp();
      place[k] = seen + __popc(before);
      if (in && before == 0) cnt[warp][d] = seen + __popc(peers);
      __syncwarp();
    }
    __syncthreads();
    // counts of the warps before, four threads a digit
    {
      constexpr int kPart = kWarps / 4;
      const int d = threadIdx.x / 4, q = threadIdx.x & 3, first = q * kPart;
      uint32_t c[kPart], sum = 0;
#pragma unroll
      for (int w = 0; w < kPart; ++w) {
        c[w] = cnt[first + w][d];
        sum += c[w];
      }
      uint32_t upto = sum;
#pragma unroll
      for (int o = 1; o < 4; o *= 2) {
        const uint32_t w = __shfl_up_sync(~0u, upto, o);
        if (q >= o) upto += w;
      }
      uint32_t at = upto - sum;
#pragma unroll
      for (int w = 0; w < kPart; ++w) {
        cnt[first + w][d] = at;
        at += c[w];
      }
      if (q == 3) total[d] = upto;
    }
    const int d = threadIdx.x;
    cluster_sync();
    // digit d's first place: digits below it, then the CTAs before this one
    uint32_t below = 0, all = 0, v = 0, mine = 0, u = 0;
    if (d < kDigits) {
#pragma unroll
      for (int r = 0; r < kCluster; ++r) {
        const uint32_t c = remote_word(&total[d], r);
        if (r < rank) below += c;
        if (r == rank) mine = c;
        all += c;
      }
      v = all;
      u = mine;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const uint32_t w = __shfl_up_sync(~0u, v, o), x = __shfl_up_sync(~0u, u, o);
        if (lane >= o) {
          v += w;
          u += x;
        }
      }
      if (lane == 31) warp_sum[warp] = make_uint2(v, u);
    }
    __syncthreads();
    if (d < kDigits) {
      uint32_t at = v - all + below, here = u - mine;
      for (int w = 0; w < warp; ++w) {
        at += warp_sum[w].x;
        here += warp_sum[w].y;
      }
      local[d] = here;
      start[d] = at - here;
    }
    __syncthreads();
    // through shared memory, so that neighbouring threads write a digit's run
#pragma unroll
    for (int k = 0; k < kClusterPerLane; ++k) {
      if (k >= s.per_lane || base + k * 32 >= s.tokens) break;
      const uint32_t digit = (rec[k].x >> shift) & (kDigits - 1);
      tile[local[digit] + cnt[warp][digit] + place[k]] = rec[k];
    }
    __syncthreads();
    const int have = min(kClusterThreads * s.per_lane, s.tokens - rank * kClusterThreads * s.per_lane);
    for (int j = threadIdx.x; j < have; j += kClusterThreads) {
      const uint2 r = tile[j];
      s.rec[pass & 1][start[(r.x >> shift) & (kDigits - 1)] + j] = r;
      if (pass == 0 && s.named != nullptr && r.x < s.vocab && (j == 0 || tile[j - 1].x != r.x)) s.named[r.x] = 1;
    }
    cluster_sync();  // the next pass reads what all wrote, and totals may change
  }
}

// ---------------------------------------------------------------------------
// Sums over runs of equal ids
// ---------------------------------------------------------------------------
// The sorted positions are cut into pieces of `piece`.  `lanes` lanes of a warp
// (a power of two) add the rows of one piece for lanes x V columns.  A run that lies inside
// a piece is finished there; of one that crosses pieces, `lead` takes the sum of
// the part that began before the piece and `trail` of the part that begins in it
// and goes on.  k_grad_join adds those in order.
// Bound by memory: 1,048,573 fp32 rows of 128 in 84 us (6.4 TB/s); 32,768 bf16 rows of
// 2,048 in 32 us (4.2 TB/s: pieces are short there), and 11 us for the joins of either.
struct GradArgs {
  const uint2* rec;  // sorted (id, position)
  long long tokens, vocab;
  int dim, lanes, piece;
  long long pieces;
  float scale;
  long long in_stride, out_stride;
  float* lead;   // [pieces][dim]
  float* trail;  // [pieces][dim]
  long long sum_blocks;  // of k_grad_sum's grid.x; the rest clears rows no id names
  const unsigned char* named;
  bool cleared;  // the table is zero already
};

constexpr int kSumThreads = 128;
constexpr int kClearRows = 16;  // rows a group of lanes looks at
constexpr int kSumUnroll = 8;

template <typename TG, int V>
__device__ __forceinline__ void store_row(TG* out, const float (&acc)[V], float scale) {
  Pack<TG, V> q;
#pragma unroll
  for (int e = 0; e < V; ++e) q.v[e] = from_f32<TG>(__fmul_rn(acc[e], scale));
  *reinterpret_cast<Pack<TG, V>*>(out) = q;
}

template <typename TI, typename TG, int V>
__global__ void __launch_bounds__(kSumThreads) k_grad_sum(GradArgs a, const TI* grad, TG* out) {
  const int groups = kSumThreads / a.lanes;
  const int lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes;
  const int col = (blockIdx.y * a.lanes + lane) * V;
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x >= a.sum_blocks) {
    // rows that no id names
    if (col >= a.dim) return;
    const long long first = (blockIdx.x - a.sum_blocks) * groups * kClearRows + group;
    const float zero[V] = {};
#pragma unroll
    for (int i = 0; i < kClearRows; ++i) {
      const long long v = first + i * groups;
      if (v < a.vocab && (a.named == nullptr || a.named[v] == 0)) store_row<TG, V>(out + v * a.out_stride + col, zero, 1.0f);
    }
    return;
  }
  const long long p = static_cast<long long>(blockIdx.x) * groups + group;
  if (p >= a.pieces || col >= a.dim) return;
  const long long begin = p * a.piece, end = min(begin + a.piece, a.tokens);
  const uint32_t none = static_cast<uint32_t>(a.vocab);
  uint32_t run = a.rec[begin].x;
  bool led = begin > 0 && a.rec[begin - 1].x == run;  // the current run began before the piece
  float acc[V] = {};
  auto flush = [&]() {
    if (run >= none) return;
    if (led) {
      Pack<float, V>* q = reinterpret_cast<Pack<float, V>*>(a.lead + p * a.dim + col);
      Pack<float, V> w;
#pragma unroll
      for (int e = 0; e < V; ++e) w.v[e] = acc[e];
      *q = w;
    } else {
      store_row<TG, V>(out + run * a.out_stride + col, acc, a.scale);
    }
  };
  const int count = static_cast<int>(end - begin);
  const uint2* rp = a.rec + begin;
  const TI* gp = grad + col;
  // a full batch without checks, its keys and positions one batch ahead
  uint2 rec[kSumUnroll];
  auto fetch = [&](int i) {
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      rec[u] = make_uint2(none, 0);
      if (i + u < count) rec[u] = rp[i + u];
    }
  };
  fetch(0);
#pragma unroll 1
  for (int i = 0; i < count; i += kSumUnroll) {
    Pack<TI, V> g[kSumUnroll];
    uint32_t now[kSumUnroll];
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      now[u] = rec[u].x;
      // (past the piece's end position 0 is read and not used)
      g[u] = *reinterpret_cast<const Pack<TI, V>*>(gp + static_cast<long long>(rec[u].y) * a.in_stride);
    }
    fetch(i + kSumUnroll);
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      if (now[u] != run) {
        if (i + u >= count) break;
        flush();
        run = now[u];
        led = false;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
      }
      if (now[u] < none) {
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += to_f32(g[u].v[e]);
      }
    }
  }
  if (run >= none) return;
  const bool goes_on = end < a.tokens && a.rec[end].x == run;
  if (goes_on && !led) {
    Pack<float, V> w;
#pragma unroll
    for (int e = 0; e < V; ++e) w.v[e] = acc[e];
    *reinterpret_cast<Pack<float, V>*>(a.trail + p * a.dim + col) = w;
  } else {
    flush();
  }
}

// Finishes runs that begin in a piece and go on past it.  A CTA looks at eight pieces, a warp each,
// and adds for every run found, 32 x V columns: warp w takes the pieces p + 1 + w, + 8, ...;
// the warps' sums are added in order.
constexpr int kJoinWarps = 8;

// Past the last of the equal keys that a[0] begins: 32 places are looked at a step.
__device__ __forceinline__ long long run_end(const uint2* a, long long n, uint32_t v) {
  const int lane = threadIdx.x & 31;
  long long lo = 0, hi = n;  // a[lo - 1] == v (or lo = 0), a[hi] > v (or hi = n)
  while (lo < hi) {
    const long long step = (hi - lo + 31) / 32;
    const long long at = lo + lane * step;
    const unsigned equal = __ballot_sync(~0u, at < hi && a[at].x == v);
    const int k = __popc(equal);  // the keys are sorted: the first k places hold v
    if (k == 0) return lo;
    const long long from = lo;
    lo = from + (k - 1) * step + 1;
    hi = min(hi, from + k * step);
  }
  return lo;
}

template <typename TG, int V>
__global__ void __launch_bounds__(kJoinWarps * 32) k_grad_join(GradArgs a, TG* out) {
  __shared__ float part[kJoinWarps][32 * V];
  __shared__ long long last_of[kJoinWarps];  // last piece of the run that begins in the warp's piece, or -1
  __shared__ uint32_t run_of[kJoinWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  {
    const long long p = static_cast<long long>(blockIdx.x) * kJoinWarps + warp;
    const long long begin = p * a.piece, end = min(begin + a.piece, a.tokens);
    long long last = -1;
    uint32_t run = 0;
    if (p < a.pieces && end < a.tokens) {
      run = a.rec[end - 1].x;
      const uint32_t next = a.rec[end].x, first = a.rec[begin].x, before = begin > 0 ? a.rec[begin - 1].x : run + 1;
      // goes on, is no padding, and did not begin earlier
      if (run < static_cast<uint32_t>(a.vocab) && next == run && !(first == run && before == run))
        last = (end + run_end(a.rec + end, a.tokens - end, run) - 1) / a.piece;
    }
    if (lane == 0) {
      last_of[warp] = last;
      run_of[warp] = run;
    }
  }
  __syncthreads();
  const int col = (blockIdx.y * 32 + lane) * V;
  const bool in = col < a.dim;
  for (int k = 0; k < kJoinWarps; ++k) {
    const long long last = last_of[k], p = static_cast<long long>(blockIdx.x) * kJoinWarps + k;
    if (last < 0) continue;
    float acc[V] = {};
    if (in) {
      if (warp == 0) {
        const Pack<float, V> w = *reinterpret_cast<const Pack<float, V>*>(a.trail + p * a.dim + col);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = w.v[e];
      }
#pragma unroll 4
      for (long long q = p + 1 + warp; q <= last; q += kJoinWarps) {
        const Pack<float, V> w = *reinterpret_cast<const Pack<float, V>*>(a.lead + q * a.dim + col);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += w.v[e];
      }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) part[warp][e * 32 + lane] = acc[e];
    __syncthreads();
    if (warp == 0 && in) {
      const long long used = last - p;  // warps with a piece (warp 0 has the first's rest too)
      for (int w = 1; w < kJoinWarps && w < used; ++w)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += part[w][e * 32 + lane];
      store_row<TG, V>(out + run_of[k] * a.out_stride + col, acc, a.scale);
    }
    __syncthreads();
  }
}

int pow2_at_most_32(long long v) {
  int l = 1;
  while (l < 32 && l < v) l *= 2;
  return l;
}

struct GradPlan {
  int per_lane, tiles, passes, piece;
  long long pieces;
  bool cluster;  // sorted in one launch
  bool clear;    // the table is cleared meanwhile
  size_t off_rec[2], off_counts, off_totals, off_named, off_lead, off_trail, bytes;
};

// Pieces: 24 to 96 warps for each SM over all column chunks, 16 to 512 rows each, so that a
// run's partial sums stay few beside the rows they stand for.
GradPlan grad_plan(long long tokens, long long vocab, int dim, int sms) {
  GradPlan g{};
  const long long n = tokens < 1 ? 1 : tokens;
  g.cluster = n <= kClusterTokens;
  g.per_lane = sort_per_lane(n);
  g.tiles = static_cast<int>((n + kSortThreads * g.per_lane - 1) / (kSortThreads * g.per_lane));
  int bits = 1;
  while (bits < 32 && (vocab >> bits) != 0) ++bits;
  g.passes = (bits + 7) / 8;
  const long long work = n * ((dim + 127) / 128);
  g.piece = 16;
  while (g.piece < 512 && work / g.piece > 96LL * sms) g.piece *= 2;
  g.pieces = (n + g.piece - 1) / g.piece;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += up256(bytes);
    return o;
  };
  for (int k = 0; k < 2; ++k) {
    g.off_rec[k] = take(n * 8);
  }
  g.off_counts = take(static_cast<size_t>(kDigits) * g.tiles * 4);
  g.off_totals = take(kDigits * 4);
  g.off_named = take(vocab);
  g.off_lead = take(static_cast<size_t>(g.pieces) * dim * 4);
  g.off_trail = take(static_cast<size_t>(g.pieces) * dim * 4);
  g.bytes = at;
  return g;
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs& a, int sms, long long* launches, cudaStream_t st) {
  if (a.tokens == 0) return cudaSuccess;
  ++*launches;
  return with_width(pack_width(a), [&](auto width) {
    constexpr int V = decltype(width)::value;
    return with_dtype(a.in_dtype, [&](auto ti) {
      return with_dtype(a.out_dtype, [&](auto to) {
        using TI = decltype(ti);
        using TO = decltype(to);
        const int packs = a.dim / V;
        const int lanes = pow2_at_most_32((packs + kUnroll - 1) / kUnroll);
        if (packs > 64 && V * (sizeof(TI) < sizeof(TO) ? sizeof(TI) : sizeof(TO)) < 16) {
          // 16 CTAs for each SM before a warp takes a second row, four rows at most
          const long long full = a.tokens / (16LL * 8 * sms);
          const int rows = full < 1 ? 1 : full > 4 ? 4 : static_cast<int>(full);
          const dim3 ctas(static_cast<unsigned>((a.tokens + 8LL * rows - 1) / (8LL * rows)));
          return launch_pdl(k_embed_rows<TI, TO, V>, ctas, dim3(256), 0, st, static_cast<const TI*>(a.table), a.in_stride,
                            a.ids, a.ids_64, a.tokens, a.vocab, a.dim, a.scale, static_cast<TO*>(a.out), a.out_stride,
                            rows, a.err);
        }
        const long long per = 256 / lanes;
        const dim3 grid(static_cast<unsigned>((a.tokens + per - 1) / per),
                        static_cast<unsigned>((packs + lanes * kUnroll - 1) / (lanes * kUnroll)));
        return launch_pdl(k_embed<TI, TO, V>, grid, dim3(256), 0, st, static_cast<const TI*>(a.table), a.in_stride,
                          a.ids, a.ids_64, a.tokens, a.vocab, a.dim, a.scale, static_cast<TO*>(a.out), a.out_stride,
                          lanes, a.err);
      });
    });
  });
}

size_t embed_grad_workspace(long long tokens, long long vocab, int dim, int sms) {
  return grad_plan(tokens, vocab, dim, sms).bytes;
}

cudaError_t launch_embed_grad(const EmbedArgs& a, int sms, long long* launches, cudaStream_t st) {
  GradPlan g = grad_plan(a.tokens, a.vocab, a.dim, sms);
  unsigned char* ws = static_cast<unsigned char*>(a.ws);
  auto u32 = [&](size_t off) { return reinterpret_cast<uint32_t*>(ws + off); };
  auto records = [&](int k) { return reinterpret_cast<uint2*>(ws + g.off_rec[k]); };
  const uint2* sorted = nullptr;
  if (a.tokens > 0 && g.cluster) {
    ClusterSort s{};
    s.ids = a.ids;
    s.ids_64 = a.ids_64;
    for (int k = 0; k < 2; ++k) s.rec[k] = records(k);
    s.tokens = static_cast<int>(a.tokens);
    s.passes = g.passes;
    s.per_lane = static_cast<int>((a.tokens + kCluster * kClusterThreads - 1) / (kCluster * kClusterThreads));
    s.vocab = a.vocab;
    // A table of up to 160 MB is zeroed by the SMs that the sort leaves idle, in about its time;
    // rows that are named are then written twice.  Of a larger one only rows not named are cleared.
    const size_t elem = dtype_size(a.out_dtype);
    g.clear = static_cast<size_t>(a.vocab) * a.dim * elem <= (size_t(160) << 20);
    s.named = g.clear ? nullptr : ws + g.off_named;
    s.table = static_cast<unsigned char*>(a.out);
    s.rows = a.vocab;
    s.row_bytes = static_cast<long long>(a.dim) * elem;
    s.stride_bytes = a.out_stride * elem;
    s.err = a.err;
    const unsigned extra = g.clear ? static_cast<unsigned>(2 * (sms - kCluster) / kCluster * kCluster) : 0;
    const size_t smem = sizeof(uint2) * kClusterThreads * s.per_lane;
    cudaError_t e = allow_smem(reinterpret_cast<const void*>(k_sort_cluster), smem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(k_sort_cluster, dim3(kCluster + extra), dim3(kClusterThreads), smem, st, s);
    if (e != cudaSuccess) return e;
    ++*launches;
    sorted = s.rec[(g.passes - 1) & 1];
  } else if (a.tokens > 0) {
    for (int k = 0; k < g.passes; ++k) {
      SortPass s{};
      s.ids = k == 0 ? a.ids : nullptr;
      s.ids_64 = a.ids_64;
      s.in = sorted;
      s.out = records(k & 1);
      s.counts = u32(g.off_counts);
      s.totals = u32(g.off_totals);
      s.tokens = a.tokens;
      s.vocab = a.vocab;
      s.tiles = g.tiles;
      s.shift = 8 * k;
      s.err = a.err;
      s.named = k == 0 ? ws + g.off_named : nullptr;
      const dim3 grid(g.tiles), block(kSortThreads);
      cudaError_t e = g.per_lane == 8 ? launch_pdl(k_sort_count<8>, grid, block, 0, st, s)
                                      : launch_pdl(k_sort_count<2>, grid, block, 0, st, s);
      if (e != cudaSuccess) return e;
      e = launch_pdl(k_sort_scan, dim3(kDigits), dim3(256), 0, st, s.counts, s.totals, g.tiles);
      if (e != cudaSuccess) return e;
      const size_t smem = sizeof(uint2) * kSortThreads * g.per_lane;
      e = allow_smem(g.per_lane == 8 ? reinterpret_cast<const void*>(k_sort_scatter<8>)
                                     : reinterpret_cast<const void*>(k_sort_scatter<2>),
                     smem);
      if (e != cudaSuccess) return e;
      e = g.per_lane == 8 ? launch_pdl(k_sort_scatter<8>, grid, block, smem, st, s)
                          : launch_pdl(k_sort_scatter<2>, grid, block, smem, st, s);
      if (e != cudaSuccess) return e;
      *launches += 3;
      sorted = s.out;
    }
  }
  GradArgs q{};
  q.rec = sorted;
  q.tokens = a.tokens;
  q.vocab = a.vocab;
  q.dim = a.dim;
  q.piece = g.piece;
  q.pieces = a.tokens > 0 ? g.pieces : 0;
  q.cleared = g.clear;
  q.named = a.tokens > 0 && !g.clear ? ws + g.off_named : nullptr;
  q.scale = a.scale;
  q.in_stride = a.in_stride;
  q.out_stride = a.out_stride;
  q.lead = reinterpret_cast<float*>(ws + g.off_lead);
  q.trail = reinterpret_cast<float*>(ws + g.off_trail);
  return with_width(pack_width(a), [&](auto width) {
    constexpr int V = decltype(width)::value;
    return with_dtype(a.in_dtype, [&](auto ti) {
      return with_dtype(a.out_dtype, [&](auto to) {
        using TI = decltype(ti);
        using TO = decltype(to);
        const int packs = a.dim / V;
        q.lanes = pow2_at_most_32(packs);
        const long long groups = kSumThreads / q.lanes;
        q.sum_blocks = (q.pieces + groups - 1) / groups;
        const unsigned chunks = static_cast<unsigned>((packs + q.lanes - 1) / q.lanes);
        const dim3 grid(static_cast<unsigned>(q.sum_blocks + (q.cleared ? 0 : (a.vocab + groups * kClearRows - 1) / (groups * kClearRows))), chunks);
        cudaError_t e = launch_pdl(k_grad_sum<TI, TO, V>, grid, dim3(kSumThreads), 0, st, q,
                                   static_cast<const TI*>(a.table), static_cast<TO*>(a.out));
        if (e != cudaSuccess) return e;
        ++*launches;
        if (q.pieces < 2) return cudaSuccess;
        ++*launches;
        return launch_pdl(k_grad_join<TO, V>, dim3(static_cast<unsigned>((q.pieces + kJoinWarps - 1) / kJoinWarps), (packs + 31) / 32),
                          dim3(kJoinWarps * 32), 0, st, q, static_cast<TO*>(a.out));
      });
    });
  });
}

}  // namespace mlt
