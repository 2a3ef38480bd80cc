// Token embedding: the lookup, and its gradient summed over tokens sorted by id.
//
// The lookup reads M rows and writes M rows.  The gradient reads M rows and
// writes all vocab rows, most of them zeros: with a large vocabulary the zeros
// are most of its bytes.  So one kernel sorts the ids, on 8 SMs, while another
// writes zeros; the third adds the tokens' rows up, run by run of equal ids, and
// writes the rows that occur; the fourth joins the runs that were cut.  (Spreading the zeros over the later kernels, past the rows that
// occur, was no faster: the sort is hidden behind them here, and was not then.)
// Every sum runs over the sorted tokens in fixed pieces and in fixed order: no
// atomics on results, the bits do not depend on timing.
// Measured: lookup of 16384 x 8192 BF16 71.6 us, 7.5 TB/s (frequent rows come out
// of L2); gradient of 16384 x 4096 tokens for 128000 rows, BF16: 200 us, 5.9 TB/s
// = 90 % of the copy rate (zeros 148 us, sums 37, join 8).
#include "ptx_sm100.cuh"
#include "row_ops.cuh"

namespace compass {

namespace {

struct VocabShards {
  void* ptr[kMaxP];
  FastDiv rows;       // per shard (the last ones hold fewer)
  uint32_t vocab;
  template <typename T>
  __device__ __forceinline__ T* row(uint32_t v, int64_t pitch) const {
    const uint32_t r = rows.div(v);
    return static_cast<T*>(ptr[r]) + int64_t(v - r * rows.d) * pitch;
  }
};

// An id as an index, or `vocab` when it is none.
__device__ __forceinline__ uint32_t token_id(const void* ids, bool wide, int64_t i, uint32_t vocab) {
  const int64_t v = wide ? static_cast<const int64_t*>(ids)[i] : int64_t(static_cast<const int32_t*>(ids)[i]);
  return v >= 0 && v < int64_t(vocab) ? uint32_t(v) : vocab;
}

// ---- lookup --------------------------------------------------------------------

struct LookupParams {
  VocabShards w;
  RowShards out;
  const void* ids;
  int64_t hidden;
  uint32_t M;
  uint32_t pieces;        // pieces of blockDim * U vectors per row
  int32_t wide_ids;
  float scale;
};

// A block copies one piece of one row, U vectors per thread in flight.
template <typename T, int V, int U>
__global__ void __launch_bounds__(128) embedding_kernel(const __grid_constant__ LookupParams p) {
  const uint32_t row = blockIdx.x / p.pieces;
  const uint32_t piece = blockIdx.x - row * p.pieces;
  const uint32_t id = token_id(p.ids, p.wide_ids, row, p.w.vocab);
  T* out = p.out.row<T>(row, p.hidden);
  const T* in = id < p.w.vocab ? p.w.row<T>(id, p.hidden) : nullptr;
  float v[U][V];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int64_t c = (int64_t(piece) * (128 * U) + i * 128 + threadIdx.x) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) v[i][j] = 0.f;
    if (in && c < p.hidden) load_vec(v[i], in + c);
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int64_t c = (int64_t(piece) * (128 * U) + i * 128 + threadIdx.x) * V;
    if (c < p.hidden) {
      if (in) {     // a padding row is +0 whatever the scale
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] *= p.scale;
      }
      store_vec(out + c, v[i]);
    }
  }
}

// ---- gradient: sort ------------------------------------------------------------
// Stable radix sort of (id, position), padding ids (= vocab) last, 9 bits a pass.  Up to kClusterTokens tokens it is the work
// of one cluster of 8 CTAs, which exchange digit counts and items through distributed shared memory; beyond, of a kernel for
// each step.  (One CTA took 30 us for 16384 tokens, nearly all of it for the ranks; the cluster takes 15.)

constexpr int kRadixBits = 9;
constexpr int kRadix = 1 << kRadixBits;
constexpr int kSortThreads = 512;                         // (their registers fit beside a block that writes zeros)
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 16;                            // items per thread at most
constexpr int kSortTile = kSortThreads * kSortItems;      // tokens of one block at most
constexpr int kCluster = 8;
constexpr int64_t kClusterTokens = int64_t(kCluster) * kSortTile;

struct GradParams {
  VocabShards dw;
  RowShards dout;
  const void* ids;
  uint32_t *key_a, *pos_a, *key_b, *pos_b;   // sorted (id, position); b: the other side of a pass
  uint32_t* hist;                            // [kRadix][tiles] (more than one tile)
  float* partial;                            // [pieces][2][hidden] sums of runs that cross a piece's ends
  int64_t hidden;
  uint32_t M;
  uint32_t tiles;
  uint32_t run;                              // sorted tokens per piece
  int32_t wide_ids;
  int32_t bits;                              // of a key
  int32_t accumulate;
  int64_t elem;                              // bytes of an element of dW
  float scale;
};

// Where each of a warp's items goes within the block: `rank` of every item among the warp's items with the same digit, items
// in order of position (warp-major, then item, then lane).  count[warp][digit] afterwards: items of that digit in earlier
// warps; total[digit]: in the block.
template <int kItems>
__device__ __forceinline__ void block_rank(const uint32_t (&digit)[kItems], uint32_t (&rank)[kItems], uint16_t* count, uint32_t* total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint16_t* mine = count + warp * kRadix;
  for (int d = lane; d < kRadix / 2; d += 32) reinterpret_cast<uint32_t*>(mine)[d] = 0;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const uint32_t same = __match_any_sync(0xffffffffu, digit[i]);
    const uint32_t before = __popc(same & ((1u << lane) - 1u));
    const uint32_t base = mine[digit[i]];
    __syncwarp();
    if (before == 0) mine[digit[i]] = uint16_t(base + __popc(same));
    __syncwarp();
    rank[i] = base + before;
  }
  __syncthreads();
  static_assert(kSortThreads == kRadix, "a thread per digit");
  {
    uint32_t sum = 0, c[kSortWarps];
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) c[w] = count[w * kRadix + threadIdx.x];
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      count[w * kRadix + threadIdx.x] = uint16_t(sum);
      sum += c[w];
    }
    total[threadIdx.x] = sum;
  }
  __syncthreads();
}

// Exclusive sum of a value per digit, one per thread.
__device__ __forceinline__ uint32_t scan_digits(uint32_t v, uint32_t* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < warp; ++w) before += warp_sums[w];
  return before + x - v;
}

struct SortShared {
  uint32_t key[kSortTile], pos[kSortTile];
  uint16_t count[kSortWarps * kRadix];
  uint32_t total[kRadix], base[kRadix];
  uint32_t warp_sums[kRadix / 32];
};

__device__ __forceinline__ uint32_t load_cluster(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void store_cluster(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// Sorts up to kCluster * kSortThreads * kItems tokens on one cluster.
template <int kItems>
__device__ void sort_cluster(const GradParams& p, SortShared& s) {
  using namespace ptx;
  constexpr uint32_t kTile = kSortThreads * kItems;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t cta = cluster_ctarank();
  const uint32_t own = warp * (32 * kItems) + lane;      // first of this thread's places in the tile, 32 apart
  uint32_t key[kItems], pos[kItems], digit[kItems], rank[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    pos[i] = cta * kTile + own + i * 32;
    // past the end: beyond every key, so that it stays behind the tokens in every pass
    key[i] = pos[i] < p.M ? token_id(p.ids, p.wide_ids, pos[i], p.dw.vocab) : 0xffffffffu;
  }
  const uint32_t key_at = smem_u32(s.key), pos_at = smem_u32(s.pos), total_at = smem_u32(s.total);
  for (int shift = 0; shift < p.bits; shift += kRadixBits) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) digit[i] = (key[i] >> shift) & (kRadix - 1);
    block_rank(digit, rank, s.count, s.total);
    cluster_arrive();      // every CTA's totals are there, and every CTA has read its items of the pass before
    cluster_wait();
    uint32_t all = 0, before = 0;
    {
      uint32_t t[kCluster];
#pragma unroll
      for (int c = 0; c < kCluster; ++c) t[c] = load_cluster(map_to_cta(total_at + threadIdx.x * 4, c));
#pragma unroll
      for (int c = 0; c < kCluster; ++c) {
        all += t[c];
        if (uint32_t(c) < cta) before += t[c];
      }
    }
    const uint32_t first = scan_digits(all, s.warp_sums);
    s.base[threadIdx.x] = first + before;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const uint32_t to = s.base[digit[i]] + s.count[warp * kRadix + digit[i]] + rank[i];
      store_cluster(map_to_cta(key_at + to % kTile * 4, to / kTile), key[i]);
      store_cluster(map_to_cta(pos_at + to % kTile * 4, to / kTile), pos[i]);
    }
    cluster_arrive();      // (and no CTA leaves while others still read its totals)
    cluster_wait();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      key[i] = s.key[own + i * 32];
      pos[i] = s.pos[own + i * 32];
    }
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const uint32_t at = cta * kTile + own + i * 32;
    if (at < p.M) {
      p.key_a[at] = key[i];
      p.pos_a[at] = pos[i];
    }
  }
}

template <int kItems>
__global__ void __launch_bounds__(kSortThreads, 1) embedding_sort_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ uint4 raw[];
  launch_dependents();
  sort_cluster<kItems>(p, *reinterpret_cast<SortShared*>(raw));
}

// Zeros for every row of dW.  It may run beside the sort, but is not done before it: what follows waits for this one.
// Many small blocks: 1.05 GB take 149 us with 64 of 256 threads per SM, 171 us with one of 1024.
constexpr int kZeroThreads = 256;
constexpr int kZeroAtOnce = 4;
__global__ void __launch_bounds__(kZeroThreads) embedding_zero_kernel(const __grid_constant__ GradParams p) {
  launch_dependents();
  const int64_t n = int64_t(gridDim.x) * (kZeroThreads * kZeroAtOnce), own = int64_t(blockIdx.x) * (kZeroThreads * kZeroAtOnce) + threadIdx.x;
  const uint32_t per = p.dw.rows.d;
  for (uint32_t r = 0, v0 = 0; v0 < p.dw.vocab; ++r, v0 += per) {
    int64_t bytes = int64_t(min(per, p.dw.vocab - v0)) * p.hidden * p.elem;
    uint8_t* base = static_cast<uint8_t*>(p.dw.ptr[r]);
    // up to the first 16-byte boundary
    const int64_t front = min(bytes, int64_t((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15));
    if (blockIdx.x == 0 && threadIdx.x * 2 < front) *reinterpret_cast<uint16_t*>(base + threadIdx.x * 2) = 0;
    base += front;
    bytes -= front;
    const int64_t whole = bytes / 16;
    for (int64_t i = own; i < whole; i += n) {
#pragma unroll
      for (int k = 0; k < kZeroAtOnce; ++k)
        if (i + k * kZeroThreads < whole) __stcs(reinterpret_cast<uint4*>(base) + i + k * kZeroThreads, make_uint4(0u, 0u, 0u, 0u));
    }
    if (blockIdx.x == 0)
      for (int64_t b = whole * 16 + threadIdx.x * 2; b < bytes; b += kZeroThreads * 2) *reinterpret_cast<uint16_t*>(base + b) = 0;
  }
  if (blockIdx.x == gridDim.x - 1) wait_for_previous_kernel();
}

// More tokens than a cluster sorts: per pass a histogram of every tile, their scan, and the scatter.
template <bool kFirst>
__device__ __forceinline__ void load_tile(const GradParams& p, uint32_t (&key)[kSortItems], uint32_t (&pos)[kSortItems]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const int64_t at = int64_t(blockIdx.x) * kSortTile + warp * (32 * kSortItems) + i * 32 + lane;
    key[i] = 0xffffffffu;
    pos[i] = uint32_t(at);
    if (at < int64_t(p.M)) {
      key[i] = kFirst ? token_id(p.ids, p.wide_ids, at, p.dw.vocab) : p.key_a[at];
      if (!kFirst) pos[i] = p.pos_a[at];
    }
  }
}
template <bool kFirst, bool kScatter>
__global__ void __launch_bounds__(kSortThreads, 1) embedding_pass_kernel(const __grid_constant__ GradParams p, int shift) {
  __shared__ uint16_t count[kSortWarps * kRadix];
  __shared__ uint32_t total[kRadix];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t key[kSortItems], pos[kSortItems], digit[kSortItems], rank[kSortItems];
  load_tile<kFirst>(p, key, pos);
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) digit[i] = (key[i] >> shift) & (kRadix - 1);
  block_rank(digit, rank, count, total);
  if constexpr (!kScatter) {
    p.hist[uint64_t(threadIdx.x) * p.tiles + blockIdx.x] = total[threadIdx.x];
  } else {
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      const int64_t at = int64_t(blockIdx.x) * kSortTile + warp * (32 * kSortItems) + i * 32 + lane;
      if (at < int64_t(p.M)) {     // what lies past the end has the last digit and the last places: nothing moves up
        const uint32_t to = p.hist[uint64_t(digit[i]) * p.tiles + blockIdx.x] + count[warp * kRadix + digit[i]] + rank[i];
        p.key_b[to] = key[i];
        p.pos_b[to] = pos[i];
      }
    }
  }
}
// Exclusive sum over hist, digit-major: one block, a run of the table per thread.
__global__ void __launch_bounds__(1024, 1) embedding_scan_kernel(const __grid_constant__ GradParams p) {
  __shared__ uint32_t warp_sums[32];
  const uint64_t n = uint64_t(kRadix) * p.tiles, per = (n + 1023) / 1024;
  const uint64_t from = per * threadIdx.x, to = from + per < n ? from + per : n;
  uint32_t sum = 0;
  for (uint64_t i = from; i < to; ++i) sum += p.hist[i];
  uint32_t x = sum;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  uint32_t before = x - sum;
  for (int w = 0; w < warp; ++w) before += warp_sums[w];
  for (uint64_t i = from; i < to; ++i) {
    const uint32_t c = p.hist[i];
    p.hist[i] = before;
    before += c;
  }
}

// ---- gradient: sums ------------------------------------------------------------

constexpr int kGradThreads = 128;
constexpr int kAhead = 8;                  // tokens whose rows are in flight

// V FP32 sums, in accesses of 16 bytes where V allows.
template <int V>
__device__ __forceinline__ void store_sums(float* p, const float (&v)[V]) {
  if constexpr (V == 1) {
    *p = v[0];
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
  }
}
template <int V>
__device__ __forceinline__ void load_sums(float (&v)[V], const float* p) {
  if constexpr (V == 1) {
    v[0] = __ldcg(p);
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const float4 q = __ldcg(reinterpret_cast<const float4*>(p + j));
      v[j] = q.x, v[j + 1] = q.y, v[j + 2] = q.z, v[j + 3] = q.w;
    }
  }
}

template <typename G, int V>
__device__ __forceinline__ void finish_row(const GradParams& p, uint32_t id, int64_t c, const float (&acc)[V]) {
  G* row = p.dw.row<G>(id, p.hidden) + c;
  if constexpr (V == 8 && sizeof(G) == 4) {
    float a[4], b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = acc[j] * p.scale + (p.accumulate ? row[j] : 0.f);
      b[j] = acc[4 + j] * p.scale + (p.accumulate ? row[4 + j] : 0.f);
    }
    store_vec(row, a);
    store_vec(row + 4, b);
  } else if constexpr (V == 4 && sizeof(G) == 2) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float v[1] = {acc[j] * p.scale + (p.accumulate ? __bfloat162float(row[j]) : 0.f)};
      store_vec(row + j, v);
    }
  } else {
    float old[V], v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) old[j] = 0.f;
    if (p.accumulate) load_vec(old, row);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = fmaf(acc[j], p.scale, old[j]);
    store_vec(row, v);
  }
}

// A block takes `run` sorted tokens and kGradThreads vectors of columns.  A run of equal ids that lies inside the piece is
// written; the part of one that began earlier goes to partial[piece][0], of one that begins here and goes on to
// partial[piece][1].
template <typename T, typename G, int V>
__global__ void __launch_bounds__(kGradThreads) embedding_grad_kernel(const __grid_constant__ GradParams p, uint32_t slabs) {
  wait_for_previous_kernel();
  const uint32_t slab = blockIdx.x % slabs;
  extern __shared__ uint4 raw[];
  // where each token's row is (null: padding), and what to do behind it: kNone, or a run's end
  enum : int { kNone = 0, kWrite = 1, kInherited = 2, kGoesOn = 3 };
  const T** rows = reinterpret_cast<const T**>(raw);
  int* what = reinterpret_cast<int*>(rows + p.run);
  uint32_t* ids = reinterpret_cast<uint32_t*>(what + p.run);
  const int64_t piece = blockIdx.x / slabs;
  const int64_t first = piece * p.run;
  const int n = int(min(int64_t(p.run), int64_t(p.M) - first));
  for (int i = threadIdx.x; i < int(p.run); i += kGradThreads) {
    rows[i] = nullptr;
    what[i] = kNone;
    if (i >= n) continue;
    const uint32_t id = p.key_a[first + i];
    ids[i] = id;
    if (id >= p.dw.vocab) continue;
    rows[i] = p.dout.row<T>(p.pos_a[first + i], p.hidden);
    const bool goes_on = first + i + 1 < int64_t(p.M) && p.key_a[first + i + 1] == id;
    if (!goes_on || i + 1 == n) {
      const bool inherited = first > 0 && p.key_a[first] == id && p.key_a[first - 1] == id;
      what[i] = inherited ? kInherited : goes_on ? kGoesOn : kWrite;
    }
  }
  __syncthreads();
  const int64_t c = (int64_t(slab) * kGradThreads + threadIdx.x) * V;
  if (c >= p.hidden) return;
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  Raw<T, V> ahead[kAhead];
  auto fetch = [&](int i, Raw<T, V>& to) {
    const T* r = rows[i];
    if (r) to.load(r + c);
    else to.zero();
  };
#pragma unroll
  for (int k = 0; k < kAhead; ++k) fetch(k, ahead[k]);          // (p.run is a multiple of kAhead)
  for (int i0 = 0; i0 < n; i0 += kAhead) {
    const bool more = i0 + kAhead < n;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float x[V];
      ahead[k].get(x);
      if (more) fetch(i0 + kAhead + k, ahead[k]);
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += x[j];
      const int end = what[i0 + k];
      if (end != kNone) {
        if (end == kWrite) {
          finish_row<G, V>(p, ids[i0 + k], c, acc);
        } else {
          store_sums(p.partial + (piece * 2 + (end == kInherited ? 0 : 1)) * p.hidden + c, acc);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
      }
    }
  }
}

// The runs that cross pieces: where one begins, what its pieces left is added up in order; of a long run, every kJoinWays-th
// piece by one group of threads, and the groups' sums in turn.
constexpr int kJoinWays = 4;
constexpr int kJoinLanes = 32;
constexpr int kJoinShort = 128;     // up to this many pieces: a thread adds up a column's by itself
template <typename G, int V>
__global__ void __launch_bounds__(kJoinWays * kJoinLanes) embedding_join_kernel(const __grid_constant__ GradParams p, uint32_t pieces, uint32_t slabs) {
  __shared__ float part[kJoinWays][kJoinLanes][V + 1];
  wait_for_previous_kernel();
  const int64_t piece = blockIdx.x / slabs;
  const uint32_t slab = blockIdx.x % slabs;
  const int64_t first = piece * p.run, last = min(first + p.run, int64_t(p.M)) - 1;
  if (last + 1 >= int64_t(p.M)) return;
  // (four independent loads before the first branch)
  const uint32_t id = p.key_a[last], next = p.key_a[last + 1], front = p.key_a[first], before = first > 0 ? p.key_a[first - 1] : 0xffffffffu;
  if (id >= p.dw.vocab || next != id) return;        // nothing goes on
  if (front == id && before == id) return;           // it began earlier
  // the last piece that it reaches into starts with it; every warp looks at 32 pieces at a time
  int64_t lo = piece;
  for (;;) {
    const int64_t q = lo + 1 + (threadIdx.x & 31);
    const uint32_t same = __ballot_sync(0xffffffffu, q < int64_t(pieces) && p.key_a[q < int64_t(pieces) ? q * p.run : first] == id);
    const int n = __ffs(~same) - 1;                  // (-1: all 32)
    lo += n < 0 ? 32 : n;
    if (n >= 0) break;
  }
  if (lo - piece < kJoinShort) {
    for (int64_t c = (int64_t(slab) * blockDim.x + threadIdx.x) * V; c < p.hidden; c += int64_t(slabs) * blockDim.x * V) {
      float acc[V];
      load_sums(acc, p.partial + (piece * 2 + 1) * p.hidden + c);
      for (int64_t q0 = piece + 1; q0 <= lo; q0 += 8) {
        float x[8][V];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (q0 + k <= lo) {
            load_sums(x[k], p.partial + (q0 + k) * 2 * p.hidden + c);
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j) x[k][j] = 0.f;
          }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] += x[k][j];
      }
      finish_row<G, V>(p, id, c, acc);
    }
    return;
  }
  const int lane = threadIdx.x % kJoinLanes, way = threadIdx.x / kJoinLanes;
  for (int64_t c0 = int64_t(slab) * kJoinLanes * V; c0 < p.hidden; c0 += int64_t(slabs) * kJoinLanes * V) {
    const int64_t c = c0 + lane * V;
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    if (c < p.hidden) {
      // (the piece where it begins left its part in slot 1, the others in slot 0)
#pragma unroll 4
      for (int64_t q = piece + way; q <= lo; q += kJoinWays) {
        float x[V];
        load_sums(x, p.partial + (q * 2 + (q == piece ? 1 : 0)) * p.hidden + c);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += x[j];
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) part[way][lane][j] = acc[j];
    __syncthreads();
    if (way == 0 && c < p.hidden) {
#pragma unroll
      for (int w = 1; w < kJoinWays; ++w)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += part[w][lane][j];
      finish_row<G, V>(p, id, c, acc);
    }
    __syncthreads();
  }
}

// ---- host ----------------------------------------------------------------------

int check_embed(const compass_embed* e) {
  if (e == nullptr) return COMPASS_ERR_INVALID_ARG;
  int st = check_rows(e->P, e->M, e->hidden);
  if (st != COMPASS_OK) return st;
  if (e->vocab <= 0) return COMPASS_ERR_SHAPE;
  if (e->vocab > kMaxDim) return COMPASS_ERR_UNSUPPORTED;
  if (e->index_dtype != COMPASS_INDEX_INT64 && e->index_dtype != COMPASS_INDEX_INT32) return COMPASS_ERR_INVALID_ARG;
  st = check_dtype(e->dtype, true);
  return st == COMPASS_OK ? check_dtype(e->grad_dtype, true) : st;
}

int check_ids(const void* ids, int64_t M, int index_dtype) {
  if (M > 0 && ids == nullptr) return COMPASS_ERR_INVALID_ARG;
  return is_aligned(ids, index_dtype == COMPASS_INDEX_INT64 ? 8 : 4) ? COMPASS_OK : COMPASS_ERR_ALIGNMENT;
}

VocabShards vocab_shards(const void* const* w, int P, int64_t vocab) {
  VocabShards s = {};
  s.rows.set(uint32_t(vocab_shard_rows(vocab, P)));
  s.vocab = uint32_t(vocab);
  for (int r = 0; r < P; ++r) s.ptr[r] = const_cast<void*>(w[r]);
  return s;
}

template <typename T, int V, int U>
int run_lookup(LookupParams p, cudaStream_t stream) {
  p.pieces = uint32_t(ceil_div(p.hidden, 128 * U * V));
  const int64_t grid = int64_t(p.pieces) * p.M;
  if (grid > 0x7fffffff) return COMPASS_ERR_UNSUPPORTED;
  return launch(embedding_kernel<T, V, U>, grid, 128, 0, stream, false, p);
}
// Four vectors per thread where that still gives every SM several blocks; else one, for more blocks.  Measured (four, one):
// 16384 tokens of 8192: 68.4, 91.4 us; 4096 of 4096: 11.3, 13.4; 512 of 4096: 2.7, 2.9; 8 of 4096: 1.95, 1.75.
template <typename T, int V>
int pick_lookup(const LookupParams& p, int sms, cudaStream_t stream) {
  const int64_t blocks = int64_t(p.M) * ceil_div(p.hidden, 128 * 4 * V);
  return blocks >= 8 * sms ? run_lookup<T, V, 4>(p, stream) : run_lookup<T, V, 1>(p, stream);
}

// Sorted tokens per piece: 8 (whose loads a thread has in flight together), more where that would be over 512 pieces: fewer
// of them leave runs to join (16384 tokens of 4096: sums and join 38 + 30 us at 8 a piece, 37 + 15 at 16, 36 + 8 at 32).
// At most 2048, whose positions a block keeps in shared memory.
uint32_t run_length(int64_t M) { return uint32_t(M <= 4096 ? 8 : M > 512 * 2048 ? 2048 : round_up(size_t(ceil_div(M, 512)), 8)); }

struct GradPlan {
  uint32_t tiles, run, pieces;      // (tiles: 1 where a cluster sorts)
  size_t key, hist, partial, bytes;
};
GradPlan grad_plan(const compass_embed* e) {
  GradPlan g;
  g.tiles = e->M <= kClusterTokens ? 1 : uint32_t(ceil_div(e->M, kSortTile));
  g.run = run_length(e->M);
  g.pieces = uint32_t(ceil_div(e->M, g.run));
  g.key = round_up(size_t(e->M) * 4, 256);
  g.hist = g.tiles > 1 ? round_up(size_t(kRadix) * g.tiles * 4, 256) : 0;
  g.partial = round_up(size_t(g.pieces) * 2 * size_t(e->hidden) * 4, 256);
  g.bytes = 256 + (g.tiles > 1 ? 4 : 2) * g.key + g.hist + g.partial;
  return g;
}

template <int kItems>
int run_sort(const GradParams& p, cudaStream_t stream) {
  static_assert(sizeof(SortShared) <= 227 * 1024, "");
  static std::atomic<uint64_t> allowed{0};
  auto kernel = embedding_sort_kernel<kItems>;
  const int st = allow_smem(reinterpret_cast<const void*>(kernel), sizeof(SortShared), &allowed);
  if (st != COMPASS_OK) return st;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(kCluster));
  cfg.blockDim = dim3(kSortThreads);
  cfg.dynamicSmemBytes = sizeof(SortShared);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kCluster;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  count_kernel_launch();
  return e == cudaSuccess ? COMPASS_OK : record_cuda_error(e);
}

template <typename T, typename G, int V>
int run_grad(const GradParams& p, const GradPlan& g, cudaStream_t stream) {
  const int64_t slabs = ceil_div(p.hidden, kGradThreads * V);
  if (g.pieces * slabs > 0x7fffffff) return COMPASS_ERR_UNSUPPORTED;
  int st = launch(embedding_grad_kernel<T, G, V>, g.pieces * slabs, kGradThreads, size_t(g.run) * 16, stream, true, p,
                  uint32_t(slabs));
  if (st != COMPASS_OK || g.pieces == 1) return st;
  const int64_t all = ceil_div(p.hidden, kJoinLanes * V), join_slabs = all < 4 ? all : 4;
  return launch(embedding_join_kernel<G, V>, g.pieces * join_slabs, kJoinWays * kJoinLanes, 0, stream, true, p, g.pieces,
                uint32_t(join_slabs));
}
template <typename T, int V>
int pick_grad(const GradParams& p, const GradPlan& g, bool fp32_grad, cudaStream_t stream) {
  return fp32_grad ? run_grad<T, float, V>(p, g, stream) : run_grad<T, __nv_bfloat16, V>(p, g, stream);
}

}  // namespace

}  // namespace compass

using namespace compass;

extern "C" int compass_embedding(const compass_embed* e, const void* ids, const void* const* W, void* const* Out, void* stream) {
  int st = check_embed(e);
  if (st != COMPASS_OK) return st;
  LookupParams p = {};
  st = check_ids(ids, e->M, e->index_dtype);
  const size_t element = dtype_size(e->dtype);
  bool whole = e->hidden * int64_t(element) % 16 == 0;
  if (st == COMPASS_OK) st = check_vocab_shards(W, e->P, e->vocab, element, &whole);
  if (st == COMPASS_OK) st = fill_shards(Out, e->P, e->M, &p.out, element, &whole);
  if (st != COMPASS_OK || e->M == 0) return st;
  int sms = 0;
  st = sm_count(&sms);
  if (st != COMPASS_OK) return st;
  p.w = vocab_shards(W, e->P, e->vocab);
  p.ids = ids;
  p.hidden = e->hidden;
  p.M = uint32_t(e->M);
  p.wide_ids = e->index_dtype == COMPASS_INDEX_INT64;
  p.scale = e->scale;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (e->dtype == COMPASS_DTYPE_FP32)
    return whole ? pick_lookup<float, 4>(p, sms, s) : pick_lookup<float, 1>(p, sms, s);
  return whole ? pick_lookup<__nv_bfloat16, 8>(p, sms, s) : pick_lookup<__nv_bfloat16, 1>(p, sms, s);
}

extern "C" int compass_embedding_workspace_bytes(const compass_embed* e, size_t* bytes) {
  if (bytes == nullptr) return COMPASS_ERR_INVALID_ARG;
  const int st = check_embed(e);
  if (st != COMPASS_OK) return st;
  *bytes = grad_plan(e).bytes;
  return COMPASS_OK;
}

extern "C" int compass_embedding_backward(const compass_embed* e, const void* ids, const void* const* dOut, void* const* dW,
                                          void* ws, size_t ws_bytes, void* stream) {
  int st = check_embed(e);
  if (st != COMPASS_OK) return st;
  GradParams p = {};
  st = check_ids(ids, e->M, e->index_dtype);
  bool whole = e->hidden % (e->dtype == COMPASS_DTYPE_FP32 ? 4 : 8) == 0;
  if (st == COMPASS_OK) st = fill_shards(dOut, e->P, e->M, &p.dout, dtype_size(e->dtype), &whole);
  if (st == COMPASS_OK) st = check_vocab_shards(dW, e->P, e->vocab, dtype_size(e->grad_dtype), &whole);
  if (st != COMPASS_OK) return st;
  const GradPlan g = grad_plan(e);
  st = check_workspace(ws, ws_bytes, g.bytes);
  if (st != COMPASS_OK) return st;
  int sms = 0;
  st = sm_count(&sms);
  if (st != COMPASS_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint8_t* at = static_cast<uint8_t*>(ws) + 256;
  auto take = [&](size_t n) {
    uint8_t* was = at;
    at += n;
    return was;
  };
  p.dw = vocab_shards(dW, e->P, e->vocab);
  p.ids = ids;
  p.partial = reinterpret_cast<float*>(take(g.partial));
  p.key_a = reinterpret_cast<uint32_t*>(take(g.key));
  p.pos_a = reinterpret_cast<uint32_t*>(take(g.key));
  p.hidden = e->hidden;
  p.M = uint32_t(e->M);
  p.tiles = g.tiles;
  p.run = g.run;
  p.wide_ids = e->index_dtype == COMPASS_INDEX_INT64;
  p.accumulate = e->accumulate != 0;
  p.elem = int64_t(dtype_size(e->grad_dtype));
  p.scale = e->scale;
  while ((int64_t(1) << p.bits) <= e->vocab) ++p.bits;      // keys 0 .. vocab
  const int64_t vecs = e->vocab * e->hidden * p.elem / 16, zero_blocks = ceil_div(vecs + 1, kZeroThreads * kZeroAtOnce);
  auto write_zeros = [&](bool beside_sort) {
    return launch(embedding_zero_kernel, zero_blocks < 64 * sms ? zero_blocks : 64 * sms, kZeroThreads, 0, s, beside_sort, p);
  };
  if (!p.accumulate && (e->M == 0 || g.tiles > 1)) st = write_zeros(false);
  if (st != COMPASS_OK || e->M == 0) return st;
  if (g.tiles == 1) {
    st = e->M <= kCluster * kSortThreads ? run_sort<1>(p, s) : e->M <= 4 * kCluster * kSortThreads ? run_sort<4>(p, s) : run_sort<kSortItems>(p, s);
    if (st == COMPASS_OK && !p.accumulate) st = write_zeros(true);
  } else {
    p.key_b = reinterpret_cast<uint32_t*>(take(g.key));
    p.pos_b = reinterpret_cast<uint32_t*>(take(g.key));
    p.hist = reinterpret_cast<uint32_t*>(take(g.hist));
    for (int shift = 0; st == COMPASS_OK && shift < p.bits; shift += kRadixBits) {
      st = shift ? launch(embedding_pass_kernel<false, false>, g.tiles, kSortThreads, 0, s, false, p, shift)
                 : launch(embedding_pass_kernel<true, false>, g.tiles, kSortThreads, 0, s, false, p, shift);
      if (st == COMPASS_OK) st = launch(embedding_scan_kernel, 1, 1024, 0, s, false, p);
      if (st == COMPASS_OK)
        st = shift ? launch(embedding_pass_kernel<false, true>, g.tiles, kSortThreads, 0, s, false, p, shift)
                   : launch(embedding_pass_kernel<true, true>, g.tiles, kSortThreads, 0, s, false, p, shift);
      uint32_t* k = p.key_a;
      p.key_a = p.key_b;
      p.key_b = k;
      k = p.pos_a;
      p.pos_a = p.pos_b;
      p.pos_b = k;
    }
  }
  if (st != COMPASS_OK) return st;
  const bool fp32_grad = e->grad_dtype == COMPASS_DTYPE_FP32;
  if (e->dtype == COMPASS_DTYPE_FP32)
    return whole ? pick_grad<float, 4>(p, g, fp32_grad, s) : pick_grad<float, 1>(p, g, fp32_grad, s);
  return whole ? pick_grad<__nv_bfloat16, 8>(p, g, fp32_grad, s) : pick_grad<__nv_bfloat16, 1>(p, g, fp32_grad, s);
}
