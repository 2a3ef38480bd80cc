// Token embedding: the lookup, and its gradient summed over tokens sorted by id.
//
// The lookup reads M rows and writes M rows.  The gradient reads M rows and
// writes all vocab rows, most of them zeros: with a large vocabulary the zeros
// are most of its bytes.  So one kernel sorts the ids on one SM while the other
// SMs write the zeros, and a second one adds the tokens' rows up, run by run of
// equal ids, and writes only the rows that occur.  Every sum runs over the sorted
// tokens in fixed pieces and in fixed order: no atomics on results, the bits do
// not depend on timing.
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
// Stable radix sort of (id, position), padding ids (= vocab) last, 9 bits a pass.

constexpr int kRadixBits = 9;
constexpr int kRadix = 1 << kRadixBits;
constexpr int kSortThreads = 1024;
constexpr int kSortItems = 16;
constexpr int kSortTile = kSortThreads * kSortItems;      // tokens one block sorts in its registers and shared memory
constexpr int kSortWarps = kSortThreads / 32;

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
  int32_t fill;                              // zeros are written beside the sort
  int64_t elem;                              // bytes of an element of dW
  float scale;
};

// Where each of a warp's items goes within the block: `rank` of every item among the block's items with the same digit,
// items in order of position (warp-major, then item, then lane).  count[warp][digit] afterwards: items of that digit in
// earlier warps; total[digit]: in the block.
__device__ __forceinline__ void block_rank(const uint32_t (&digit)[kSortItems], uint32_t (&rank)[kSortItems], uint16_t* count,
                                           uint32_t* total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint16_t* mine = count + warp * kRadix;
  for (int d = lane; d < kRadix; d += 32) mine[d] = 0;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t same = __match_any_sync(0xffffffffu, digit[i]);
    const uint32_t before = __popc(same & ((1u << lane) - 1u));
    const uint32_t base = mine[digit[i]];
    __syncwarp();
    if (before == 0) mine[digit[i]] = uint16_t(base + __popc(same));
    __syncwarp();
    rank[i] = base + before;
  }
  __syncthreads();
  if (threadIdx.x < kRadix) {
    uint32_t sum = 0;
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = count[w * kRadix + threadIdx.x];
      count[w * kRadix + threadIdx.x] = uint16_t(sum);
      sum += c;
    }
    total[threadIdx.x] = sum;
  }
  __syncthreads();
}

// Exclusive sum over the kRadix totals of a block.
__device__ __forceinline__ void scan_digits(uint32_t* total, uint32_t* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t v = 0, x = 0;
  if (threadIdx.x < kRadix) {
    v = x = total[threadIdx.x];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) warp_sums[warp] = x;
  }
  __syncthreads();
  if (threadIdx.x < kRadix) {
    uint32_t before = 0;
    for (int w = 0; w < warp; ++w) before += warp_sums[w];
    total[threadIdx.x] = before + x - v;
  }
  __syncthreads();
}

struct SortShared {
  uint32_t key[kSortTile], pos[kSortTile];
  uint16_t count[kSortWarps * kRadix];
  uint32_t total[kRadix];
  uint32_t warp_sums[kRadix / 32];
};

// Sorts up to kSortTile tokens on one block.
__device__ void sort_tile(const GradParams& p, SortShared& s) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t key[kSortItems], pos[kSortItems], digit[kSortItems], rank[kSortItems];
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t at = warp * (32 * kSortItems) + i * 32 + lane;
    pos[i] = at;
    // past the end: beyond every key, so that it stays behind the tokens in every pass
    key[i] = at < p.M ? token_id(p.ids, p.wide_ids, at, p.dw.vocab) : 0xffffffffu;
  }
  for (int shift = 0; shift < p.bits; shift += kRadixBits) {
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) digit[i] = (key[i] >> shift) & (kRadix - 1);
    block_rank(digit, rank, s.count, s.total);
    scan_digits(s.total, s.warp_sums);
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      const uint32_t to = s.total[digit[i]] + s.count[warp * kRadix + digit[i]] + rank[i];
      s.key[to] = key[i];
      s.pos[to] = pos[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      const uint32_t at = warp * (32 * kSortItems) + i * 32 + lane;
      key[i] = s.key[at];
      pos[i] = s.pos[at];
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t at = warp * (32 * kSortItems) + i * 32 + lane;
    if (at < p.M) {
      p.key_a[at] = key[i];
      p.pos_a[at] = pos[i];
    }
  }
}

// Zeros for every row of dW, by blocks first .. first + n - 1 of the grid.
__device__ __forceinline__ void write_zeros(const GradParams& p, int64_t first, int64_t n) {
  const uint32_t per = p.dw.rows.d;
  for (uint32_t r = 0, v0 = 0; v0 < p.dw.vocab; ++r, v0 += per) {
    const int64_t rows = min(per, p.dw.vocab - v0);
    const int64_t bytes = rows * p.hidden * p.elem;
    uint8_t* base = static_cast<uint8_t*>(p.dw.ptr[r]);
    const int64_t whole = bytes / 16;
    for (int64_t i = (int64_t(blockIdx.x) - first) * blockDim.x + threadIdx.x; i < whole; i += n * blockDim.x)
      __stcs(reinterpret_cast<uint4*>(base) + i, make_uint4(0u, 0u, 0u, 0u));
    if (int64_t(blockIdx.x) == first)
      for (int64_t b = whole * 16 + threadIdx.x * 2; b < bytes; b += blockDim.x * 2) *reinterpret_cast<uint16_t*>(base + b) = 0;
  }
}

// Block 0 sorts; the others write the zeros meanwhile.
__global__ void __launch_bounds__(kSortThreads, 1) embedding_sort_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ uint4 raw[];
  launch_dependents();
  if (blockIdx.x == 0) sort_tile(p, *reinterpret_cast<SortShared*>(raw));
  else write_zeros(p, 1, int64_t(gridDim.x) - 1);
}

// More tokens than one block sorts: per pass a histogram of every tile, their scan, and the scatter.
__global__ void __launch_bounds__(kSortThreads, 1) embedding_zero_kernel(const __grid_constant__ GradParams p) {
  write_zeros(p, 0, gridDim.x);
}
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
    if (threadIdx.x < kRadix) p.hist[uint64_t(threadIdx.x) * p.tiles + blockIdx.x] = total[threadIdx.x];
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
__global__ void __launch_bounds__(kGradThreads) embedding_grad_kernel(const __grid_constant__ GradParams p) {
  wait_for_previous_kernel();
  extern __shared__ uint4 raw[];
  // where each token's row is (null: padding), and what to do behind it: kNone, or a run's end
  enum : int { kNone = 0, kWrite = 1, kInherited = 2, kGoesOn = 3 };
  const T** rows = reinterpret_cast<const T**>(raw);
  int* what = reinterpret_cast<int*>(rows + p.run);
  uint32_t* ids = reinterpret_cast<uint32_t*>(what + p.run);
  const int64_t piece = blockIdx.x;
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
  const int64_t c = (int64_t(blockIdx.y) * kGradThreads + threadIdx.x) * V;
  if (c >= p.hidden) return;
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  for (int i0 = 0; i0 < n; i0 += kAhead) {
    Raw<T, V> ahead[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const T* r = rows[i0 + k];          // (p.run is a multiple of kAhead)
      if (r) ahead[k].load(r + c);
      else ahead[k].zero();
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float x[V];
      ahead[k].get(x);
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
constexpr int kJoinShort = 16;      // up to this many pieces: a thread adds up a column's by itself
template <typename G, int V>
__global__ void __launch_bounds__(kJoinWays * kJoinLanes) embedding_join_kernel(const __grid_constant__ GradParams p, uint32_t pieces) {
  __shared__ float part[kJoinWays][kJoinLanes][V + 1];
  wait_for_previous_kernel();
  const int64_t piece = blockIdx.x;
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
    for (int64_t c = (int64_t(blockIdx.y) * blockDim.x + threadIdx.x) * V; c < p.hidden; c += int64_t(gridDim.y) * blockDim.x * V) {
      float acc[V];
      load_sums(acc, p.partial + (piece * 2 + 1) * p.hidden + c);
#pragma unroll 4
      for (int64_t q = piece + 1; q <= lo; ++q) {
        float x[V];
        load_sums(x, p.partial + q * 2 * p.hidden + c);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += x[j];
      }
      finish_row<G, V>(p, id, c, acc);
    }
    return;
  }
  const int lane = threadIdx.x % kJoinLanes, way = threadIdx.x / kJoinLanes;
  for (int64_t c0 = int64_t(blockIdx.y) * kJoinLanes * V; c0 < p.hidden; c0 += int64_t(gridDim.y) * kJoinLanes * V) {
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
// Four vectors per thread where that still gives every SM several blocks; else one, for more blocks in flight.
template <typename T, int V>
int pick_lookup(const LookupParams& p, int sms, cudaStream_t stream) {
  const int64_t blocks = int64_t(p.M) * ceil_div(p.hidden, 128 * 4 * V);
  return blocks >= 8 * sms ? run_lookup<T, V, 4>(p, stream) : run_lookup<T, V, 1>(p, stream);
}

// Sorted tokens per piece: 8 (whose loads a thread has in flight together), more where that would be over 1024 pieces.
uint32_t run_length(int64_t M) { return uint32_t(M <= 8192 ? 8 : round_up(size_t(ceil_div(M, 1024)), 8)); }

struct GradPlan {
  uint32_t tiles, run, pieces;
  size_t key, hist, partial, bytes;
};
GradPlan grad_plan(const compass_embed* e) {
  GradPlan g;
  g.tiles = uint32_t(ceil_div(e->M, kSortTile));
  g.run = run_length(e->M);
  g.pieces = uint32_t(ceil_div(e->M, g.run));
  g.key = round_up(size_t(e->M) * 4, 256);
  g.hist = g.tiles > 1 ? round_up(size_t(kRadix) * g.tiles * 4, 256) : 0;
  g.partial = round_up(size_t(g.pieces) * 2 * size_t(e->hidden) * 4, 256);
  g.bytes = 256 + (g.tiles > 1 ? 4 : 2) * g.key + g.hist + g.partial;
  return g;
}

template <typename T, typename G, int V>
int run_grad(const GradParams& p, const GradPlan& g, cudaStream_t stream) {
  const unsigned slabs = unsigned(ceil_div(p.hidden, kGradThreads * V));
  if (slabs > 65535) return COMPASS_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(g.pieces, slabs);
  cfg.blockDim = dim3(kGradThreads);
  cfg.dynamicSmemBytes = size_t(g.run) * 16;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, embedding_grad_kernel<T, G, V>, p);
  count_kernel_launch();
  if (e != cudaSuccess) return record_cuda_error(e);
  if (g.pieces == 1) return COMPASS_OK;
  cfg.dynamicSmemBytes = 0;
  cfg.gridDim = dim3(g.pieces, unsigned(ceil_div(p.hidden, kJoinLanes * V) < 4 ? ceil_div(p.hidden, kJoinLanes * V) : 4));
  cfg.blockDim = dim3(kJoinWays * kJoinLanes);
  e = cudaLaunchKernelEx(&cfg, embedding_join_kernel<G, V>, p, g.pieces);
  count_kernel_launch();
  return e == cudaSuccess ? COMPASS_OK : record_cuda_error(e);
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
  if (st == COMPASS_OK) st = check_vocab_shards(W, e->P, e->vocab);
  if (st == COMPASS_OK) st = fill_shards(Out, e->P, e->M, &p.out);
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
    return e->hidden % 4 == 0 ? pick_lookup<float, 4>(p, sms, s) : pick_lookup<float, 1>(p, sms, s);
  return e->hidden % 8 == 0 ? pick_lookup<__nv_bfloat16, 8>(p, sms, s) : pick_lookup<__nv_bfloat16, 1>(p, sms, s);
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
  if (st == COMPASS_OK) st = fill_shards(dOut, e->P, e->M, &p.dout);
  if (st == COMPASS_OK) st = check_vocab_shards(dW, e->P, e->vocab);
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
  p.fill = !p.accumulate;
  p.elem = int64_t(dtype_size(e->grad_dtype));
  p.scale = e->scale;
  while ((int64_t(1) << p.bits) <= e->vocab) ++p.bits;      // keys 0 .. vocab
  if (e->M == 0) return p.fill ? launch(embedding_zero_kernel, 2 * sms, kSortThreads, 0, s, false, p) : COMPASS_OK;
  if (g.tiles == 1) {
    static_assert(sizeof(SortShared) <= 227 * 1024, "");
    static std::atomic<uint64_t> allowed{0};
    st = allow_smem(reinterpret_cast<const void*>(embedding_sort_kernel), sizeof(SortShared), &allowed);
    if (st != COMPASS_OK) return st;
    st = launch(embedding_sort_kernel, p.fill ? sms : 1, kSortThreads, sizeof(SortShared), s, false, p);
  } else {
    p.key_b = reinterpret_cast<uint32_t*>(take(g.key));
    p.pos_b = reinterpret_cast<uint32_t*>(take(g.key));
    p.hist = reinterpret_cast<uint32_t*>(take(g.hist));
    if (p.fill) st = launch(embedding_zero_kernel, 2 * sms, kSortThreads, 0, s, false, p);
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
    return e->hidden % 4 == 0 ? pick_grad<float, 4>(p, g, fp32_grad, s) : pick_grad<float, 1>(p, g, fp32_grad, s);
  return e->hidden % 8 == 0 ? pick_grad<__nv_bfloat16, 8>(p, g, fp32_grad, s) : pick_grad<__nv_bfloat16, 1>(p, g, fp32_grad, s);
}
