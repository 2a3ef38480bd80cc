// Root-mean-square norm, forward (with the residual sum of a block, its output in full precision, in 8 bits with scales, or
// both) and backward:
//   h = X (+ residual),  rstd = 1 / sqrt(mean(h^2) + eps),  y = h * rstd * gamma
//   dX = rstd * (g dY - xhat * mean(g dY xhat)) (+ dsum),  dgamma = sum over the rows of dY * xhat,  xhat = X * rstd
//
// Bound by HBM.  A row is read once into registers; the rows after it are copied ahead through shared memory.  The output in 8
// bits is made from the FP32 values: a run of 128 columns lies in 16 neighbouring lanes (32 in FP32), so that its maximum is four
// (five) shuffles away, and it costs 1 + 1/128 bytes an element instead of a second pass over 2.
// 16384 x 8192 in BF16 with the residual to 8 bits: 138 us, 6.8 TB/s; without 80, by instructions; to BF16 with the residual 185, 5.8
// TB/s.  Backward with the residual's gradient, 8192 x 4096: 46 us, 5.8 TB/s, both kernels.
#include "norm_rows.cuh"
#include "scaled8.cuh"

namespace compass {

namespace {

struct RmsParams {
  RowShards x, residual, summed, y, y8, scale;      // forward
  RowShards dy, dsum, dx;                           // backward (x above: the normalised input)
  const void* gamma;
  float* rstd;
  float* partial;                                   // backward: [n_partial][hidden] sums of dY * xhat
  float* row_sums;                                  // backward, wide rows: a sum per row
  int64_t hidden;
  int64_t blocks;                                   // scales per row
  uint32_t M;
  int32_t has_residual, has_dsum, has_y;
  int32_t param_fp32;
  float eps;
  int32_t n_partial;
};

constexpr int kNone = -1;      // no output in 8 bits

// NVT vectors of V neighbouring values times `factor`, `step` elements apart, to 8 bits; a run of 128 lies in 128 / V neighbouring
// lanes.  All lanes of the warp take part; the first `live` vectors are stored.  (The factor comes in behind the maximum, which is
// that of the products all the same: rounding keeps their order.)
template <int kFormat, int V, int NVT>
__device__ __forceinline__ void store_8bit(F2 (&x)[V * NVT / 2], float factor, uint8_t* to, uint8_t* scale, int step, int live) {
  constexpr int kLanes = 128 / V, kPer = V / 2;
  float top[NVT];
  auto largest = [&] {
    bool infinite = false;
#pragma unroll
    for (int i = 0; i < NVT; ++i) {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const float2 q = of(x[i * kPer + j]);
        m = fmaxf(m, fmaxf(fabsf(q.x), fabsf(q.y)));
      }
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      top[i] = m * factor;
      infinite |= !(top[i] < INFINITY);
    }
    return infinite;
  };
  if (__any_sync(0xffffffffu, largest())) {
    // (times the factor now: a product with it may be what is infinite)
    auto finite = [&](float a) { return fabsf(a * factor) < INFINITY ? a * factor : __uint_as_float(0x7FC00000u); };
#pragma unroll
    for (int j = 0; j < kPer * NVT; ++j) {
      const float2 q = of(x[j]);
      x[j] = f2(finite(q.x), finite(q.y));
    }
    factor = 1.f;
    largest();
  }
#pragma unroll
  for (int i = 0; i < NVT; ++i) {
    if (i >= live) break;
    const uint32_t b = scale_byte_of<kFormat>(__float_as_uint(top[i]));
    const F2 f = f2(inverse_scale(b));
    uint32_t w[V / 4];
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const F2 g = f2(factor);
      const float2 lo = of(x[i * kPer + 2 * j] * g * f), hi = of(x[i * kPer + 2 * j + 1] * g * f);
      w[j] = pack8x4<kFormat>(lo.x, lo.y, hi.x, hi.y);
    }
    if constexpr (V == 8) *reinterpret_cast<uint2*>(to + i * step) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(to + i * step) = w[0];
    if (threadIdx.x % kLanes == 0) scale[i * step / 128] = uint8_t(b);
  }
}

// ---- forward -------------------------------------------------------------------
// A row per group of kTpr threads, NVT vectors of V elements a thread.  kKeep: gamma stays in registers.
// Elements of a row per thread: what a row costs every thread is shared by this many.  The output in 8 bits alone is bound by
// instructions, and takes 32 in BF16; with the residual, four streams of memory, it goes better with more threads a row.  To 8 bits, us,
// 16 and 32: 16384 x 8192: 98 and 79, with the residual 140 and 159; 16384 x 4096: 53 and 41, 76 and 81; with the values restored again
// 16384 x 1024: 23.5 and 22.4, 29.4 and 28.9.  In BF16: 16384 x 4096: 44 and 48, with the residual 95 and 91; 4096 x 8192: 25 and 23, 47
// and 47.
template <typename T, int V, bool kResidual, int kFormat>
constexpr int kForwardElems = V == 8 ? (kFormat != kNone && !kResidual ? 32 : 16) : V == 4 ? 16 : 8;
template <typename T, int V, int NVT, int kThreads, bool kResidual>
using ForwardRing = RowRing<T, V, NVT, kResidual ? 2 : 1, kThreads, 200 * 1024>;
template <typename T, int V, int NVT, int kThreads, int kTpr, bool kKeep, bool kResidual, int kFormat>
__global__ void __launch_bounds__(kThreads, 1) rms_forward_kernel(const __grid_constant__ RmsParams p) {
  using Ring = ForwardRing<T, V, NVT, kThreads, kResidual>;
  __shared__ float red[2][32];
  extern __shared__ uint4 raw[];
  const int groups = blockDim.x / kTpr, group = threadIdx.x / kTpr, t = threadIdx.x - group * kTpr;
  const int H = int(p.hidden);
  const float inv = 1.0f / float(H);
  Ring ring(raw);
  auto fetch = [&](int which, uint32_t row) {
    const bool live = row < p.M;
    const RowAt at = p.x.at(row, H);
    if constexpr (kResidual) {
      const T* const from[2] = {live ? p.x.row<T>(at) : nullptr, live ? p.residual.row<T>(at) : nullptr};
      ring.fetch(which, from, kTpr, t, H);
    } else {
      const T* const from[1] = {live ? p.x.row<T>(at) : nullptr};
      ring.fetch(which, from, kTpr, t, H);
    }
  };
  launch_dependents();
  wait_for_previous_kernel();
  const uint32_t stride = gridDim.x * groups;
  uint32_t row = blockIdx.x * groups + group;
#pragma unroll 1
  for (int k = 0; k < Ring::kDepth; ++k) fetch(k, row + k * stride);
  constexpr int kPairs = V * NVT / 2;
  F2 g[kPairs];
  if constexpr (kKeep) load_params<V, NVT>(g, p.gamma, p.param_fp32, 1.f, kTpr, t, H);
  const int own = min(NVT, max(0, (H / V - t + kTpr - 1) / kTpr));      // vectors of a row that this thread holds
  for (uint32_t turn = 0; row < p.M; ++turn, row += stride) {
    const RowAt at = p.x.at(row, H);
    Words<T, V, NVT> x;
    ring.wait();
#pragma unroll
    for (int i = 0; i < NVT; ++i) ring.take(x.w[i], 0, i, kTpr, t, H);
    if constexpr (kResidual) {
      // what is stored is normalised, so that the backward pass, which reads it, sees the same values
      Words<T, V, NVT> r;
#pragma unroll
      for (int i = 0; i < NVT; ++i) ring.take(r.w[i], 1, i, kTpr, t, H);
      x.add(r);
      x.store(p.summed.row<T>(at), kTpr, t, H);
    }
    ring.advance();
    fetch(Ring::kDepth - 1, row + Ring::kDepth * stride);
    F2 h[kPairs], sq[2] = {f2(0.f), f2(0.f)};
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      h[k] = x.pair(k);
      sq[k & 1] = fma2(h[k], h[k], sq[k & 1]);
    }
    const float rstd = 1.0f / sqrtf(row_sum(sum_of(sq[0] + sq[1]), kTpr, red[turn & 1]) * inv + p.eps);
    if constexpr (!kKeep) load_params<V, NVT>(g, p.gamma, p.param_fp32, 1.f, kTpr, t, H);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) h[k] = h[k] * g[k];
    if (kFormat == kNone || p.has_y) {
      F2 y[kPairs];
#pragma unroll
      for (int k = 0; k < kPairs; ++k) y[k] = h[k] * f2(rstd);
      x.set(y);
      x.store(p.y.row<T>(at), kTpr, t, H);
    }
    if constexpr (kFormat != kNone) {
      uint8_t* scale = static_cast<uint8_t*>(p.scale.ptr[at.shard]) + (row - at.shard * p.x.rows.d) * p.blocks + t * V / 128;
      store_8bit<kFormat, V, NVT>(h, rstd, p.y8.row<uint8_t>(at) + t * V, scale, kTpr * V, own);
    }
    if (t == 0 && p.rstd) p.rstd[row] = rstd;
  }
}

// Rows that do not fit the registers of a block: one block per row, two passes over it (the second out of L2).
template <typename T, int V, int kFormat>
__global__ void __launch_bounds__(1024) rms_forward_wide_kernel(const __grid_constant__ RmsParams p) {
  __shared__ float red[32];
  launch_dependents();
  wait_for_previous_kernel();
  const uint32_t row = blockIdx.x;
  const int64_t H = p.hidden;
  const T* x = p.x.row<T>(row, H);
  const T* r = p.has_residual ? p.residual.row<T>(row, H) : nullptr;
  T* s = p.has_residual ? p.summed.row<T>(row, H) : nullptr;
  float a[V], b[V], sq = 0.f;
  for (int64_t c = threadIdx.x * V; c < H; c += 1024 * V) {
    load_vec(a, x + c);
    if (r) {
      load_vec(b, r + c);
#pragma unroll
      for (int j = 0; j < V; ++j) a[j] = round_to<T>(a[j] + b[j]);
      store_vec(s + c, a);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sq = fmaf(a[j], a[j], sq);
  }
  const T* h = r ? s : x;       // a thread reads back only what it wrote itself
  const float rstd = 1.0f / sqrtf(row_sum(sq, 1024, red) / float(H) + p.eps);
  for (int64_t c0 = 0; c0 < H; c0 += 1024 * V) {
    const int64_t c = c0 + threadIdx.x * V;
    const bool live = c < H;
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] = 0.f;
    if (live) {
      float g[V];
      load_vec(a, h + c);
      load_param(g, p.gamma, p.param_fp32, c, 1.f);
#pragma unroll
      for (int j = 0; j < V; ++j) a[j] = a[j] * rstd * g[j];
      if (kFormat == kNone || p.has_y) store_vec(p.y.row<T>(row, H) + c, a);
    }
    if constexpr (kFormat != kNone) {
      F2 x[V / 2];
#pragma unroll
      for (int j = 0; j < V / 2; ++j) x[j] = f2(a[2 * j], a[2 * j + 1]);
      store_8bit<kFormat, V, 1>(x, 1.f, p.y8.row<uint8_t>(row, H) + c, p.scale.row<uint8_t>(row, p.blocks) + (c >> 7), 0, live);
    }
  }
  if (threadIdx.x == 0 && p.rstd) p.rstd[row] = rstd;
}

// ---- backward ------------------------------------------------------------------
// One block per SM walks the rows; a thread keeps its columns' sums of dY * xhat in registers while the next rows are on their
// way.  A block's rows add their sums up in shared memory and leave one partial row for rms_reduce_kernel: fixed order, so the
// bits do not depend on timing.
template <typename T, int V, int NVT, int kThreads, int kTpr, bool kDsum>
__global__ void __launch_bounds__(kThreads, 1) rms_backward_kernel(const __grid_constant__ RmsParams p) {
  static_assert(V * NVT == kElems<T, V>, "");
  using Ring = RowRing<T, V, NVT, kDsum ? 3 : 2, kThreads>;
  __shared__ float red[2][32];
  extern __shared__ uint4 raw[];
  const int groups = blockDim.x / kTpr, group = threadIdx.x / kTpr, t = threadIdx.x - group * kTpr;
  const int H = int(p.hidden);
  const float inv = 1.0f / float(H);
  constexpr int kPairs = V * NVT / 2;
  launch_dependents();
  wait_for_previous_kernel();
  F2 dg[kPairs];
#pragma unroll
  for (int k = 0; k < kPairs; ++k) dg[k] = f2(0.f);
  // gamma in FP32, every thread its own elements (in registers they would spill); the ring behind it
  F2* gamma = reinterpret_cast<F2*>(raw) + threadIdx.x;
  {
    F2 g[kPairs];
    load_params<V, NVT>(g, p.gamma, p.param_fp32, 1.f, kTpr, t, H);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) gamma[k * kThreads] = g[k];
  }
  Ring ring(reinterpret_cast<F2*>(raw) + kPairs * kThreads);
  auto fetch = [&](int which, uint32_t row) {
    const bool live = row < p.M;
    const RowAt at = p.x.at(row, H);
    if constexpr (kDsum) {
      const T* const from[3] = {live ? p.x.row<T>(at) : nullptr, live ? p.dy.row<T>(at) : nullptr, live ? p.dsum.row<T>(at) : nullptr};
      ring.fetch(which, from, kTpr, t, H);
    } else {
      const T* const from[2] = {live ? p.x.row<T>(at) : nullptr, live ? p.dy.row<T>(at) : nullptr};
      ring.fetch(which, from, kTpr, t, H);
    }
  };
  const uint32_t stride = gridDim.x * groups;
  uint32_t row = blockIdx.x * groups + group;
#pragma unroll 1
  for (int k = 0; k < Ring::kDepth; ++k) fetch(k, row + k * stride);
  float rstd = row < p.M ? p.rstd[row] : 0.f;
  for (uint32_t turn = 0; row < p.M; ++turn, row += stride) {
    F2 xh[kPairs], d[kPairs];
    const F2 r2 = f2(rstd);
    const RowAt at = p.x.at(row, H);
    if (row + stride < p.M) rstd = p.rstd[row + stride];
    Words<T, V, NVT> w;
    ring.wait();
#pragma unroll
    for (int i = 0; i < NVT; ++i) ring.take(w.w[i], 0, i, kTpr, t, H);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) xh[k] = w.pair(k) * r2;
#pragma unroll
    for (int i = 0; i < NVT; ++i) ring.take(w.w[i], 1, i, kTpr, t, H);
    F2 c[2] = {f2(0.f), f2(0.f)};
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const F2 dy = w.pair(k);
      dg[k] = fma2(dy, xh[k], dg[k]);
      d[k] = gamma[k * kThreads] * dy;
      c[k & 1] = fma2(d[k], xh[k], c[k & 1]);
    }
    const F2 a2 = f2(-row_sum(sum_of(c[0] + c[1]), kTpr, red[turn & 1]) * inv);
    if constexpr (kDsum) {
#pragma unroll
      for (int i = 0; i < NVT; ++i) ring.take(w.w[i], 2, i, kTpr, t, H);
    }
    ring.advance();
    fetch(Ring::kDepth - 1, row + Ring::kDepth * stride);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const F2 v = fma2(xh[k], a2, d[k]);
      d[k] = kDsum ? fma2(v, r2, w.pair(k)) : v * r2;
    }
    w.set(d);
    w.store(p.dx.row<T>(at), kTpr, t, H);
  }
  float* sums = reinterpret_cast<float*>(raw);      // [groups][hidden], over gamma and the ring, whose last copies were of no row
  asm volatile("cp.async.wait_all;" ::: "memory");
  float* out = p.partial + int64_t(blockIdx.x) * H;
  if (groups > 1) __syncthreads();
  float* to = groups > 1 ? sums + group * H : out;
#pragma unroll
  for (int i = 0; i < NVT; ++i) {
    const int c = (i * kTpr + t) * V;
    if (c < H) {
      float x[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float2 q = of(dg[(i * V + j) / 2]);
        x[j] = (i * V + j) & 1 ? q.y : q.x;
      }
      if constexpr (V == 1) {
        to[c] = x[0];
      } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(to + c + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
      }
    }
  }
  if (groups > 1) {
    __syncthreads();
    for (int c = threadIdx.x; c < H; c += blockDim.x) {
      float a = 0.f;
      for (int k = 0; k < groups; ++k) a += sums[k * H + c];
      out[c] = a;
    }
  }
}

// Sums over the partial rows: 32 columns per block, kReduceWays threads a column (each a fixed share of the rows, all of whose
// loads are in flight together: the kernel is a load's latency long), and their sums in turn.
constexpr int kReduceWays = 16;
template <typename PT>
__global__ void __launch_bounds__(32 * kReduceWays) rms_reduce_kernel(const __grid_constant__ RmsParams p, PT* dgamma) {
  __shared__ float part[kReduceWays][33];
  launch_dependents();
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int64_t c = int64_t(blockIdx.x) * 32 + lane;
  const float* in = p.partial + c;
  float a = 0.f;
  if (c < p.hidden) {
    for (int r0 = k; r0 < p.n_partial; r0 += 10 * kReduceWays) {
      float x[10];
#pragma unroll
      for (int i = 0; i < 10; ++i) {
        const int r = r0 + i * kReduceWays;
        x[i] = r < p.n_partial ? __ldcg(in + int64_t(r) * p.hidden) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 10; ++i) a += x[i];
    }
  }
  part[k][lane] = a;
  __syncthreads();
  if (k == 0 && c < p.hidden) {
    float v[1] = {0.f};
#pragma unroll
    for (int i = 0; i < kReduceWays; ++i) v[0] += part[i][lane];
    store_vec(dgamma + c, v);
  }
}

// Wide rows: the row sums first (one block per row), then dX and the column sums by slabs of columns.
template <typename T, int V>
__global__ void __launch_bounds__(1024) rms_backward_rows_kernel(const __grid_constant__ RmsParams p) {
  __shared__ float red[32];
  launch_dependents();
  wait_for_previous_kernel();
  const uint32_t row = blockIdx.x;
  const int64_t H = p.hidden;
  const T* x = p.x.row<T>(row, H);
  const T* dy = p.dy.row<T>(row, H);
  float s = 0.f, a[V], d[V], g[V];
  for (int64_t c = threadIdx.x * V; c < H; c += 1024 * V) {
    load_vec(a, x + c);
    load_vec(d, dy + c);
    load_param(g, p.gamma, p.param_fp32, c, 1.f);
#pragma unroll
    for (int j = 0; j < V; ++j) s = fmaf(d[j] * g[j], a[j], s);
  }
  s = row_sum(s, 1024, red);
  if (threadIdx.x == 0) p.row_sums[row] = s * p.rstd[row] / float(H);      // mean(g dY xhat)
}
template <typename T, int V>
__global__ void __launch_bounds__(256) rms_backward_columns_kernel(const __grid_constant__ RmsParams p) {
  launch_dependents();
  wait_for_previous_kernel();
  const int64_t H = p.hidden;
  const int64_t slabs = (H + 256 * V - 1) / (256 * V);
  const int64_t c = (int64_t(blockIdx.x) % slabs * 256 + threadIdx.x) * V;
  const uint32_t part = uint32_t(blockIdx.x / slabs);
  if (c >= H) return;
  float g[V], dg[V];
  load_param(g, p.gamma, p.param_fp32, c, 1.f);
#pragma unroll
  for (int j = 0; j < V; ++j) dg[j] = 0.f;
#pragma unroll 2
  for (uint32_t row = part; row < p.M; row += uint32_t(p.n_partial)) {
    float a[V], d[V], s[V];
    const RowAt at = p.x.at(row, H);
    load_vec(a, p.x.row<T>(at) + c);
    load_vec(d, p.dy.row<T>(at) + c);
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    if (p.has_dsum) load_vec(s, p.dsum.row<T>(at) + c);
    const float r = p.rstd[row], mean = p.row_sums[row];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float xh = a[j] * r;
      dg[j] = fmaf(d[j], xh, dg[j]);
      s[j] = fmaf(r, fmaf(-xh, mean, d[j] * g[j]), s[j]);
    }
    store_vec(p.dx.row<T>(at) + c, s);
  }
  float* out = p.partial + int64_t(part) * H + c;
#pragma unroll
  for (int j = 0; j < V; ++j) out[j] = dg[j];
}

// ---- host ----------------------------------------------------------------------

int check_norm(const compass_norm* n) {
  if (n == nullptr) return COMPASS_ERR_INVALID_ARG;
  int st = check_rows(n->P, n->M, n->hidden);
  if (st == COMPASS_OK) st = check_dtype(n->dtype, true);
  if (st == COMPASS_OK) st = check_dtype(n->param_dtype, true);
  if (st != COMPASS_OK) return st;
  return n->eps >= 0.f ? COMPASS_OK : COMPASS_ERR_INVALID_ARG;      // (NaN is refused too)
}

// Rows of whole 16-byte vectors; with pointers on 16-byte boundaries they are accessed as such.
bool whole_vectors(const compass_norm* n) { return n->hidden % (n->dtype == COMPASS_DTYPE_FP32 ? 4 : 8) == 0; }

constexpr int kSms = 148;           // blocks are counted for a B200; fewer SMs only take them in turns
constexpr int64_t kWidest = 8192;   // elements of a row that stay in the registers of a block
constexpr int kWideParts = 64;      // row ranges of the wide form's column sums

struct BackwardPlan {
  bool wide;
  int tpr, groups, threads, n_partial;
};
BackwardPlan backward_plan(const compass_norm* n, bool whole) {
  BackwardPlan b;
  const bool packed = n->dtype == COMPASS_DTYPE_BF16 && whole;
  b.wide = n->hidden > kWidest;
  b.tpr = b.wide ? 1024 : threads_per_row(n->hidden, packed ? 16 : 8);
  b.threads = b.tpr > 512 ? 1024 : 512;        // 128 registers a thread unless a row needs more than 512 threads
  b.groups = b.wide ? 1 : rows_per_block(b.tpr, b.threads);
  const int64_t most = b.wide ? kWideParts : kSms;
  const int64_t need = b.wide ? n->M : ceil_div(n->M, b.groups);
  b.n_partial = int(need < most ? need : most);
  return b;
}

template <typename T, int V, int NVT, int kThreads, int kTpr, bool kKeep, bool kResidual, int kFormat>
int run_forward(const RmsParams& p, cudaStream_t stream) {
  constexpr size_t smem = ForwardRing<T, V, NVT, kThreads, kResidual>::kSmemBytes;
  auto kernel = rms_forward_kernel<T, V, NVT, kThreads, kTpr, kKeep, kResidual, kFormat>;
  static std::atomic<uint64_t> allowed{0};
  const int st = allow_smem(reinterpret_cast<const void*>(kernel), smem, &allowed);
  if (st != COMPASS_OK) return st;
  // few rows: a block each, for the shortest way through; else blocks of several that walk the rows
  const int groups = p.M <= kSms || kTpr * 2 > kThreads ? 1 : rows_per_block(kTpr, kThreads);
  const int64_t need = ceil_div(p.M, groups), most = kSms * (smem ? 1 : kThreads / (kTpr * groups));
  return launch(kernel, need < most ? need : most, kTpr * groups, smem, stream, true, p);
}

// Up to 8192 elements a row (or 16384, at 32 a thread): gamma in registers.  Up to 16384: 16 elements per thread.
template <typename T, int V, bool kResidual, int kFormat>
int pick_forward(const RmsParams& p, cudaStream_t stream) {
  constexpr int E = kForwardElems<T, V, kResidual, kFormat>, kThreads = V == 1 ? 1024 : 512;
  if constexpr (E * kThreads < 2 * kWidest) {
    if (p.hidden > kWidest) return run_forward<T, V, 16 / V, 1024, 1024, false, kResidual, kFormat>(p, stream);
  }
  return with_tpr<kThreads>(threads_per_row(p.hidden, E), [&](auto tpr) {
    return run_forward<T, V, E / V, kThreads, decltype(tpr)::value, true, kResidual, kFormat>(p, stream);
  });
}
template <typename T, int V, int kFormat>
int forward_of(const RmsParams& p, cudaStream_t stream) {
  if (p.hidden > 2 * kWidest) return launch(rms_forward_wide_kernel<T, V, kFormat>, p.M, 1024, 0, stream, true, p);
  return p.has_residual ? pick_forward<T, V, true, kFormat>(p, stream) : pick_forward<T, V, false, kFormat>(p, stream);
}
template <typename T>
int forward_of(const RmsParams& p, bool vec, int format, cudaStream_t stream) {
  constexpr int V = 16 / int(sizeof(T));
  if (format == E4M3) return forward_of<T, V, E4M3>(p, stream);
  if (format == E5M2) return forward_of<T, V, E5M2>(p, stream);
  return vec ? forward_of<T, V, kNone>(p, stream) : forward_of<T, 1, kNone>(p, stream);
}

template <typename T, int V, int kThreads, int kTpr, bool kDsum>
int run_backward(const RmsParams& p, const BackwardPlan& b, cudaStream_t stream) {
  constexpr int NVT = kElems<T, V> / V;
  constexpr size_t ring = RowRing<T, V, NVT, kDsum ? 3 : 2, kThreads>::kSmemBytes + size_t(kElems<T, V>) * kThreads * 4;
  auto kernel = rms_backward_kernel<T, V, NVT, kThreads, kTpr, kDsum>;
  constexpr size_t sums = size_t(kThreads) * kElems<T, V> * 4;      // [groups][hidden] at most
  constexpr size_t smem = ring > sums ? ring : sums;
  static std::atomic<uint64_t> allowed{0};
  const int st = allow_smem(reinterpret_cast<const void*>(kernel), smem, &allowed);
  if (st != COMPASS_OK) return st;
  return launch(kernel, b.n_partial, b.tpr * b.groups, smem, stream, true, p);
}
template <typename T, int V, int kThreads, int kTpr>
int run_backward(const RmsParams& p, const BackwardPlan& b, cudaStream_t stream) {
  return p.has_dsum ? run_backward<T, V, kThreads, kTpr, true>(p, b, stream) : run_backward<T, V, kThreads, kTpr, false>(p, b, stream);
}
template <typename T, int V>
int backward_of(const RmsParams& p, const BackwardPlan& b, cudaStream_t stream) {
  if (b.wide) {
    const int st = launch(rms_backward_rows_kernel<T, V>, p.M, 1024, 0, stream, true, p);
    if (st != COMPASS_OK) return st;
    return launch(rms_backward_columns_kernel<T, V>, ceil_div(p.hidden, 256 * V) * b.n_partial, 256, 0, stream, true, p);
  }
  if constexpr (V != 8) {
    if (b.tpr > 512) return run_backward<T, V, 1024, 1024>(p, b, stream);
  }
  return with_tpr<512>(b.tpr, [&](auto tpr) { return run_backward<T, V, 512, decltype(tpr)::value>(p, b, stream); });
}
template <typename T>
int backward_of(const RmsParams& p, const BackwardPlan& b, bool vec, cudaStream_t stream) {
  return vec ? backward_of<T, 16 / int(sizeof(T))>(p, b, stream) : backward_of<T, 1>(p, b, stream);
}

}  // namespace

}  // namespace compass

using namespace compass;

extern "C" int compass_rms_norm(const compass_norm* n, const void* const* X, const void* const* residual, const void* gamma, void* const* summed,
                                void* const* Y, int format, void* const* Y8, void* const* scale, float* rstd, void* stream) {
  int st = check_norm(n);
  if (st != COMPASS_OK) return st;
  if ((residual == nullptr) != (summed == nullptr) || (Y8 == nullptr) != (scale == nullptr) || (Y == nullptr && Y8 == nullptr))
    return COMPASS_ERR_INVALID_ARG;
  if (Y8 && format_of(format) < 0) return COMPASS_ERR_UNSUPPORTED;
  if (Y8 && n->hidden % 16 != 0) return COMPASS_ERR_ALIGNMENT;
  RmsParams p = {};
  const size_t element = dtype_size(n->dtype), param = dtype_size(n->param_dtype);
  const size_t align = Y8 ? 16 : element;      // the output in 8 bits is made by whole vectors
  bool whole = whole_vectors(n) && is_aligned(gamma, 16);
  st = fill_shards(X, n->P, n->M, &p.x, align, &whole);
  if (st == COMPASS_OK && Y) st = fill_shards(Y, n->P, n->M, &p.y, align, &whole);
  if (st == COMPASS_OK && residual) st = fill_shards(residual, n->P, n->M, &p.residual, align, &whole);
  if (st == COMPASS_OK && summed) st = fill_shards(summed, n->P, n->M, &p.summed, align, &whole);
  if (st == COMPASS_OK && Y8) st = fill_shards(Y8, n->P, n->M, &p.y8, 16);
  if (st == COMPASS_OK && Y8) st = fill_shards(scale, n->P, n->M, &p.scale, 1);
  if (st != COMPASS_OK) return st;
  if (!is_aligned(gamma, Y8 ? 16 : param) || !is_aligned(rstd, 4)) return COMPASS_ERR_ALIGNMENT;
  if (n->M == 0) return COMPASS_OK;
  p.gamma = gamma;
  p.rstd = rstd;
  p.hidden = n->hidden;
  p.blocks = scale_blocks(n->hidden);
  p.M = uint32_t(n->M);
  p.has_residual = residual != nullptr;
  p.has_y = Y != nullptr;
  p.param_fp32 = n->param_dtype == COMPASS_DTYPE_FP32;
  p.eps = n->eps;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int f = Y8 ? format_of(format) : kNone;
  return n->dtype == COMPASS_DTYPE_FP32 ? forward_of<float>(p, whole, f, s) : forward_of<__nv_bfloat16>(p, whole, f, s);
}

// Workspace: the partial column sums, then (wide rows) a sum per row.
extern "C" int compass_rms_norm_workspace_bytes(const compass_norm* n, size_t* bytes) {
  if (bytes == nullptr) return COMPASS_ERR_INVALID_ARG;
  const int st = check_norm(n);
  if (st != COMPASS_OK) return st;
  // (whether the pointers will be on 16-byte boundaries is not known yet)
  const BackwardPlan a = backward_plan(n, false), b = backward_plan(n, whole_vectors(n));
  const int most = a.n_partial > b.n_partial ? a.n_partial : b.n_partial;
  *bytes = 256 + round_up(size_t(most) * size_t(n->hidden) * 4, 256) + (b.wide ? size_t(n->M) * 4 : 0);
  return COMPASS_OK;
}

extern "C" int compass_rms_norm_backward(const compass_norm* n, const void* const* dY, const void* const* X, const void* gamma, const float* rstd,
                                         const void* const* dsum, void* const* dX, void* dgamma, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  int st = compass_rms_norm_workspace_bytes(n, &need);
  if (st != COMPASS_OK) return st;
  RmsParams p = {};
  const size_t element = dtype_size(n->dtype), param = dtype_size(n->param_dtype);
  bool whole = whole_vectors(n) && is_aligned(gamma, 16);
  st = fill_shards(dY, n->P, n->M, &p.dy, element, &whole);
  if (st == COMPASS_OK) st = fill_shards(X, n->P, n->M, &p.x, element, &whole);
  if (st == COMPASS_OK) st = fill_shards(dX, n->P, n->M, &p.dx, element, &whole);
  if (st == COMPASS_OK && dsum) st = fill_shards(dsum, n->P, n->M, &p.dsum, element, &whole);
  if (st != COMPASS_OK) return st;
  if (n->M > 0 && rstd == nullptr) return COMPASS_ERR_INVALID_ARG;
  if (!is_aligned(gamma, param) || !is_aligned(dgamma, param) || !is_aligned(rstd, 4)) return COMPASS_ERR_ALIGNMENT;
  st = check_workspace(ws, ws_bytes, need);
  if (st != COMPASS_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (n->M == 0) {
    if (dgamma == nullptr) return COMPASS_OK;
    const cudaError_t e = cudaMemsetAsync(dgamma, 0, size_t(n->hidden) * dtype_size(n->param_dtype), s);
    return e == cudaSuccess ? COMPASS_OK : record_cuda_error(e);
  }
  const BackwardPlan b = backward_plan(n, whole);
  p.gamma = gamma;
  p.rstd = const_cast<float*>(rstd);
  p.hidden = n->hidden;
  p.M = uint32_t(n->M);
  p.has_dsum = dsum != nullptr;
  p.param_fp32 = n->param_dtype == COMPASS_DTYPE_FP32;
  p.n_partial = b.n_partial;
  p.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + 256);
  p.row_sums = p.partial + round_up(size_t(b.n_partial) * size_t(n->hidden) * 4, 256) / 4;
  st = n->dtype == COMPASS_DTYPE_FP32 ? backward_of<float>(p, b, whole, s) : backward_of<__nv_bfloat16>(p, b, whole, s);
  if (st != COMPASS_OK || dgamma == nullptr) return st;
  const int64_t grid = ceil_div(n->hidden, 32);
  if (n->param_dtype == COMPASS_DTYPE_FP32) return launch(rms_reduce_kernel<float>, grid, 32 * kReduceWays, 0, s, true, p, static_cast<float*>(dgamma));
  return launch(rms_reduce_kernel<__nv_bfloat16>, grid, 32 * kReduceWays, 0, s, true, p, static_cast<__nv_bfloat16*>(dgamma));
}
