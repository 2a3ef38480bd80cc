// Layer norm, forward (with the residual sum of a block) and backward.
//
// Both passes should be bound by HBM: forward reads X (and the residual) and
// writes Y (and the sum), backward reads dY and X (and the gradient of the
// residual path) and writes dX.  A row is read once into registers, where its
// statistics are taken from the values themselves (the variance from the centred
// ones), so no element travels twice.  What stood in the way was the number of
// instructions per element (55 in the first form, and most of the time): hence
// FP32 in pairs, one position per row for all tensors, row widths compiled in,
// 16 elements a thread.  Measured (of the copy rate, 6.55 TB/s): forward with
// residual, 16384 x 8192 BF16: 168 to 192 us, 98 to 86 %, from box to box and run
// to run (the same code; no cause found); backward with the residual's
// gradient, 8192 x 4096 BF16: 51 us, 80 % (half of its issue slots are busy, and
// a row's sums hold up the rest); backward, 4095 x 1001 FP32, an element per
// access: 21 us, 35 %; 8192 x 1001 BF16, whose rows are not copied ahead either:
// 33 us, 30 %; backward beyond 8192 elements, which passes over X and dY twice, an
// element per access, 8192 x 12288 BF16: 665 us, 18 %, FP32 705 us, 35 %; forward,
// 8 x 4096: 3.5 us, one way through.
#include <mutex>
#include <type_traits>

#include "norm_rows.cuh"

namespace compass {

namespace {

struct NormParams {
  RowShards x, residual, summed, y;      // forward
  RowShards dy, dsum, dx;                // backward (x above: the normalised input)
  const void* gamma;
  const void* beta;
  float* mean;
  float* rstd;
  float* partial;                        // backward: [2][n_partial][hidden] sums of dY * xhat and of dY
  float* row_sums;                       // backward, wide rows: [M][2]
  int64_t hidden;
  uint32_t M;
  int32_t has_residual, has_dsum;
  int32_t param_fp32;
  float eps;
  int32_t n_partial;
};

// ---- forward -------------------------------------------------------------------
// A row per group of kTpr threads, NVT vectors of V elements a thread, all in registers; the rows after it are on their way
// meanwhile.  kKeep: gamma and beta stay in registers too.
template <typename T, int V, int NVT, int kThreads, int kTpr, bool kKeep, bool kResidual>
__global__ void __launch_bounds__(kThreads, 1) norm_forward_kernel(const __grid_constant__ NormParams p) {
  using Ring = RowRing<T, V, NVT, kResidual ? 2 : 1, kThreads>;
  __shared__ float red[4][32];
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
  const uint32_t stride = gridDim.x * groups;
  uint32_t row = blockIdx.x * groups + group;
#pragma unroll 1
  for (int k = 0; k < Ring::kDepth; ++k) fetch(k, row + k * stride);
  constexpr int kPairs = V * NVT / 2;
  F2 g[kPairs], b[kPairs];
  if constexpr (kKeep) {
    load_params<V, NVT>(g, p.gamma, p.param_fp32, 1.f, kTpr, t, H);
    load_params<V, NVT>(b, p.beta, p.param_fp32, 0.f, kTpr, t, H);
  }
  const int own = min(NVT, max(0, (H / V - t + kTpr - 1) / kTpr)) * V;      // elements of a row that this thread holds
  const bool ragged = kTpr * (NVT * V) != H;
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
    F2 h[kPairs], sum[2] = {f2(0.f), f2(0.f)};
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      h[k] = x.pair(k);
      sum[k & 1] = sum[k & 1] + h[k];
    }
    const float mean = row_sum(sum_of(sum[0] + sum[1]), kTpr, red[2 * (turn & 1)]) * inv;
    F2 sq[2] = {f2(0.f), f2(0.f)};
    const F2 minus = f2(-mean);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) h[k] = h[k] + minus;
    if (ragged) {
#pragma unroll
      for (int k = 0; k < kPairs; ++k)
        if (2 * k + 1 >= own) h[k] = 2 * k < own ? f2(of(h[k]).x, 0.f) : f2(0.f);      // past the row's end
    }
#pragma unroll
    for (int k = 0; k < kPairs; ++k) sq[k & 1] = fma2(h[k], h[k], sq[k & 1]);
    const float var = row_sum(sum_of(sq[0] + sq[1]), kTpr, red[2 * (turn & 1) + 1]) * inv;
    const float rstd = 1.0f / sqrtf(var + p.eps);
    if constexpr (!kKeep) {
      load_params<V, NVT>(g, p.gamma, p.param_fp32, 1.f, kTpr, t, H);
      load_params<V, NVT>(b, p.beta, p.param_fp32, 0.f, kTpr, t, H);
    }
#pragma unroll
    for (int k = 0; k < kPairs; ++k) h[k] = fma2(h[k] * f2(rstd), g[k], b[k]);
    x.set(h);
    x.store(p.y.row<T>(at), kTpr, t, H);
    if (t == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
  }
}

// Rows that do not fit the registers of a block: one block per row, three passes over it (the later ones out of L2).
template <typename T, int V>
__global__ void __launch_bounds__(1024) norm_forward_wide_kernel(const __grid_constant__ NormParams p) {
  __shared__ float red[2][32];
  const uint32_t row = blockIdx.x;
  const int64_t H = p.hidden;
  const T* x = p.x.row<T>(row, H);
  const T* r = p.has_residual ? p.residual.row<T>(row, H) : nullptr;
  T* s = p.has_residual ? p.summed.row<T>(row, H) : nullptr;
  float a[V], b[V], sum = 0.f, sq = 0.f;
  for (int64_t c = threadIdx.x * V; c < H; c += 1024 * V) {
    load_vec(a, x + c);
    if (r) {
      load_vec(b, r + c);
#pragma unroll
      for (int j = 0; j < V; ++j) a[j] = round_to<T>(a[j] + b[j]);
      store_vec(s + c, a);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sum += a[j];
  }
  const T* h = r ? s : x;       // a thread reads back only what it wrote itself
  const float inv = 1.0f / float(H);
  const float mean = row_sum(sum, 1024, red[0]) * inv;
  for (int64_t c = threadIdx.x * V; c < H; c += 1024 * V) {
    load_vec(a, h + c);
#pragma unroll
    for (int j = 0; j < V; ++j) sq = fmaf(a[j] - mean, a[j] - mean, sq);
  }
  const float rstd = 1.0f / sqrtf(row_sum(sq, 1024, red[1]) * inv + p.eps);
  T* y = p.y.row<T>(row, H);
  for (int64_t c = threadIdx.x * V; c < H; c += 1024 * V) {
    float g[V];
    load_vec(a, h + c);
    load_param(g, p.gamma, p.param_fp32, c, 1.f);
    load_param(b, p.beta, p.param_fp32, c, 0.f);
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] = fmaf((a[j] - mean) * rstd, g[j], b[j]);
    store_vec(y + c, a);
  }
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// ---- backward ------------------------------------------------------------------
// One block per SM walks the rows; a thread keeps its columns' sums of dY * xhat and dY in registers while the next rows are
// on their way.  A block's rows add their sums up in shared memory and leave one partial row for norm_reduce_kernel: fixed
// order, so the bits do not depend on timing.
template <typename T, int V, int NVT, int kThreads, int kTpr, bool kDsum>
__global__ void __launch_bounds__(kThreads, 1) norm_backward_kernel(const __grid_constant__ NormParams p) {
  static_assert(V * NVT == kElems<T, V>, "");
  using Ring = RowRing<T, V, NVT, kDsum ? 3 : 2, kThreads>;
  __shared__ float2 red[2][32];
  extern __shared__ uint4 raw[];
  const int groups = blockDim.x / kTpr, group = threadIdx.x / kTpr, t = threadIdx.x - group * kTpr;
  const int H = int(p.hidden);
  const float inv = 1.0f / float(H);
  constexpr int kPairs = V * NVT / 2;
  F2 dg[kPairs], db[kPairs];
#pragma unroll
  for (int k = 0; k < kPairs; ++k) dg[k] = db[k] = f2(0.f);
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
  float mean = row < p.M ? p.mean[row] : 0.f, rstd = row < p.M ? p.rstd[row] : 0.f;
  for (uint32_t turn = 0; row < p.M; ++turn, row += stride) {
    F2 xh[kPairs], d[kPairs];
    const float r = rstd;
    const F2 minus = f2(-mean), r2 = f2(r);
    const RowAt at = p.x.at(row, H);
    if (row + stride < p.M) {
      mean = p.mean[row + stride];
      rstd = p.rstd[row + stride];
    }
    Words<T, V, NVT> w;
    ring.wait();
#pragma unroll
    for (int i = 0; i < NVT; ++i) ring.take(w.w[i], 0, i, kTpr, t, H);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) xh[k] = (w.pair(k) + minus) * r2;
#pragma unroll
    for (int i = 0; i < NVT; ++i) ring.take(w.w[i], 1, i, kTpr, t, H);
    F2 c1 = f2(0.f), c2 = f2(0.f);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const F2 dy = w.pair(k);      // (past the row's end: 0, so that xhat's value there does not matter)
      dg[k] = fma2(dy, xh[k], dg[k]);
      db[k] = db[k] + dy;
      d[k] = gamma[k * kThreads] * dy;
      c1 = c1 + d[k];
      c2 = fma2(d[k], xh[k], c2);
    }
    const float2 c = row_sum(sum_of(c1), sum_of(c2), kTpr, red[turn & 1]);
    const F2 a1 = f2(-c.x * inv), a2 = f2(-c.y * inv);
    if constexpr (kDsum) {
#pragma unroll
      for (int i = 0; i < NVT; ++i) ring.take(w.w[i], 2, i, kTpr, t, H);
    }
    ring.advance();
    fetch(Ring::kDepth - 1, row + Ring::kDepth * stride);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const F2 v = fma2(xh[k], a2, d[k] + a1);
      d[k] = kDsum ? fma2(v, r2, w.pair(k)) : v * r2;
    }
    w.set(d);
    w.store(p.dx.row<T>(at), kTpr, t, H);
  }
  float* sums = reinterpret_cast<float*>(raw);      // [groups][hidden], over the ring, whose last copies were of no row
  asm volatile("cp.async.wait_all;" ::: "memory");
  // this block's sums, one array after the other through shared memory
  launch_dependents();
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* out = p.partial + (int64_t(which) * p.n_partial + blockIdx.x) * H;
    if (groups > 1) __syncthreads();
    float* to = groups > 1 ? sums + group * H : out;
#pragma unroll
    for (int i = 0; i < NVT; ++i) {
      const int c = (i * kTpr + t) * V;
      if (c < H) {
        float x[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float2 q = of(which ? db[(i * V + j) / 2] : dg[(i * V + j) / 2]);
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
}

// Sums over the partial rows: 32 columns per block, kReduceWays threads a column (each a fixed share of the rows, all of whose
// loads are in flight together: the kernel is a load's latency long), and their sums in turn.
constexpr int kReduceWays = 16;
template <typename PT>
__global__ void __launch_bounds__(32 * kReduceWays) norm_reduce_kernel(const __grid_constant__ NormParams p, PT* dgamma, PT* dbeta) {
  __shared__ float part[kReduceWays][33];
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int64_t c = int64_t(blockIdx.x >> 1) * 32 + lane;
  PT* out = blockIdx.x & 1 ? dbeta : dgamma;
  if (out == nullptr) return;
  const float* in = p.partial + int64_t(blockIdx.x & 1) * p.n_partial * p.hidden + c;
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
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kReduceWays; ++i) s += part[i][lane];
    float v[1] = {s};
    store_vec(out + c, v);
  }
}

// Wide rows: the row sums first (one block per row), then dX and the column sums by slabs of columns.
template <typename T>
__global__ void __launch_bounds__(1024) norm_backward_rows_kernel(const __grid_constant__ NormParams p) {
  __shared__ float2 red[32];
  const uint32_t row = blockIdx.x;
  const int64_t H = p.hidden;
  const T* x = p.x.row<T>(row, H);
  const T* dy = p.dy.row<T>(row, H);
  const float m = p.mean[row], r = p.rstd[row];
  float c1 = 0.f, c2 = 0.f, a[1], d[1], g[1];
  for (int64_t c = threadIdx.x; c < H; c += blockDim.x) {
    load_vec(a, x + c);
    load_vec(d, dy + c);
    load_param(g, p.gamma, p.param_fp32, c, 1.f);
    c1 += d[0] * g[0];
    c2 = fmaf(d[0] * g[0], (a[0] - m) * r, c2);
  }
  const float2 s = row_sum(c1, c2, 1024, red);
  if (threadIdx.x == 0) {
    p.row_sums[2 * int64_t(row)] = s.x;
    p.row_sums[2 * int64_t(row) + 1] = s.y;
  }
}
template <typename T>
__global__ void __launch_bounds__(256) norm_backward_columns_kernel(const __grid_constant__ NormParams p) {
  wait_for_previous_kernel();
  const int64_t H = p.hidden;
  const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (c >= H) return;
  const float inv = 1.0f / float(H);
  float g[1], dg = 0.f, db = 0.f;
  load_param(g, p.gamma, p.param_fp32, c, 1.f);
  for (uint32_t row = blockIdx.y; row < p.M; row += gridDim.y) {
    float a[1], d[1], s[1] = {0.f};
    load_vec(a, p.x.row<T>(row, H) + c);
    load_vec(d, p.dy.row<T>(row, H) + c);
    if (p.has_dsum) load_vec(s, p.dsum.row<T>(row, H) + c);
    const float r = p.rstd[row], xh = (a[0] - p.mean[row]) * r;
    const float c1 = p.row_sums[2 * int64_t(row)] * inv, c2 = p.row_sums[2 * int64_t(row) + 1] * inv;
    dg = fmaf(d[0], xh, dg);
    db += d[0];
    s[0] = fmaf(r, d[0] * g[0] - c1 - xh * c2, s[0]);
    store_vec(p.dx.row<T>(row, H) + c, s);
  }
  p.partial[int64_t(blockIdx.y) * H + c] = dg;
  p.partial[(int64_t(p.n_partial) + blockIdx.y) * H + c] = db;
}

// ---- host ----------------------------------------------------------------------

int check_norm(const compass_norm* n) {
  if (n == nullptr) return COMPASS_ERR_INVALID_ARG;
  int st = check_rows(n->P, n->M, n->hidden);
  if (st != COMPASS_OK) return st;
  st = check_dtype(n->dtype, true);
  if (st == COMPASS_OK) st = check_dtype(n->param_dtype, true);
  if (st != COMPASS_OK) return st;
  return n->eps >= 0.f ? COMPASS_OK : COMPASS_ERR_INVALID_ARG;      // (NaN is refused too)
}

// Rows of whole 16-byte vectors; with pointers on 16-byte boundaries they are accessed as such.
bool whole_vectors(const compass_norm* n) { return n->hidden % (n->dtype == COMPASS_DTYPE_FP32 ? 4 : 8) == 0; }

constexpr int kSms = 148;           // blocks are counted for a B200; fewer SMs only take them in turns
constexpr int64_t kWidest = 8192;   // elements of a row that stay in the registers of a block
// Row ranges of the wide form's column sums: more of them are more threads, and more partial sums to read back.  Backward, us,
// with 16, 32, 64, 128: 64 x 32768 BF16: 23.6, 25.5, 30.4, 30.4; 512 x 16384: 54.3, 51.8, 51.7, 54.0; 4096 x 12288: 301, 294,
// 263, 260, in FP32 312, 304, 275, 272; 16384 x 8200 BF16: 994, 818, 763, 720.
constexpr int kWideParts = 64;

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

template <typename T, int V, int NVT, int kThreads, int kTpr, bool kKeep, bool kResidual>
int run_forward(const NormParams& p, cudaStream_t stream) {
  constexpr size_t smem = RowRing<T, V, NVT, kResidual ? 2 : 1, kThreads>::kSmemBytes;
  constexpr int tpr = kTpr;
  auto kernel = norm_forward_kernel<T, V, NVT, kThreads, kTpr, kKeep, kResidual>;
  static std::atomic<uint64_t> allowed{0};
  const int st = allow_smem(reinterpret_cast<const void*>(kernel), smem, &allowed);
  if (st != COMPASS_OK) return st;
  // few rows: a block each, for the shortest way through; else blocks of several that walk the rows (8 rows of 4096: 3.5 us
  // with a block each, 4.2 with shared ones)
  const int groups = p.M <= kSms || tpr * 2 > kThreads ? 1 : rows_per_block(tpr, kThreads);
  const int64_t need = ceil_div(p.M, groups), most = smem ? kSms : kSms * (kThreads / (tpr * groups));
  return launch(kernel, need < most ? need : most, tpr * groups, smem, stream, false, p);
}

// Up to 8192 elements a row: gamma and beta in registers.  Up to 16384: 16 elements per thread.
template <typename T, int V, bool kResidual>
int pick_forward(const NormParams& p, cudaStream_t stream) {
  const int64_t H = p.hidden;
  constexpr int E = kElems<T, V>, kThreads = int(kWidest) / E;
  if (H > kWidest) return run_forward<T, V, 16 / V, 1024, 1024, false, kResidual>(p, stream);
  return with_tpr<kThreads>(threads_per_row(H, E), [&](auto tpr) {
    return run_forward<T, V, E / V, kThreads, decltype(tpr)::value, true, kResidual>(p, stream);
  });
}
template <typename T, int V>
int pick_forward(const NormParams& p, cudaStream_t stream) {
  return p.has_residual ? pick_forward<T, V, true>(p, stream) : pick_forward<T, V, false>(p, stream);
}

template <typename T>
int forward_of(const NormParams& p, bool vec, cudaStream_t stream) {
  if (p.hidden > 2 * kWidest) {
    return vec ? launch(norm_forward_wide_kernel<T, 16 / int(sizeof(T))>, p.M, 1024, 0, stream, false, p)
               : launch(norm_forward_wide_kernel<T, 1>, p.M, 1024, 0, stream, false, p);
  }
  return vec ? pick_forward<T, 16 / int(sizeof(T))>(p, stream) : pick_forward<T, 1>(p, stream);
}

template <typename T, int V, int kThreads, int kTpr, bool kDsum>
int run_backward(const NormParams& p, const BackwardPlan& b, cudaStream_t stream) {
  constexpr int NVT = kElems<T, V> / V;
  constexpr size_t ring = RowRing<T, V, NVT, kDsum ? 3 : 2, kThreads>::kSmemBytes + size_t(kElems<T, V>) * kThreads * 4;
  auto kernel = norm_backward_kernel<T, V, NVT, kThreads, kTpr, kDsum>;
  constexpr size_t sums = size_t(kThreads) * kElems<T, V> * 4;      // [groups][hidden] at most
  constexpr size_t smem = ring > sums ? ring : sums;
  static std::atomic<uint64_t> allowed{0};
  const int st = allow_smem(reinterpret_cast<const void*>(kernel), smem, &allowed);
  if (st != COMPASS_OK) return st;
  return launch(kernel, b.n_partial, b.tpr * b.groups, smem, stream, false, p);
}
template <typename T, int V, int kThreads, int kTpr>
int run_backward(const NormParams& p, const BackwardPlan& b, cudaStream_t stream) {
  return p.has_dsum ? run_backward<T, V, kThreads, kTpr, true>(p, b, stream) : run_backward<T, V, kThreads, kTpr, false>(p, b, stream);
}
template <typename T, int V>
int pick_backward(const NormParams& p, const BackwardPlan& b, cudaStream_t stream) {
  if constexpr (V != 8) {
    if (b.tpr > 512) return run_backward<T, V, 1024, 1024>(p, b, stream);
  }
  return with_tpr<512>(b.tpr, [&](auto tpr) { return run_backward<T, V, 512, decltype(tpr)::value>(p, b, stream); });
}

template <typename T>
int backward_of(const NormParams& p, const BackwardPlan& b, bool vec, cudaStream_t stream) {
  if (b.wide) {
    int st = launch(norm_backward_rows_kernel<T>, p.M, 1024, 0, stream, false, p);
    if (st != COMPASS_OK) return st;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ceil_div(p.hidden, 256)), unsigned(b.n_partial));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, norm_backward_columns_kernel<T>, p);
    count_kernel_launch();
    return e == cudaSuccess ? COMPASS_OK : record_cuda_error(e);
  }
  return vec ? pick_backward<T, 16 / int(sizeof(T))>(p, b, stream) : pick_backward<T, 1>(p, b, stream);
}

}  // namespace

int allow_smem(const void* kernel, size_t bytes, std::atomic<uint64_t>* done) {
  if (bytes <= 48 * 1024) return COMPASS_OK;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return record_cuda_error(e);
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev < 64 && (done->load(std::memory_order_acquire) & bit)) return COMPASS_OK;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes));
  if (e != cudaSuccess) return record_cuda_error(e);
  if (dev < 64) done->fetch_or(bit, std::memory_order_release);
  return COMPASS_OK;
}

int sm_count(int* out) {
  constexpr int kMaxDevices = 64;
  static int counts[kMaxDevices] = {};
  static std::mutex mu;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return record_cuda_error(e);
  if (dev < 0 || dev >= kMaxDevices) return COMPASS_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(mu);
  if (counts[dev] == 0) {
    e = cudaDeviceGetAttribute(&counts[dev], cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return record_cuda_error(e);
  }
  *out = counts[dev];
  return COMPASS_OK;
}

}  // namespace compass

using namespace compass;

extern "C" int compass_layer_norm(const compass_norm* n, const void* const* X, const void* const* residual, const void* gamma,
                                  const void* beta, void* const* summed, void* const* Y, float* mean, float* rstd, void* stream) {
  int st = check_norm(n);
  if (st != COMPASS_OK) return st;
  if ((residual == nullptr) != (summed == nullptr)) return COMPASS_ERR_INVALID_ARG;
  NormParams p = {};
  const size_t element = dtype_size(n->dtype), param = dtype_size(n->param_dtype);
  bool whole = whole_vectors(n) && is_aligned(gamma, 16) && is_aligned(beta, 16);
  st = fill_shards(X, n->P, n->M, &p.x, element, &whole);
  if (st == COMPASS_OK) st = fill_shards(Y, n->P, n->M, &p.y, element, &whole);
  if (st == COMPASS_OK && residual) st = fill_shards(residual, n->P, n->M, &p.residual, element, &whole);
  if (st == COMPASS_OK && summed) st = fill_shards(summed, n->P, n->M, &p.summed, element, &whole);
  if (st != COMPASS_OK) return st;
  if (!is_aligned(gamma, param) || !is_aligned(beta, param) || !is_aligned(mean, 4) || !is_aligned(rstd, 4)) return COMPASS_ERR_ALIGNMENT;
  if (n->M == 0) return COMPASS_OK;
  p.gamma = gamma;
  p.beta = beta;
  p.mean = mean;
  p.rstd = rstd;
  p.hidden = n->hidden;
  p.M = uint32_t(n->M);
  p.has_residual = residual != nullptr;
  p.param_fp32 = n->param_dtype == COMPASS_DTYPE_FP32;
  p.eps = n->eps;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return n->dtype == COMPASS_DTYPE_FP32 ? forward_of<float>(p, whole, s) : forward_of<__nv_bfloat16>(p, whole, s);
}

// Workspace: the partial column sums, then (wide rows) two sums per row.
extern "C" int compass_layer_norm_workspace_bytes(const compass_norm* n, size_t* bytes) {
  if (bytes == nullptr) return COMPASS_ERR_INVALID_ARG;
  const int st = check_norm(n);
  if (st != COMPASS_OK) return st;
  // (whether the pointers will be on 16-byte boundaries is not known yet)
  const BackwardPlan a = backward_plan(n, false), b = backward_plan(n, whole_vectors(n));
  const int most = a.n_partial > b.n_partial ? a.n_partial : b.n_partial;
  *bytes = 256 + round_up(size_t(2 * most) * size_t(n->hidden) * 4, 256) + (b.wide ? size_t(n->M) * 8 : 0);
  return COMPASS_OK;
}

extern "C" int compass_layer_norm_backward(const compass_norm* n, const void* const* dY, const void* const* X, const void* gamma,
                                           const float* mean, const float* rstd, const void* const* dsum, void* const* dX,
                                           void* dgamma, void* dbeta, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  int st = compass_layer_norm_workspace_bytes(n, &need);
  if (st != COMPASS_OK) return st;
  NormParams p = {};
  const size_t element = dtype_size(n->dtype), param = dtype_size(n->param_dtype);
  bool whole = whole_vectors(n) && is_aligned(gamma, 16);
  st = fill_shards(dY, n->P, n->M, &p.dy, element, &whole);
  if (st == COMPASS_OK) st = fill_shards(X, n->P, n->M, &p.x, element, &whole);
  if (st == COMPASS_OK) st = fill_shards(dX, n->P, n->M, &p.dx, element, &whole);
  if (st == COMPASS_OK && dsum) st = fill_shards(dsum, n->P, n->M, &p.dsum, element, &whole);
  if (st != COMPASS_OK) return st;
  if (n->M > 0 && (mean == nullptr || rstd == nullptr)) return COMPASS_ERR_INVALID_ARG;
  if (!is_aligned(gamma, param) || !is_aligned(dgamma, param) || !is_aligned(dbeta, param) || !is_aligned(mean, 4) || !is_aligned(rstd, 4))
    return COMPASS_ERR_ALIGNMENT;
  st = check_workspace(ws, ws_bytes, need);
  if (st != COMPASS_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (n->M == 0) {
    for (void* g : {dgamma, dbeta})
      if (g) {
        const cudaError_t e = cudaMemsetAsync(g, 0, size_t(n->hidden) * dtype_size(n->param_dtype), s);
        if (e != cudaSuccess) return record_cuda_error(e);
      }
    return COMPASS_OK;
  }
  const BackwardPlan b = backward_plan(n, whole);
  p.gamma = gamma;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.hidden = n->hidden;
  p.M = uint32_t(n->M);
  p.has_dsum = dsum != nullptr;
  p.param_fp32 = n->param_dtype == COMPASS_DTYPE_FP32;
  p.n_partial = b.n_partial;
  p.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + 256);
  p.row_sums = p.partial + round_up(size_t(2 * b.n_partial) * size_t(n->hidden) * 4, 256) / 4;
  st = n->dtype == COMPASS_DTYPE_FP32 ? backward_of<float>(p, b, whole, s) : backward_of<__nv_bfloat16>(p, b, whole, s);
  if (st != COMPASS_OK || (dgamma == nullptr && dbeta == nullptr)) return st;
  const int64_t grid = 2 * ceil_div(n->hidden, 32);
  if (n->param_dtype == COMPASS_DTYPE_FP32)
    return launch(norm_reduce_kernel<float>, grid, 32 * kReduceWays, 0, s, true, p, static_cast<float*>(dgamma), static_cast<float*>(dbeta));
  return launch(norm_reduce_kernel<__nv_bfloat16>, grid, 32 * kReduceWays, 0, s, true, p, static_cast<__nv_bfloat16*>(dgamma),
                static_cast<__nv_bfloat16*>(dbeta));
}
