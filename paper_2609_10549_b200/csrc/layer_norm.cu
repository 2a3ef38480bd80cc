// Layer norm, forward (with the residual sum of a block) and backward.
//
// Both passes are bound by HBM: forward reads X (and the residual) and writes Y
// (and the sum), backward reads dY and X (and the gradient of the residual path)
// and writes dX.  A row is read once into registers, where its statistics are
// taken from the values themselves (the variance from the centred ones), so no
// element travels twice.
#include <mutex>

#include "row_ops.cuh"

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
  int32_t tpr;                           // threads per row, a multiple of 32
  int32_t n_partial;
};

// V parameters (gamma or beta) from element c on; `none` where the pointer is NULL.
template <int V>
__device__ __forceinline__ void load_param(float (&out)[V], const void* p, bool fp32, int64_t c, float none) {
  if (p == nullptr) {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = none;
  } else if (fp32) {
    const float* q = static_cast<const float*>(p) + c;
    if constexpr (V == 8) {
      const float4 a = *reinterpret_cast<const float4*>(q), b = *reinterpret_cast<const float4*>(q + 4);
      out[0] = a.x, out[1] = a.y, out[2] = a.z, out[3] = a.w;
      out[4] = b.x, out[5] = b.y, out[6] = b.z, out[7] = b.w;
    } else {
      load_vec(out, q);
    }
  } else {
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p) + c;
    if constexpr (V == 4) {
      const uint2 a = *reinterpret_cast<const uint2*>(q);
      out[0] = __uint_as_float(a.x << 16), out[1] = __uint_as_float(a.x & 0xFFFF0000u);
      out[2] = __uint_as_float(a.y << 16), out[3] = __uint_as_float(a.y & 0xFFFF0000u);
    } else {
      load_vec(out, q);
    }
  }
}

// Sum of two values over the `tpr` threads of a row; every thread gets it.  `red`: two floats per warp of the block, a
// buffer that no earlier call since the last barrier used.  All threads of the block take part.
__device__ __forceinline__ float2 row_sum(float a, float b, int tpr, float2* red) {
  a = warp_sum(a);
  b = warp_sum(b);
  if (tpr == 32) return make_float2(a, b);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) red[warp] = make_float2(a, b);
  __syncthreads();
  const int n = tpr >> 5, first = warp / n * n;
  const float2 v = lane < n ? red[first + lane] : make_float2(0.f, 0.f);
  return make_float2(warp_sum(v.x), warp_sum(v.y));
}

// ---- forward -------------------------------------------------------------------
// One row per group of `tpr` threads, NVT vectors of V elements per thread, all in registers.
template <typename T, int V, int NVT>
__global__ void __launch_bounds__(1024) norm_forward_kernel(const __grid_constant__ NormParams p) {
  __shared__ float2 red[2][32];
  const int t = threadIdx.x % p.tpr;
  const uint32_t row = uint32_t(blockIdx.x) * (blockDim.x / p.tpr) + threadIdx.x / p.tpr;
  const bool live = row < p.M;
  const int64_t H = p.hidden;
  float h[NVT][V];
  float sum = 0.f;
  if (live) {
    const T* x = p.x.row<T>(row, H);
    const T* r = p.has_residual ? p.residual.row<T>(row, H) : nullptr;
    T* s = p.has_residual ? p.summed.row<T>(row, H) : nullptr;
    Raw<T, V> xr[NVT], rr[NVT];
#pragma unroll
    for (int i = 0; i < NVT; ++i) {
      const int64_t c = int64_t(i * p.tpr + t) * V;
      xr[i].zero();
      rr[i].zero();
      if (c < H) {
        xr[i].load(x + c);
        if (r) rr[i].load(r + c);
      }
    }
#pragma unroll
    for (int i = 0; i < NVT; ++i) {
      const int64_t c = int64_t(i * p.tpr + t) * V;
      xr[i].get(h[i]);
      if (r) {
        float b[V];
        rr[i].get(b);
        // what is stored is normalised, so that the backward pass, which reads it, sees the same values
#pragma unroll
        for (int j = 0; j < V; ++j) h[i][j] = round_to<T>(h[i][j] + b[j]);
        if (c < H) store_vec(s + c, h[i]);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sum += h[i][j];
    }
  }
  const float inv = 1.0f / float(H);
  const float mean = row_sum(sum, 0.f, p.tpr, red[0]).x * inv;
  float sq = 0.f;
  if (live) {
#pragma unroll
    for (int i = 0; i < NVT; ++i)
      if (int64_t(i * p.tpr + t) * V < H) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          h[i][j] -= mean;
          sq = fmaf(h[i][j], h[i][j], sq);
        }
      }
  }
  const float var = row_sum(sq, 0.f, p.tpr, red[1]).x * inv;
  const float rstd = 1.0f / sqrtf(var + p.eps);
  if (!live) return;
  T* y = p.y.row<T>(row, H);
#pragma unroll
  for (int i = 0; i < NVT; ++i) {
    const int64_t c = int64_t(i * p.tpr + t) * V;
    if (c < H) {
      float g[V], b[V];
      load_param(g, p.gamma, p.param_fp32, c, 1.f);
      load_param(b, p.beta, p.param_fp32, c, 0.f);
#pragma unroll
      for (int j = 0; j < V; ++j) g[j] = fmaf(h[i][j] * rstd, g[j], b[j]);
      store_vec(y + c, g);
    }
  }
  if (t == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// Rows that do not fit the registers of a block: one block per row, three passes over it (the later ones out of L2).
template <typename T>
__global__ void __launch_bounds__(1024) norm_forward_wide_kernel(const __grid_constant__ NormParams p) {
  __shared__ float2 red[2][32];
  const uint32_t row = blockIdx.x;
  const int64_t H = p.hidden;
  const T* x = p.x.row<T>(row, H);
  const T* r = p.has_residual ? p.residual.row<T>(row, H) : nullptr;
  T* s = p.has_residual ? p.summed.row<T>(row, H) : nullptr;
  float a[1], b[1], sum = 0.f, sq = 0.f;
  for (int64_t c = threadIdx.x; c < H; c += blockDim.x) {
    load_vec(a, x + c);
    if (r) {
      load_vec(b, r + c);
      a[0] = round_to<T>(a[0] + b[0]);
      store_vec(s + c, a);
    }
    sum += a[0];
  }
  const T* h = r ? s : x;       // a thread reads back only what it wrote itself
  const float inv = 1.0f / float(H);
  const float mean = row_sum(sum, 0.f, p.tpr, red[0]).x * inv;
  for (int64_t c = threadIdx.x; c < H; c += blockDim.x) {
    load_vec(a, h + c);
    sq = fmaf(a[0] - mean, a[0] - mean, sq);
  }
  const float rstd = 1.0f / sqrtf(row_sum(sq, 0.f, p.tpr, red[1]).x * inv + p.eps);
  T* y = p.y.row<T>(row, H);
  for (int64_t c = threadIdx.x; c < H; c += blockDim.x) {
    float g[1];
    load_vec(a, h + c);
    load_param(g, p.gamma, p.param_fp32, c, 1.f);
    load_param(b, p.beta, p.param_fp32, c, 0.f);
    a[0] = fmaf((a[0] - mean) * rstd, g[0], b[0]);
    store_vec(y + c, a);
  }
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// ---- backward ------------------------------------------------------------------
// One block per SM walks the rows; a thread keeps its columns' sums of dY * xhat and dY in registers and has the next
// row's loads in flight while it works on this one.  The block's groups add their sums up in shared memory and leave one
// partial row each for norm_reduce_kernel: fixed order, so the bits do not depend on timing.
constexpr int kBackThreads = 512;
constexpr int kBackElems = 16;      // elements of a row per thread

template <typename T, int V, int NVT>
__global__ void __launch_bounds__(kBackThreads, 1) norm_backward_kernel(const __grid_constant__ NormParams p) {
  static_assert(V * NVT <= kBackElems, "");
  __shared__ float2 red[2][32];
  extern __shared__ float sums[];           // [groups][hidden], only with more than one group
  const int groups = blockDim.x / p.tpr, group = threadIdx.x / p.tpr, t = threadIdx.x % p.tpr;
  const int64_t H = p.hidden;
  const float inv = 1.0f / float(H);
  float g[NVT][V], dg[NVT][V], db[NVT][V];
#pragma unroll
  for (int i = 0; i < NVT; ++i) {
    const int64_t c = int64_t(i * p.tpr + t) * V;
    if (c < H) load_param(g[i], p.gamma, p.param_fp32, c, 1.f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (c >= H) g[i][j] = 0.f;
      dg[i][j] = db[i][j] = 0.f;
    }
  }
  Raw<T, V> xr[NVT], yr[NVT], sr[NVT];
  float mean = 0.f, rstd = 0.f;
  auto fetch = [&](uint32_t row) {
    const bool live = row < p.M;
    const T* x = live ? p.x.row<T>(row, H) : nullptr;
    const T* dy = live ? p.dy.row<T>(row, H) : nullptr;
    const T* ds = live && p.has_dsum ? p.dsum.row<T>(row, H) : nullptr;
#pragma unroll
    for (int i = 0; i < NVT; ++i) {
      const int64_t c = int64_t(i * p.tpr + t) * V;
      xr[i].zero();
      yr[i].zero();
      sr[i].zero();
      if (live && c < H) {
        xr[i].load(x + c);
        yr[i].load(dy + c);
        if (ds) sr[i].load(ds + c);
      }
    }
    mean = live ? p.mean[row] : 0.f;
    rstd = live ? p.rstd[row] : 0.f;
  };
  const uint32_t stride = gridDim.x * groups;
  uint32_t row = blockIdx.x * groups + group;
  fetch(row);
  // every group takes the same number of turns: the row sums have barriers in them
  const uint32_t turns = (p.M - blockIdx.x * groups + stride - 1) / stride;
  for (uint32_t turn = 0; turn < turns; ++turn, row += stride) {
    float xh[NVT][V], d[NVT][V], s[NVT][V];
    const float r = rstd, m = mean;
    float c1 = 0.f, c2 = 0.f;
#pragma unroll
    for (int i = 0; i < NVT; ++i) {
      const bool in = int64_t(i * p.tpr + t) * V < H;
      xr[i].get(xh[i]);
      yr[i].get(d[i]);
      sr[i].get(s[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        xh[i][j] = in ? (xh[i][j] - m) * r : 0.f;
        dg[i][j] = fmaf(d[i][j], xh[i][j], dg[i][j]);
        db[i][j] += d[i][j];
        d[i][j] *= g[i][j];
        c1 += d[i][j];
        c2 = fmaf(d[i][j], xh[i][j], c2);
      }
    }
    const bool live = row < p.M;
    fetch(row + stride);
    const float2 c = row_sum(c1, c2, p.tpr, red[turn & 1]);
    if (live) {
      T* dx = p.dx.row<T>(row, H);
#pragma unroll
      for (int i = 0; i < NVT; ++i) {
        const int64_t col = int64_t(i * p.tpr + t) * V;
        if (col < H) {
#pragma unroll
          for (int j = 0; j < V; ++j) d[i][j] = fmaf(r, d[i][j] - c.x * inv - xh[i][j] * (c.y * inv), s[i][j]);
          store_vec(dx + col, d[i]);
        }
      }
    }
  }
  // this block's sums, one array after the other through shared memory
  launch_dependents();
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* out = p.partial + (int64_t(which) * p.n_partial + blockIdx.x) * H;
    if (groups == 1) {
#pragma unroll
      for (int i = 0; i < NVT; ++i) {
        const int64_t c = int64_t(i * p.tpr + t) * V;
        if (c < H) {
#pragma unroll
          for (int j = 0; j < V; ++j) out[c + j] = which ? db[i][j] : dg[i][j];
        }
      }
    } else {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NVT; ++i) {
        const int64_t c = int64_t(i * p.tpr + t) * V;
        if (c < H) {
#pragma unroll
          for (int j = 0; j < V; ++j) sums[group * H + c + j] = which ? db[i][j] : dg[i][j];
        }
      }
      __syncthreads();
      for (int64_t c = threadIdx.x; c < H; c += blockDim.x) {
        float a = 0.f;
        for (int k = 0; k < groups; ++k) a += sums[k * H + c];
        out[c] = a;
      }
    }
  }
}

// Sums over the partial rows, in their order: 32 columns per block, 8 threads a column.
template <typename PT>
__global__ void __launch_bounds__(256) norm_reduce_kernel(const __grid_constant__ NormParams p, PT* dgamma, PT* dbeta) {
  __shared__ float part[8][33];
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int64_t c = int64_t(blockIdx.x >> 1) * 32 + lane;
  PT* out = blockIdx.x & 1 ? dbeta : dgamma;
  if (out == nullptr) return;
  const float* in = p.partial + int64_t(blockIdx.x & 1) * p.n_partial * p.hidden + c;
  float a = 0.f;
  if (c < p.hidden) {
#pragma unroll 4
    for (int r = k; r < p.n_partial; r += 8) a += in[int64_t(r) * p.hidden];
  }
  part[k][lane] = a;
  __syncthreads();
  if (k == 0 && c < p.hidden) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += part[i][lane];
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
  const float2 s = row_sum(c1, c2, p.tpr, red);
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

bool vectorised(const compass_norm* n) { return n->hidden % (n->dtype == COMPASS_DTYPE_FP32 ? 4 : 8) == 0; }

// Threads per row, a multiple of 32, when each holds `elems` elements.
int threads_per_row(int64_t hidden, int elems) { return int(round_up(size_t(ceil_div(hidden, elems)), 32)); }

// The backward pass keeps a row in the registers of at most kBackThreads threads.
constexpr int64_t kBackWidest = int64_t(kBackThreads) * kBackElems;
constexpr int kWideParts = 64;      // row ranges of the wide form's column sums

struct BackwardPlan {
  bool wide;
  int tpr, groups, grid, n_partial;
};
int backward_plan(const compass_norm* n, BackwardPlan* b) {
  int sms = 0;
  const int st = sm_count(&sms);
  if (st != COMPASS_OK) return st;
  b->wide = n->hidden > kBackWidest;
  if (b->wide) {
    b->tpr = 1024;
    b->groups = 1;
    b->n_partial = int(n->M < kWideParts ? n->M : kWideParts);
    b->grid = 0;
    return COMPASS_OK;
  }
  b->tpr = threads_per_row(n->hidden, kBackElems);
  b->groups = kBackThreads / b->tpr;
  const int64_t need = ceil_div(n->M, b->groups);
  b->grid = int(need < sms ? need : sms);
  b->n_partial = b->grid;
  return COMPASS_OK;
}

template <typename T, int V, int NVT>
int run_forward(const NormParams& p, int tpr, cudaStream_t stream) {
  NormParams q = p;
  q.tpr = tpr;
  const int groups = tpr >= 128 ? 1 : 128 / tpr;
  return launch(norm_forward_kernel<T, V, NVT>, ceil_div(p.M, groups), tpr * groups, 0, stream, false, q);
}

// Elements per thread: few where rows are few (latency: more threads a row, shorter chains), else 16 (32 where a row would
// need more than 1024 threads).
template <typename T, int V>
int pick_forward(const NormParams& p, int sms, cudaStream_t stream) {
  const int64_t H = p.hidden;
  constexpr int one = V == 1 ? 4 : V, two = V == 1 ? 16 : 16, four = 32;
  if (int64_t(p.M) <= 2 * sms && H <= one * 1024) return run_forward<T, V, one / V>(p, threads_per_row(H, one), stream);
  if (H <= two * 512) return run_forward<T, V, two / V>(p, threads_per_row(H, two), stream);
  return run_forward<T, V, four / V>(p, threads_per_row(H, four), stream);
}

template <typename T>
int forward_of(const NormParams& p, bool vec, int sms, cudaStream_t stream) {
  if (p.hidden > 32 * 1024) {
    NormParams q = p;
    q.tpr = 1024;
    return launch(norm_forward_wide_kernel<T>, p.M, 1024, 0, stream, false, q);
  }
  return vec ? pick_forward<T, 16 / int(sizeof(T))>(p, sms, stream) : pick_forward<T, 1>(p, sms, stream);
}

template <typename T, int V, int NVT>
int run_backward(const NormParams& p, const BackwardPlan& b, cudaStream_t stream) {
  return launch(norm_backward_kernel<T, V, NVT>, b.grid, b.tpr * b.groups, b.groups > 1 ? size_t(b.groups) * p.hidden * 4 : 0, stream,
                false, p);
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
  constexpr int V = 16 / int(sizeof(T));
  return vec ? run_backward<T, V, kBackElems / V>(p, b, stream) : run_backward<T, 1, kBackElems>(p, b, stream);
}

}  // namespace

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
  st = fill_shards(X, n->P, n->M, &p.x);
  if (st == COMPASS_OK) st = fill_shards(Y, n->P, n->M, &p.y);
  if (st == COMPASS_OK && residual) st = fill_shards(residual, n->P, n->M, &p.residual);
  if (st == COMPASS_OK && summed) st = fill_shards(summed, n->P, n->M, &p.summed);
  if (st != COMPASS_OK) return st;
  if (!is_aligned(gamma, 16) || !is_aligned(beta, 16) || !is_aligned(mean, 4) || !is_aligned(rstd, 4)) return COMPASS_ERR_ALIGNMENT;
  if (n->M == 0) return COMPASS_OK;
  int sms = 0;
  st = sm_count(&sms);
  if (st != COMPASS_OK) return st;
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
  return n->dtype == COMPASS_DTYPE_FP32 ? forward_of<float>(p, vectorised(n), sms, s) : forward_of<__nv_bfloat16>(p, vectorised(n), sms, s);
}

// Workspace: the partial column sums, then (wide rows) two sums per row.
extern "C" int compass_layer_norm_workspace_bytes(const compass_norm* n, size_t* bytes) {
  if (bytes == nullptr) return COMPASS_ERR_INVALID_ARG;
  const int st = check_norm(n);
  if (st != COMPASS_OK) return st;
  // an upper bound that needs no device: a block per SM at most (kWideParts row ranges with wide rows)
  const bool wide = n->hidden > kBackWidest;
  const int64_t parts = wide ? kWideParts : 256;
  const int64_t most = n->M < parts ? n->M : parts;
  *bytes = 256 + round_up(size_t(2 * most) * size_t(n->hidden) * 4, 256) + (wide ? size_t(n->M) * 8 : 0);
  return COMPASS_OK;
}

extern "C" int compass_layer_norm_backward(const compass_norm* n, const void* const* dY, const void* const* X, const void* gamma,
                                           const float* mean, const float* rstd, const void* const* dsum, void* const* dX,
                                           void* dgamma, void* dbeta, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  int st = compass_layer_norm_workspace_bytes(n, &need);
  if (st != COMPASS_OK) return st;
  NormParams p = {};
  st = fill_shards(dY, n->P, n->M, &p.dy);
  if (st == COMPASS_OK) st = fill_shards(X, n->P, n->M, &p.x);
  if (st == COMPASS_OK) st = fill_shards(dX, n->P, n->M, &p.dx);
  if (st == COMPASS_OK && dsum) st = fill_shards(dsum, n->P, n->M, &p.dsum);
  if (st != COMPASS_OK) return st;
  if (n->M > 0 && (mean == nullptr || rstd == nullptr)) return COMPASS_ERR_INVALID_ARG;
  if (!is_aligned(gamma, 16) || !is_aligned(dgamma, 16) || !is_aligned(dbeta, 16) || !is_aligned(mean, 4) || !is_aligned(rstd, 4))
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
  BackwardPlan b;
  st = backward_plan(n, &b);
  if (st != COMPASS_OK) return st;
  if (b.n_partial > 256) return COMPASS_ERR_UNSUPPORTED;
  p.gamma = gamma;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.hidden = n->hidden;
  p.M = uint32_t(n->M);
  p.has_dsum = dsum != nullptr;
  p.param_fp32 = n->param_dtype == COMPASS_DTYPE_FP32;
  p.tpr = b.tpr;
  p.n_partial = b.n_partial;
  p.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + 256);
  p.row_sums = p.partial + round_up(size_t(2 * b.n_partial) * size_t(n->hidden) * 4, 256) / 4;
  st = n->dtype == COMPASS_DTYPE_FP32 ? backward_of<float>(p, b, vectorised(n), s) : backward_of<__nv_bfloat16>(p, b, vectorised(n), s);
  if (st != COMPASS_OK || (dgamma == nullptr && dbeta == nullptr)) return st;
  const int64_t grid = 2 * ceil_div(n->hidden, 32);
  if (n->param_dtype == COMPASS_DTYPE_FP32)
    return launch(norm_reduce_kernel<float>, grid, 256, 0, s, true, p, static_cast<float*>(dgamma), static_cast<float*>(dbeta));
  return launch(norm_reduce_kernel<__nv_bfloat16>, grid, 256, 0, s, true, p, static_cast<__nv_bfloat16*>(dgamma),
                static_cast<__nv_bfloat16*>(dbeta));
}
