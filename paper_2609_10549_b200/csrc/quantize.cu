// Tensors kept in 8 bits: E4M3 or E5M2 values with a power of two for each run of 128 columns of a row (activations), or for
// each block of 128 x 128 (weights, whose transpose then has the same scales), and back.
//
// Bound by HBM: a BF16 element is 2 bytes read and 1 + 1/128 written, or the reverse.  A thread takes 16 elements, so that 8
// neighbouring lanes hold a run and its maximum is three shuffles away; two (four, back) such units a thread are in flight.
// 16384 x 8192 in BF16: 64 us there (6.3 TB/s), 61 back (6.6), 72 by blocks of 128 x 128.
#include "row_ops.cuh"
#include "scaled8.cuh"

namespace compass {

namespace {

constexpr int kThreads = 256;
constexpr int kUnit = 16;            // elements of a thread's unit: 8 units are a run of 128
constexpr int kItems = 4;            // units of a thread that are in flight together
constexpr int kRowItems = 2;         // the same where runs are brought to 8 bits: fewer registers, more blocks (16384 x 8192 BF16, 2, 4, 8: 64, 77, 71 us)
constexpr int kChunkUnits = 1024;    // units of a row that one block takes at most

struct QuantParams {
  RowShards x, q, s;       // full precision, 8 bits, scales
  int64_t cols;
  int64_t blocks;          // scales per row
  uint32_t M;
  FastDiv units;           // of a row (of 16 columns, whole runs) that a block takes
  FastDiv chunks;          // blocks side by side along a row
  uint32_t rows;           // that a block takes
  int32_t wide;            // the full-precision tensors lie on 32-byte boundaries
  FastDiv block_rows;      // 128 x 128 blocks: of them along a shard's rows, and along its columns
  FastDiv block_cols;
};

// 16 elements as they lie in memory.
template <typename T>
struct Unit {
  static constexpr int kWords = kUnit * int(sizeof(T)) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p, bool wide) {
#pragma unroll
    for (int i = 0; i < kWords; i += 8) {
      const uint32_t* a = reinterpret_cast<const uint32_t*>(p) + i;
      if (wide) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]), "=r"(w[i + 6]), "=r"(w[i + 7])
                     : "l"(a));
      } else {
        const uint4 b = *reinterpret_cast<const uint4*>(a), c = *reinterpret_cast<const uint4*>(a + 4);
        w[i] = b.x, w[i + 1] = b.y, w[i + 2] = b.z, w[i + 3] = b.w;
        w[i + 4] = c.x, w[i + 5] = c.y, w[i + 6] = c.z, w[i + 7] = c.w;
      }
    }
  }
  __device__ __forceinline__ void store(T* p, bool wide) const {
#pragma unroll
    for (int i = 0; i < kWords; i += 8) {
      uint32_t* a = reinterpret_cast<uint32_t*>(p) + i;
      if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(a), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]),
                     "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7])
                     : "memory");
      } else {
        reinterpret_cast<uint4*>(a)[0] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        reinterpret_cast<uint4*>(a)[1] = make_uint4(w[i + 4], w[i + 5], w[i + 6], w[i + 7]);
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ void get(float (&x)[kUnit]) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[i] = __uint_as_float(w[i]);
      } else {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  }
  __device__ __forceinline__ void set(const float (&x)[kUnit]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
      else w[i] = bf16x2_of(x[2 * i], x[2 * i + 1]);
    }
  }
};

// Largest |x|, NaN left out.
__device__ __forceinline__ float largest(const float (&x)[kUnit]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < kUnit; ++i) m = fmaxf(m, fabsf(x[i]));
  return m;
}
__device__ __forceinline__ void infinite_to_nan(float (&x)[kUnit]) {
#pragma unroll
  for (int i = 0; i < kUnit; ++i) x[i] = fabsf(x[i]) < INFINITY ? x[i] : __uint_as_float(0x7FC00000u);
}
__device__ __forceinline__ float largest_of_8(float m) {
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}
template <int kFormat>
__device__ __forceinline__ uint4 pack16(const float (&x)[kUnit], float f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack8x4<kFormat>(x[4 * i] * f, x[4 * i + 1] * f, x[4 * i + 2] * f, x[4 * i + 3] * f);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Where a unit of a block lies.
struct Place {
  RowAt at;          // row (offset 0 of it)
  uint32_t row;
  int64_t col;
  bool live;
};
__device__ __forceinline__ Place place_of(const QuantParams& p, uint32_t i) {
  const uint32_t group = p.chunks.div(blockIdx.x), chunk = blockIdx.x - group * p.chunks.d;
  const uint32_t r = p.units.div(i);
  Place q;
  q.row = group * p.rows + r;
  q.col = (int64_t(chunk) * p.units.d + (i - r * p.units.d)) * kUnit;
  q.live = r < p.rows && q.row < p.M && q.col < p.cols;
  return q;
}

template <typename T, int kFormat>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const __grid_constant__ QuantParams p) {
  launch_dependents();
  wait_for_previous_kernel();
  const uint32_t n = p.rows * p.units.d;
  for (uint32_t i0 = threadIdx.x; i0 < n + threadIdx.x; i0 += kThreads * kRowItems) {      // (the same number of turns for all lanes)
    Unit<T> u[kRowItems];
    Place at[kRowItems];
#pragma unroll
    for (int k = 0; k < kRowItems; ++k) {
      at[k] = place_of(p, i0 + k * kThreads);
      if (at[k].live) u[k].load(p.x.row<T>(at[k].row, p.cols) + at[k].col, p.wide);
      else u[k].zero();
    }
#pragma unroll
    for (int k = 0; k < kRowItems; ++k) {
      float x[kUnit];
      u[k].get(x);
      float top = largest_of_8(largest(x));
      if (__any_sync(0xffffffffu, !(top < INFINITY))) {
        infinite_to_nan(x);
        top = largest_of_8(largest(x));
      }
      const uint32_t b = scale_byte_of<kFormat>(__float_as_uint(top));
      if (at[k].live) {
        *reinterpret_cast<uint4*>(p.q.row<uint8_t>(at[k].row, p.cols) + at[k].col) = pack16<kFormat>(x, inverse_scale(b));
        if ((threadIdx.x & 7) == 0) p.s.row<uint8_t>(at[k].row, p.blocks)[at[k].col >> 7] = uint8_t(b);
      }
    }
  }
}

constexpr int kBlockItems = 2, kBlockThreads = 1024 / kBlockItems;
// A block of 128 x 128, two units a thread.
template <typename T, int kFormat>
__global__ void __launch_bounds__(kBlockThreads) quantize_blocks_kernel(const __grid_constant__ QuantParams p) {
  __shared__ float tops[2][kBlockThreads / 32];
  launch_dependents();
  wait_for_previous_kernel();
  const uint32_t line = p.block_cols.div(blockIdx.x), col = blockIdx.x - line * p.block_cols.d;
  const uint32_t shard = p.block_rows.div(line), row0 = (line - shard * p.block_rows.d) * 128;
  const T* x = static_cast<const T*>(p.x.ptr[shard]);
  uint8_t* q = static_cast<uint8_t*>(p.q.ptr[shard]);
  const int64_t c = int64_t(col) * 128 + (threadIdx.x & 7) * kUnit;
  Unit<T> u[kBlockItems];
  float top = 0.f;
  auto row_of = [&](int k) { return row0 + k * (kBlockThreads / 8) + (threadIdx.x >> 3); };
#pragma unroll
  for (int k = 0; k < kBlockItems; ++k) {
    if (row_of(k) < p.x.rows.d && c < p.cols) u[k].load(x + int64_t(row_of(k)) * p.cols + c, p.wide);
    else u[k].zero();
  }
  auto block_top = [&](float m, float* part) {
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
    m = largest_of_8(fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16)));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBlockThreads / 32; ++i) m = fmaxf(m, part[i]);
    return m;
  };
  float y[kUnit];
#pragma unroll
  for (int k = 0; k < kBlockItems; ++k) {
    u[k].get(y);
    top = fmaxf(top, largest(y));
  }
  top = block_top(top, tops[0]);
  const bool infinite = !(top < INFINITY);      // (the same for all)
  if (infinite) {
    top = 0.f;
#pragma unroll
    for (int k = 0; k < kBlockItems; ++k) {
      u[k].get(y);
      infinite_to_nan(y);
      top = fmaxf(top, largest(y));
    }
    top = block_top(top, tops[1]);
  }
  const uint32_t b = scale_byte_of<kFormat>(__float_as_uint(top));
#pragma unroll
  for (int k = 0; k < kBlockItems; ++k) {
    u[k].get(y);
    if (infinite) infinite_to_nan(y);
    if (row_of(k) < p.x.rows.d && c < p.cols)
      *reinterpret_cast<uint4*>(q + int64_t(row_of(k)) * p.cols + c) = pack16<kFormat>(y, inverse_scale(b));
  }
  if (threadIdx.x == 0) static_cast<uint8_t*>(p.s.ptr[shard])[int64_t(row0 >> 7) * p.blocks + col] = uint8_t(b);
}

template <typename T, int kFormat>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const __grid_constant__ QuantParams p) {
  launch_dependents();
  wait_for_previous_kernel();
  const uint32_t n = p.rows * p.units.d;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kThreads * kItems) {
    uint4 w[kItems];
    uint32_t b[kItems];
    Place at[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      at[k] = place_of(p, i0 + k * kThreads);
      if (!at[k].live) continue;
      w[k] = *reinterpret_cast<const uint4*>(p.q.row<uint8_t>(at[k].row, p.cols) + at[k].col);
      // (128 x 128 blocks: the row of scales goes by the row within the shard)
      if (p.block_rows.d == 0) {
        b[k] = p.s.row<uint8_t>(at[k].row, p.blocks)[at[k].col >> 7];
      } else {
        const uint32_t shard = p.x.rows.div(at[k].row), r = at[k].row - shard * p.x.rows.d;
        b[k] = static_cast<const uint8_t*>(p.s.ptr[shard])[int64_t(r >> 7) * p.blocks + (at[k].col >> 7)];
      }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (!at[k].live) continue;
      const float f = scale_value(b[k]);
      const uint32_t v[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
      float x[kUnit];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 lo = unpack8x2<kFormat>(v[i]), hi = unpack8x2<kFormat>(v[i] >> 16);
        x[4 * i] = lo.x * f, x[4 * i + 1] = lo.y * f, x[4 * i + 2] = hi.x * f, x[4 * i + 3] = hi.y * f;
      }
      Unit<T> u;
      u.set(x);
      u.store(p.x.row<T>(at[k].row, p.cols) + at[k].col, p.wide);
    }
  }
}

// ---- host ----------------------------------------------------------------------

int check_quant(const compass_quant* q) {
  if (q == nullptr) return COMPASS_ERR_INVALID_ARG;
  int st = check_rows(q->P, q->M, q->cols);
  if (st == COMPASS_OK) st = check_dtype(q->dtype, true);
  if (st != COMPASS_OK) return st;
  if (format_of(q->format) < 0) return COMPASS_ERR_UNSUPPORTED;
  if (q->block_rows != 1 && q->block_rows != 128) return COMPASS_ERR_INVALID_ARG;
  return q->cols % 16 == 0 ? COMPASS_OK : COMPASS_ERR_ALIGNMENT;
}

int fill(const compass_quant* q, const void* const* X, const void* const* Q, const void* const* S, QuantParams* p) {
  int st = check_quant(q);
  if (st == COMPASS_OK) st = fill_shards(X, q->P, q->M, &p->x);
  if (st == COMPASS_OK) st = fill_shards(Q, q->P, q->M, &p->q);
  if (st == COMPASS_OK) st = fill_shards(S, q->P, q->M, &p->s, 1);
  if (st != COMPASS_OK) return st;
  p->wide = 1;
  for (int r = 0; r < q->P && q->M > 0; ++r)
    if (!is_aligned(X[r], 32)) p->wide = 0;
  p->cols = q->cols;
  p->blocks = scale_blocks(q->cols);
  p->M = uint32_t(q->M);
  // a block takes about kChunkUnits units: several short rows, or a piece of a long one
  const int64_t units = p->blocks * 8, take = units < kChunkUnits ? units : kChunkUnits;
  p->units.set(uint32_t(take));
  p->chunks.set(uint32_t(ceil_div(units, take)));
  p->rows = uint32_t(kChunkUnits / take);
  return COMPASS_OK;
}

template <typename T, int kFormat>
int run_quantize(const compass_quant* q, QuantParams& p, cudaStream_t stream) {
  if (q->block_rows == 128) {
    const int64_t lines = ceil_div(q->M / q->P, 128);
    p.block_rows.set(uint32_t(lines));
    p.block_cols.set(uint32_t(p.blocks));
    return launch(quantize_blocks_kernel<T, kFormat>, q->P * lines * p.blocks, kBlockThreads, 0, stream, true, p);
  }
  return launch(quantize_rows_kernel<T, kFormat>, ceil_div(q->M, p.rows) * p.chunks.d, kThreads, 0, stream, true, p);
}
template <typename T, int kFormat>
int run_dequantize(const compass_quant* q, QuantParams& p, cudaStream_t stream) {
  p.block_rows.d = q->block_rows == 128;
  return launch(dequantize_kernel<T, kFormat>, ceil_div(q->M, p.rows) * p.chunks.d, kThreads, 0, stream, true, p);
}

}  // namespace

}  // namespace compass

using namespace compass;

extern "C" int compass_quantize(const compass_quant* q, const void* const* X, void* const* Q, void* const* scale, void* stream) {
  QuantParams p = {};
  const int st = fill(q, X, Q, scale, &p);
  if (st != COMPASS_OK || q->M == 0) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool e4 = q->format == COMPASS_DTYPE_E4M3;
  if (q->dtype == COMPASS_DTYPE_FP32) return e4 ? run_quantize<float, E4M3>(q, p, s) : run_quantize<float, E5M2>(q, p, s);
  return e4 ? run_quantize<__nv_bfloat16, E4M3>(q, p, s) : run_quantize<__nv_bfloat16, E5M2>(q, p, s);
}

extern "C" int compass_dequantize(const compass_quant* q, const void* const* Q, const void* const* scale, void* const* X, void* stream) {
  QuantParams p = {};
  const int st = fill(q, X, Q, scale, &p);
  if (st != COMPASS_OK || q->M == 0) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool e4 = q->format == COMPASS_DTYPE_E4M3;
  if (q->dtype == COMPASS_DTYPE_FP32) return e4 ? run_dequantize<float, E4M3>(q, p, s) : run_dequantize<float, E5M2>(q, p, s);
  return e4 ? run_dequantize<__nv_bfloat16, E4M3>(q, p, s) : run_dequantize<__nv_bfloat16, E5M2>(q, p, s);
}
