// What the embedding, the layer norm and the output-layer loss share: row shards,
// typed vector access, warp sums, argument checks and launches that overlap
// their start with the end of the kernel before them.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>

#include "internal.h"

namespace compass {

// Activations split by rows over the ranks.  A 32-bit division finds the shard: M <= 2^30.
struct RowShards {
  void* ptr[kMaxP];
  uint32_t rows;      // per shard
  template <typename T>
  __device__ __forceinline__ T* row(uint32_t i, int64_t pitch) const {
    const uint32_t r = i / rows;
    return static_cast<T*>(ptr[r]) + int64_t(i - r * rows) * pitch;
  }
};

// V elements of type T as one access (V * sizeof(T) is 16 bytes, or one element).
template <typename T, int V>
struct Vec {
  T v[V];
};

template <int V>
__device__ __forceinline__ void load_vec(float (&out)[V], const float* p) {
  if constexpr (V == 4) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    out[0] = q.x, out[1] = q.y, out[2] = q.z, out[3] = q.w;
  } else {
    static_assert(V == 1, "");
    out[0] = *p;
  }
}
__device__ __forceinline__ void unpack_bf16x8(float (&out)[8], const uint4& q) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    out[2 * i] = __uint_as_float(w[i] << 16);
    out[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
template <int V>
__device__ __forceinline__ void load_vec(float (&out)[V], const __nv_bfloat16* p) {
  if constexpr (V == 8) {
    unpack_bf16x8(out, *reinterpret_cast<const uint4*>(p));
  } else {
    static_assert(V == 1, "");
    out[0] = __bfloat162float(*p);
  }
}
template <int V>
__device__ __forceinline__ void store_vec(float* p, const float (&in)[V]) {
  if constexpr (V == 4) *reinterpret_cast<float4*>(p) = make_float4(in[0], in[1], in[2], in[3]);
  else *p = in[0];
}
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <int V>
__device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float (&in)[V]) {
  if constexpr (V == 8)
    *reinterpret_cast<uint4*>(p) =
        make_uint4(bf16x2_of(in[0], in[1]), bf16x2_of(in[2], in[3]), bf16x2_of(in[4], in[5]), bf16x2_of(in[6], in[7]));
  else *p = __float2bfloat16_rn(in[0]);
}
template <typename T>
__device__ __forceinline__ float round_to(float x) {
  if constexpr (sizeof(T) == 2) return __bfloat162float(__float2bfloat16_rn(x));
  else return x;
}

// Raw 16 bytes (or one element) kept as loaded until they are needed: half the registers for BF16.
template <typename T, int V>
struct Raw {
  uint32_t w[V * sizeof(T) >= 4 ? V * sizeof(T) / 4 : 1];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (V * sizeof(T) == 16) {
      const uint4 q = __ldcs(reinterpret_cast<const uint4*>(p));
      w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    } else if constexpr (sizeof(T) == 4) {
      w[0] = __float_as_uint(__ldcs(reinterpret_cast<const float*>(p)));
    } else {
      w[0] = uint32_t(__ldcs(reinterpret_cast<const unsigned short*>(p)));
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (auto& x : w) x = 0u;
  }
  __device__ __forceinline__ void get(float (&out)[V]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) out[i] = __uint_as_float(w[i]);
    } else if constexpr (V == 1) {
      out[0] = __uint_as_float(w[0] << 16);
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        out[2 * i] = __uint_as_float(w[i] << 16);
        out[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  }
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// The next kernel of the stream may be launched already; it waits before it reads what this one writes.
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- host ----------------------------------------------------------------------

inline bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t dtype_size(int dtype) { return dtype == COMPASS_DTYPE_FP32 ? 4 : 2; }

constexpr int64_t kMaxDim = int64_t(1) << 30;

inline int check_dtype(int dtype, bool fp32) {
  if (dtype == COMPASS_DTYPE_BF16 || (fp32 && dtype == COMPASS_DTYPE_FP32)) return COMPASS_OK;
  return COMPASS_ERR_UNSUPPORTED;
}
inline int check_rows(int P, int64_t M, int64_t hidden) {
  if (P < 1) return COMPASS_ERR_INVALID_ARG;
  if (P > kMaxP) return COMPASS_ERR_UNSUPPORTED;
  if (M < 0 || hidden <= 0 || M % P != 0) return COMPASS_ERR_SHAPE;
  if (M > kMaxDim || hidden > kMaxDim) return COMPASS_ERR_UNSUPPORTED;
  return COMPASS_OK;
}
inline int64_t vocab_shard_rows(int64_t vocab, int P) { return ceil_div(vocab, P); }
inline int64_t rows_of_vocab_shard(int64_t vocab, int P, int r) {
  const int64_t s = vocab_shard_rows(vocab, P);
  const int64_t left = vocab - s * r;
  return left < 0 ? 0 : (left < s ? left : s);
}
// P row shards; with rows == 0 nothing is read and nothing is asked of the pointers.
inline int fill_shards(const void* const* p, int P, int64_t M, RowShards* out) {
  out->rows = uint32_t(M / P);
  if (M == 0) return COMPASS_OK;
  if (p == nullptr) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < P; ++r) {
    if (p[r] == nullptr) return COMPASS_ERR_INVALID_ARG;
    out->ptr[r] = const_cast<void*>(p[r]);
  }
  for (int r = 0; r < P; ++r)
    if (!is_aligned(p[r], 16)) return COMPASS_ERR_ALIGNMENT;
  return COMPASS_OK;
}
inline int check_vocab_shards(const void* const* p, int P, int64_t vocab) {
  if (p == nullptr) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < P; ++r)
    if (p[r] == nullptr && rows_of_vocab_shard(vocab, P, r) > 0) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < P; ++r)
    if (!is_aligned(p[r], 16)) return COMPASS_ERR_ALIGNMENT;
  return COMPASS_OK;
}
inline int check_workspace(const void* ws, size_t have, size_t need) {
  if (ws == nullptr) return COMPASS_ERR_INVALID_ARG;
  if (!is_aligned(ws, 256)) return COMPASS_ERR_ALIGNMENT;
  return have < need ? COMPASS_ERR_BUFFER_TOO_SMALL : COMPASS_OK;
}

// Launch; `overlap`: the kernel begins with wait_for_previous_kernel() and may start while its predecessor ends.
template <typename... Params, typename... Args>
int launch(void (*kernel)(Params...), int64_t grid, int block, size_t smem, cudaStream_t stream, bool overlap, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(grid));
  cfg.blockDim = dim3(unsigned(block));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = overlap ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
  count_kernel_launch();
  return e == cudaSuccess ? COMPASS_OK : record_cuda_error(e);
}

// Streaming multiprocessors of the current device (148 on a B200), looked up once per device.
int sm_count(int* out);

}  // namespace compass
