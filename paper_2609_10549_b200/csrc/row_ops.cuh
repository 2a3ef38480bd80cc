// What the embedding, the layer norm and the output-layer loss share: row shards,
// typed vector access, warp sums, argument checks and launches that overlap
// their start with the end of the kernel before them.
#pragma once

#include <atomic>
#include <cstdint>
#include <cuda_bf16.h>

#include "internal.h"

namespace compass {

// Division of n < 2^31 by a divisor that the host knows: (n * mul) >> shift with shift = 31 + ceil(log2 d) and mul =
// floor(2^shift / d) + 1, which is below 2^32 (exact: Granlund and Montgomery's bound).  A quarter of the instructions of a
// division, which rows of a few elements per thread feel.
struct FastDiv {
  uint32_t d, mul, shift;
  __host__ void set(uint32_t divisor) {
    d = divisor;
    uint32_t l = 0;
    while ((uint64_t(1) << l) < d) ++l;
    shift = 31 + l;
    mul = d ? uint32_t((uint64_t(1) << shift) / d + 1) : 0;
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return uint32_t((uint64_t(n) * mul) >> shift); }
};

// Activations split by rows over the ranks (M <= 2^30), `rows` each.
struct RowAt {
  uint32_t shard;
  int64_t offset;      // elements from the shard's start
};
struct RowShards {
  void* ptr[kMaxP];
  FastDiv rows;
  __device__ __forceinline__ RowAt at(uint32_t i, int64_t pitch) const {
    const uint32_t r = rows.div(i);
    return RowAt{r, int64_t(i - r * rows.d) * pitch};
  }
  template <typename T>
  __device__ __forceinline__ T* row(const RowAt& a) const {
    return static_cast<T*>(ptr[a.shard]) + a.offset;
  }
  template <typename T>
  __device__ __forceinline__ T* row(uint32_t i, int64_t pitch) const {
    return row<T>(at(i, pitch));
  }
};

// V elements of a type as one access (16 bytes, or one element), as FP32.
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

// The next rows of kArrays tensors on their way from HBM: every thread copies its own elements to shared memory, kDepth rows
// ahead, and reads back only what it copied, so that no barrier is needed and nothing is held in registers.  Elements of two
// bytes (rows that are not whole vectors) cannot be copied this way: those are loaded when they are taken.
template <typename T, int V, int NVT, int kArrays, int kThreads>
struct RowRing {
  static constexpr int kBytes = V * int(sizeof(T));
  static constexpr bool kAsync = kBytes >= 4;
  static constexpr int kRowBytes = kArrays * NVT * kThreads * kBytes;
  static constexpr int kRoom = 160 * 1024;
  static constexpr int kDepth = !kAsync ? 1 : kRoom / kRowBytes > 8 ? 8 : kRoom / kRowBytes < 1 ? 1 : kRoom / kRowBytes;
  static constexpr size_t kSmemBytes = kAsync ? size_t(kDepth) * kRowBytes : 0;
  uint32_t base;      // this thread's slot 0
  int at = 0;         // oldest row
  const T* src[kArrays] = {};
  __device__ __forceinline__ explicit RowRing(void* smem)
      : base(static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + threadIdx.x * kBytes) {}
  // Row `which` (0 = the oldest) is to come from `p` (elements of this row; null: no row).
  __device__ __forceinline__ void fetch(int which, const T* const (&p)[kArrays], int tpr, int t, int H) {
    if constexpr (kAsync) {
      const int slot = at + which >= kDepth ? at + which - kDepth : at + which;
#pragma unroll
      for (int a = 0; a < kArrays; ++a)
#pragma unroll
        for (int i = 0; i < NVT; ++i) {
          const int c = (i * tpr + t) * V;
          if (p[a] != nullptr && c < H) {
            const uint32_t to = base + ((slot * kArrays + a) * NVT + i) * (kThreads * kBytes);
            if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p[a] + c) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(p[a] + c) : "memory");
          }
        }
      asm volatile("cp.async.commit_group;" ::: "memory");
    } else {
#pragma unroll
      for (int a = 0; a < kArrays; ++a) src[a] = p[a];
    }
  }
  // The oldest row has landed.
  __device__ __forceinline__ void wait() {
    if constexpr (kAsync) asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
  }
  // V elements of it as they are stored (zeros past the row's end): one word per 4 bytes.
  static constexpr int kWords = kBytes >= 4 ? kBytes / 4 : 1;
  __device__ __forceinline__ void take(uint32_t (&w)[kWords], int array, int i, int tpr, int t, int H) const {
    const int c = (i * tpr + t) * V;
#pragma unroll
    for (int k = 0; k < kWords; ++k) w[k] = 0u;
    if (c < H) {
      if constexpr (kAsync) {
        const uint32_t from = base + ((at * kArrays + array) * NVT + i) * (kThreads * kBytes);
        if constexpr (kBytes == 16)
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from) : "memory");
        else
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(from) : "memory");
      } else {
        w[0] = uint32_t(*reinterpret_cast<const unsigned short*>(src[array] + c));
      }
    }
  }
  __device__ __forceinline__ void advance() { at = at + 1 == kDepth ? 0 : at + 1; }
};

// Two FP32 values per instruction (add, mul and fma on pairs).
struct F2 {
  unsigned long long v;
};
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ F2 f2(float a) { return f2(a, a); }
__device__ __forceinline__ float2 of(F2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
  return r;
}
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ float sum_of(F2 a) {
  const float2 q = of(a);
  return q.x + q.y;
}

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
// P row shards; with rows == 0 nothing is read and nothing is asked of the pointers.  They are aligned to `align` bytes at
// least; *whole is cleared where one is not to 16 (then every access is of one element).
inline int fill_shards(const void* const* p, int P, int64_t M, RowShards* out, size_t align = 16, bool* whole = nullptr) {
  out->rows.set(uint32_t(M / P));
  if (M == 0) return COMPASS_OK;
  if (p == nullptr) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < P; ++r) {
    if (p[r] == nullptr) return COMPASS_ERR_INVALID_ARG;
    out->ptr[r] = const_cast<void*>(p[r]);
  }
  for (int r = 0; r < P; ++r) {
    if (!is_aligned(p[r], align)) return COMPASS_ERR_ALIGNMENT;
    if (whole && !is_aligned(p[r], 16)) *whole = false;
  }
  return COMPASS_OK;
}
inline int check_vocab_shards(const void* const* p, int P, int64_t vocab, size_t align = 16, bool* whole = nullptr) {
  if (p == nullptr) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < P; ++r)
    if (p[r] == nullptr && rows_of_vocab_shard(vocab, P, r) > 0) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < P; ++r) {
    if (!is_aligned(p[r], align)) return COMPASS_ERR_ALIGNMENT;
    if (whole && !is_aligned(p[r], 16)) *whole = false;
  }
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

// Lets a kernel have this much dynamic shared memory on the current device; `done`: the devices where it does already.
int allow_smem(const void* kernel, size_t bytes, std::atomic<uint64_t>* done);
// Streaming multiprocessors of the current device (148 on a B200), looked up once per device.
int sm_count(int* out);

}  // namespace compass
