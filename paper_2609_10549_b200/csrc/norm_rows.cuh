// What the layer norm and the root-mean-square norm share: a row's elements in the registers of the threads that hold it, its
// sums over them, and how many threads a row gets.
#pragma once

#include <type_traits>

#include "row_ops.cuh"

namespace compass {

// Elements of a row per thread: what a row costs every thread (sums over the row, addresses) is shared by this many.  16 where
// they are loaded packed, two to a register; 8 in FP32 and in rows that are not whole vectors.
template <typename T, int V>
constexpr int kElems = V == 8 ? 16 : 8;

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

// Sum of two values over the `tpr` threads of a row; every thread gets it.  `red`: a float2 per warp of the block, a buffer
// that no call since the last but one used.  The rows of a block do not wait for one another: each has a barrier of its own.
__device__ __forceinline__ float2 row_sum(float a, float b, int tpr, float2* red) {
  a = warp_sum(a);
  b = warp_sum(b);
  if (tpr == 32) return make_float2(a, b);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = tpr >> 5, group = warp / n;
  if (lane == 0) red[warp] = make_float2(a, b);
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(tpr) : "memory");
  const float2 v = lane < n ? red[group * n + lane] : make_float2(0.f, 0.f);
  return make_float2(warp_sum(v.x), warp_sum(v.y));
}

__device__ __forceinline__ float row_sum(float a, int tpr, float* red) {
  a = warp_sum(a);
  if (tpr == 32) return a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = tpr >> 5, group = warp / n;
  if (lane == 0) red[warp] = a;
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(tpr) : "memory");
  return warp_sum(lane < n ? red[group * n + lane] : 0.f);
}

// NVT vectors of V elements of type T, a word per 4 bytes, and their values two by two.  (BF16 in rows that are not whole
// vectors: an element a word.)
template <typename T, int V, int NVT>
struct Words {
  static constexpr int kPer = V * int(sizeof(T)) >= 4 ? V * int(sizeof(T)) / 4 : 1;
  static constexpr int kPairs = V * NVT / 2;
  uint32_t w[NVT][kPer];
  __device__ __forceinline__ F2 pair(int k) const {
    if constexpr (V == 8) {
      const uint32_t q = w[k / 4][k % 4];
      return f2(__uint_as_float(q << 16), __uint_as_float(q & 0xFFFF0000u));
    } else if constexpr (sizeof(T) == 2) {
      return f2(__uint_as_float(w[2 * k][0] << 16), __uint_as_float(w[2 * k + 1][0] << 16));
    } else {
      return f2(__uint_as_float(w[2 * k / V][2 * k % V]), __uint_as_float(w[(2 * k + 1) / V][(2 * k + 1) % V]));
    }
  }
  // a + b, rounded to T
  __device__ __forceinline__ void add(const Words& o) {
#pragma unroll
    for (int i = 0; i < NVT; ++i)
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        if constexpr (sizeof(T) == 2) asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(w[i][k]) : "r"(w[i][k]), "r"(o.w[i][k]));
        else w[i][k] = __float_as_uint(__uint_as_float(w[i][k]) + __uint_as_float(o.w[i][k]));
      }
  }
  __device__ __forceinline__ void set(const F2 (&v)[kPairs]) {
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const float2 q = of(v[k]);
      if constexpr (V == 8) {
        w[k / 4][k % 4] = bf16x2_of(q.x, q.y);
      } else if constexpr (sizeof(T) == 2) {
        w[2 * k][0] = bf16x2_of(q.x, 0.f);
        w[2 * k + 1][0] = bf16x2_of(q.y, 0.f);
      } else {
        w[2 * k / V][2 * k % V] = __float_as_uint(q.x);
        w[(2 * k + 1) / V][(2 * k + 1) % V] = __float_as_uint(q.y);
      }
    }
  }
  __device__ __forceinline__ void store(T* row, int tpr, int t, int H) const {
#pragma unroll
    for (int i = 0; i < NVT; ++i) {
      const int c = (i * tpr + t) * V;
      if (c < H) {
        if constexpr (kPer == 4) *reinterpret_cast<uint4*>(row + c) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
        else if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(row + c) = w[i][0];
        else *reinterpret_cast<unsigned short*>(row + c) = static_cast<unsigned short>(w[i][0]);
      }
    }
  }
};
// A row's gamma or beta, two by two.
template <int V, int NVT>
__device__ __forceinline__ void load_params(F2 (&out)[V * NVT / 2], const void* p, bool fp32, float none, int tpr, int t, int H) {
  float v[NVT][V];
#pragma unroll
  for (int i = 0; i < NVT; ++i) {
    const int c = (i * tpr + t) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) v[i][j] = 0.f;
    if (c < H) load_param(v[i], p, fp32, c, none);
  }
#pragma unroll
  for (int k = 0; k < V * NVT / 2; ++k) out[k] = f2(v[2 * k / V][2 * k % V], v[(2 * k + 1) / V][(2 * k + 1) % V]);
}

// ---- host ----------------------------------------------------------------------

// Threads per row when each holds `elems` elements: a power of two from 32 on, which the kernels are compiled for (their
// addresses are then a register and a constant; with an odd hidden size, an element per access, that is half their time).
inline int threads_per_row(int64_t hidden, int elems) {
  int tpr = 32;
  while (int64_t(tpr) * elems < hidden) tpr *= 2;
  return tpr;
}
// Rows a block of at most `threads` works on side by side (each has a named barrier, but for single warps: 8 at most).
inline int rows_per_block(int tpr, int threads) { return tpr == 32 || tpr * 8 >= threads ? threads / tpr : 8; }
// f(threads per row as a constant), up to kMost of them.
template <int kMost, typename F>
inline int with_tpr(int tpr, F f) {
  switch (tpr) {
    case 32: return f(std::integral_constant<int, 32>{});
    case 64: return f(std::integral_constant<int, 64>{});
    case 128: return f(std::integral_constant<int, 128>{});
    case 256: return f(std::integral_constant<int, 256>{});
    case 512: return f(std::integral_constant<int, 512>{});
    default: return f(std::integral_constant<int, kMost>{});
  }
}

}  // namespace compass
