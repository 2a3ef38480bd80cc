// Gradient of a tensor-parallel product's weights from the activations as they were kept, in 8 bits:
//   dW[n][k] (+)= sum_m G[m][n] * 2^s[m][k / 128] * x[m][k]
// The contraction runs over the rows, along which the scales differ, so the tensor cores cannot apply them (they take one scale
// for 32 elements of the contraction): the 8-bit tile is turned into BF16 in shared memory, which holds scale times value
// exactly, and the products are BF16 ones with FP32 sums.  The activations cross HBM and L2 in 8 bits.
//
// Pairs of CTAs, 512 rows (n) x 256 columns (k) a tile as long as they fill whole rounds of the pairs (two accumulators that share
// one converted tile), 256 x 256 for the rest; 64 rows of the contraction a stage.  Both operands lie across the contraction
// (MN-major).  Warp 0 loads G (TMA), warp 18 X, warp 1 issues the products, warps 2..9 are the epilogue, warps 10..17
// convert: four groups of two warps, which take the stages in turn; a thread has its CTA's 128 columns of one row of a stage, so one
// scale.  Rows past a rank's last one are zeros of the tensor maps.
//
// The tensor cores cut off what their FP32 sums cannot hold, a little at each step: up to 2^-23 of the sum so far for 16 rows.  For a
// result in FP32 the sums are therefore 1024 rows long, and added up in FP32, in tensor memory: 256 x 256 tiles whose second accumulator
// keeps the total.  For one in BF16 the same is done with sums of 65536 rows, in which the cut-off stays below 2^-12 of growing sums, an
// eighth of BF16's half step (as one sum each, the shares of 4 million positive rows came out up to 0.6 % too small, where half a step is 0.2 %;
// sums of 65536 rows cost 4096 x 4096 over 131072 rows 4350 us instead of 3880, having no 512 x 256 tiles).
//
// Bound by the tensor cores and the board's power: 4 ranks' 2752 x 4096 over 8192 rows 505 to 515 us in a burst (1.45 PFLOP/s, tensor pipe
// busy 88 %) and 560 to 600 in loops.  In FP32 8192 x 8192 over 8192 rows takes 1060 to 1110 against 790 to 840 us: the products wait for the sums of 1024 rows,
// and tiles of 256 x 256 take shared memory's bandwidth (160 bytes a clock).
#include <mutex>

#include "pipeline.cuh"
#include "row_ops.cuh"
#include "scaled8.cuh"

namespace compass {

using namespace ptx;

namespace {

constexpr int kThreads = 608;
constexpr int kEpiWarps = 8;
constexpr int kConvWarps = 2;                         // of a group
constexpr int kGroups = 4;
constexpr int kRows = 64;                             // of the contraction in a stage
constexpr int kGBytes = 256 * kRows * 2;              // this CTA's 256 (or 128) columns of G: boxes of 64
constexpr int kXBytes = 128 * kRows;                  // its 128 columns of X
constexpr int kCBytes = 128 * kRows * 2;              // the same in BF16: two chunks of 64
constexpr int kChunk = 64 * kRows * 2;
constexpr int kStages = 4;                            // of G and of X in BF16
constexpr int kXStages = 4;
constexpr int kSkew = 3;                              // stages at a 512 x 256 tile's ends in which accumulator 0 runs ahead
// Stages of one sum: of one that goes to FP32, and of one that is rounded to BF16 (65536 rows).
constexpr int kFp32Range = 16, kBf16Range = 1024;
constexpr int kMostSplits = 4;                        // pairs of a cluster
constexpr int kRowGroup = 8;                          // row tiles that go through the columns together

struct GradParams {
  CUtensorMap g[kMaxP];
  CUtensorMap x[kMaxP];
  const uint8_t* sx[kMaxP];
  void* dw[kMaxP];
  StatusBlock* status;
  int64_t N, K;
  int32_t ag;              // AllGather: X in row shards, G whole; else the other way round
  int32_t P;
  int32_t m;               // rows per shard
  int32_t blocks;          // scales per row
  int32_t stages;          // per shard
  int32_t box;             // rows of a load
  int32_t big_rows, col_tiles;      // rows of 512 x 256 tiles
  int32_t odd;                      // and one more of 256 x 256
  int32_t n_big, left, total;       // 512 x 256 tiles; places left over, two 256 x 256 tiles each
  int32_t splits;                   // pairs of a cluster, which share a tile's contraction
  int32_t accumulate, fp32;
  int32_t range;           // stages of one sum at most
  int32_t wide;            // results lie on 32-byte boundaries
  uint32_t wait_limit_us;
};

struct Control {
  uint64_t ready[kStages];      // leader's: both CTAs' G has landed and both CTAs' X is converted
  uint64_t empty[kStages];
  uint64_t x_full[kXStages], x_empty[kXStages];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t drain;
  uint32_t signal[kGroups * kConvWarps];
  uint32_t tmem_base;
  int abort;
};
constexpr int kXAt = kStages * kGBytes, kCAt = kXAt + kXStages * kXBytes, kControlAt = kCAt + kStages * kCBytes;
constexpr size_t kSmemBytes = 1024 + kControlAt + sizeof(Control);
static_assert(kSmemBytes <= 227 * 1024 && keeps_tmem_apart(kSmemBytes) && kGroups <= kStages && kStages <= kXStages, "");

struct Tile {
  bool big;
  int rank;
  int row0, col0;
};
__device__ __forceinline__ Tile tile_of(const GradParams& p, int t) {
  Tile c;
  c.big = t < p.n_big;
  int slot = t, half = 0;
  const int u = t - p.n_big;
  if (!c.big && u >= 2 * p.left) {
    const int w = u - 2 * p.left;
    c.rank = w / p.col_tiles;
    c.col0 = (w - c.rank * p.col_tiles) * 256;
    c.row0 = p.big_rows * 512;
    return c;
  }
  if (!c.big) {
    slot = p.n_big + (u >> 1);
    half = u & 1;
  }
  const int per_rank = p.big_rows * p.col_tiles;
  c.rank = slot / per_rank;
  int w = slot - c.rank * per_rank;
  const int g = w / (kRowGroup * p.col_tiles);
  w -= g * kRowGroup * p.col_tiles;
  const int high = min(kRowGroup, p.big_rows - g * kRowGroup);
  const int nt = w / high;
  c.row0 = (g * kRowGroup + w - nt * high) * 512 + half * 256;
  c.col0 = nt * 256;
  return c;
}

// 16 values of 8 bits times a scale, in BF16 (`scale`: two of it), those of each four in the order 0, 2, 1, 3, which the epilogue
// undoes.  The bits of an 8-bit number, its exponent moved to where BF16 has its own, are that number times 2^-120 (E5M2: 2^-112),
// subnormal ones too; the factors are powers of two, so nothing is rounded above BF16's subnormal range.  What is not a number in
// 8 bits has now the size of one past the largest: times kPast it overflows, and infinity times 0 is added, in E4M3 to the value, in E5M2,
// whose infinities are to stay such, to `odd`: a row with any is converted again by convert16_rare.  (By the conversion
// instructions this took three quarters of the kernel's time; with the NaN looked for among the bits, the integer pipe was full.)
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ void st_global_b32x8(void* to, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
               "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void ld_global_f32x8(float* v, const float* from) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "l"(from)
               : "memory");
}
template <int kFormat>
__device__ __forceinline__ uint32_t scaled_pair(uint32_t bits, uint32_t scale, uint32_t& odd) {
  constexpr uint32_t kBias = kFormat == E4M3 ? 0x7B807B80u : 0x77807780u;       // 2^120, 2^112
  // E4M3: 448 kPast is finite, 480 kPast is not: 1.109375 * 2^119.  E5M2: 57344 kPast, 65536 kPast: 1.0625 * 2^112.
  constexpr uint32_t kPast = kFormat == E4M3 ? 0x7B0E7B0Eu : 0x77887788u;
  const uint32_t y = mul_bf16x2(bits, kBias);
  if constexpr (kFormat == E5M2) {
    odd = fma_bf16x2(mul_bf16x2(y, kPast), 0u, odd);
    return mul_bf16x2(y, scale);
  }
  return fma_bf16x2(y, scale, mul_bf16x2(mul_bf16x2(y, kPast), 0u));
}
template <int kFormat>
__device__ __forceinline__ void convert16(const uint4& w, uint32_t scale, uint4& lo, uint4& hi, uint32_t& odd) {
  constexpr int kShift = kFormat == E4M3 ? 4 : 3;
  constexpr uint32_t kMask = (0x7F00u >> kShift) * 0x10001u;
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = scaled_pair<kFormat>(((v[i] << 8) & 0x80008000u) | ((v[i] << (8 - kShift)) & kMask), scale, odd);      // numbers 0 and 2
    o[2 * i + 1] = scaled_pair<kFormat>((v[i] & 0x80008000u) | ((v[i] >> kShift) & kMask), scale, odd);               // 1 and 3
  }
  lo = make_uint4(o[0], o[1], o[2], o[3]);
  hi = make_uint4(o[4], o[5], o[6], o[7]);
}
// The same by the conversion instructions, of E5M2 with what is infinite or no number.
__device__ __forceinline__ void convert16_rare(const uint4& w, uint32_t scale, uint4& lo, uint4& hi) {
  const float s = __uint_as_float(scale << 16);
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = unpack8x2<E5M2>(v[i]), b = unpack8x2<E5M2>(v[i] >> 16);
    o[2 * i] = bf16x2_of(a.x * s, b.x * s);
    o[2 * i + 1] = bf16x2_of(a.y * s, b.y * s);
  }
  lo = make_uint4(o[0], o[1], o[2], o[3]);
  hi = make_uint4(o[4], o[5], o[6], o[7]);
}
// 2^(b - 127) in BF16, twice; 255 is NaN.
__device__ __forceinline__ uint32_t scale_bf16x2(uint32_t b) { return (b == 0 ? 0x0040u : b == 255 ? 0x7FC0u : b << 7) * 0x10001u; }

// kSplit: tiles shared by the pairs of a cluster (of its own, for the instructions: 0.4 us a call otherwise).
template <int kFormat, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) weight_grad_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  Control* ctl = reinterpret_cast<Control*>(smem + kControlAt);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // (ranks by the block's index, which is known to be the same for all threads)
  const int splits = kSplit ? p.splits : 1;
  const int unit = int(blockIdx.x) / (2 * splits), units = int(gridDim.x) / (2 * splits), place = int(blockIdx.x) - unit * 2 * splits;
  const int cta = place & 1, pair = place >> 1;
  const uint32_t first_cta = uint32_t(2 * pair);      // of this pair in its cluster
  const bool leader = cta == 0;
  const WaitContext wc{p.status, &ctl->abort, p.wait_limit_us};
  // this pair's stages of a tile
  const int from = p.P * p.stages * pair / splits, all = p.P * p.stages * (pair + 1) / splits - from;
  const int range = p.range, parts = (all + range - 1) / range;      // stages of one sum, and how many sums

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&ctl->ready[s], kConvWarps + 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int s = 0; s < kXStages; ++s) {
      mbar_init(&ctl->x_full[s], 1);
      mbar_init(&ctl->x_empty[s], kConvWarps);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->acc_full[b], 1);
      mbar_init(&ctl->acc_empty[b], 2 * kEpiWarps);
    }
    mbar_init(&ctl->drain, 1);
    ctl->abort = 0;
    fence_mbar_init();
  }
  if (p.box < kRows) {
    // Shards of fewer rows than a stage has: loads bring those that there are (rows outside a matrix of a few made them several times
    // as long), the others are zeros from the start.
    for (int i = threadIdx.x; i < kCAt / 16; i += kThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    tmem_alloc_pair(&ctl->tmem_base, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after_sync();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, ctl->tmem_base, 0);
  launch_dependents();
  wait_for_previous_kernel();

  if (warp == 0 || warp == 2 + kEpiWarps + kGroups * kConvWarps) {
    // ----------------------------------------------------------- TMA producers
    if (lane == 0) {
      const bool of_g = warp == 0;
      const uint64_t pol = make_l2_policy(L2_EVICT_NORMAL);
      const uint32_t depth = of_g ? kStages : kXStages;
      uint64_t* full = of_g ? ctl->ready : ctl->x_full;
      uint64_t* empty = of_g ? ctl->empty : ctl->x_empty;
      uint32_t j = 0;
      bool ok = true;
      for (int t = unit; ok && t < p.total; t += units) {
        const Tile c = tile_of(p, t);
        const int boxes = c.big ? 4 : 2, n0 = c.row0 + cta * boxes * 64, k0 = c.col0 + cta * 128;
        int s = from / p.stages, i = from - s * p.stages;
        for (int a = 0; a < all; ++a, ++j) {
            const uint32_t slot = j % depth;
            if (j >= depth && !(ok = wait_phase(&empty[slot], (j / depth - 1) & 1u, wc, SITE_EMPTY, t))) break;
            if (of_g) {
              const uint32_t bar = map_to_cta(smem_u32(&full[slot]), first_cta);
              if (leader) mbar_arrive_expect_tx(&full[slot], uint32_t(2 * boxes * p.box * 128) + kConvWarps * kSignalBytes);
              const CUtensorMap* g = &p.g[p.ag ? c.rank : s];
              for (int b = 0; b < boxes; ++b)
                tma_load_3d_pair_hint(smem + slot * kGBytes + b * kChunk, g, bar, n0 + b * 64, i * kRows, p.ag ? s : 0, pol);
            } else {
              mbar_arrive_expect_tx(&full[slot], uint32_t(p.box * 128));
              tma_load_3d_hint(smem + kXAt + slot * kXBytes, &p.x[p.ag ? s : c.rank], &full[slot], k0, i * kRows, p.ag ? 0 : s, pol);
            }
            if (++i == p.stages) {
              i = 0;
              ++s;
            }
        }
      }
      // leave only when the last stages have been read (the leader's products read both CTAs' memory)
      const uint32_t back = j < depth ? j : depth;
      for (uint32_t i = 1; i <= back; ++i) {
        const uint32_t r = j - i;
        if (!wait_phase(&empty[r % depth], (r / depth) & 1u, wc, SITE_DRAIN, -1)) {
          // (G's copies of both CTAs are counted with the conversions, which may never come: then after the 100 ms)
          if (!of_g || leader)
            for (uint32_t k = 1; k <= back; ++k) wait_settled(&full[(j - k) % depth], ((j - k) / depth) & 1u);
          break;
        }
      }
    }
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA issuer
    // (the whole warp goes through the loop and one lane issues, as in the products of 8-bit operands)
    if (leader) {
      constexpr uint32_t idesc = umma_idesc_bf16_f32(256, 256) | kUmmaIdescAMnMajor | kUmmaIdescBMnMajor;
      const uint64_t desc_g = umma_smem_desc_sw128_mn(smem_u32(smem), kChunk);
      const uint64_t desc_c = umma_smem_desc_sw128_mn(smem_u32(smem + kCAt), kChunk);
      uint32_t j = 0, uses[2] = {0, 0}, small = 0;
      bool ok = true;
      int t = unit;
      auto acc_free = [&](int b) {
        if (!wait_warp(&ctl->acc_empty[b], (uses[b] & 1u) ^ 1u, wc, SITE_ACC_EMPTY, t)) return false;
        tc_fence_after_sync();
        return true;
      };
      auto commit = [&](uint64_t* bar) {
        if (elect_one()) umma_commit_both(bar, first_cta + 1);
        __syncwarp();
      };
      auto landed = [&](uint32_t s) {
        if (!wait_warp<true>(&ctl->ready[s % kStages], (s / kStages) & 1u, wc, SITE_FULL, t)) return false;
        tc_fence_after_sync();
        return true;
      };
      // Products of stage `s` of a tile (the `s0 + s`-th of all) with columns 128 `block` on of G; a step of 16 rows of the contraction
      // is two groups of 8 (2048 bytes).  `first`: 0 where a sum begins.
      auto issue = [&](uint32_t acc, uint32_t at, int block, int s, uint32_t first) {
        const uint32_t slot = at % kStages;
        const uint64_t da = desc_g + uint64_t((slot * kGBytes + block * 2 * kChunk) >> 4), db = desc_c + uint64_t((slot * kCBytes) >> 4);
        const int rows = p.m - (from + s) % p.stages * kRows;
        if (!elect_one()) return;
        if (rows >= kRows) {
#pragma unroll
          for (int k = 0; k < kRows / 16; ++k) umma_bf16_pair(acc, da + k * (2048 >> 4), db + k * (2048 >> 4), idesc, k ? 1u : first);
        } else {
          for (int k = 0; k < (rows + 15) / 16; ++k) umma_bf16_pair(acc, da + k * (2048 >> 4), db + k * (2048 >> 4), idesc, k ? 1u : first);
        }
      };
      for (; ok && t < p.total; t += units) {
        if (tile_of(p, t).big) {
          // Both accumulators are live for the whole tile, so nothing would hide the epilogue's reads if they ended together: for the
          // first and last kSkew stages accumulator 0's products go first.  It is then complete early (its epilogue runs under
          // accumulator 1's last products), and the next tile begins on it while accumulator 1 is still being read.
          const int skew = all >= 2 * kSkew ? kSkew : 0;
          auto skewed = [&](int s0, bool begin) {
            for (int s = 0; s < kSkew; ++s) {
              if (!landed(j + s)) return false;
              issue(tmem_base, j + s, 0, s0 + s, s0 + s ? 1u : 0u);
            }
            if (begin) {
              if (!acc_free(1)) return false;
            } else {
              commit(&ctl->acc_full[0]);
            }
            for (int s = 0; s < kSkew; ++s) {
              issue(tmem_base + 256, j + s, 1, s0 + s, s0 + s ? 1u : 0u);
              commit(&ctl->empty[(j + s) % kStages]);
            }
            j += kSkew;
            return true;
          };
          ok = acc_free(0);
          if (ok) ok = skew ? skewed(0, true) : acc_free(1);
          for (int s = skew; ok && s < all - skew; ++s, ++j) {
            if (!(ok = landed(j))) break;
            issue(tmem_base, j, 0, s, s ? 1u : 0u);
            issue(tmem_base + 256, j, 1, s, s ? 1u : 0u);
            commit(&ctl->empty[j % kStages]);
          }
          if (ok && skew) ok = skewed(all - skew, false);
          else if (ok) commit(&ctl->acc_full[0]);
          if (!ok) break;
          commit(&ctl->acc_full[1]);
          ++uses[0];
          ++uses[1];
        } else {
          for (int s = 0; ok && s < all;) {
            // one sum: the accumulators in turn; several: the first goes where the total is kept
            const int b = parts > 1 ? (s == 0 ? 1 : 0) : int(small & 1u);
            const int begin = s, to = min(all, s + range);
            if (!(ok = acc_free(b))) break;
            for (; s < to; ++s, ++j) {
              if (!(ok = landed(j))) break;
              issue(tmem_base + b * 256, j, 0, s, s != begin ? 1u : 0u);
              commit(&ctl->empty[j % kStages]);
            }
            if (!ok) break;
            commit(&ctl->acc_full[b]);
            ++uses[b];
          }
          ++small;
        }
      }
      // leave only when the accumulators' last signals have come: the other CTA's may be on their way to this one's memory still
      for (int b = 0; ok && b < 2; ++b)
        if (uses[b] > 0) ok = wait_warp(&ctl->acc_empty[b], (uses[b] - 1) & 1u, wc, SITE_DRAIN, -1);
      if (__any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&ctl->abort) != 0)) {
        if (elect_one()) umma_commit_pair(&ctl->drain, 0x1);
        wait_settled(&ctl->drain, 0);
      }
    }
  } else if (warp >= 2 + kEpiWarps) {
    // ------------------------------------------------------------- 8 bits -> BF16
    const int w = warp - 2 - kEpiWarps, group = w / kConvWarps;
    const int row = (w & 1) * 32 + lane;
    const int swizzle = row & 7;
    uint32_t j = 0;
    bool ok = true;
    for (int t = unit; ok && t < p.total; t += units) {
      const Tile c = tile_of(p, t);
      const int block = (c.col0 >> 7) + cta;
      // (scales of columns that do not exist: 1, their values are zeros)
      auto scale_at = [&](int a) -> uint32_t {
        const int s = (from + a) / p.stages, r = (from + a - s * p.stages) * kRows + row;
        if (a >= all || r >= p.m || block >= p.blocks) return 127u;
        const uint8_t* sx = p.ag ? p.sx[s] + int64_t(r) * p.blocks : p.sx[c.rank] + (int64_t(s) * p.m + r) * p.blocks;
        return sx[block];
      };
      int a = int((uint32_t(group) - j) & (kGroups - 1));      // this group's first stage of the tile
      uint32_t next = scale_at(a);
      for (; a < all; a += kGroups) {
        const uint32_t scale = scale_bf16x2(next);
        next = scale_at(a + kGroups);
        const uint32_t at = j + uint32_t(a), xs = at % kXStages, slot = at % kStages;
        // In this order: a parity tells a phase from the one before it only, and the other groups' stages in between may be late.
        // This group's last stage waited for the products of stage at - kGroups - kStages, so it is the phase before that can be
        // missing at worst; and when those of stage at - kStages are done, the load before this one into its place has landed.
        if (at >= kStages) ok = wait_phase(&ctl->empty[slot], (at / kStages - 1) & 1u, wc, SITE_EMPTY, t);
        if (ok) ok = wait_phase(&ctl->x_full[xs], (at / kXStages) & 1u, wc, SITE_FULL, t);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint8_t* from = smem + kXAt + xs * kXBytes + row * 128;
        uint8_t* to = smem + kCAt + slot * kCBytes + row * 128;
        uint4 in[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) in[u] = *reinterpret_cast<const uint4*>(from + ((u ^ swizzle) << 4));
        auto put = [&](int u, const uint4& lo, const uint4& hi) {
          uint8_t* chunk = to + (u >> 2) * kChunk;
          const int at16 = 2 * (u & 3);
          *reinterpret_cast<uint4*>(chunk + ((at16 ^ swizzle) << 4)) = lo;
          *reinterpret_cast<uint4*>(chunk + (((at16 + 1) ^ swizzle) << 4)) = hi;
        };
        uint4 lo, hi;
        uint32_t odd = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          convert16<kFormat>(in[u], scale, lo, hi, odd);
          put(u, lo, hi);
        }
        // (0 times anything finite has added nothing)
        if (kFormat == E5M2 && (odd & 0x7FFF7FFFu) != 0) {
#pragma unroll 1
          for (int u = 0; u < 8; ++u) {
            convert16_rare(*reinterpret_cast<const uint4*>(from + ((u ^ swizzle) << 4)), scale, lo, hi);
            put(u, lo, hi);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&ctl->x_empty[xs]);
          if (leader) mbar_arrive(&ctl->ready[slot]);
          else mbar_signal_cluster(map_to_cta(smem_u32(&ctl->signal[w]), first_cta), map_to_cta(smem_u32(&ctl->ready[slot]), first_cta));
        }
      }
      j += uint32_t(all);
    }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint32_t uses[2] = {0, 0}, small = 0;
    bool ok = true;
    const uint32_t lanes = tmem_base + (uint32_t(quarter * 32) << 16) + half * 128;
    for (int t = unit; ok && t < p.total; t += units) {
      const Tile c = tile_of(p, t);
      auto filled = [&](int b) {
        ok = wait_warp(&ctl->acc_full[b], uses[b] & 1u, wc, SITE_ACC_FULL, t);
        tc_fence_after_sync();
        ++uses[b];
        return ok;
      };
      auto give_back = [&](int b) {
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(map_to_cta(smem_u32(&ctl->acc_empty[b]), first_cta));
      };
      if (parts > 1) {
        // the total is in accumulator 1; all sums but the last are added to it
        if (!filled(1)) break;
        for (int s = 2; ok && s < parts; ++s) {
          if (!filled(0)) break;
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            uint32_t v[32], w[32];
            tmem_ld_32x32b_x32(lanes + q * 32, v);
            tmem_ld_32x32b_x32(lanes + 256 + q * 32, w);
            tmem_ld_wait();
            if (q == 3) give_back(0);
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) + __uint_as_float(v[i]));
            tmem_st_32x32b_x32(lanes + 256 + q * 32, w);
          }
          tmem_st_wait();
        }
        if (!ok || !filled(0)) break;
      }
      const int64_t k0 = c.col0 + half * 128;
      const int cols = int(min(int64_t(128), p.K - k0));      // a multiple of 16, or none
      const bool add = p.accumulate;
      for (int block = 0; block < (c.big ? 2 : 1); ++block) {
        const int b = parts > 1 ? 0 : c.big ? block : int(small & 1u);
        if (parts == 1 && !filled(b)) break;
        const int64_t n = c.row0 + (c.big ? cta * 256 + block * 128 : cta * 128) + quarter * 32 + lane;
        const int64_t at = n * p.K + k0;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          uint32_t v[32];
          tmem_ld_32x32b_x32(lanes + b * 256 + q * 32, v);
          tmem_ld_wait();
          if (parts > 1) {
            uint32_t w[32];
            tmem_ld_32x32b_x32(lanes + 256 + q * 32, w);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(w[i]) + __uint_as_float(v[i]));
          }
          if (q == 3) {
            give_back(b);
            if (parts > 1) give_back(1);
          }
          if (!kSplit && (n >= p.N || q * 32 >= cols)) continue;
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const uint32_t x = v[i + 1];
            v[i + 1] = v[i + 2];
            v[i + 2] = x;
          }
          if constexpr (kSplit) {
            // to the cluster: 128 rows of 256, over G's stages, which have been read
            const int row = quarter * 32 + lane;
#pragma unroll
            for (int g = 0; g < 8; ++g)
              *reinterpret_cast<uint4*>(smem + row * 1024 + (((half * 32 + q * 8 + g) ^ (row & 7)) << 4)) =
                  make_uint4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
            continue;
          }
          if (p.fp32) {
            float* out = static_cast<float*>(p.dw[c.rank]) + at + q * 32;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (q * 32 + h * 16 >= cols) break;
              uint32_t* x = v + h * 16;
              if (add) {
                // the loads of 16 columns before the first store
                float old[16];
                if (p.wide) {
                  ld_global_f32x8(old, out + h * 16);
                  ld_global_f32x8(old + 8, out + h * 16 + 8);
                } else {
#pragma unroll
                  for (int g = 0; g < 4; ++g) {
                    const float4 o = reinterpret_cast<const float4*>(out + h * 16)[g];
                    old[4 * g] = o.x, old[4 * g + 1] = o.y, old[4 * g + 2] = o.z, old[4 * g + 3] = o.w;
                  }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) + old[i]);
              }
              // (whole sectors of 32 bytes: in stores of 16 bytes an 8192 x 8192 gradient of 64 rows took 149 us, so 68)
              if (p.wide) {
                st_global_b32x8(out + h * 16, x);
                st_global_b32x8(out + h * 16 + 8, x + 8);
              } else {
#pragma unroll
                for (int g = 0; g < 4; ++g) reinterpret_cast<uint4*>(out + h * 16)[g] = make_uint4(x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]);
              }
            }
          } else {
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.dw[c.rank]) + at + q * 32;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              if (q * 32 + g * 16 >= cols) break;
              float x[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(v[g * 16 + i]);
              if (add) {
                float old[8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  unpack_bf16x8(old, reinterpret_cast<const uint4*>(out + g * 16)[h]);
#pragma unroll
                  for (int i = 0; i < 8; ++i) x[h * 8 + i] += old[i];
                }
              }
              uint32_t w[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
              if (p.wide) {
                st_global_b32x8(out + g * 16, w);
              } else {
                reinterpret_cast<uint4*>(out + g * 16)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint4*>(out + g * 16)[1] = make_uint4(w[4], w[5], w[6], w[7]);
              }
            }
          }
        }
      }
      if (!c.big) ++small;
    }
  }

  if constexpr (kSplit) {
    // The pairs' sums of the cluster's tile: each adds up its part of the rows, in the pairs' order.  A warp reads 512 bytes in
    // a row of a CTA's memory at a time (eight neighbouring columns a thread, every other 16 bytes: 3.5 us more).
    __syncthreads();
    if (warp == 0) cluster_arrive();
    else cluster_arrive_relaxed();
    cluster_wait();
    if (*reinterpret_cast<volatile int*>(&ctl->abort) == 0) {
      const Tile c = tile_of(p, unit);
      // (128 columns are read only where a lane stores some of them: then they have been read before the warp says that the others may leave.)
      const bool second = c.col0 + 128 < p.K;
      for (int row = pair + splits * warp; row < 128; row += splits * (kThreads / 32)) {
        const int64_t n = c.row0 + cta * 128 + row;
        if (n >= p.N) break;
        const uint32_t at = smem_u32(smem + row * 1024);
        float4 y[kMostSplits][2];
#pragma unroll
        for (int q = 0; q < kMostSplits; ++q)
          if (q < splits)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (h == 0 || second) asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                           : "=f"(y[q][h].x), "=f"(y[q][h].y), "=f"(y[q][h].z), "=f"(y[q][h].w)
                           : "r"(map_to_cta(at + (uint32_t((h * 32 + lane) ^ (row & 7)) << 4), uint32_t(2 * q + cta))));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float4 x = y[0][h];
#pragma unroll
          for (int q = 1; q < kMostSplits; ++q)
            if (q < splits) x.x += y[q][h].x, x.y += y[q][h].y, x.z += y[q][h].z, x.w += y[q][h].w;
          const int64_t k = c.col0 + h * 128 + lane * 4;
          if (k >= p.K) continue;
          if (p.fp32) {
            float4* out = reinterpret_cast<float4*>(static_cast<float*>(p.dw[c.rank]) + n * p.K + k);
            if (p.accumulate) {
              const float4 a = *out;
              x.x += a.x, x.y += a.y, x.z += a.z, x.w += a.w;
            }
            *out = x;
          } else {
            uint2* out = reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.dw[c.rank]) + n * p.K + k);
            if (p.accumulate) {
              const uint2 a = *out;
              x.x += __uint_as_float(a.x << 16), x.y += __uint_as_float(a.x & 0xFFFF0000u);
              x.z += __uint_as_float(a.y << 16), x.w += __uint_as_float(a.y & 0xFFFF0000u);
            }
            *out = make_uint2(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w));
          }
        }
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_arrive_relaxed();      // nobody's memory goes while it is read
  cluster_wait();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// ---- host ----------------------------------------------------------------------

using GradKernel = void (*)(const GradParams);
GradKernel grad_kernel(int format, bool split) {
  if (format == E4M3) return split ? weight_grad_kernel<E4M3, true> : weight_grad_kernel<E4M3, false>;
  return split ? weight_grad_kernel<E5M2, true> : weight_grad_kernel<E5M2, false>;
}

// Clusters of n pairs that the device holds at once, in [n].
struct Clusters {
  int of[kMostSplits + 1];
};
int device_clusters(Clusters* out) {
  constexpr int kMaxDevices = 64;
  static Clusters known[kMaxDevices] = {};
  static std::mutex mu;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return record_cuda_error(e);
  if (dev < 0 || dev >= kMaxDevices) return COMPASS_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(mu);
  if (known[dev].of[1] == 0) {
    for (GradKernel k : {grad_kernel(E4M3, false), grad_kernel(E5M2, false), grad_kernel(E4M3, true), grad_kernel(E5M2, true)})
      if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmemBytes));
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    Clusters found = {};
    for (int n = 1; n <= kMostSplits; ++n) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(unsigned(sms / (2 * n) * 2 * n));
      cfg.blockDim = dim3(kThreads);
      cfg.dynamicSmemBytes = kSmemBytes;
      cudaLaunchAttribute attr;
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = unsigned(2 * n);
      attr.val.clusterDim.y = 1;
      attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&found.of[n], grad_kernel(E4M3, n > 1), &cfg);
      if (e != cudaSuccess) return record_cuda_error(e);
    }
    if (found.of[1] < 1) return COMPASS_ERR_UNSUPPORTED;
    known[dev] = found;
  }
  *out = known[dev];
  return COMPASS_OK;
}

}  // namespace

}  // namespace compass

using namespace compass;

extern "C" int compass_weight_grad_8bit(const compass_problem* g, int grad_dtype, int accumulate, const void* const* G, const void* const* X,
                                        const void* const* X_scale, void* const* dW, void* ws, size_t ws_bytes, void* stream) {
  if (g == nullptr) return COMPASS_ERR_INVALID_ARG;
  int st = check_problem_8bit(g);
  if (st == COMPASS_OK) st = check_dtype(grad_dtype, true);
  if (st != COMPASS_OK) return st;
  if (g->b_layout != COMPASS_B_NK) return COMPASS_ERR_UNSUPPORTED;
  if (g->N % 8 != 0) return COMPASS_ERR_ALIGNMENT;
  if (!G || !X || !X_scale || !dW) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < g->P; ++r)
    if (!G[r] || !X[r] || !X_scale[r] || !dW[r]) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < g->P; ++r)
    if (!is_aligned(G[r], 16) || !is_aligned(X[r], 16) || !is_aligned(dW[r], 16)) return COMPASS_ERR_ALIGNMENT;
  st = check_workspace(ws, ws_bytes, COMPASS_STATUS_BYTES);
  if (st != COMPASS_OK) return st;
  const int64_t row_tiles = ceil_div(g->N, 256), col_tiles = ceil_div(g->K, 256);
  if (row_tiles * col_tiles * g->P > kMaxDim || g->M + 2 * kRows * g->P > kMaxDim) return COMPASS_ERR_UNSUPPORTED;
  Clusters clusters;
  st = device_clusters(&clusters);
  if (st != COMPASS_OK) return st;
  GradParams p = {};
  p.ag = g->op == COMPASS_OP_AG_GEMM;
  p.P = g->P;
  p.m = int32_t(g->M / g->P);
  p.N = g->N;
  p.K = g->K;
  p.blocks = int32_t(scale_blocks(g->K));
  p.stages = int32_t(ceil_div(p.m, kRows));
  p.box = p.m < kRows ? p.m : kRows;
  p.accumulate = accumulate != 0;
  p.fp32 = grad_dtype == COMPASS_DTYPE_FP32;
  // whole rounds of the pairs take 512 x 256 tiles, what is left, and all where a tile has several sums, 256 x 256 ones
  p.big_rows = int32_t(row_tiles / 2);
  p.odd = int32_t(row_tiles % 2);
  p.col_tiles = int32_t(col_tiles);
  const int32_t places = int32_t(p.big_rows * col_tiles * g->P);
  const int pairs = clusters.of[1];
  const int64_t stages = int64_t(p.stages) * g->P;
  p.range = p.fp32 ? kFp32Range : kBf16Range;
  p.left = stages > p.range ? places : places % pairs;
  p.n_big = places - p.left;
  p.total = int32_t(p.n_big + 2 * p.left + p.odd * col_tiles * g->P);
  // Tiles that leave pairs without work: several pairs share a tile's contraction.  A stage of a tile takes some 770 cycles, the sum
  // over the cluster some 5000 (and the next kernel begins no earlier on SMs without work).  Measured with one pair and with several: 1024 x
  // 1024 over 4096 rows 30.9 us : 18.6, over 1024 12.5 : 12.2, 4 ranks' 232 x 480 over 5552 rows 42 : 17.8, 768 x 768 over 2048 rows in FP32
  // 25.6 : 12.6; 512 x 512 over 512 rows 9.0 : 9.8.
  p.splits = 1;
  int64_t least = stages * 770;
  for (int n = 2; n <= kMostSplits && n <= stages; ++n)
    if (p.n_big == 0 && p.total <= clusters.of[n] && ceil_div(stages, n) * 770 + 5000 < least) {
      p.splits = n;
      least = ceil_div(stages, n) * 770 + 5000;
    }
  p.wide = 1;
  p.status = static_cast<StatusBlock*>(ws);
  p.wait_limit_us = default_wait_limit_us() ? default_wait_limit_us() : 2000000u;
  bool ok = true;
  for (int r = 0; r < g->P; ++r) {
    p.sx[r] = static_cast<const uint8_t*>(X_scale[r]);
    p.dw[r] = dW[r];
    if (!is_aligned(dW[r], 32)) p.wide = 0;
    ok = ok && encode_tensor_map_slabs(&p.g[r], G[r], p.ag ? g->P : 1, p.m, g->N, 2, p.box);
    ok = ok && encode_tensor_map_slabs(&p.x[r], X[r], p.ag ? 1 : g->P, p.m, g->K, 1, p.box);
  }
  if (!ok) return record_cuda_error(cudaErrorUnknown);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(2 * p.splits * (p.total < pairs ? p.total : pairs)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(2 * p.splits);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, grad_kernel(format_of(g->dtype), p.splits > 1), p);
  count_kernel_launch();
  return e == cudaSuccess ? COMPASS_OK : record_cuda_error(e);
}
