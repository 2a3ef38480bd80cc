// Tensor-parallel products of 8-bit operands with a scale for each block of 128, for sm_100a:
//   C[i][j] = sum_b 2^(sa[i][b] + sb[j / 128][b]) * sum_{k in block b} a[i][k] * w[j][k]
// a: activations in E4M3 or E5M2, a scale per row and 128 columns; w: weights in E4M3, a scale per 128 x 128.  The scales are
// powers of two (E8M0), which the tensor core applies itself to every 32 products (kind::mxf8f6f4); one for 128 is four times the
// same.  (With scales of any value the accumulator would have to leave tensor memory every 128 elements.)
//
//   AllGather+GEMM      rank r's tiles read the row shards of all ranks, its own first (gather by address)
//   GEMM+ReduceScatter  a tile's contraction runs over the ranks' slices in ring order, ending near the owner, into one accumulator
//
// Two kernels.  gemm8_pair_kernel: pairs of CTAs, 256 rows x up to 256 columns a tile, for batches.  gemm8_few_kernel: weights on
// the products' M side, 128 rows a tile, and up to 256 activation rows on the N side, the contraction split over a cluster, for
// few rows, where the weights' bytes are all the work, and for few tiles of a long contraction.  Which one by what they are estimated
// to take (few_plan, pair_plan).
#include <mutex>

#include "pipeline.cuh"
#include "row_ops.cuh"
#include "scaled8.cuh"

namespace compass {

using namespace ptx;

namespace {

constexpr int kAtom = 128;                    // elements = bytes of the contraction in one swizzle row: what a scale covers
constexpr int kChunkBytes = 128 * kAtom;      // 128 rows (or, contraction across: 128 columns) of one atom
constexpr int kGroupAtoms = 4;                // atoms whose scales are one 32-bit word
constexpr uint32_t kOne = 0x7F7F7F7Fu;        // scales of 1

struct Gemm8Params {
  CUtensorMap a[kMaxP];
  CUtensorMap b[kMaxP];
  const uint8_t* sa[kMaxP];
  const uint8_t* sb[kMaxP];
  __nv_bfloat16* out[kMaxP];
  StatusBlock* status;
  int64_t N;
  int32_t rs;              // GEMM+ReduceScatter
  int32_t P;
  int32_t m;               // rows per shard
  int32_t K;
  int32_t atoms;           // of a slice of the contraction
  int32_t kn;              // weights are [K][N]
  int32_t n_blocks;        // scales along N
  int32_t a_format;
  int32_t whole_words;     // rows of the activations' scales are whole aligned words of four
  int32_t wide;            // output rows: 2: whole 32-byte sectors, 1: whole 16-byte vectors, 0: neither
  uint32_t wait_limit_us;
  // pair kernel
  int32_t frags;           // 128-row fragments per shard
  int32_t row_tiles;       // pairs of fragments
  int32_t col_tiles, bn;   // tiles of bn columns
  int32_t n_step;          // whose number is a multiple of this, at the end too: both CTAs load half of them from a 16-byte boundary on
  int32_t total;
  // rows of a load, those of a matrix of fewer (rows outside one made its loads several times as long); [K][N] weights: 128 of the
  // contraction, zero behind it
  int32_t a_box, b_box;
  FastDiv per_rank, per_group, by_frags;      // tiles of a rank, of a group of rows
  // few-rows kernel
  FastDiv each;            // rows per shard
  FastDiv by_rows;         // row tiles of a rank's 128-row tile of weights
  FastDiv pieces;          // of a shard's rows, a row tile each
  int32_t tile_shards;     // shards of a row tile (AllGather, shards in one piece)
  int32_t tile_rows;       // rows of a shard in it, what is loaded together
  FastDiv slot;            // accumulator columns for them: rounded up to 8
  int32_t cols;            // accumulator columns, a multiple of 16
  int32_t n_tiles;         // 128-row tiles of one rank's weights
  int32_t splits;          // CTAs of a cluster, which share a tile's contraction
  int32_t all;             // atoms of the whole contraction
  FastDiv by_splits, by_tiles;
  int32_t stages;
  int32_t tmem_cols;
};

// The scales of a row's `count` (1..4) blocks from `p` on, as they are loaded: a word where rows are whole aligned words (`words`,
// the same for a warp), else bytes (past the last one that again: not used).  Nothing is done with them before word() is called, and
// no lane leaves a load out, so that all of a group's loads are in flight together: waiting for each in turn, the scales took longer
// than the products (4096 x 4736, contraction 4224 instead of 4096: 1.50 and 1.80 PFLOP/s).
struct RowScales {
  uint32_t b[4];
  __device__ __forceinline__ void load(const uint8_t* p, int count, bool words) {
    if (words) {
      b[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i] = p[min(i, count - 1)];
    }
  }
  __device__ __forceinline__ uint32_t word(bool words) const { return words ? b[0] : b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24; }
};
// The weights' scales of 8 blocks along N from `j` on, for `count` blocks of the contraction from atom `a` on: a byte a lane, and
// the word of block j + k from lanes 4 k on.
__device__ __forceinline__ uint32_t weight_byte(const Gemm8Params& p, int rank, int64_t j, int a, int count, int lane) {
  const int64_t n = min(j + (lane >> 2), int64_t(p.n_blocks - 1));
  const int at = a + min(lane & 3, count - 1);
  return p.sb[rank][p.kn ? int64_t(at) * p.n_blocks + n : n * p.atoms + at];
}
__device__ __forceinline__ uint32_t weight_words(uint32_t byte, int lane) {
  uint32_t w = byte << (8 * (lane & 3));
  w |= __shfl_xor_sync(0xffffffffu, w, 1);
  return w | __shfl_xor_sync(0xffffffffu, w, 2);
}
// MMAs (32 elements each) in atom `a` of a slice.
__device__ __forceinline__ int steps_of(const Gemm8Params& p, int a) { return min(4, (p.K - a * kAtom + 31) / 32); }

// ---- batches -------------------------------------------------------------------
// Warp 0 loads (TMA), warp 1 issues the products, warps 2..9 are the epilogue (two per quarter of the rows, 128 columns each),
// warp 10 brings the scales.  Tensor memory holds two accumulators of 256 columns and the scales only because the accumulators
// share 32 columns: each is emptied from the shared ones on, and the next tile's products begin once these are read.
// Bound by the tensor cores, then by the board's power: 8 ranks' 8192 x 1376 x 4096 254 to 264 us in a burst (2.8 to 2.9 PFLOP/s, tensor pipe busy
// 85 % of the cycles) and 305 to 340 in loops; GEMM+ReduceScatter of 4 ranks 8192 x 4096 x 2752, [K][N], 251 to 263 and 320 to 350.  256 x 256 takes the fewest
// operand bytes that tensor memory has room for with two accumulators.
constexpr int kPairThreads = 352;
constexpr int kEpiWarps = 8;
constexpr int kPairStages = 3;
constexpr int kStageAtoms = 2;
constexpr int kPairStageBytes = kStageAtoms * 2 * kChunkBytes;
constexpr uint32_t kAcc1 = 224;               // second accumulator's first column; the first's last 32 are shared
constexpr uint32_t kScaleCols = 480;          // scales of A: 2 x 4 columns, of B: 2 x 8 behind them
constexpr int kRowGroup = 16;                 // row tiles that go through the columns together (their A stays in L2; 8: 3 % slower at 8192 x 8192 x 8192)
constexpr int kPitch = 17;                    // words of a staged row of 32 columns
struct PairControl {
  uint64_t full[kPairStages], empty[kPairStages];
  uint64_t scales_full[2], scales_empty[2];      // (full: the leader's, by both CTAs)
  uint64_t acc_full, acc_early;
  uint64_t drain;
  uint32_t signal;
  uint32_t tmem_base;
  int abort;
};
struct PairShared {
  uint4 scales[2][3][32];                     // [buffer][A, B's columns 0.., B's columns 128..][lane]
  uint32_t rows[kEpiWarps][32 * kPitch];
  PairControl ctl;
};
constexpr size_t kPairSmemBytes = 1024 + size_t(kPairStages) * kPairStageBytes + sizeof(PairShared);
static_assert(kPairSmemBytes <= 227 * 1024, "");

struct PairTile {
  int rank;            // whose weights and output (AllGather)
  int chunk, row0;     // this CTA's fragment: row shard, first row in it
  int rows;            // rows of it that exist
  int first;           // GEMM+ReduceScatter: rank whose slice comes first
  int64_t col0;
  int n;               // columns, a multiple of n_step
};
__device__ __forceinline__ PairTile pair_tile(const Gemm8Params& p, int t, int cta) {
  PairTile c;
  c.rank = int(p.per_rank.div(uint32_t(t)));
  int w = t - c.rank * int(p.per_rank.d);
  const int g = int(p.per_group.div(uint32_t(w)));
  w -= g * int(p.per_group.d);
  const int high = min(kRowGroup, p.row_tiles - g * kRowGroup);
  const int nt = high == kRowGroup ? w / kRowGroup : w / high;
  const int f = 2 * (g * kRowGroup + w - nt * high) + cta;
  c.col0 = int64_t(nt) * p.bn;
  c.n = int(min(int64_t(p.bn), (p.N - c.col0 + p.n_step - 1) / p.n_step * p.n_step));
  const int all = p.frags * p.P, mine = min(f, all - 1);
  const int s = int(p.by_frags.div(uint32_t(mine)));
  c.chunk = p.rs ? s : c.rank + s - (c.rank + s >= p.P ? p.P : 0);
  c.row0 = (mine - s * p.frags) * 128;
  c.rows = f < all ? min(128, p.m - c.row0) : 0;
  c.first = int(p.by_frags.div(uint32_t(f - cta))) + 1;
  if (c.first == p.P) c.first = 0;
  return c;
}
// Tensor of slice `seg`, the row in it where this CTA's fragment begins.
__device__ __forceinline__ int slice_of(const Gemm8Params& p, const PairTile& c, int seg) {
  return p.rs ? c.first + seg - (c.first + seg >= p.P ? p.P : 0) : c.chunk;
}
__device__ __forceinline__ int slice_row(const Gemm8Params& p, const PairTile& c) { return p.rs ? c.chunk * p.m + c.row0 : c.row0; }

__global__ void __launch_bounds__(kPairThreads, 1) gemm8_pair_kernel(const __grid_constant__ Gemm8Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  PairShared* sh = reinterpret_cast<PairShared*>(smem + kPairStages * kPairStageBytes);
  PairControl* ctl = &sh->ctl;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = int(blockIdx.x & 1);      // (the rank in the cluster, known to be the same for all threads)
  const bool leader = cta == 0;
  const int unit = int(blockIdx.x >> 1), units = int(gridDim.x >> 1);
  const WaitContext wc{p.status, &ctl->abort, p.wait_limit_us};
  const int segs = p.rs ? p.P : 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kPairStages; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->scales_full[b], 1);
      mbar_init(&ctl->scales_empty[b], 1);
    }
    mbar_init(&ctl->acc_full, 1);
    mbar_init(&ctl->acc_early, 2 * kEpiWarps);
    mbar_init(&ctl->drain, 1);
    ctl->abort = 0;
    fence_mbar_init();
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

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    // (the whole warp goes through the loop and one lane issues, as below)
    const uint64_t pol = make_l2_policy(L2_EVICT_NORMAL);
    const int bytes = (p.a_box + p.b_box) * kAtom;
    uint32_t j = 0, slot = 0, turn = 0;
    bool ok = true;
    for (int t = unit; ok && t < p.total; t += units) {
      const PairTile c = pair_tile(p, t, cta);
      const int b0 = int(c.col0) + cta * (c.n / 2);
      for (int seg = 0; ok && seg < segs; ++seg) {
        const int q = slice_of(p, c, seg), row = slice_row(p, c), br = p.rs ? q : c.rank;
        for (int a = 0; a < p.atoms; a += kStageAtoms) {
          if (turn > 0 && !(ok = wait_warp(&ctl->empty[slot], (turn - 1) & 1u, wc, SITE_EMPTY, t))) break;
          if (elect_one()) {
            const int n = min(kStageAtoms, p.atoms - a);
            const uint32_t bar = map_to_cta(smem_u32(&ctl->full[slot]), 0);
            if (leader) mbar_arrive_expect_tx(&ctl->full[slot], uint32_t(2 * n * bytes));
            uint8_t* dst = smem + slot * kPairStageBytes;
#pragma unroll
            for (int i = 0; i < kStageAtoms; ++i) {
              if (i >= n) break;
              tma_load_2d_pair_hint(dst + i * 2 * kChunkBytes, &p.a[q], bar, (a + i) * kAtom, row, pol);
              if (p.kn) tma_load_2d_pair_hint(dst + (i * 2 + 1) * kChunkBytes, &p.b[br], bar, b0, (a + i) * kAtom, pol);
              else tma_load_2d_pair_hint(dst + (i * 2 + 1) * kChunkBytes, &p.b[br], bar, (a + i) * kAtom, b0, pol);
            }
          }
          __syncwarp();
          ++j;
          if (++slot == kPairStages) {
            slot = 0;
            ++turn;
          }
        }
      }
    }
    // leave only when the last stages have been read (the leader's products read both CTAs' memory)
    const uint32_t back = j < uint32_t(kPairStages) ? j : uint32_t(kPairStages);
    ok = true;
    for (uint32_t i = 1; ok && i <= back; ++i) ok = wait_warp(&ctl->empty[(j - i) % kPairStages], ((j - i) / kPairStages) & 1u, wc, SITE_DRAIN, -1);
    if (!ok && leader)
      for (uint32_t k = 1; k <= back; ++k) wait_settled(&ctl->full[(j - k) % kPairStages], ((j - k) / kPairStages) & 1u);
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA issuer
    // The whole warp goes through the loop and one lane issues: descriptors and addresses are then the warp's, in the registers that
    // the instructions take them from.  (With the loop in one lane, each was moved there for every MMA: 180 cycles each, whatever
    // their size; a full one takes 128.)
    if (leader) {
      const uint64_t desc_a0 = umma_smem_desc_sw128(smem_u32(smem));
      const uint64_t desc_b0 = p.kn ? umma_smem_desc_sw128_mn(smem_u32(smem + kChunkBytes), kChunkBytes) : umma_smem_desc_sw128(smem_u32(smem + kChunkBytes));
      // a step of 32 elements: 32 bytes of a row, or (contraction across) four groups of 8 rows
      const uint64_t bk = p.kn ? 4096 >> 4 : 2;
      const uint64_t desc_s = smem_desc_scales(smem_u32(sh->scales));
      uint32_t j = 0, it = 0, g = 0;
      bool ok = true;
      for (int t = unit; ok && t < p.total; t += units, ++it) {
        const PairTile c = pair_tile(p, t, 0);
        const uint32_t idesc0 = umma_idesc_mx8(256, uint32_t(c.n), uint32_t(p.a_format), E4M3) | (p.kn ? kUmmaIdescBMnMajor : 0u);
        const uint32_t acc = tmem_base + (it & 1u ? kAcc1 : 0u);
        if (it > 0) {
          if (!(ok = wait_warp(&ctl->acc_early, (it - 1) & 1u, wc, SITE_ACC_EMPTY, t))) break;
          tc_fence_after_sync();
        }
        for (int seg = 0; ok && seg < segs; ++seg) {
          uint32_t buf = 0;
          for (int a = 0; a < p.atoms; a += kStageAtoms, ++j) {
            if (a % kGroupAtoms == 0) {
              buf = g & 1u;
              if (!(ok = wait_warp<true>(&ctl->scales_full[buf], (g >> 1) & 1u, wc, SITE_SCALES_FULL, t))) break;
              tc_fence_after_sync();
              const uint64_t from = desc_s + uint64_t(buf * (3 * 512 >> 4));
              if (elect_one()) {
                tmem_copy_scales<true>(tmem_base + kScaleCols + buf * 4, from);
                tmem_copy_scales<true>(tmem_base + kScaleCols + 8 + buf * 8, from + (512 >> 4));
                tmem_copy_scales<true>(tmem_base + kScaleCols + 12 + buf * 8, from + (1024 >> 4));
              }
              ++g;
            }
            const uint32_t slot = j % kPairStages;
            if (!(ok = wait_warp(&ctl->full[slot], (j / kPairStages) & 1u, wc, SITE_FULL, t))) break;
            tc_fence_after_sync();
            const uint32_t sa = tmem_base + kScaleCols + buf * 4, sb = tmem_base + kScaleCols + 8 + buf * 8;
            if (elect_one()) {
#pragma unroll
              for (int i = 0; i < kStageAtoms; ++i) {
                if (a + i >= p.atoms) break;
                const uint64_t da = desc_a0 + uint64_t((slot * kPairStageBytes + i * 2 * kChunkBytes) >> 4);
                const uint64_t db = desc_b0 + uint64_t((slot * kPairStageBytes + i * 2 * kChunkBytes) >> 4);
                const uint32_t idesc = idesc0 | umma_scale_byte(uint32_t(a + i) % kGroupAtoms);
                const uint32_t first = (seg | a | i) != 0 ? 1u : 0u;
                const int steps = steps_of(p, a + i);
                if (steps == 4) {
#pragma unroll
                  for (int k = 0; k < 4; ++k) umma_mx8<true>(acc, da + k * 2, db + k * bk, idesc, sa, sb, k ? 1u : first);
                } else {
                  for (int k = 0; k < steps; ++k) umma_mx8<true>(acc, da + k * 2, db + k * bk, idesc, sa, sb, k ? 1u : first);
                }
              }
              umma_commit_pair(&ctl->empty[slot], 0x3);
              if (a % kGroupAtoms == kGroupAtoms - kStageAtoms || a + kStageAtoms >= p.atoms) umma_commit_pair(&ctl->scales_empty[buf], 0x3);
            }
            __syncwarp();
          }
        }
        if (ok && elect_one()) umma_commit_pair(&ctl->acc_full, 0x3);
        __syncwarp();
      }
      if (__any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&ctl->abort) != 0)) {
        // gave up somewhere: let the tensor core finish what it still has before tensor memory is released
        if (elect_one()) umma_commit_pair(&ctl->drain, 0x1);
        wait_settled(&ctl->drain, 0);
      }
    }
  } else if (warp == 10) {
    // ------------------------------------------------------------------ scales
    // A word of four blocks' scales per row; the loads of the next group are in flight while this one's buffer is waited for.
    struct Group {
      RowScales a[4];
      uint32_t b;
      int64_t col0;
    };
    struct Cursor {
      int t, seg, a;
    };
    PairTile c = {};
    auto load = [&](const Cursor& at, Group& x) {
      if (at.t >= p.total) return;
      if (at.seg == 0 && at.a == 0) c = pair_tile(p, at.t, cta);
      const int q = slice_of(p, c, at.seg), n = min(kGroupAtoms, p.atoms - at.a);
      const uint8_t* sa = p.sa[q] + int64_t(slice_row(p, c)) * p.atoms + at.a;
      const int last = max(c.rows - 1, 0);      // (the scales of rows that do not exist do not matter)
#pragma unroll
      for (int i = 0; i < 4; ++i) x.a[i].load(sa + int64_t(min(i * 32 + lane, last)) * p.atoms, n, p.whole_words);
      x.b = weight_byte(p, p.rs ? q : c.rank, c.col0 >> 7, at.a, n, lane);
      x.col0 = c.col0;
    };
    uint32_t g = 0;
    bool ok = true;
    Cursor at{unit, 0, 0};
    Group x, next;
    load(at, x);
    for (; at.t < p.total; ++g) {
      const int t = at.t;
      at.a += kGroupAtoms;
      if (at.a >= p.atoms) {
        at.a = 0;
        if (++at.seg == segs) {
          at.seg = 0;
          at.t += units;
        }
      }
      load(at, next);
      uint32_t a[4], b[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = x.a[i].word(p.whole_words);
      const uint32_t w = weight_words(x.b, lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = __shfl_sync(0xffffffffu, w, 4 * int(((x.col0 + 32 * i + lane) >> 7) - (x.col0 >> 7)));
      const uint32_t buf = g & 1u;
      if (g >= 2) {
        ok = wait_warp(&ctl->scales_empty[buf], ((g >> 1) - 1) & 1u, wc, SITE_SCALES_EMPTY, t);
        if (!ok) break;
      }
      sh->scales[buf][0][lane] = make_uint4(a[0], a[1], a[2], a[3]);
      sh->scales[buf][1][lane] = make_uint4(b[0], b[1], b[2], b[3]);
      sh->scales[buf][2][lane] = make_uint4(b[4], b[5], b[6], b[7]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        if (leader) mbar_arrive_expect_tx(&ctl->scales_full[buf], kSignalBytes);
        else mbar_signal_cluster(map_to_cta(smem_u32(&ctl->signal), 0), map_to_cta(smem_u32(&ctl->scales_full[buf]), 0));
      }
      x = next;
    }
    // leave only when the last groups' signals have come
    for (uint32_t i = g < 2u ? g : 2u; ok && i > 0; --i)
      ok = wait_warp(&ctl->scales_empty[(g - i) & 1u], ((g - i) >> 1) & 1u, wc, SITE_DRAIN, -1);
  } else {
    // ---------------------------------------------------------------- epilogue
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint32_t it = 0;
    for (int t = unit; t < p.total; t += units, ++it) {
      const PairTile c = pair_tile(p, t, cta);
      uint32_t v[4][32];
      const bool got = wait_phase(&ctl->acc_full, it & 1u, wc, SITE_ACC_FULL, t);
      if (!__all_sync(0xffffffffu, got)) break;
      tc_fence_after_sync();
      const uint32_t taddr = tmem_base + (uint32_t(quarter * 32) << 16) + (it & 1u ? kAcc1 : 0u) + half * 128;
      // The shared columns first: the last 32 of the first accumulator, the first 32 of the second.  The others, of the accumulator
      // that the next tile does not touch, may be read later.
      const bool second = it & 1u;
      if (second) tmem_ld_32x32b_x32(taddr, v[0]);
      else tmem_ld_32x32b_x32(taddr + 96, v[3]);
      tmem_ld_wait();
      tc_fence_before_sync();
      __syncwarp();
      // (not of the last tile: nobody would wait for the signal, and the CTA that it goes to may have left)
      if (lane == 0 && t + units < p.total) mbar_arrive_cluster_relaxed(map_to_cta(smem_u32(&ctl->acc_early), 0));
      if (second) tmem_ld_32x32b_x32(taddr + 96, v[3]);
      else tmem_ld_32x32b_x32(taddr, v[0]);
      tmem_ld_32x32b_x32(taddr + 32, v[1]);
      tmem_ld_32x32b_x32(taddr + 64, v[2]);
      tmem_ld_wait();

      const int64_t left = p.N - c.col0 - half * 128;
      const int cols = int(min(int64_t(min(128, c.n - half * 128)), left));      // of this warp's 128
      const int rank = p.rs ? c.chunk : c.rank;
      const int64_t row0 = (p.rs ? c.row0 : c.chunk * int64_t(p.m) + c.row0) + quarter * 32;
      __nv_bfloat16* out = p.out[rank] + row0 * p.N + c.col0 + half * 128;
      if (p.wide) {
        if (quarter * 32 + lane < c.rows) {
          __nv_bfloat16* mine = out + int64_t(lane) * p.N;
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            if (g * 16 >= cols) break;
            uint32_t q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
              q[i] = pack_bf16x2(__uint_as_float(v[g >> 1][(g & 1) * 16 + 2 * i]), __uint_as_float(v[g >> 1][(g & 1) * 16 + 2 * i + 1]));
            if (p.wide == 2) {
              asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(mine + g * 16), "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3]),
                           "r"(q[4]), "r"(q[5]), "r"(q[6]), "r"(q[7])
                           : "memory");
            } else {
              *reinterpret_cast<uint4*>(mine + g * 16) = make_uint4(q[0], q[1], q[2], q[3]);
              if (g * 16 + 8 < cols) *reinterpret_cast<uint4*>(mine + g * 16 + 8) = make_uint4(q[4], q[5], q[6], q[7]);
            }
          }
        }
      } else {
        // rows that are not whole vectors: through shared memory, so that a warp writes an element each of one row's 32
        uint32_t* rows = sh->rows[warp - 2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (k * 32 >= cols) break;
#pragma unroll
          for (int i = 0; i < 16; ++i) rows[lane * kPitch + i] = pack_bf16x2(__uint_as_float(v[k][2 * i]), __uint_as_float(v[k][2 * i + 1]));
          __syncwarp();
          if (k * 32 + lane < cols) {
            const int shift = 16 * (lane & 1);
            for (int r = 0; r < min(32, c.rows - quarter * 32); ++r)
              reinterpret_cast<unsigned short*>(out + int64_t(r) * p.N)[k * 32 + lane] = static_cast<unsigned short>(rows[r * kPitch + (lane >> 1)] >> shift);
          }
          __syncwarp();
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

// ---- few rows ------------------------------------------------------------------
// Bound by the weights' bytes where they are many (one row of 8192 x 8192: 67 MB in 15 us), by launch, first loads and the cluster's sum
// where not (4096 x 4096: 16.8 MB in 6.0 us, of which a kernel that does next to nothing takes 3.5).  Weights on the M side, because the
// tensor cores take no fewer than 128 rows there but as few columns as 16; the contraction split so that all SMs load.
// Warp 0 loads, warp 1 multiplies, warp 2 brings the scales, warps 4..7 read the accumulator.  The CTAs of a cluster take a share
// of the contraction each and add their FP32 sums up, rank by rank, through each other's shared memory.
constexpr int kFewThreads = 256;
constexpr int kFewMostCols = 256;
constexpr int kFewMostStages = 12;
constexpr int kFewRoom = 200 * 1024;          // of stages, with one CTA per SM
constexpr int kFewHalfRoom = 96 * 1024;       // with two
constexpr int kMostSplits = 8;
constexpr size_t kFewAll = 152 * 1024;        // shared memory of a cluster's CTA with more than half of tensor memory, at least
static_assert(keeps_tmem_apart(kFewAll) && keeps_tmem_apart(kPairSmemBytes), "");
struct FewControl {
  uint64_t full[kFewMostStages], empty[kFewMostStages];
  uint64_t scales_full[2], scales_empty[2];
  uint64_t acc_full, drain;
  uint32_t tmem_base;
  int abort;
};
struct FewShared {
  uint4 scales[2][3][32];
  FewControl ctl;
};
// This CTA's atoms one after the other: slice, atom in it, place in the ring and its turn.  (By divisions, about 100 cycles each, an
// atom took the issuing warp 1000 cycles.)
struct FewWalk {
  int seg, a, left, slot;
  uint32_t turn;
  __device__ __forceinline__ FewWalk(const Gemm8Params& p, int from, int to) : left(to - from), slot(0), turn(0) {
    seg = from >= p.atoms ? from / p.atoms : 0;
    a = from - seg * p.atoms;
  }
  __device__ __forceinline__ void next(const Gemm8Params& p) {
    --left;
    if (++a == p.atoms) {
      a = 0;
      ++seg;
    }
    if (++slot == p.stages) {
      slot = 0;
      ++turn;
    }
  }
  // atoms of the group of scales that begins here
  __device__ __forceinline__ int group(const Gemm8Params& p) const { return min(min(kGroupAtoms, p.atoms - a), left); }
};
__host__ __device__ constexpr int few_stage_bytes(int cols) { return kChunkBytes + cols * kAtom; }
__host__ __device__ constexpr size_t few_smem_bytes(int cols, int stages) { return 1024 + size_t(stages) * few_stage_bytes(cols) + sizeof(FewShared); }

__global__ void __launch_bounds__(kFewThreads, 2) gemm8_few_kernel(const __grid_constant__ Gemm8Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int stage_bytes = few_stage_bytes(p.cols), stages = p.stages;
  FewShared* sh = reinterpret_cast<FewShared*>(smem + stages * stage_bytes);
  FewControl* ctl = &sh->ctl;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // (the rank in the cluster by the block's index, which is known to be the same for all threads: what goes by it stays in the
  // registers that the issuing instructions take)
  const int t = int(p.by_splits.div(blockIdx.x)), part = int(blockIdx.x) - t * p.splits;
  const int wt = int(p.by_rows.div(uint32_t(t))), rt = t - wt * int(p.by_rows.d);
  const int rank = p.rs ? 0 : int(p.by_tiles.div(uint32_t(wt)));
  const int64_t n0 = int64_t(wt - rank * p.n_tiles) * 128;
  // the tile's activation rows: `rows` from row0 on of `shards` shards (GEMM+ReduceScatter: of all rows)
  const int piece = p.rs ? rt : int(p.pieces.d) == 1 ? 0 : rt - int(p.pieces.div(uint32_t(rt))) * int(p.pieces.d);
  const int shard0 = p.rs ? 0 : int(p.pieces.div(uint32_t(rt))) * p.tile_shards, row0 = piece * p.tile_rows;
  const int shards = p.rs ? 1 : min(p.tile_shards, p.P - shard0);
  const int rows = min(p.tile_rows, (p.rs ? p.m * p.P : p.m) - row0);
  const WaitContext wc{p.status, &ctl->abort, p.wait_limit_us};
  // this CTA's atoms of the whole contraction
  const int from = int(p.by_splits.div(uint32_t(p.all * part))), to = int(p.by_splits.div(uint32_t(p.all * (part + 1))));

  if (warp == 0 && lane == 0) {
    prefetch_tensormap(&p.b[rank]);
    prefetch_tensormap(&p.a[0]);
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->scales_full[b], 1);
      mbar_init(&ctl->scales_empty[b], 1);
    }
    mbar_init(&ctl->acc_full, 1);
    mbar_init(&ctl->drain, 1);
    ctl->abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&ctl->tmem_base, uint32_t(p.tmem_cols));
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, ctl->tmem_base, 0);
  const uint32_t scale_a = tmem_base + uint32_t(p.cols), scale_b = scale_a + 8;      // 2 x 4 and 2 x 8 columns
  launch_dependents();
  // Scales of the activations in column `i * 32 + lane` (columns without any: any): the row in its tensor, and with AllGather, where the
  // tensors differ from lane to lane, its address.
  int64_t row_at[8];
  if (warp == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int col = i * 32 + lane, s = int(p.slot.div(uint32_t(col)));
      row_at[i] = int64_t(row0 + min(col - s * int(p.slot.d), rows - 1)) * p.atoms;
      if (!p.rs) row_at[i] += reinterpret_cast<int64_t>(p.sa[shard0 + min(s, shards - 1)]);
    }
  }
  wait_for_previous_kernel();

  if (warp == 0) {
    const uint64_t pol = make_l2_policy(L2_EVICT_NORMAL);
    const uint32_t bytes = uint32_t((p.b_box + shards * p.tile_rows) * kAtom);
    FewWalk w(p, from, to);
    for (; w.left > 0; w.next(p)) {
      if (w.turn > 0 && !wait_warp(&ctl->empty[w.slot], (w.turn - 1) & 1u, wc, SITE_EMPTY, t)) break;
      if (elect_one()) {
        uint8_t* dst = smem + w.slot * stage_bytes;
        mbar_arrive_expect_tx(&ctl->full[w.slot], bytes);
        const CUtensorMap* b = &p.b[p.rs ? w.seg : rank];
        if (p.kn) tma_load_2d_hint(dst, b, &ctl->full[w.slot], int(n0), w.a * kAtom, pol);
        else tma_load_2d_hint(dst, b, &ctl->full[w.slot], w.a * kAtom, int(n0), pol);
        for (int s = 0; s < shards; ++s)
          tma_load_2d_hint(dst + kChunkBytes + s * p.slot.d * kAtom, &p.a[p.rs ? w.seg : shard0 + s], &ctl->full[w.slot], w.a * kAtom, row0, pol);
      }
      __syncwarp();
    }
    // leave only when everything that was loaded has landed and been read: the last turn's places before this one's, the one's before
    // it from here on
    bool ok = true;
    for (int i = 0; ok && i < stages; ++i) {
      const int turn = int(w.turn) - (i < w.slot ? 0 : 1);
      if (turn >= 0) ok = wait_warp(&ctl->empty[i], uint32_t(turn) & 1u, wc, SITE_DRAIN, -1);
    }
    for (int i = 0; !ok && i < stages; ++i) {
      const int turn = int(w.turn) - (i < w.slot ? 0 : 1);
      if (turn >= 0) wait_settled(&ctl->full[i], uint32_t(turn) & 1u);
    }
  } else if (warp == 1) {
    // (the whole warp goes through the loop and one lane issues, as above)
    const uint32_t idesc0 = umma_idesc_mx8(128, uint32_t(p.cols), E4M3, uint32_t(p.a_format)) | (p.kn ? kUmmaIdescAMnMajor : 0u);
    const uint64_t desc_w = p.kn ? umma_smem_desc_sw128_mn(smem_u32(smem), kChunkBytes) : umma_smem_desc_sw128(smem_u32(smem));
    const uint64_t desc_x = umma_smem_desc_sw128(smem_u32(smem + kChunkBytes));
    const uint64_t desc_s = smem_desc_scales(smem_u32(sh->scales));
    const uint64_t wk = p.kn ? 4096 >> 4 : 2;
    uint32_t group = 0, buf = 0, more = 0;
    int in_group = 0, left = 0;
    bool ok = true;
    for (FewWalk w(p, from, to); w.left > 0; w.next(p)) {
      if (left == 0) {
        // a group of scales: up to four atoms of one slice
        left = w.group(p);
        in_group = 0;
        buf = group & 1u;
        if (!(ok = wait_warp(&ctl->scales_full[buf], (group >> 1) & 1u, wc, SITE_SCALES_FULL, t))) break;
        tc_fence_after_sync();
        const uint64_t src = desc_s + uint64_t(buf * (3 * 512 >> 4));
        if (elect_one()) {
          tmem_copy_scales<false>(scale_a + buf * 4, src);
          tmem_copy_scales<false>(scale_b + buf * 8, src + (512 >> 4));
          if (p.cols > 128) tmem_copy_scales<false>(scale_b + buf * 8 + 4, src + (1024 >> 4));
        }
        ++group;
      }
      if (!(ok = wait_warp(&ctl->full[w.slot], w.turn & 1u, wc, SITE_FULL, t))) break;
      tc_fence_after_sync();
      const uint64_t dw = desc_w + uint64_t((w.slot * stage_bytes) >> 4), dx = desc_x + uint64_t((w.slot * stage_bytes) >> 4);
      const uint32_t idesc = idesc0 | umma_scale_byte(uint32_t(in_group));
      const int steps = steps_of(p, w.a);
      ++in_group;
      --left;
      if (elect_one()) {
        if (steps == 4) {
#pragma unroll
          for (int k = 0; k < 4; ++k) umma_mx8<false>(tmem_base, dw + k * wk, dx + k * 2, idesc, scale_a + buf * 4, scale_b + buf * 8, k ? 1u : more);
        } else {
          for (int k = 0; k < steps; ++k) umma_mx8<false>(tmem_base, dw + k * wk, dx + k * 2, idesc, scale_a + buf * 4, scale_b + buf * 8, k ? 1u : more);
        }
        umma_commit(&ctl->empty[w.slot]);
        if (left == 0) umma_commit(&ctl->scales_empty[buf]);
      }
      __syncwarp();
      more = 1;
    }
    if (ok && elect_one()) umma_commit(&ctl->acc_full);
    __syncwarp();
    if (__any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&ctl->abort) != 0)) {
      if (elect_one()) umma_commit(&ctl->drain);
      wait_settled(&ctl->drain, 0);
    }
  } else if (warp == 2) {
    struct Group {
      RowScales x[8];
      uint32_t w;
      bool words;
      int n;         // 0: behind the last
    };
    FewWalk at(p, from, to);
    auto load = [&](Group& x) {      // of the group that begins here, and on behind it
      x.n = 0;
      if (at.left == 0) return;
      const int a = at.a, n = x.n = at.group(p);
      x.words = p.whole_words && n == 4 && (a & 3) == 0;
      x.w = weight_byte(p, p.rs ? at.seg : rank, n0 >> 7, a, n, lane);
      const int64_t base = p.rs ? reinterpret_cast<int64_t>(p.sa[at.seg]) : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i * 32 < p.cols) x.x[i].load(reinterpret_cast<const uint8_t*>(row_at[i] + base) + a, n, x.words);
      at.a += n;
      at.left -= n;
      if (at.a == p.atoms) {
        at.a = 0;
        ++at.seg;
      }
    };
    uint32_t group = 0;
    bool ok = true;
    Group x[2];      // (two, so that what is on its way is not moved)
    load(x[0]);
    load(x[1]);
    while (ok && x[0].n > 0) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (!ok || x[u].n == 0) break;
        const uint32_t v = __shfl_sync(0xffffffffu, weight_words(x[u].w, lane), 0);
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = i * 32 < p.cols ? x[u].x[i].word(x[u].words) : kOne;
        load(x[u]);
        const uint32_t buf = group & 1u;
        if (group >= 2) {
          ok = wait_warp(&ctl->scales_empty[buf], ((group >> 1) - 1) & 1u, wc, SITE_SCALES_EMPTY, t);
          if (!ok) break;
        }
        sh->scales[buf][0][lane] = make_uint4(v, v, v, v);
        sh->scales[buf][1][lane] = make_uint4(w[0], w[1], w[2], w[3]);
        sh->scales[buf][2][lane] = make_uint4(w[4], w[5], w[6], w[7]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl->scales_full[buf]);
        ++group;
      }
    }
    for (uint32_t i = group < 2u ? group : 2u; ok && i > 0; --i)
      ok = wait_warp(&ctl->scales_empty[(group - i) & 1u], ((group - i) >> 1) & 1u, wc, SITE_DRAIN, -1);
  }

  // The sums: lanes are weight rows, columns are activation rows.
  const int quarter = warp & 3;
  bool ok = true;
  float* sums = reinterpret_cast<float*>(smem);      // [column][128], over the stages
  if (warp >= 4) {
    ok = wait_warp(&ctl->acc_full, 0, wc, SITE_ACC_FULL, t);
    tc_fence_after_sync();
    if (ok) {
      for (int c = 0; c < p.cols; c += 16) {
        uint32_t v[16];
        tmem_ld_32x32b_x16(tmem_base + (uint32_t(quarter * 32) << 16) + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[(c + i) * 128 + quarter * 32 + lane] = __uint_as_float(v[i]);
      }
    }
    tc_fence_before_sync();
  }
  __syncthreads();
  if (p.splits > 1) {
    // One warp's release stands for all, behind the block's barrier.  (A warp arrives as one: its threads must not part here.)
    if (warp == 0) cluster_arrive();
    else cluster_arrive_relaxed();
    cluster_wait();
  }
  if (*reinterpret_cast<volatile int*>(&ctl->abort) == 0) {
    // four neighbouring sums a thread, those of all CTAs of a cluster in flight together
    const uint32_t base = smem_u32(sums);
    const int n = lane * 4;
    for (int i = part + p.splits * warp; i < shards * rows; i += p.splits * (kFewThreads / 32)) {
      // the i-th row of the tile: of which shard, and its accumulator column
      const int s = shards == 1 ? 0 : int(p.each.div(uint32_t(i))), row = i - s * rows;
      const uint32_t at = base + uint32_t((s * int(p.slot.d) + row) * 128 + n) * 4;
      if (n0 + n >= p.N) continue;      // (only what is stored is read, and so has been read before the warp says that the others may leave)
      float4 y[kMostSplits];
#pragma unroll
      for (int k = 0; k < kMostSplits; ++k)
        if (k < p.splits)
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(y[k].x), "=f"(y[k].y), "=f"(y[k].z), "=f"(y[k].w)
                       : "r"(map_to_cta(at, uint32_t(k))));
      float4 x = y[0];
#pragma unroll
      for (int k = 1; k < kMostSplits; ++k)
        if (k < p.splits) x.x += y[k].x, x.y += y[k].y, x.z += y[k].z, x.w += y[k].w;
      __nv_bfloat16* out;
      if (p.rs) {
        const int chunk = int(p.each.div(uint32_t(row0 + row)));
        out = p.out[chunk] + int64_t(row0 + row - chunk * p.m) * p.N;
      } else {
        out = p.out[rank] + (int64_t(shard0 + s) * p.m + row0 + row) * p.N;
      }
      out += n0 + n;
      if (p.wide) {      // (N is a multiple of 8)
        *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w));
      } else {
        const float z[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (n0 + n + k < p.N) out[k] = __float2bfloat16_rn(z[k]);
      }
    }
  }
  if (p.splits > 1) {
    __syncwarp();
    cluster_arrive_relaxed();      // nobody's memory goes while it is read
    cluster_wait();
  }
  if (warp == 1) {
    __syncwarp();
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, uint32_t(p.tmem_cols));
  }
}

// ---- host ----------------------------------------------------------------------

int check_problem8(const compass_problem* g, int op) {
  if (g == nullptr) return COMPASS_ERR_INVALID_ARG;
  if (g->op != op) return COMPASS_ERR_INVALID_ARG;
  const int st = check_problem_8bit(g);
  if (st != COMPASS_OK) return st;
  // weights [K][N] are read along N
  return g->b_layout == COMPASS_B_KN && g->N % 16 != 0 ? COMPASS_ERR_ALIGNMENT : COMPASS_OK;
}

struct DeviceFacts {
  bool ready = false;
  int pairs = 0, sms = 0;
  int few[kMostSplits + 1] = {};      // clusters of n CTAs of the few-rows kernel that fit, one CTA per SM
};
int device_facts(DeviceFacts** out) {
  constexpr int kMaxDevices = 64;
  static DeviceFacts facts[kMaxDevices];
  static std::mutex mu;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return record_cuda_error(e);
  if (dev < 0 || dev >= kMaxDevices) return COMPASS_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(mu);
  DeviceFacts& f = facts[dev];
  if (!f.ready) {
    e = cudaFuncSetAttribute(gemm8_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kPairSmemBytes));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gemm8_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&f.sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(f.sms / 2 * 2));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kPairSmemBytes;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&f.pairs, gemm8_pair_kernel, &cfg);
    if (e != cudaSuccess) return record_cuda_error(e);
    if (f.pairs < 1) return COMPASS_ERR_UNSUPPORTED;
    for (int n = 1; n <= kMostSplits; ++n) {
      cfg.gridDim = dim3(unsigned(f.sms / n * n));
      cfg.blockDim = dim3(kFewThreads);
      cfg.dynamicSmemBytes = 1024 + size_t(kFewRoom) + sizeof(FewShared);
      attr.val.clusterDim.x = unsigned(n);
      e = cudaOccupancyMaxActiveClusters(&f.few[n], gemm8_few_kernel, &cfg);
      if (e != cudaSuccess) return record_cuda_error(e);
      if (f.few[n] < 1) return COMPASS_ERR_UNSUPPORTED;
    }
    f.ready = true;
  }
  *out = &f;
  return COMPASS_OK;
}

// How long a call takes, in cycles, by what an atom of a tile takes: the products, or its operands at 60 bytes a clock from L2 (2.1
// cycles a row of 128 bytes), whatever is more; and what a tile takes besides.  Of the widths, splits and kernels the one with the
// shortest time is taken.  Measured, the pair kernel against the other: 1024 x 1024 x 256 rows 5.6 us : 14, 4096 x 4096 x 512 rows 13.0 :
// 18.5, 2 ranks' 5003 x 2064 x 59 rows 12.8 : 15.9; GEMM+ReduceScatter of 8 ranks 752 x 4096 x 1136 rows 66 : 36, [K][N] 87 : 39; 82 x
// 7392 x 1571 rows 17.6 : 12.0, 4096 x 4096 x 1 row 17 : 6.
double atom_cycles(double products, double rows) { return products > 2.1 * rows ? products : 2.1 * rows; }

// Columns of a pair's tile: 2 cycles of products each.  For each CTA 128 rows of A and half of its columns of B, or (weights [K][N])
// 128 of the contraction whatever the width.  Tiles are of equal width as far as n_step allows, so that none is a narrow rest that
// still loads all of A.
struct PairPlan {
  int bn;
  double cost;
};
PairPlan pair_plan(int64_t N, int64_t row_tiles, int64_t atoms, int step, bool kn, int pairs) {
  PairPlan best = {256, 0};
  for (int most = 256; most >= 64; most -= 32) {
    const int64_t tiles = ceil_div(N, most);
    const int bn = int(ceil_div(ceil_div(N, tiles), step) * step);
    const double tile = double(atoms) * atom_cycles(2.0 * bn, 128 + (kn ? 128 : bn / 2)) + 1500;
    const double cost = double(ceil_div(row_tiles * ceil_div(N, bn), pairs)) * tile;
    if (best.cost == 0 || cost < 0.98 * best.cost) best = {bn, cost};
  }
  return best;
}

// The other kernel's row tiles: whole shards, as many as fit, or equal pieces of one; and over how many CTAs each one's contraction is
// split.  Their sums cost two barriers of the cluster and some 30 cycles a column.
bool few_two(int64_t cols, int64_t ctas, int sms) { return ctas > sms && cols <= 128; }      // two CTAs per SM
// Clusters of n CTAs that run at once.  The occupancy query answers for one CTA per SM, whatever its shared memory.  With two, twice as many
// fit, and some on what is left of the SMs: one for n SMs, but no more than there are clusters of n / 2, whose SMs one of n takes; where n
// is odd, two thirds of that.  Clusters of 2, 3 .. 8: 148, 92, 70, 54, 45, 34, 33, where in time 148, 92, 71, 55, 45, 37, 33 do (one more, and
// a token's product takes 9.5 to 10 us instead of 5.6 to 6.1).
int64_t few_fit(const DeviceFacts& d, int n, bool two) {
  if (!two) return d.few[n];
  const int left = d.sms - n * d.few[n];
  if (n % 2 != 0) return 2 * d.few[n] + 2 * left / n / 3;
  return 2 * d.few[n] + left / n < d.few[n / 2] ? 2 * d.few[n] + left / n : d.few[n / 2];
}
struct FewPlan {
  int64_t shards, pieces, rows, slot, cols, row_tiles;
  int splits;
  double cost;
};
FewPlan few_plan(bool rs, int P, int64_t m, int64_t n_tiles, int64_t all, const DeviceFacts& d) {
  FewPlan f = {};
  const int64_t whole = rs ? m * P : m;      // rows of a tensor of activations
  f.shards = f.pieces = 1;
  f.rows = whole;
  if (whole > kFewMostCols) {
    f.pieces = ceil_div(whole, kFewMostCols);
    f.rows = int64_t(round_up(size_t(ceil_div(whole, f.pieces)), 8));
    f.pieces = ceil_div(whole, f.rows);
  }
  f.slot = int64_t(round_up(size_t(f.rows), 8));
  if (!rs && f.pieces == 1) {
    f.shards = kFewMostCols / f.slot < P ? kFewMostCols / f.slot : P;
    f.shards = ceil_div(P, ceil_div(P, f.shards));
  }
  f.cols = int64_t(round_up(size_t(f.shards * f.slot), 16));
  f.row_tiles = f.pieces * (rs ? 1 : ceil_div(P, f.shards));
  const int64_t tiles = n_tiles * f.row_tiles * (rs ? 1 : P);
  double atom = atom_cycles(2.0 * double(f.cols), 128 + double(f.shards * f.rows));
  if (atom < 550) atom = 550;      // (measured, whatever the columns)
  for (int n = 1; n <= kMostSplits && (n == 1 || 2 * n <= all); ++n) {
    // Clusters that do not fit at once take as long again (2048 x 8192 x 16 rows, 16 clusters of 8 where 15 fit: 13.4 us, of 6 8.8; two CTAs
    // per SM, 4096 x 5760 x 1 row, 45 of 6: 7.6 us, 46 12.8), which can still be the least (4096 x 25600 x 1 row, 200 of 2: 26.7 us, of 1 29).
    const double tile = double(ceil_div(all, n)) * atom + 1500;
    const double cost = n > 1 ? double(ceil_div(tiles, few_fit(d, n, few_two(f.cols, tiles * n, d.sms)))) * (tile + 2000.0 + 30.0 * double(f.cols))
                              : double(ceil_div(tiles, d.sms)) * tile + 10.0 * double(f.cols);
    if (f.splits == 0 || cost < f.cost) {
      f.splits = n;
      f.cost = cost;
    }
  }
  return f;
}

int launch_clusters(void (*kernel)(const Gemm8Params), int64_t grid, int threads, size_t smem, int cluster, const Gemm8Params& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(grid));
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(cluster);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  count_kernel_launch();
  return e == cudaSuccess ? COMPASS_OK : record_cuda_error(e);
}

int run_product(const compass_problem* g, int op, const void* const* A, const void* const* sA, const void* const* B, const void* const* sB,
                void* const* out, void* ws, size_t ws_bytes, void* stream) {
  int st = check_problem8(g, op);
  if (st != COMPASS_OK) return st;
  if (!A || !sA || !B || !sB || !out) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < g->P; ++r)
    if (!A[r] || !sA[r] || !B[r] || !sB[r] || !out[r]) return COMPASS_ERR_INVALID_ARG;
  for (int r = 0; r < g->P; ++r)
    if (!is_aligned(A[r], 16) || !is_aligned(B[r], 16) || !is_aligned(out[r], 2)) return COMPASS_ERR_ALIGNMENT;
  st = check_workspace(ws, ws_bytes, COMPASS_STATUS_BYTES);
  if (st != COMPASS_OK) return st;
  DeviceFacts* f;
  st = device_facts(&f);
  if (st != COMPASS_OK) return st;

  Gemm8Params p = {};
  p.rs = op == COMPASS_OP_GEMM_RS;
  p.P = g->P;
  p.m = int32_t(g->M / g->P);
  p.K = int32_t(g->K);
  p.N = g->N;
  p.atoms = int32_t(scale_blocks(g->K));
  p.kn = g->b_layout == COMPASS_B_KN;
  p.n_blocks = int32_t(scale_blocks(g->N));
  p.a_format = format_of(g->dtype);
  p.status = static_cast<StatusBlock*>(ws);
  p.wait_limit_us = default_wait_limit_us() ? default_wait_limit_us() : 2000000u;
  p.whole_words = 1;
  p.wide = g->N % 16 == 0 ? 2 : g->N % 8 == 0 ? 1 : 0;
  for (int r = 0; r < g->P; ++r) {
    p.sa[r] = static_cast<const uint8_t*>(sA[r]);
    p.sb[r] = static_cast<const uint8_t*>(sB[r]);
    p.out[r] = static_cast<__nv_bfloat16*>(out[r]);
    if (p.wide == 2 && !is_aligned(out[r], 32)) p.wide = 1;
    if (!is_aligned(out[r], 16)) p.wide = 0;
    if (p.atoms % 4 != 0 || !is_aligned(sA[r], 4)) p.whole_words = 0;
  }
  const int64_t a_rows = p.rs ? g->M : p.m;
  const int64_t b_rows = p.kn ? g->K : g->N, b_cols = p.kn ? g->N : g->K;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  bool ok = true;
  const int64_t n_tiles = scale_blocks(g->N), ranks = p.rs ? 1 : g->P, all = (p.rs ? g->P : 1) * int64_t(p.atoms);
  const FewPlan few = few_plan(p.rs, g->P, p.m, n_tiles, all, *f);
  p.frags = int32_t(ceil_div(p.m, 128));
  p.row_tiles = int32_t(ceil_div(int64_t(p.frags) * g->P, 2));
  p.n_step = p.kn ? 32 : 16;
  const PairPlan pair = pair_plan(g->N, p.row_tiles * ranks, all, p.n_step, p.kn, f->pairs);
  const int64_t few_tiles = n_tiles * few.row_tiles * ranks;
  if (few.cost < pair.cost && few_tiles * few.splits <= kMaxDim) {
    p.tile_shards = int32_t(few.shards);
    p.tile_rows = int32_t(few.rows);
    p.slot.set(uint32_t(few.slot));
    p.pieces.set(uint32_t(p.rs ? 1 : few.pieces));
    p.by_rows.set(uint32_t(few.row_tiles));
    p.each.set(uint32_t(p.m));
    p.by_tiles.set(uint32_t(n_tiles));
    p.cols = int32_t(few.cols);
    p.n_tiles = int32_t(n_tiles);
    p.splits = few.splits;
    const int64_t cols = few.cols, tiles = few_tiles;
    p.all = int32_t(all);
    p.by_splits.set(uint32_t(p.splits));
    const int stage = few_stage_bytes(p.cols);
    const int64_t mine = ceil_div(all, p.splits);
    const int room = few_two(cols, tiles * p.splits, f->sms) ? kFewHalfRoom : kFewRoom;
    int64_t stages = room / stage;
    if (stages > mine) stages = mine;
    if (stages > kFewMostStages) stages = kFewMostStages;
    // (the sums lie where the stages were)
    while (stages * stage < cols * 512) ++stages;
    p.stages = int32_t(stages);
    p.tmem_cols = 32;
    while (p.tmem_cols < p.cols + 24) p.tmem_cols *= 2;
    p.b_box = p.kn || g->N > 128 ? 128 : int32_t(g->N);
    for (int r = 0; r < g->P; ++r) {
      ok = ok && encode_tensor_map_bytes(&p.a[r], A[r], a_rows, g->K, p.tile_rows);
      ok = ok && encode_tensor_map_bytes(&p.b[r], B[r], b_rows, b_cols, p.b_box);
    }
    if (!ok) return record_cuda_error(cudaErrorUnknown);
    // the CTAs of a cluster wait for one another while they hold tensor memory
    size_t smem = few_smem_bytes(p.cols, p.stages);
    if (p.splits > 1) {
      const size_t least = p.tmem_cols <= 256 ? kHalfTmemShared : kFewAll;
      if (smem < least) smem = least;
    }
    return launch_clusters(gemm8_few_kernel, tiles * p.splits, kFewThreads, smem, p.splits, p, s);
  }
  p.bn = pair.bn;
  p.col_tiles = int32_t(ceil_div(g->N, p.bn));
  const int64_t total = int64_t(p.row_tiles) * p.col_tiles * (p.rs ? 1 : g->P);
  if (total > kMaxDim) return COMPASS_ERR_UNSUPPORTED;
  p.total = int32_t(total);
  p.per_rank.set(uint32_t(p.row_tiles) * uint32_t(p.col_tiles));
  p.per_group.set(uint32_t(kRowGroup) * uint32_t(p.col_tiles));
  p.by_frags.set(uint32_t(p.frags));
  p.a_box = a_rows < 128 ? int32_t(a_rows) : 128;
  p.b_box = p.kn ? 128 : g->N < p.bn / 2 ? int32_t(g->N) : p.bn / 2;
  for (int r = 0; r < g->P; ++r) {
    ok = ok && encode_tensor_map_bytes(&p.a[r], A[r], a_rows, g->K, p.a_box);
    ok = ok && encode_tensor_map_bytes(&p.b[r], B[r], b_rows, b_cols, p.b_box);
  }
  if (!ok) return record_cuda_error(cudaErrorUnknown);
  return launch_clusters(gemm8_pair_kernel, 2 * (total < f->pairs ? total : f->pairs), kPairThreads, kPairSmemBytes, 2, p, s);
}

}  // namespace

// What the products and the weight gradient of 8-bit activations ask of a description.
int check_problem_8bit(const compass_problem* g) {
  if (g->P < 1 || (g->op != COMPASS_OP_AG_GEMM && g->op != COMPASS_OP_GEMM_RS)) return COMPASS_ERR_INVALID_ARG;
  if (g->P > kMaxP) return COMPASS_ERR_UNSUPPORTED;
  if (g->M <= 0 || g->N <= 0 || g->K <= 0 || g->M % g->P != 0) return COMPASS_ERR_SHAPE;
  if (g->M > kMaxDim || g->N > kMaxDim || g->K > kMaxDim) return COMPASS_ERR_UNSUPPORTED;
  if (format_of(g->dtype) < 0 || g->rs_variant != COMPASS_RS_SEGMENTED_K) return COMPASS_ERR_UNSUPPORTED;
  if (g->b_layout != COMPASS_B_NK && g->b_layout != COMPASS_B_KN) return COMPASS_ERR_INVALID_ARG;
  return g->K % 16 == 0 ? COMPASS_OK : COMPASS_ERR_ALIGNMENT;
}

}  // namespace compass

using namespace compass;

extern "C" int compass_8bit_workspace_bytes(const compass_problem* g, size_t* bytes) {
  if (g == nullptr || bytes == nullptr) return COMPASS_ERR_INVALID_ARG;
  const int st = check_problem_8bit(g);
  if (st != COMPASS_OK) return st;
  *bytes = COMPASS_STATUS_BYTES;
  return COMPASS_OK;
}

extern "C" int compass_ag_gemm_8bit(const compass_problem* g, const void* const* A, const void* const* A_scale, const void* const* B,
                                    const void* const* B_scale, void* const* C, void* ws, size_t ws_bytes, void* stream) {
  return run_product(g, COMPASS_OP_AG_GEMM, A, A_scale, B, B_scale, C, ws, ws_bytes, stream);
}

extern "C" int compass_gemm_rs_8bit(const compass_problem* g, const void* const* A, const void* const* A_scale, const void* const* B,
                                    const void* const* B_scale, void* const* Out, void* ws, size_t ws_bytes, void* stream) {
  return run_product(g, COMPASS_OP_GEMM_RS, A, A_scale, B, B_scale, Out, ws, ws_bytes, stream);
}
