// Softmax cross entropy of the vocabulary-parallel output layer, forward and
// backward, without the logits.
//
// Rows whose target lies outside the vocabulary take no part: head_count_kernel
// counts the others and head_gather_kernel copies them together, so that the
// products run over real rows only, whatever the mask and the ranks' shards.
// Then one kernel in three forms (tcgen05 products of BF16 with FP32 sums):
//   STATS  logits of 256 vocabulary columns at a time; what leaves the epilogue
//          is each row's maximum and sum of exponentials over 128 columns
//   GRAD   the same product again; the epilogue writes the logits' gradient
//          (BF16) of one piece of the vocabulary
//   SUMS   the two products of that piece, in one launch, so that the one's
//          tiles fill the other's last round: DX, the piece times the table,
//          added to the FP32 sums of dX, and DW, the piece, transposed, times X:
//          dW of the piece
// The backward pass is bound by the tensor cores: 6 M hidden vocab operations.
// Measured: forward, 7392 rows, 4096 x 32000, 1.28 ms alone = 1.52 PFLOP/s (the
// library's 8192^3 product reaches 1.65), 1.51 ms = 1.29 in a loop at the power
// limit (1.37); backward, 7392 rows, 4096 x 128000, 18.1 ms = 1.28 PFLOP/s at that
// limit; backward, 401 rows, 1024 x 50001, 200 us = 0.62 PFLOP/s (every tile's part
// of the table comes from HBM, and three launches ramp up and down).
// With few rows or a small hidden size it is far from either bound: one row tile
// takes 256 rows' work, launches and epilogues are what takes the time (backward,
// 8 rows, 4096 x 32000: 232 us, 2.9 times the table's bytes; 8192 rows, 64 x 32000:
// 685 us, 11 times its operations).
// The tensor cores' FP32 sums cut off what they cannot hold, a little at each step.
// The statistics' sums are therefore short, 1024 elements of the contraction, and
// added up in FP32: losses and lse are 5e-7 to 7e-7 off (relative, root mean
// square), as with FP32 arithmetic; in one sum they were 2.5e-6 off over 4096
// elements and 5.5e-6 over 8192. What goes to BF16 afterwards keeps one sum.
// The logits' gradient is rounded to BF16 because its products take BF16 operands
// (in two BF16 halves it would double both products, 4 of 6 M hidden vocab). What
// that costs, relative and root mean square: dW in FP32 is 0.9e-3 to 1.4e-3 off,
// gradients in BF16 1.9e-3 to 2.2e-3, of which their own rounding is 1.7e-3.
//
// Tiles are computed by pairs of CTAs: 512 x 256 as long as they fill whole
// rounds of the pairs (two accumulators that share one tile of B: 48 bytes of
// operands per SM and clock at the tensor cores' full rate, against 64 for
// 256 x 256), 256 x 256 for the rest, and for all of the statistics, whose short
// sums need registers and the second accumulator for a tile.  Warp 0 loads (TMA), warp 1 issues the
// products, warps 2..9 are the epilogue: two per quarter of the rows, 128
// columns each, so that a whole accumulator is in registers, and its tensor
// memory free again, before the exponentials begin.
#include <mutex>
#include <type_traits>

#include "ptx_sm100.cuh"
#include "row_ops.cuh"

namespace compass {

using namespace ptx;

namespace {

enum Form : int { STATS = 0, GRAD = 1, SUMS = 2, DX = 3, DW = 4 };      // (DX and DW: of a SUMS tile)

constexpr int kThreads = 320;
constexpr int kEpiWarps = 8;
constexpr int kSlots = 4;
constexpr int kChunkBytes = 128 * BK * 2;       // 16 KB: 128 rows (or columns) of one 64-wide k-atom
constexpr int kHalfChunk = kChunkBytes / 2;     // an MN-major operand is two boxes of 64 columns x 64 k-rows
constexpr int kChunks = 12;
constexpr int kGroup = 8;                       // row tiles that go through the columns together (their A stays in L2)
constexpr int kSkew = 3;                        // stages at a tile's ends in which accumulator 0 runs ahead
// The statistics' logits are summed up in ranges of the contraction, this many 64-wide k-atoms each, which the epilogue adds in
// FP32.  8192 (7392) rows, 4096 x 32000, in one range with 512 x 256 tiles, in one with 256 x 256, in ranges of 32, 16 and 8:
// 1470, 1495, 1550, 1572, 1634 us (before the additions were rid of spilled registers, which brought 16 to 1515); losses
// 2.9e-6, 2.9e-6, 1.5e-6, 6.9e-7, 3.3e-7 off.  FP32 arithmetic: 6.4e-7.
constexpr int kRangeAtoms = 16;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// 2^x, relative error 2^-22; results below 2^-126 are zero (of a sum that is at least 1, or of a BF16 gradient).
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What the kernels before the products found out.
struct Found {
  int32_t rows;      // that take part
  float top;         // max |dloss| over them (1 if that is not finite)
};

struct HeadParams {
  CUtensorMap x_k;              // gathered X [pad][hidden]: boxes of 128 rows (A of the logits), of few_cols with few rows
  CUtensorMap x_mn;             // boxes of 64 rows (B of dW)
  CUtensorMap d_k, d_mn;        // the piece's gradient [pad][piece_cols]: A of dX; A of dW
  CUtensorMap w_k[kMaxP], w_mn[kMaxP];
  void* dw[kMaxP];
  const Found* found;
  const int32_t* target;        // of the gathered rows
  const float* lse2;            // in units of log 2
  const float* weight;          // dloss of the gathered rows
  float2* part;                 // [2 * vocab tiles][pad] (maximum, sum), in units of log 2
  float* part_sum;              // [2 * vocab tiles][pad] sum of logits (label smoothing)
  float* target_logit;          // [pad]
  __nv_bfloat16* d;             // the piece's gradient
  float4* acc;                  // FP32 sums of dX, in the order the epilogue's lanes hold them
  StatusBlock* status;
  int64_t hidden;
  int32_t pad;                  // rows of the workspace's arrays, a multiple of 512
  int32_t vocab_rows;           // rows per shard
  int32_t vocab;
  int32_t tiles_per_shard;
  int32_t vt0, n_vt;            // the piece: vocabulary tiles [vt0, vt0 + n_vt)
  int32_t piece_cols;           // row pitch of d
  int32_t hidden_tiles;
  int32_t splits;               // of dX's contraction
  int32_t first_piece;
  int32_t one_row_tile;         // M <= 256
  int32_t few_cols;             // head_few_kernel: M rounded up to a multiple of 16
  int32_t grad_fp32;
  int32_t dw_wide;              // dW's rows are whole 32-byte sectors
  float z_scale;                // logit_scale * log2(e)
  float out_scale;              // logit_scale
  float smoothing, uniform;     // label_smoothing, label_smoothing / vocab
  uint32_t wait_limit_us;
};

struct Control {
  uint64_t full[kSlots], empty[kSlots];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t drain;
  uint32_t tmem_base;
  int abort;
};

constexpr size_t kSmemBytes = 1024 + size_t(kChunks) * kChunkBytes + sizeof(Control);
static_assert(keeps_tmem_apart(kSmemBytes), "");

enum Site : int { SITE_EMPTY = 1, SITE_FULL = 2, SITE_ACC_EMPTY = 3, SITE_ACC_FULL = 4, SITE_DRAIN = 5 };

__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, Control* ctl, const HeadParams& p, int site, int tile) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  const uint64_t limit = uint64_t(p.wait_limit_us) * 1000ull;
  for (uint32_t spins = 1; spins < (1u << 30); ++spins) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((spins & 0xFF) == 0) {
      if (*reinterpret_cast<volatile int*>(&ctl->abort)) return false;
      if (globaltimer_ns() - t0 > limit) break;
    }
  }
  *reinterpret_cast<volatile int*>(&ctl->abort) = 1;
  if (atomicCAS(&p.status->code, 0, int(COMPASS_ERR_TIMEOUT)) == 0) {
    p.status->detail = site;
    p.status->block_idx = int(blockIdx.x);
    p.status->tile = tile;
  }
  return false;
}

// After giving up: wait for copies or products in flight, whatever the others do, before this CTA's memory may go (100 ms at
// most).
__device__ __forceinline__ void wait_landed(uint64_t* bar, uint32_t parity) {
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t spins = 1; spins < (1u << 30) && !mbar_try_wait(bar, parity); ++spins)
    if ((spins & 0xFF) == 0 && globaltimer_ns() - t0 > 100000000ull) break;
}

// How a product's output is cut into tiles; the number of rows is known on the device only.
struct Part {
  int big_rows;        // row tiles of 512
  int odd;             // one more of 256
  int cols;            // column tiles (of all splits)
  int n_big, left;     // 512 x 256 tiles; slots left over, two 256 x 256 tiles each
  int total;
  int atoms;           // 64-wide k-atoms of a tile (an even number)
};
// Whole rounds of the units take 512 x 256 tiles, what is left, and all of STATS, 256 x 256 ones.  `before`: tiles of the launch that come first;
// the tiles go to the units in turn, so that a unit that has had one of its last, smaller ones gets its share of these later.
__device__ __forceinline__ Part make_part(const HeadParams& p, int form, int units, int before) {
  Part q;
  const int found = max(p.found->rows, 1);      // at least one tile: its zeros are what dW reads when no row takes part
  const int halves = form == DW ? p.n_vt : (found + 255) / 256;
  q.big_rows = halves / 2;
  q.odd = halves & 1;
  q.cols = form == DW ? p.hidden_tiles : form == DX ? p.hidden_tiles * p.splits : p.n_vt;
  const int slots = q.big_rows * q.cols;
  q.left = form == STATS ? slots : min(slots, (before + slots) % units);
  q.n_big = slots - q.left;
  q.total = q.n_big + 2 * q.left + q.odd * q.cols;
  q.atoms = form == DW ? (found + 127) / 128 * 2 : form == DX ? 4 * p.n_vt : int((p.hidden + 127) / 128) * 2;
  return q;
}
// Ranges of a 256 x 256 tile's contraction, the last one shorter.
__device__ __forceinline__ int ranges_of(int form, int atoms) { return form == STATS ? (atoms + kRangeAtoms - 1) / kRangeAtoms : 1; }
struct Plan {
  Part part[2];        // SUMS: DX, DW; else the first alone
  int total;
};
template <int kForm>
__device__ __forceinline__ Plan make_plan(const HeadParams& p, int units) {
  Plan q = {};
  if (kForm == SUMS) {
    q.part[0] = make_part(p, DX, units, 0);
    q.part[1] = make_part(p, DW, units, q.part[0].total);
  } else {
    q.part[0] = make_part(p, kForm, units, 0);
  }
  q.total = q.part[0].total + q.part[1].total;
  return q;
}
struct Tile {
  int form;
  bool big;
  int row0;            // first of 512 or 256 rows
  int col;             // column tile
  int atom0, atoms;    // range of the contraction
};
template <int kForm>
__device__ __forceinline__ Tile tile_of(const HeadParams& p, const Plan& plan, int t) {
  Tile c;
  const bool second = kForm == SUMS && t >= plan.part[0].total;
  const Part& q = plan.part[second ? 1 : 0];
  if (second) t -= plan.part[0].total;
  c.form = kForm != SUMS ? kForm : second ? int(DW) : int(DX);
  c.big = t < q.n_big;
  int slot = t, half = 0;
  const int u = t - q.n_big;
  if (!c.big && u >= 2 * q.left) {
    c.row0 = q.big_rows * 512;
    c.col = u - 2 * q.left;
  } else {
    if (!c.big) {
      slot = q.n_big + (u >> 1);
      half = u & 1;
    }
    const int g = slot / (kGroup * q.cols);
    const int rest = slot - g * (kGroup * q.cols);
    const int wide = min(kGroup, q.big_rows - g * kGroup);
    c.col = rest / wide;
    c.row0 = (g * kGroup + rest - c.col * wide) * 512 + half * 256;
  }
  c.atom0 = 0;
  c.atoms = q.atoms;
  if (c.form == DX && p.splits > 1) {
    // whole vocabulary tiles (4 atoms) per split
    const int s = c.col / p.hidden_tiles;
    const int from = int(int64_t(p.n_vt) * s / p.splits), to = int(int64_t(p.n_vt) * (s + 1) / p.splits);
    c.atom0 = 4 * from;
    c.atoms = 4 * (to - from);
  }
  return c;
}

// This CTA's 128 rows of A of one k-atom.
__device__ __forceinline__ void load_a(const HeadParams& p, int form, uint8_t* dst, uint32_t bar, int row, int atom, uint64_t pol) {
  if (form == DW) {
    tma_load_2d_pair_hint(dst, &p.d_mn, bar, row, atom * BK, pol);
    tma_load_2d_pair_hint(dst + kHalfChunk, &p.d_mn, bar, row + 64, atom * BK, pol);
  } else {
    tma_load_2d_pair_hint(dst, form == DX ? &p.d_k : &p.x_k, bar, atom * BK, row, pol);
  }
}
// This CTA's 128 columns of B of one k-atom.
__device__ __forceinline__ void load_b(const HeadParams& p, int form, uint8_t* dst, uint32_t bar, int col_tile, int cta, int atom, uint64_t pol) {
  if (form == DW) {
    const int col = col_tile * 256 + cta * 128;
    tma_load_2d_pair_hint(dst, &p.x_mn, bar, col, atom * BK, pol);
    tma_load_2d_pair_hint(dst + kHalfChunk, &p.x_mn, bar, col + 64, atom * BK, pol);
  } else if (form == DX) {
    const int col = (p.splits > 1 ? col_tile % p.hidden_tiles : col_tile) * 256 + cta * 128;
    const int vt = p.vt0 + (atom >> 2);
    const int shard = vt / p.tiles_per_shard;
    const int row = (vt - shard * p.tiles_per_shard) * 256 + (atom & 3) * BK;
    tma_load_2d_pair_hint(dst, &p.w_mn[shard], bar, col, row, pol);
    tma_load_2d_pair_hint(dst + kHalfChunk, &p.w_mn[shard], bar, col + 64, row, pol);
  } else {
    const int vt = p.vt0 + col_tile;
    const int shard = vt / p.tiles_per_shard;
    tma_load_2d_pair_hint(dst, &p.w_k[shard], bar, atom * BK, (vt - shard * p.tiles_per_shard) * 256 + cta * 128, pol);
  }
}

// 32 bytes, one sector, at a 32-byte boundary.  (Measured and not kept: the results of an accumulator held back until the
// next one has been read, so that its tensor memory is free before they are stored: 200 -> 209 us at 401 x 1024 x 50001.)
__device__ __forceinline__ void store_32(void* p, const uint32_t (&q)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3]), "r"(q[4]),
               "r"(q[5]), "r"(q[6]), "r"(q[7])
               : "memory");
}
// The same at a 16-byte boundary where rows are not whole sectors, `both` halves or the first.
__device__ __forceinline__ void store_row_piece(void* p, const uint32_t (&q)[8], bool wide, bool both) {
  if (wide) {
    store_32(p, q);
  } else {
    uint4* o = static_cast<uint4*>(p);
    o[0] = make_uint4(q[0], q[1], q[2], q[3]);
    if (both) o[1] = make_uint4(q[4], q[5], q[6], q[7]);
  }
}

// Vocabulary columns that exist in a tile.
__device__ __forceinline__ int vocab_cols(const HeadParams& p, int vt, int* shard, int* row) {
  *shard = vt / p.tiles_per_shard;
  *row = (vt - *shard * p.tiles_per_shard) * 256;
  const int64_t rows = min(int64_t(p.vocab_rows), int64_t(p.vocab) - int64_t(*shard) * p.vocab_rows);
  return int(min(int64_t(256), rows - *row));
}

template <int kForm>
__global__ void __launch_bounds__(kThreads, 1) head_kernel(const __grid_constant__ HeadParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  Control* ctl = reinterpret_cast<Control*>(smem + kChunks * kChunkBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t cta = cluster_ctarank();
  const bool leader = cta == 0;
  const int unit = int(blockIdx.x >> 1), units = int(gridDim.x >> 1);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->acc_full[b], 1);
      mbar_init(&ctl->acc_empty[b], 2 * kEpiWarps);
    }
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
  const uint32_t tmem_base = ctl->tmem_base;
  launch_dependents();
  const uint64_t pol = make_l2_policy(L2_EVICT_NORMAL);
  // The first stages' tiles of the table do not depend on the kernels before (which list and gather the rows): with one row
  // tile, whose place among the tiles is known, they are on their way before those are done.
  int early = 0;
  if ((kForm == STATS || kForm == GRAD) && p.one_row_tile && threadIdx.x == 0 && unit < p.n_vt) {
    const int stages = min(3, int((p.hidden + 127) / 128));
    for (; early < stages; ++early) {
      const uint32_t bar = map_to_cta(smem_u32(&ctl->full[early]), 0);
      if (leader) mbar_arrive_expect_tx(&ctl->full[early], uint32_t(8 * kChunkBytes));
      for (int i = 0; i < 2; ++i)
        load_b(p, kForm, smem + (early * 4 + 2 + i) * kChunkBytes, bar, unit, int(cta), early * 2 + i, pol);
    }
  }
  wait_for_previous_kernel();
  const Plan plan = make_plan<kForm>(p, units);

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      uint32_t j = 0;          // stages so far
      uint32_t last_small = 0u - 4u;   // the last 256x256 one
      int chunk = 0;           // ring cursor
      bool ok = true;
      for (int t = unit; ok && t < plan.total; t += units) {
        const Tile tile = tile_of<kForm>(p, plan, t);
        const int row = tile.row0 + int(cta) * (tile.big ? 256 : 128);
        const int step = tile.big ? 1 : 2;
        for (int a = 0; a < tile.atoms; a += step, ++j) {
          // Four 512x256 stages (3 chunks each) fill the ring; with a 256x256 stage (4 chunks) among the last three, a stage
          // must not overwrite anything newer than the third before it.
          const uint32_t depth = tile.big && j - last_small > 3u ? 4u : 3u;
          if (!tile.big) last_small = j;
          if (j >= depth) {
            const uint32_t r = j - depth;
            if (!wait_bar(&ctl->empty[r & 3u], (r >> 2) & 1u, ctl, p, SITE_EMPTY, t)) {
              ok = false;
              break;
            }
          }
          const uint32_t slot = j & 3u;
          const uint32_t bar = map_to_cta(smem_u32(&ctl->full[slot]), 0);
          const int n = tile.big ? 3 : 4;
          const bool b_sent = j < uint32_t(early);
          if (leader && !b_sent) mbar_arrive_expect_tx(&ctl->full[slot], uint32_t(2 * n * kChunkBytes));
          uint8_t* c[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) c[i] = smem + ((chunk + i) % kChunks) * kChunkBytes;
          const int atom = tile.atom0 + a;
          if (tile.big) {
            load_a(p, tile.form, c[0], bar, row, atom, pol);
            load_a(p, tile.form, c[1], bar, row + 128, atom, pol);
            load_b(p, tile.form, c[2], bar, tile.col, int(cta), atom, pol);
          } else {
            load_a(p, tile.form, c[0], bar, row, atom, pol);
            if (!b_sent) load_b(p, tile.form, c[2], bar, tile.col, int(cta), atom, pol);
            load_a(p, tile.form, c[1], bar, row, atom + 1, pol);
            if (!b_sent) load_b(p, tile.form, c[3], bar, tile.col, int(cta), atom + 1, pol);
          }
          chunk = (chunk + n) % kChunks;
        }
      }
      // leave only when the last stages have been read (the leader's products read both CTAs' chunks)
      const uint32_t back = j < 4u ? j : 4u;
      for (uint32_t i = 1; i <= back; ++i) {
        const uint32_t r = j - i;
        if (!wait_bar(&ctl->empty[r & 3u], (r >> 2) & 1u, ctl, p, SITE_DRAIN, -1)) {
          // (the leader's barriers count both CTAs' copies, and neither CTA ends before the other)
          if (leader)
            for (uint32_t k = 1; k <= back; ++k) wait_landed(&ctl->full[(j - k) & 3u], ((j - k) >> 2) & 1u);
          break;
        }
      }
    }
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA issuer
    if (leader && lane == 0) {
      const uint64_t desc_k = umma_smem_desc_sw128(smem_u32(smem));
      const uint64_t desc_mn = umma_smem_desc_sw128_mn(smem_u32(smem), kHalfChunk);
      uint32_t j = 0, uses[2] = {0, 0}, small = 0;
      int chunk = 0;
      auto at = [&](uint64_t base, int c) { return base + uint64_t(((c % kChunks) * kChunkBytes) >> 4); };
      auto acc_free = [&](int b, int t) {
        if (!wait_bar(&ctl->acc_empty[b], (uses[b] & 1u) ^ 1u, ctl, p, SITE_ACC_EMPTY, t)) return false;
        tc_fence_after_sync();
        return true;
      };
      auto landed = [&](uint32_t s, int t) {
        if (!wait_bar(&ctl->full[s & 3u], (s >> 2) & 1u, ctl, p, SITE_FULL, t)) return false;
        tc_fence_after_sync();
        return true;
      };
      bool ok = true;
      // Operands are contiguous along the contraction, or (B of both sums, A of DW) across it: then an atom is two boxes, and
      // a step of 16 k-elements is two groups of 8 rows (2048 bytes) instead of 32 bytes of a row.
      auto run = [&](auto across, const Tile& tile, int t) {
        constexpr bool kAMn = decltype(across)::value, kBMn = kForm == SUMS;
        constexpr uint32_t idesc = umma_idesc_bf16_f32(256, 256) | (kAMn ? kUmmaIdescAMnMajor : 0u) | (kBMn ? kUmmaIdescBMnMajor : 0u);
        constexpr uint64_t ak = kAMn ? 2048 >> 4 : 2, bk = kBMn ? 2048 >> 4 : 2;
        const uint64_t desc_a = kAMn ? desc_mn : desc_k, desc_b = kBMn ? desc_mn : desc_k;
        auto issue = [&](uint32_t acc, int a_chunk, int b_chunk, uint32_t first) {
          const uint64_t da = at(desc_a, a_chunk), db = at(desc_b, b_chunk);
#pragma unroll
          for (int k = 0; k < BK / UMMA_K; ++k) umma_bf16_pair(acc, da + k * ak, db + k * bk, idesc, k ? 1u : first);
        };
        if (kForm != STATS && tile.big) {
          // Both accumulators are live for the whole tile, so nothing would hide the epilogue's reads if they ended
          // together: for the first and last kSkew stages accumulator 0's products go first.  It is then complete early
          // (its epilogue runs under accumulator 1's last products), and the next tile begins on it while accumulator 1
          // is still being read.
          const int n = tile.atoms;
          const int skew = n >= 2 * kSkew ? kSkew : 0;
          auto skewed = [&](int kb, bool begin) {
            for (int s = 0; s < kSkew; ++s) {
              if (!landed(j + s, t)) return false;
              issue(tmem_base, chunk + 3 * s, chunk + 3 * s + 2, (kb + s) != 0 ? 1u : 0u);
            }
            if (begin) {
              if (!acc_free(1, t)) return false;
            } else {
              umma_commit_pair(&ctl->acc_full[0], 0x3);
            }
            for (int s = 0; s < kSkew; ++s) {
              issue(tmem_base + 256, chunk + 3 * s + 1, chunk + 3 * s + 2, (kb + s) != 0 ? 1u : 0u);
              umma_commit_pair(&ctl->empty[(j + s) & 3u], 0x3);
            }
            j += kSkew;
            chunk = (chunk + 3 * kSkew) % kChunks;
            return true;
          };
          ok = acc_free(0, t);
          if (ok) ok = skew ? skewed(0, true) : acc_free(1, t);
          for (int kb = skew; ok && kb < n - skew; ++kb, ++j) {
            if (!(ok = landed(j, t))) break;
            const uint64_t a0 = at(desc_a, chunk), a1 = at(desc_a, chunk + 1), b = at(desc_b, chunk + 2);
            const uint32_t first = kb != 0 ? 1u : 0u;
#pragma unroll
            for (int k = 0; k < BK / UMMA_K; ++k) {
              umma_bf16_pair(tmem_base, a0 + k * ak, b + k * bk, idesc, k ? 1u : first);
              umma_bf16_pair(tmem_base + 256, a1 + k * ak, b + k * bk, idesc, k ? 1u : first);
            }
            chunk = (chunk + 3) % kChunks;
            umma_commit_pair(&ctl->empty[j & 3u], 0x3);
          }
          if (ok && skew) ok = skewed(n - skew, false);
          else if (ok) umma_commit_pair(&ctl->acc_full[0], 0x3);
          if (!ok) return;
          umma_commit_pair(&ctl->acc_full[1], 0x3);
          ++uses[0];
          ++uses[1];
        } else {
          const int ranges = ranges_of(kForm, tile.atoms);
          for (int r = 0; r < ranges; ++r) {
            const int b = int(small & 1u);
            const int from = r * kRangeAtoms, to = ranges > 1 ? min(tile.atoms, from + kRangeAtoms) : tile.atoms;
            if (!(ok = acc_free(b, t))) return;
            for (int a = from; a < to; a += 2, ++j) {
              if (!(ok = landed(j, t))) return;
              issue(tmem_base + b * 256, chunk, chunk + 2, a != from ? 1u : 0u);
              issue(tmem_base + b * 256, chunk + 1, chunk + 3, 1u);
              chunk = (chunk + 4) % kChunks;
              umma_commit_pair(&ctl->empty[j & 3u], 0x3);
            }
            umma_commit_pair(&ctl->acc_full[b], 0x3);
            ++uses[b];
            ++small;
          }
        }
      };
      for (int t = unit; ok && t < plan.total; t += units) {
        const Tile tile = tile_of<kForm>(p, plan, t);
        if (kForm == SUMS && tile.form == DW) run(std::true_type{}, tile, t);
        else run(std::false_type{}, tile, t);
      }
      if (*reinterpret_cast<volatile int*>(&ctl->abort)) {
        // gave up somewhere: let the tensor core finish what it still has before tensor memory is released
        umma_commit_pair(&ctl->drain, 0x1);
        wait_landed(&ctl->drain, 0);
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const int rows = p.found->rows;
    const float out_scale = kForm == SUMS ? p.out_scale * p.found->top : 0.f;
    const float top_weight = kForm == GRAD ? p.found->top : 1.f;
    uint32_t uses[2] = {0, 0}, small = 0;
    bool ok = true;
    for (int t = unit; ok && t < plan.total; t += units) {
      const Tile tile = tile_of<kForm>(p, plan, t);
      const int ranges = tile.big ? 1 : ranges_of(kForm, tile.atoms);
      for (int a = 0; a < (tile.big ? 2 : 1); ++a) {
        int b = tile.big ? a : int(small & 1u);
        const int frag0 = tile.row0 + (tile.big ? int(cta) * 256 + a * 128 : int(cta) * 128);    // this CTA's 128 rows
        const int row = frag0 + quarter * 32 + lane;
        int target = -1;
        float lse2 = 0.f, w = 0.f;
        if (kForm == STATS || kForm == GRAD) {
          if (row < rows) {
            target = p.target[row];
            if (kForm == GRAD) {
              lse2 = p.lse2[row];
              w = p.weight[row] / top_weight;
            }
          }
        }
        // (A wait that gives up is looked at behind the last range: what is read until then is dropped.  Leaving in between cost
        // 220 bytes of spilled registers a thread.)
        uint32_t v[4][32];
        bool gave_up = false;
        auto take = [&](auto add) {
          gave_up |= !wait_bar(&ctl->acc_full[b], uses[b] & 1u, ctl, p, SITE_ACC_FULL, t);
          __syncwarp();
          tc_fence_after_sync();
          const uint32_t taddr = tmem_base + (uint32_t(quarter * 32) << 16) + b * 256 + half * 128;
          if constexpr (decltype(add)::value) {
#pragma unroll
            for (int c = 0; c < 8; ++c) {      // (32 columns at a time would spill)
              uint32_t more[16];
              tmem_ld_32x32b_x16(taddr + c * 16, more);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                uint32_t& x = v[c >> 1][(c & 1) * 16 + i];
                x = __float_as_uint(__uint_as_float(x) + __uint_as_float(more[i]));
              }
            }
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(taddr + c * 32, v[c]);
            tmem_ld_wait();
          }
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster_relaxed(map_to_cta(smem_u32(&ctl->acc_empty[b]), 0));
          ++uses[b];
        };
        take(std::false_type{});
        if constexpr (kForm == STATS) {
          for (int r = 1; r < ranges; ++r) {
            ++small;
            b = int(small & 1u);
            take(std::true_type{});
          }
        }
        ok = __all_sync(0xffffffffu, !gave_up);      // (a warp goes on as one)
        if (!ok) break;

        if (kForm == STATS || kForm == GRAD) {
          int shard, vrow;
          const int cols = vocab_cols(p, p.vt0 + tile.col, &shard, &vrow) - half * 128;      // of this thread's 128
          const int hit = target - (shard * p.vocab_rows + vrow + half * 128);               // the target among them?
          const bool mine = target >= 0 && hit >= 0 && hit < min(cols, 128);
          const bool any = __any_sync(0xffffffffu, mine);
          if (kForm == STATS) {
            float m = -INFINITY, sum = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                float z = __uint_as_float(v[c][i]) * p.z_scale;
                if (cols < 128 && c * 32 + i >= cols) z = -INFINITY;
                else if (p.smoothing != 0.f) sum += z;
                v[c][i] = __float_as_uint(z);
                m = fmaxf(m, z);
              }
            const float top = m == -INFINITY ? 0.f : m;
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i) s[i & 3] += exp2_fast(__uint_as_float(v[c][i]) - top);
            if (any) {
              float z = 0.f;
#pragma unroll
              for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (hit == c * 32 + i) z = __uint_as_float(v[c][i]);
              if (mine) p.target_logit[row] = z;
            }
            if (row < rows) {
              const int64_t at = int64_t(2 * (p.vt0 + tile.col) + half) * p.pad + row;
              p.part[at] = make_float2(m, (s[0] + s[1]) + (s[2] + s[3]));
              if (p.smoothing != 0.f) p.part_sum[at] = sum;
            }
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                v[c][i] = __float_as_uint((exp2_fast(fmaf(__uint_as_float(v[c][i]), p.z_scale, -lse2)) - p.uniform) * w);
            if (any) {
              const float off = (1.f - p.smoothing) * w;
#pragma unroll
              for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (mine && hit == c * 32 + i) v[c][i] = __float_as_uint(__uint_as_float(v[c][i]) - off);
            }
            // Zeros past the shard's last row, and in the rows past the last that takes part, which DW sums over: selected, not
            // computed, because such a row's X is zero, but 0 * inf is NaN where the table has an infinite entry (a word
            // masked out).
            const int live = row < rows ? cols : 0;
            if (live < 128) {
#pragma unroll
              for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (c * 32 + i >= live) v[c][i] = 0u;
            }
            // straight from the registers, 32 bytes of a row per lane: through shared memory the tensor cores' operand
            // reads, which take most of its bandwidth, made this phase several times as long
            __nv_bfloat16* out = p.d + int64_t(row) * p.piece_cols + tile.col * 256 + half * 128;
#pragma unroll
            for (int g = 0; g < 8; ++g) {
              uint32_t q[8];
#pragma unroll
              for (int i = 0; i < 8; ++i)
                q[i] = pack_bf16x2(__uint_as_float(v[g >> 1][(g & 1) * 16 + 2 * i]), __uint_as_float(v[g >> 1][(g & 1) * 16 + 2 * i + 1]));
              store_32(out + g * 16, q);
            }
          }
        } else if (tile.form == DX) {
          // sums in the order the lanes hold them: 32 groups of 4 columns per warp, each group the lanes' 16 bytes in a row
          const int64_t frag = (int64_t(frag0 >> 7) * plan.part[0].cols + tile.col) * 8 + quarter * 2 + half;
          float4* sum = p.acc + frag * (32 * 32) + lane;
          if (tile.atoms == 0) continue;      // a last piece of fewer vocabulary tiles than splits: nothing to add
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            float4 old[4];
            if (!p.first_piece) {
#pragma unroll
              for (int g = 0; g < 4; ++g) old[g] = __ldcg(sum + (c * 4 + g) * 32);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const uint32_t* q = &v[c >> 1][(c & 1) * 16 + g * 4];
              float4 x = make_float4(__uint_as_float(q[0]), __uint_as_float(q[1]), __uint_as_float(q[2]), __uint_as_float(q[3]));
              if (!p.first_piece) {
                x.x += old[g].x;
                x.y += old[g].y;
                x.z += old[g].z;
                x.w += old[g].w;
              }
              sum[(c * 4 + g) * 32] = x;
            }
          }
        } else {
          // rows are vocabulary rows: this CTA's fragment lies in one vocabulary tile
          int shard, vrow;
          const int vt_rows = vocab_cols(p, p.vt0 + (frag0 >> 8), &shard, &vrow);
          const int in_tile = (frag0 & 255) + quarter * 32;
          const int col0 = tile.col * 256 + half * 128;
          if (in_tile + lane < vt_rows) {
            const int bytes = p.grad_fp32 ? 4 : 2;
            uint8_t* out = static_cast<uint8_t*>(p.dw[shard]) + ((int64_t(vrow) + in_tile + lane) * p.hidden + col0) * bytes;
            const int left = int(p.hidden) - col0;            // columns, a multiple of 8
            if (p.grad_fp32) {
#pragma unroll
              for (int g = 0; g < 16; ++g) {
                uint32_t q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) q[i] = __float_as_uint(__uint_as_float(v[g >> 2][(g & 3) * 8 + i]) * out_scale);
                if (g * 8 < left) store_row_piece(out + g * 32, q, p.dw_wide, true);
              }
            } else {
#pragma unroll
              for (int g = 0; g < 8; ++g) {
                uint32_t q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  q[i] = pack_bf16x2(__uint_as_float(v[g >> 1][(g & 1) * 16 + 2 * i]) * out_scale,
                                     __uint_as_float(v[g >> 1][(g & 1) * 16 + 2 * i + 1]) * out_scale);
                if (g * 16 < left) store_row_piece(out + g * 32, q, p.dw_wide, g * 16 + 8 < left);
              }
            }
          }
        }
      }
      if (!tile.big) ++small;
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// ---- statistics of few rows ----------------------------------------------------
// Up to kFewRows rows the forward product only has to read the table.  Here the table's rows are the products' M side (128 at
// a time) and X's the N side, so that all the loads but a few are of the table and fill the whole ring (the form above spends
// half of its ring on rows of X that are not there).  Single CTAs; warp 0 loads, warp 1 multiplies, warps 2..5 transpose the
// accumulator through shared memory and take each row's statistics over their 32 vocabulary rows.
// Measured, whole calls in a graph, the form above and this one: 1 row, 4096 x 128000: 216 and 179 us (the table's bytes take
// 160); 16 rows, 512 x 128000: 114 and 35; 64 rows, 4096 x 32000: 67 and 56, 200 x 65286: 42 and 28.  With more rows it is
// this form's epilogue that takes the time: 128 rows, 512 x 128000: 43 and 58, 4096 x 32000: 66 and 62.
constexpr int kFewRows = 64;
constexpr int kFewThreads = 192;
// A tile's contraction goes to this many accumulators in turn, which are added up in FP32: the tensor cores cut off what their
// sums cannot hold, a little at each step, and shorter sums lose less (16 rows, hidden = 4096: losses 2e-6 to 4e-6 off with one
// accumulator, 6e-7 with four, as with FP32 arithmetic).  The time is the table's either way.
constexpr int kFewParts = 4;
// Steps of 128 elements whose sums are read back together, so that an accumulator's are never longer than 1024 elements (64 rows,
// 8192 x 8000: lse 7e-7 off, 1.5e-6 with all of them together; 8192 x 32000: 99.7 and 101.0 us).
constexpr int kFewRange = 32;
constexpr int kFewAhead = 8;              // stages behind the ring whose part of the table is fetched into L2 meanwhile
constexpr int kFewRoom = 192 * 1024;
struct FewControl {
  uint64_t full[8], empty[8];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t drain;
  uint32_t tmem_base;
  int abort;
};
struct FewShared {
  float z[4][32][33];        // [warp][token][vocabulary row]
  float2 part[4][32];
  float sum[4][32];
};
__host__ __device__ constexpr int few_stage_bytes(int n) { return 2 * (kChunkBytes + n * BK * 2); }      // two k-atoms
__host__ __device__ constexpr int few_stages(int n) { return kFewRoom / few_stage_bytes(n) < 8 ? kFewRoom / few_stage_bytes(n) : 8; }
constexpr size_t kFewSmemBytes = 1024 + kFewRoom + sizeof(FewControl) + 16 + sizeof(FewShared);

__device__ __forceinline__ bool wait_few(uint64_t* bar, uint32_t parity, FewControl* ctl, const HeadParams& p, int site, int tile) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  const uint64_t limit = uint64_t(p.wait_limit_us) * 1000ull;
  for (uint32_t spins = 1; spins < (1u << 30); ++spins) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((spins & 0xFF) == 0) {
      if (*reinterpret_cast<volatile int*>(&ctl->abort)) return false;
      if (globaltimer_ns() - t0 > limit) break;
    }
  }
  *reinterpret_cast<volatile int*>(&ctl->abort) = 1;
  if (atomicCAS(&p.status->code, 0, int(COMPASS_ERR_TIMEOUT)) == 0) {
    p.status->detail = site;
    p.status->block_idx = int(blockIdx.x);
    p.status->tile = tile;
  }
  return false;
}

// Whether a wait of the four epilogue warps succeeded for all of them.  They meet at barrier 1 for every tile: a warp that gave
// up alone, just before the others' wait was over, would leave them there for good.
__device__ __forceinline__ bool few_agree(bool ok) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"(uint32_t(ok)) : "memory");
  return all != 0;
}

__global__ void __launch_bounds__(kFewThreads, 1) head_few_kernel(const __grid_constant__ HeadParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  FewControl* ctl = reinterpret_cast<FewControl*>(smem + kFewRoom);
  FewShared* sh = reinterpret_cast<FewShared*>((reinterpret_cast<uintptr_t>(ctl + 1) + 15) & ~uintptr_t(15));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_cols = p.few_cols;
  const int stage_bytes = few_stage_bytes(n_cols), stages = few_stages(n_cols);
  const int tiles = 2 * p.n_vt;                        // of 128 vocabulary rows
  const int ksteps = int((p.hidden + 127) / 128);
  const int ranges = (ksteps + kFewRange - 1) / kFewRange;
  if (threadIdx.x == 0) {
    for (int s = 0; s < 8; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->acc_full[b], 1);
      mbar_init(&ctl->acc_empty[b], 4);
    }
    mbar_init(&ctl->drain, 1);
    ctl->abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&ctl->tmem_base, 2 * kFewParts * kFewRows);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = ctl->tmem_base;
  launch_dependents();
  // the vocabulary rows of a tile that exist (0: none, the tile is left out by everyone)
  auto rows_of = [&](int t, int* shard, int* row) {
    const int rows = vocab_cols(p, t >> 1, shard, row) - (t & 1) * 128;
    *row += (t & 1) * 128;
    return max(0, min(128, rows));
  };

  if (warp == 0) {
    if (lane == 0) {
      const uint64_t pol = make_l2_policy(L2_EVICT_NORMAL);
      auto load_table = [&](uint8_t* dst, uint64_t* bar, int shard, int row, int k) {
        mbar_arrive_expect_tx(bar, uint32_t(stage_bytes));
        tma_load_2d_hint(dst, &p.w_k[shard], bar, k * 2 * BK, row, pol);
        tma_load_2d_hint(dst + kChunkBytes, &p.w_k[shard], bar, (k * 2 + 1) * BK, row, pol);
      };
      // the first stages' part of the table is on its way before the rows of X are gathered
      int shard, row, early = 0;
      if (int(blockIdx.x) < tiles && rows_of(blockIdx.x, &shard, &row) > 0)
        for (; early < min(stages, ksteps); ++early) load_table(smem + early * stage_bytes, &ctl->full[early], shard, row, early);
      for (int i = 2 * early; early > 0 && i < min(2 * (early + kFewAhead), 2 * ksteps); ++i) tma_prefetch_l2_2d(&p.w_k[shard], i * BK, row);
      wait_for_previous_kernel();
      int j = 0;
      bool ok = true;
      for (int t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
        if (rows_of(t, &shard, &row) == 0) continue;
        for (int k = 0; k < ksteps; ++k, ++j) {
          const int slot = j % stages;
          if (j >= stages && !wait_few(&ctl->empty[slot], uint32_t(j / stages - 1) & 1u, ctl, p, SITE_EMPTY, t)) {
            ok = false;
            break;
          }
          uint8_t* dst = smem + slot * stage_bytes;
          if (j >= early) load_table(dst, &ctl->full[slot], shard, row, k);
          for (int i = 0; i < 2; ++i)
            tma_load_2d_hint(dst + 2 * kChunkBytes + i * n_cols * BK * 2, &p.x_k, &ctl->full[slot], (k * 2 + i) * BK, 0, pol);
        }
      }
      // leave only when everything that was loaded has landed and been read
      for (int i = max(0, j - stages); i < j; ++i)
        if (!wait_few(&ctl->empty[i % stages], uint32_t(i / stages) & 1u, ctl, p, SITE_DRAIN, -1)) {
          for (int k = max(0, j - stages); k < j; ++k) wait_landed(&ctl->full[k % stages], uint32_t(k / stages) & 1u);
          break;
        }
    } else {
      wait_for_previous_kernel();
    }
  } else if (warp == 1) {
    wait_for_previous_kernel();
    if (lane == 0) {
      const uint32_t idesc = umma_idesc_bf16_f32(128, uint32_t(n_cols));
      const uint64_t desc = umma_smem_desc_sw128(smem_u32(smem));
      int j = 0;
      uint32_t it = 0;
      bool ok = true;
      for (int t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
        int shard, row;
        if (rows_of(t, &shard, &row) == 0) continue;
        for (int r = 0; ok && r < ranges; ++r) {
          const int steps = min(kFewRange, ksteps - r * kFewRange);
          const uint32_t b = it & 1u;
          if (!(ok = wait_few(&ctl->acc_empty[b], ((it >> 1) & 1u) ^ 1u, ctl, p, SITE_ACC_EMPTY, t))) break;
          tc_fence_after_sync();
          for (int k = 0; k < steps; ++k, ++j) {
            const int slot = j % stages;
            if (!(ok = wait_few(&ctl->full[slot], uint32_t(j / stages) & 1u, ctl, p, SITE_FULL, t))) break;
            tc_fence_after_sync();
            const uint64_t da = desc + uint64_t((slot * stage_bytes) >> 4), db = da + uint64_t((2 * kChunkBytes) >> 4);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              umma_bf16(tmem_base + (b * kFewParts + k % kFewParts) * kFewRows, da + uint64_t((i >> 2) * (kChunkBytes >> 4) + (i & 3) * 2),
                        db + uint64_t((i >> 2) * ((n_cols * BK * 2) >> 4) + (i & 3) * 2), idesc, k >= kFewParts || i ? 1u : 0u);
            umma_commit(&ctl->empty[slot]);
          }
          if (!ok) break;
          umma_commit(&ctl->acc_full[b]);
          ++it;
        }
      }
      if (*reinterpret_cast<volatile int*>(&ctl->abort)) {
        umma_commit(&ctl->drain);
        wait_landed(&ctl->drain, 0);
      }
    }
  } else {
    wait_for_previous_kernel();
    const int quarter = warp & 3;
    const int rows = p.found->rows;
    uint32_t it = 0;
    bool ok = true;
    for (int t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
      int shard, vrow;
      const int live = rows_of(t, &shard, &vrow) - quarter * 32;        // of this warp's 32 vocabulary rows
      const bool empty = live + quarter * 32 == 0;
      float v[kFewRows / 32][32] = {};      // the logits, 32 tokens at a time
      for (int r = 0; !empty && ok && r < ranges; ++r) {
        const uint32_t b = it & 1u;
        ok = few_agree(__all_sync(0xffffffffu, wait_few(&ctl->acc_full[b], (it >> 1) & 1u, ctl, p, SITE_ACC_FULL, t)));
        if (!ok) continue;
        tc_fence_after_sync();
        const int parts = min(kFewParts, ksteps - r * kFewRange);
#pragma unroll
        for (int c = 0; c < kFewRows / 32; ++c) {
          if (c * 32 >= n_cols) continue;
          const uint32_t taddr = tmem_base + (uint32_t(quarter * 32) << 16) + b * kFewParts * kFewRows + c * 32;
          for (int part = 0; part < parts; ++part) {
            uint32_t w[32];
            tmem_ld_32x32b_x32(taddr + part * kFewRows, w);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[c][i] += __uint_as_float(w[i]);
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl->acc_empty[b]);
        ++it;
      }
      if (!ok) break;
#pragma unroll
      for (int c = 0; c < kFewRows / 32; ++c) {
        if (c * 32 >= n_cols) continue;
        const int token = c * 32 + lane;
        float m = -INFINITY, s = 0.f, sum = 0.f;
        if (!empty) {
#pragma unroll
          for (int i = 0; i < 32; ++i) sh->z[quarter][i][lane] = v[c][i] * p.z_scale;
          __syncwarp();
          const float* z = sh->z[quarter][lane];
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i < live) m = fmaxf(m, z[i]);
          const float top = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i < live) {
              s += exp2_fast(z[i] - top);
              sum += z[i];
            }
          if (token < rows) {
            const int hit = p.target[token] - (shard * p.vocab_rows + vrow + quarter * 32);
            if (hit >= 0 && hit < min(live, 32)) p.target_logit[token] = z[hit];
          }
        }
        // the four warps' statistics as one
        sh->part[quarter][lane] = make_float2(m, s);
        sh->sum[quarter][lane] = sum;
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (quarter == 0 && token < rows) {
          float top = -INFINITY;
          s = sum = 0.f;
#pragma unroll
          for (int w = 0; w < 4; ++w) top = fmaxf(top, sh->part[w][lane].x);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float2 x = sh->part[w][lane];
            s += top == -INFINITY || x.x == -INFINITY ? x.y : x.y * exp2_fast(x.x - top);
            sum += sh->sum[w][lane];
          }
          const int64_t at = int64_t(t) * p.pad + token;
          p.part[at] = make_float2(top, s);
          if (p.smoothing != 0.f) p.part_sum[at] = sum;
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 2 * kFewParts * kFewRows);
  }
}

// ---- which rows take part ------------------------------------------------------

constexpr int kCountRows = 1024;      // rows counted together
constexpr int kGatherRows = 4;        // rows a block copies, two warps each
constexpr int kFewestRows = 16;       // rows that are always there behind the gathered ones' beginning, zeros past the last

struct RowParams {
  RowShards x, dx;          // dx: backward, zeros for the rows that take no part
  const void* targets;
  const float* lse;         // backward
  const float* dloss;
  float* loss_out;          // forward: zeros for the rows that take no part
  float* lse_out;
  int32_t* counts;          // [ceil(M / kCountRows)] rows that take part
  float* tops;              // the same: max |dloss| over them, infinite where one is not finite
  Found* found;
  int32_t* origin;          // [pad] row that a gathered one comes from
  int32_t* target;
  float* lse2;
  float* weight;
  uint4* gathered;
  uint32_t M;
  uint32_t vecs;            // 16-byte vectors per row
  int32_t vocab;
  int32_t wide;
};

// A row's target, or -1 when it takes no part.
__device__ __forceinline__ int32_t target_of(const RowParams& p, uint32_t i) {
  const int64_t y = p.wide ? static_cast<const int64_t*>(p.targets)[i] : int64_t(static_cast<const int32_t*>(p.targets)[i]);
  return y >= 0 && y < p.vocab ? int32_t(y) : -1;
}

// |g|, infinite where g is not finite.
__device__ __forceinline__ float finite_size(float g) { return fabsf(g) < INFINITY ? fabsf(g) : INFINITY; }

__global__ void __launch_bounds__(256) head_count_kernel(const __grid_constant__ RowParams p) {
  __shared__ int32_t counts[8];
  __shared__ float tops[8];
  launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t n = 0;
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < kCountRows / 256; ++k) {
    const uint32_t i = blockIdx.x * kCountRows + k * 256 + threadIdx.x;
    if (i >= p.M) continue;
    const float g = p.dloss ? finite_size(p.dloss[i]) : 0.f;
    if (target_of(p, i) >= 0) {
      ++n;
      top = fmaxf(top, g);
    } else if (p.loss_out) {
      p.loss_out[i] = 0.f;
      p.lse_out[i] = 0.f;
    }
  }
  n = __reduce_add_sync(0xffffffffu, n);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) {
    counts[warp] = n;
    tops[warp] = top;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) {
      n += counts[w];
      top = fmaxf(top, tops[w]);
    }
    p.counts[blockIdx.x] = n;
    p.tops[blockIdx.x] = top;
  }
}

// Sum over the block; all its threads take part.
__device__ __forceinline__ int2 block_add(int2 v, int2* part) {
  v.x = __reduce_add_sync(0xffffffffu, v.x);
  v.y = __reduce_add_sync(0xffffffffu, v.y);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < 8; ++w) {
    v.x += part[w].x;
    v.y += part[w].y;
  }
  return v;
}

// The rows that take part, together and in order.  The k-th row that takes none zeroes the k-th row behind them, up to a
// multiple of 512 (dW contracts over whole tiles of these rows), and its own dX.
__global__ void __launch_bounds__(256) head_gather_kernel(const __grid_constant__ RowParams p) {
  __shared__ int2 part[8];
  __shared__ int32_t places[kGatherRows];
  launch_dependents();
  wait_for_previous_kernel();
  const uint32_t row0 = blockIdx.x * kGatherRows;
  int2 sum = make_int2(0, 0);       // rows that take part: before row0, in all
  float top = 0.f;
  if (p.M <= kCountRows) {
    // few enough for every block to count them (there was no head_count_kernel)
    for (uint32_t i = threadIdx.x; i < p.M; i += 256) {
      const bool in = target_of(p, i) >= 0;
      sum.x += in && i < row0;
      sum.y += in;
      if (p.dloss && in) top = fmaxf(top, finite_size(p.dloss[i]));
      if (p.loss_out && !in && i - row0 < kGatherRows) {
        p.loss_out[i] = 0.f;
        p.lse_out[i] = 0.f;
      }
    }
  } else {
    const uint32_t chunk = row0 / kCountRows, chunks = (p.M + kCountRows - 1) / kCountRows;
    for (uint32_t b = threadIdx.x; b < chunks; b += 256) {
      const int32_t n = p.counts[b];
      if (b < chunk) sum.x += n;
      sum.y += n;
      top = fmaxf(top, p.tops[b]);
    }
    for (uint32_t i = chunk * kCountRows + threadIdx.x; i < row0; i += 256) sum.x += target_of(p, i) >= 0;
  }
  sum = block_add(sum, part);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x == 0) {
    __shared__ float tops[8];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) tops[warp] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < 8; ++w) top = fmaxf(top, tops[w]);
      p.found->rows = sum.y;
      p.found->top = top > 0.f && top < INFINITY ? top : 1.f;
    }
  }
  if (warp == 0) {
    const uint32_t i = row0 + lane;
    const bool in = lane < kGatherRows && i < p.M;
    const int32_t target = in ? target_of(p, i) : -1;
    const uint32_t valid = __ballot_sync(0xffffffffu, target >= 0);
    const int32_t at = sum.x + __popc(valid & ((1u << lane) - 1u));
    if (target >= 0) {
      p.origin[at] = int32_t(i);
      p.target[at] = target;
      if (p.dloss) {
        p.weight[at] = p.dloss[i];
        p.lse2[at] = p.lse[i] * kLog2e;
      }
    }
    // a row that takes no part, the (i - at)-th of them: its place is behind the others, as ~place
    if (lane < kGatherRows) places[lane] = target >= 0 ? at : ~(sum.y + int32_t(i) - at);
  }
  __syncthreads();
  const int32_t padded = (max(sum.y, 1) + 511) / 512 * 512;
  if (blockIdx.x == 0 && p.M < kFewestRows)
    for (uint32_t c = p.M * p.vecs + threadIdx.x; c < kFewestRows * p.vecs; c += 256) p.gathered[c] = make_uint4(0u, 0u, 0u, 0u);
  const uint32_t i = row0 + (warp >> 1);
  if (i >= p.M) return;
  const int32_t place = places[warp >> 1];
  const uint32_t c0 = threadIdx.x & 63;
  if (place >= 0) {
    const uint4* from = p.x.row<uint4>(i, p.vecs);
    uint4* to = p.gathered + int64_t(place) * p.vecs;
    uint32_t c = c0;
    for (; c + 7 * 64 < p.vecs; c += 8 * 64) {
      uint4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __ldcs(from + c + k * 64);
#pragma unroll
      for (int k = 0; k < 8; ++k) to[c + k * 64] = v[k];
    }
    for (; c < p.vecs; c += 64) to[c] = __ldcs(from + c);
  } else {
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    uint4* to = p.gathered + int64_t(~place) * p.vecs;
    if (~place < padded)
      for (uint32_t c = c0; c < p.vecs; c += 64) to[c] = zero;
    if (p.dloss) {
      to = p.dx.row<uint4>(i, p.vecs);
      for (uint32_t c = c0; c < p.vecs; c += 64) to[c] = zero;
    }
  }
}

// ---- what the statistics say ---------------------------------------------------

struct CombineParams {
  const Found* found;
  const int32_t* origin;
  const float2* part;
  const float* part_sum;
  const float* target_logit;
  float* loss;
  float* lse;
  int32_t parts, pad;
  float smoothing, uniform;
};
// 32 rows per block: every warp a share of their parts, then every warp one row.
__global__ void __launch_bounds__(1024) head_combine_kernel(const __grid_constant__ CombineParams p) {
  __shared__ float2 ms[32][33];
  __shared__ float zs[32][33];
  wait_for_previous_kernel();
  const int rows = p.found->rows;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row0 = blockIdx.x * 32;
  if (row0 >= rows) return;
  float m = -INFINITY, s = 0.f, z = 0.f;
  if (row0 + lane < rows) {
    for (int q0 = warp; q0 < p.parts; q0 += 32 * 8) {
      float2 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int q = q0 + i * 32;
        x[i] = make_float2(-INFINITY, 0.f);
        if (q < p.parts) {
          x[i] = p.part[int64_t(q) * p.pad + row0 + lane];
          if (p.smoothing != 0.f) z += p.part_sum[int64_t(q) * p.pad + row0 + lane];
        }
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i].x);
      // (no maximum: nothing but -inf, whose sum is 0, and NaN, whose sum is NaN)
      const float at = top == -INFINITY ? 0.f : top;
      s = m == -INFINITY ? s : s * exp2f(m - at);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += x[i].x == -INFINITY ? x[i].y : x[i].y * exp2f(x[i].x - at);
      m = top;
    }
  }
  ms[warp][lane] = make_float2(m, s);
  zs[warp][lane] = z;
  __syncthreads();
  const int row = row0 + warp;
  if (row >= rows) return;
  const float2 x = ms[lane][warp];
  float top = x.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  s = warp_sum(x.x == -INFINITY ? x.y : x.y * exp2f(x.x - top));
  z = warp_sum(zs[lane][warp]);
  if (lane == 0) {
    const float lse2 = top + log2f(s);
    const int to = p.origin[row];
    p.lse[to] = lse2 * kLn2;
    float l = lse2 - (1.f - p.smoothing) * p.target_logit[row];
    if (p.smoothing != 0.f) l -= p.uniform * z;
    p.loss[to] = l * kLn2;
  }
}

// ---- dX from its FP32 sums -----------------------------------------------------

struct FinishParams {
  RowShards dx;
  const Found* found;
  const int32_t* origin;
  const float4* acc;
  int64_t hidden;
  int32_t hidden_tiles, splits;
  FastDiv row_blocks;
  float out_scale;
};
// A block takes 32 gathered rows and 128 columns: what one warp of the products' epilogue holds.  (One grid axis: the second
// would end at 65535 blocks, 8.4 million columns.)
__global__ void __launch_bounds__(256) head_finish_kernel(const __grid_constant__ FinishParams p) {
  __shared__ float tile[32][129];
  wait_for_previous_kernel();
  const int rows = p.found->rows;
  const uint32_t slab = p.row_blocks.div(blockIdx.x);      // of 128 columns
  const int row0 = int(blockIdx.x - slab * p.row_blocks.d) * 32;
  if (row0 >= rows) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float scale = p.out_scale * p.found->top;
  const int64_t step = int64_t(p.hidden_tiles) * 8 * (32 * 32);            // from one split's sums to the next one's
  const int64_t frag = (int64_t(row0 >> 7) * p.hidden_tiles * p.splits + int(slab >> 1)) * 8 + ((row0 >> 5) & 3) * 2 + int(slab & 1);
  const float4* in = p.acc + frag * (32 * 32) + warp * 4 * 32 + lane;      // 4 of the 32 groups of 4 columns per warp
  float4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 y = __ldcs(in + s * step + i * 32);
      x[i].x += y.x;
      x[i].y += y.y;
      x[i].z += y.z;
      x[i].w += y.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float* t = &tile[lane][(warp * 4 + i) * 4];
    t[0] = x[i].x * scale;
    t[1] = x[i].y * scale;
    t[2] = x[i].z * scale;
    t[3] = x[i].w * scale;
  }
  __syncthreads();
  // 16 lanes a row, 8 columns each
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int r = k * 16 + (threadIdx.x >> 4);
    const int64_t c = int64_t(slab) * 128 + (threadIdx.x & 15) * 8;
    if (row0 + r < rows && c < p.hidden) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = tile[r][(threadIdx.x & 15) * 8 + i];
      store_vec(p.dx.row<__nv_bfloat16>(uint32_t(p.origin[row0 + r]), p.hidden) + c, y);
    }
  }
}

// ---- host ----------------------------------------------------------------------

int check_head(const compass_head* h) {
  if (h == nullptr) return COMPASS_ERR_INVALID_ARG;
  int st = check_rows(h->P, h->M, h->hidden);
  if (st != COMPASS_OK) return st;
  if (h->vocab <= 0) return COMPASS_ERR_SHAPE;
  if (h->vocab > kMaxDim) return COMPASS_ERR_UNSUPPORTED;
  if (h->index_dtype != COMPASS_INDEX_INT64 && h->index_dtype != COMPASS_INDEX_INT32) return COMPASS_ERR_INVALID_ARG;
  st = check_dtype(h->dtype, false);
  if (st == COMPASS_OK) st = check_dtype(h->grad_dtype, true);
  if (st != COMPASS_OK) return st;
  if (!(h->label_smoothing >= 0.f && h->label_smoothing < 1.f)) return COMPASS_ERR_INVALID_ARG;
  if (!(h->logit_scale - h->logit_scale == 0.f)) return COMPASS_ERR_INVALID_ARG;      // not finite
  return h->hidden % 8 == 0 ? COMPASS_OK : COMPASS_ERR_ALIGNMENT;
}

// Pairs of CTAs that a launch counts on (one CTA per SM of the B200's 148); fewer co-resident ones only take more rounds.
constexpr int kPairs = 74;
// Bytes of the logits' gradient that are held at a time.  Fewer, larger pieces mean fewer launches and sums read back, and that
// outweighs a piece that stays in L2 even where hidden is small.  Backward, us, with pieces of 32, 64, 128, 256, 512 MB:
// 8192 rows, 4096 x 64000: 12350, 10910, 10150, 9880, 9780; 1024 x 50000: 3040, 2740, 2460, 2270, 2180; 368 x 32000: 1390, 1250,
// 900, 810, 780; 5926 rows, 96 x 5021: 187, 125, 130, 131 to 152, 125 to 150; 1000 rows, 4096 x 50001: 1170, 1117, 1070, 1065, 1065.
// 512 would be 1 to 4 % faster on the large ones for twice the workspace.
constexpr int64_t kPieceBytes = int64_t(256) << 20;

struct HeadPlan {
  int64_t pad;
  int tiles_per_shard, vocab_tiles, hidden_tiles, splits, piece_tiles;
  size_t ints, chunks, part, part_sum, gathered, acc, d;      // sections of the workspace, in bytes
  size_t bytes;
};
// Rows that the tensor maps of the workspace's matrices have: loads of 128 rows from a matrix of 8 or fewer took four times as
// long (1 row, 4096 x 128000: 880 us forward; 16 rows: 218).
int64_t map_rows(int64_t M) { return M < kFewestRows ? kFewestRows : M; }
HeadPlan head_plan(const compass_head* h, bool backward) {
  HeadPlan q = {};
  q.pad = int64_t(round_up(size_t(h->M), 512));
  const int64_t rows = vocab_shard_rows(h->vocab, h->P);
  q.tiles_per_shard = int(ceil_div(rows, 256));
  for (int r = 0; r < h->P; ++r) q.vocab_tiles += int(ceil_div(rows_of_vocab_shard(h->vocab, h->P, r), 256));
  q.hidden_tiles = int(ceil_div(h->hidden, 256));
  // dX has few tiles when rows are few: its contraction over the vocabulary is then split over the pairs.  Backward, us, split
  // and not: 1 row, 4096 x 128000: 827, 1378; 16, 4096 x 32000: 230, 368; 64, 512 x 32000: 96, 240; 300, 4096 x 32000: 365, 421;
  // 401, 1024 x 50001: 179, 409.
  const int64_t dx_tiles = ceil_div(h->M, 256) * q.hidden_tiles;
  q.splits = dx_tiles > 0 && dx_tiles < kPairs ? int(kPairs / dx_tiles) : 1;
  if (q.splits > q.vocab_tiles) q.splits = q.vocab_tiles;
  // pieces of equal size, an even number of vocabulary tiles each (512-row tiles of dW)
  int64_t most = kPieceBytes / (q.pad * 512 + 1);
  if (most < 2) most = 2;
  const int64_t pieces = ceil_div(q.vocab_tiles, most);
  q.piece_tiles = int(round_up(size_t(ceil_div(q.vocab_tiles, pieces)), 2));
  if (q.splits > q.piece_tiles) q.splits = q.piece_tiles;
  q.ints = round_up(size_t(q.pad) * 4, 256);
  q.chunks = round_up(size_t(ceil_div(h->M, kCountRows)) * 4, 256);
  q.gathered = size_t(map_rows(h->M)) * size_t(h->hidden) * 2;
  if (backward) {
    q.acc = size_t(q.pad / 128) * size_t(q.hidden_tiles) * size_t(q.splits) * (128 * 256 * 4);
    q.d = size_t(q.pad) * size_t(q.piece_tiles) * 512;
    q.bytes = 512 + 2 * q.chunks + 4 * q.ints + round_up(q.gathered, 256) + q.acc + q.d;
  } else {
    q.part = round_up(size_t(q.pad) * size_t(q.vocab_tiles) * 2 * 8, 256);
    q.part_sum = h->label_smoothing != 0.f ? q.part / 2 : 0;
    q.part_sum = round_up(q.part_sum, 256);
    q.bytes = 512 + 2 * q.chunks + 3 * q.ints + round_up(q.gathered, 256) + q.part + q.part_sum;
  }
  return q;
}

struct DeviceFacts {
  bool ready = false;
  int pairs = 0, sms = 0;
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
    const void* kernels[] = {reinterpret_cast<const void*>(head_kernel<STATS>), reinterpret_cast<const void*>(head_kernel<GRAD>),
                             reinterpret_cast<const void*>(head_kernel<SUMS>)};
    for (const void* k : kernels) {
      e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmemBytes));
      if (e != cudaSuccess) return record_cuda_error(e);
    }
    e = cudaFuncSetAttribute(head_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kFewSmemBytes));
    if (e != cudaSuccess) return record_cuda_error(e);
    e = cudaDeviceGetAttribute(&f.sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return record_cuda_error(e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(f.sms / 2 * 2));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&f.pairs, head_kernel<STATS>, &cfg);
    if (e != cudaSuccess) return record_cuda_error(e);
    if (f.pairs < 1) return COMPASS_ERR_UNSUPPORTED;
    f.ready = true;
  }
  *out = &f;
  return COMPASS_OK;
}

int launch_form(int form, const HeadParams& p, int64_t most_tiles, const DeviceFacts& f, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(2 * (most_tiles < f.pairs ? most_tiles : f.pairs)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cudaError_t e;
  if (form == STATS) e = cudaLaunchKernelEx(&cfg, head_kernel<STATS>, p);
  else if (form == GRAD) e = cudaLaunchKernelEx(&cfg, head_kernel<GRAD>, p);
  else e = cudaLaunchKernelEx(&cfg, head_kernel<SUMS>, p);
  count_kernel_launch();
  return e == cudaSuccess ? COMPASS_OK : record_cuda_error(e);
}

// The part of both directions that lists and gathers the rows.
struct Common {
  HeadPlan q;
  DeviceFacts* facts;
  bool few;               // head_few_kernel takes the statistics
  uint8_t* at;            // next free byte of the workspace
  RowParams rows;
  HeadParams p;
  uint8_t* take(size_t n) {
    uint8_t* was = at;
    at += n;
    return was;
  }
};

int begin(const compass_head* h, const void* const* X, const void* const* W, const void* targets, void* ws, size_t ws_bytes, bool backward,
          Common* c) {
  int st = check_head(h);
  if (st != COMPASS_OK) return st;
  if (h->M > 0 && targets == nullptr) return COMPASS_ERR_INVALID_ARG;
  if (!is_aligned(targets, h->index_dtype == COMPASS_INDEX_INT64 ? 8 : 4)) return COMPASS_ERR_ALIGNMENT;
  st = fill_shards(X, h->P, h->M, &c->rows.x);
  if (st == COMPASS_OK) st = check_vocab_shards(W, h->P, h->vocab);
  if (st != COMPASS_OK) return st;
  c->q = head_plan(h, backward);
  // tiles are numbered in 32 bits
  const int64_t cols = c->q.vocab_tiles > c->q.hidden_tiles * c->q.splits ? c->q.vocab_tiles : c->q.hidden_tiles * c->q.splits;
  if ((h->M / 256 + 1) * cols > kMaxDim || int64_t(c->q.vocab_tiles) * c->q.hidden_tiles > kMaxDim) return COMPASS_ERR_UNSUPPORTED;
  return check_workspace(ws, ws_bytes, c->q.bytes);
}

int gather_rows(const compass_head* h, const void* const* W, const void* targets, void* ws, Common* c, cudaStream_t stream) {
  int st = device_facts(&c->facts);
  if (st != COMPASS_OK) return st;
  const HeadPlan& q = c->q;
  HeadParams& p = c->p;
  if (c->few) p.few_cols = int32_t(round_up(size_t(h->M), 16));
  uint8_t* base = static_cast<uint8_t*>(ws);
  Found* found = reinterpret_cast<Found*>(base + 256);
  c->at = base + 512;
  RowParams& r = c->rows;
  r.targets = targets;
  r.found = found;
  r.counts = reinterpret_cast<int32_t*>(c->take(q.chunks));
  r.tops = reinterpret_cast<float*>(c->take(q.chunks));
  r.origin = reinterpret_cast<int32_t*>(c->take(q.ints));
  r.target = reinterpret_cast<int32_t*>(c->take(q.ints));
  r.M = uint32_t(h->M);
  r.vocab = int32_t(h->vocab);
  r.wide = h->index_dtype == COMPASS_INDEX_INT64;
  if (r.dloss) {
    r.lse2 = reinterpret_cast<float*>(c->take(q.ints));
    r.weight = reinterpret_cast<float*>(c->take(q.ints));
  } else {
    p.target_logit = reinterpret_cast<float*>(c->take(q.ints));
  }
  uint8_t* gathered = c->take(round_up(q.gathered, 256));
  p.found = found;
  p.target = r.target;
  p.lse2 = r.lse2;
  p.weight = r.weight;
  p.status = static_cast<StatusBlock*>(ws);
  p.hidden = h->hidden;
  p.pad = int32_t(q.pad);
  p.vocab_rows = int32_t(vocab_shard_rows(h->vocab, h->P));
  p.vocab = int32_t(h->vocab);
  p.tiles_per_shard = q.tiles_per_shard;
  p.hidden_tiles = q.hidden_tiles;
  p.one_row_tile = h->M <= 256;
  p.splits = q.splits;
  p.z_scale = h->logit_scale * kLog2e;
  p.out_scale = h->logit_scale;
  p.smoothing = h->label_smoothing;
  p.uniform = float(double(h->label_smoothing) / double(h->vocab));
  p.wait_limit_us = default_wait_limit_us() ? default_wait_limit_us() : 2000000u;
  // (rows past these are not loaded: they read as zeros)
  bool ok = encode_tensor_map(&p.x_k, gathered, map_rows(h->M), h->hidden, c->few ? p.few_cols : 128);
  for (int s = 0; s < h->P; ++s) {
    const int64_t n = rows_of_vocab_shard(h->vocab, h->P, s);
    if (n > 0) ok = ok && encode_tensor_map(&p.w_k[s], W[s], n, h->hidden, 128);
    if (n > 0 && r.dloss) ok = ok && encode_tensor_map(&p.w_mn[s], W[s], n, h->hidden, 64);
  }
  if (r.dloss) ok = ok && encode_tensor_map(&p.x_mn, gathered, map_rows(h->M), h->hidden, 64);
  if (!ok) return record_cuda_error(cudaErrorUnknown);
  r.gathered = reinterpret_cast<uint4*>(gathered);
  r.vecs = uint32_t(h->hidden / 8);
  const bool counted = h->M > kCountRows;
  if (counted) st = launch(head_count_kernel, ceil_div(h->M, kCountRows), 256, 0, stream, false, r);
  if (st != COMPASS_OK) return st;
  return launch(head_gather_kernel, ceil_div(h->M, kGatherRows), 256, 0, stream, counted, r);
}

// Tiles of a form at most, counted as 256 x 256.
int64_t most_tiles(const compass_head* h, const HeadPlan& q, int64_t cols) { return ceil_div(h->M, 256) * cols; }

}  // namespace

}  // namespace compass

using namespace compass;

extern "C" int compass_head_workspace_bytes(const compass_head* h, int backward, size_t* bytes) {
  if (bytes == nullptr) return COMPASS_ERR_INVALID_ARG;
  const int st = check_head(h);
  if (st != COMPASS_OK) return st;
  *bytes = head_plan(h, backward != 0).bytes;
  return COMPASS_OK;
}

extern "C" int compass_head_loss(const compass_head* h, const void* const* X, const void* const* W, const void* targets, float* loss,
                                 float* lse, void* ws, size_t ws_bytes, void* stream) {
  Common c = {};
  int st = begin(h, X, W, targets, ws, ws_bytes, false, &c);
  if (st != COMPASS_OK) return st;
  if (h->M > 0 && (loss == nullptr || lse == nullptr)) return COMPASS_ERR_INVALID_ARG;
  if (!is_aligned(loss, 4) || !is_aligned(lse, 4)) return COMPASS_ERR_ALIGNMENT;
  if (h->M == 0) return COMPASS_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  c.rows.loss_out = loss;
  c.rows.lse_out = lse;
  c.few = h->M <= kFewRows;
  st = gather_rows(h, W, targets, ws, &c, s);
  if (st != COMPASS_OK) return st;
  HeadParams& p = c.p;
  p.part = reinterpret_cast<float2*>(c.take(c.q.part));
  p.part_sum = reinterpret_cast<float*>(c.take(c.q.part_sum));
  p.n_vt = c.q.vocab_tiles;
  if (c.few) {
    const int64_t tiles = 2 * int64_t(c.q.vocab_tiles);
    st = launch(head_few_kernel, tiles < c.facts->sms ? tiles : c.facts->sms, kFewThreads, kFewSmemBytes, s, true, p);
  } else {
    st = launch_form(STATS, p, most_tiles(h, c.q, c.q.vocab_tiles), *c.facts, s);
  }
  if (st != COMPASS_OK) return st;
  CombineParams m = {};
  m.found = p.found;
  m.origin = c.rows.origin;
  m.part = p.part;
  m.part_sum = p.part_sum;
  m.target_logit = p.target_logit;
  m.loss = loss;
  m.lse = lse;
  m.parts = 2 * c.q.vocab_tiles;
  m.pad = int32_t(c.q.pad);
  m.smoothing = p.smoothing;
  m.uniform = p.uniform;
  return launch(head_combine_kernel, ceil_div(h->M, 32), 1024, 0, s, true, m);
}

extern "C" int compass_head_loss_backward(const compass_head* h, const void* const* X, const void* const* W, const void* targets,
                                          const float* lse, const float* dloss, void* const* dX, void* const* dW, void* ws,
                                          size_t ws_bytes, void* stream) {
  Common c = {};
  int st = begin(h, X, W, targets, ws, ws_bytes, true, &c);
  if (st != COMPASS_OK) return st;
  if (h->M > 0 && (lse == nullptr || dloss == nullptr)) return COMPASS_ERR_INVALID_ARG;
  if (!is_aligned(lse, 4) || !is_aligned(dloss, 4)) return COMPASS_ERR_ALIGNMENT;
  st = fill_shards(dX, h->P, h->M, &c.rows.dx);
  if (st == COMPASS_OK) st = check_vocab_shards(dW, h->P, h->vocab);
  if (st != COMPASS_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (h->M == 0) {
    for (int r = 0; r < h->P; ++r) {
      const int64_t n = rows_of_vocab_shard(h->vocab, h->P, r);
      if (n == 0) continue;
      const cudaError_t e = cudaMemsetAsync(dW[r], 0, size_t(n) * size_t(h->hidden) * dtype_size(h->grad_dtype), s);
      if (e != cudaSuccess) return record_cuda_error(e);
    }
    return COMPASS_OK;
  }
  c.rows.lse = lse;
  c.rows.dloss = dloss;
  st = gather_rows(h, W, targets, ws, &c, s);
  if (st != COMPASS_OK) return st;
  const HeadPlan& q = c.q;
  HeadParams& p = c.p;
  p.acc = reinterpret_cast<float4*>(c.take(q.acc));
  p.d = reinterpret_cast<__nv_bfloat16*>(c.take(q.d));
  p.grad_fp32 = h->grad_dtype == COMPASS_DTYPE_FP32;
  p.piece_cols = q.piece_tiles * 256;
  p.dw_wide = h->hidden * int64_t(dtype_size(h->grad_dtype)) % 32 == 0;
  for (int r = 0; r < h->P; ++r) {
    p.dw[r] = dW[r];
    if (!is_aligned(dW[r], 32)) p.dw_wide = 0;
  }
  if (!encode_tensor_map(&p.d_k, p.d, map_rows(h->M), p.piece_cols, 128) || !encode_tensor_map(&p.d_mn, p.d, map_rows(h->M), p.piece_cols, 64))
    return record_cuda_error(cudaErrorUnknown);
  for (int vt = 0; vt < q.vocab_tiles; vt += q.piece_tiles) {
    p.vt0 = vt;
    p.n_vt = q.vocab_tiles - vt < q.piece_tiles ? q.vocab_tiles - vt : q.piece_tiles;
    p.first_piece = vt == 0;
    st = launch_form(GRAD, p, most_tiles(h, q, p.n_vt), *c.facts, s);
    if (st == COMPASS_OK)
      st = launch_form(SUMS, p, most_tiles(h, q, int64_t(q.hidden_tiles) * q.splits) + int64_t(p.n_vt) * q.hidden_tiles, *c.facts, s);
    if (st != COMPASS_OK) return st;
  }
  FinishParams f = {};
  f.dx = c.rows.dx;
  f.found = p.found;
  f.origin = c.rows.origin;
  f.acc = p.acc;
  f.hidden = h->hidden;
  f.hidden_tiles = q.hidden_tiles;
  f.splits = q.splits;
  f.row_blocks.set(uint32_t(ceil_div(h->M, 32)));
  f.out_scale = p.out_scale;
  return launch(head_finish_kernel, int64_t(f.row_blocks.d) * 2 * q.hidden_tiles, 256, 0, s, true, f);
}
