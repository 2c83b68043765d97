// Persistent CTA-pair matrix product on the sm_103a tensor cores, with the work on a finished
// 256 x 256 tile left to the caller:  D[m, n] = sum_k A[m, k] B[n, k]   (bf16 in, fp32 sums).
//
// Used by the head loss (logit tiles that never leave the chip, and the two gradient products), by the
// adapter projection and by the gated feed-forward (two products that share A, side by side).  Each operand
// is K-major (k contiguous) or MN-major (m or n contiguous); the tensor maps and the MMA descriptors carry the
// difference.
//
// Three shapes.  Narrow: a pair of CTAs holds a 256 x 256 fp32 tile (128 rows per CTA: half of
// TMEM); the other half of TMEM takes the next tile while eight warps read this one.  Wide: 256 x 512,
// two accumulators that share A, all of TMEM.  What bounds the narrow one is shared memory: per 64-wide
// k-block and CTA the loads write 32 KB and the MMAs read 32 KB in the 512 cycles that the MMAs take,
// 128 bytes per cycle, all that shared memory moves, and a k-block took 672 cycles (with a quarter of
// the MMAs, about 450).  The wide one writes 48 KB for 1024 cycles of MMAs.  Its epilogue is not
// hidden behind a second buffer, so the MMAs of the next tile's first four k-blocks go to the first
// accumulator, which is read first, before any goes to the second.
// Single: up to 128 rows of A in all (a few tokens against a vocabulary).  A pair would leave its odd CTA
// multiplying zero rows, so each CTA works alone on 128 x 256 tiles, with the narrow shape's segments
// and two buffers; B's read from HBM is then the bound.  With B K-major its tiles may be narrower than
// 256 columns (`width`, a multiple of 16; of twin products each `width` columns, a multiple of 8), so that the last round of CTAs is as full as the others, and
// A's loads bring only the rows there are (the MMA's other rows read what lies behind; nobody reads
// their sums): the ring is as deep as that allows, in at most 8 stages (16 or 24 gained nothing) of one, two or four
// k-blocks.
//   warp 0       TMA producer (both CTAs): its CTA's 128 rows of A and 128 rows of B per accumulator
//   warp 1       one thread of the even CTA issues the MMAs (M = 256, N = 256, K = 16)
//   warps 2..9   take the sums out of TMEM: warp w holds rows 32 (w & 3) .. + 31 of its CTA, one row
//                per lane, and 128 of an accumulator's 256 columns, in registers
// Segments (narrow and single): the tensor cores' fp32 accumulation loses a fraction of an ulp of the running
// sum at every step, always toward zero.  The sums restart every `seg_kb` k-blocks and the epilogue
// warps add the segments in registers with round-to-nearest additions, which bounds that bias whatever
// K is (a logit at K = 5120 comes out ~10x nearer to its 64-bit value than with one accumulator).  A
// segment is also the unit of the TMEM double buffer.  The wide shape never restarts, nor do twin products in
// the single one: they serve outputs that are the sum itself, rounded to bf16, with K up to kWideK (up to
// the caller's own limit where it gives pick_shape() one: 32768 for dX of the gated feed-forward).  A step loses up to 2^-22
// of the running sum, so 1024 steps lose up to 2^-12 of it and 2048 2^-11, next to the rounding's half step of 2^-8 of
// the value; where terms cancel, the loss is one of the running sum and not of the value.  They do not serve logits,
// whose exponentials turn a bias of the sum into one of the result.
// Every wait is bounded; the failure path is that of the Gram kernel: the first waiter that gives up
// records LOCA_ERR_TIMEOUT and raises the launch's abort flag, every role stops at its own point,
// the even CTA settles the copies that only one CTA issued, MMAs and copies in flight land, TMEM is
// freed and both CTAs leave together.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include <atomic>

#include "loca_internal.h"
#include "tc_ptx.cuh"

namespace loca {
namespace gp {

using namespace tc;

constexpr int TM = 256;               // tile rows per CTA pair
constexpr int TN = 256;               // columns of an accumulator
constexpr int HALF = 128;             // rows of A, and of B, loaded per CTA
constexpr int BK = 64;                // k per pipeline stage
constexpr int OPB = HALF * BK * 2;    // 16 KB: 128 rows of an operand in one stage
constexpr int SUB = 64 * BK * 2;      // one 64 x 64 swizzled box (8 KB)
constexpr int EPI_WARPS = 8;
constexpr int BOX = 4096;             // one epilogue warp's staging box: 32 rows x 128 bytes
constexpr int THREADS = 64 + 32 * EPI_WARPS;
constexpr int64_t kWideK = 16384;
constexpr int kMostPer = 4;           // k-blocks of a stage at most
enum : int { kNarrow = 0, kWide = 1, kSingle = 2 };
template <int kShape>
struct Shape {
  static constexpr int kCtas = kShape == kSingle ? 1 : 2;  // CTAs of a tile
  static constexpr int kAcc = kShape == kWide ? 2 : 1;     // accumulators of a tile
  static constexpr int kCols = TN * kAcc;
  static constexpr int kOpsB = kShape == kNarrow ? 1 : 2;  // 128-row operands of B per CTA and stage
  static constexpr int kStageBytes = (1 + kOpsB) * OPB;
  static constexpr int kStages = 12 * OPB / kStageBytes;
  static constexpr int kMostStages = kShape == kSingle ? 8 : kStages;
  static constexpr int kBars = 2 * kMostStages + 5;        // full[S], empty[S], acc_full[2], acc_empty[2], drain
};
constexpr int SMEM = 12 * OPB + EPI_WARPS * BOX + 256 + 1024;
static_assert(SMEM <= 232448, "shared memory per CTA");
static_assert(Shape<kNarrow>::kBars * 8 + 8 <= 256 && Shape<kSingle>::kBars * 8 + 8 <= 256, "barrier area");

// What the device chooses the number of k ranges by where fewer rows are live than the host planned for:
// the sums' room in row tiles, and the costs of cycles() with those of writing and adding a range's sums.
// 819 live rows of 8192 at d = 896, V = 32000: loss and dH 256 us with the host's ranges, 154 so.
// Integers throughout: the product and the kernel that adds its ranges come to the same number.
constexpr int kRangeCycles = 250;  // k_head_dh fetches four ranges at a time
struct Fit {
  int room = 0;  // row tiles x ranges that the sums' memory holds (0: the host's choice stands)
  int at_once, n_tiles, nkb;
  int kb_cycles, tile_cycles, row_tile_cycles;
};
__device__ __forceinline__ int fit_splits(const Fit& f, int planned, int m_planned, int m) {
  if (f.room == 0 || m < 1 || m >= m_planned) return planned;
  int most = f.room / m < 32 ? f.room / m : 32;
  if (most > f.nkb / 16) most = f.nkb / 16;
  const int tiles = m * f.n_tiles;
  int best = planned;
  int64_t best_c = 0;
#pragma unroll
  for (int r = 0; r <= 4; ++r) {  // as planned, or what fills one to four rounds
    int s = r == 0 ? planned : r * f.at_once / tiles;
    if (s > most) s = most;
    if (s < planned) s = planned;
    const int rounds = (tiles * s + f.at_once - 1) / f.at_once;
    const int64_t c = int64_t(rounds) * (f.kb_cycles * ((f.nkb + s - 1) / s) + f.tile_cycles) +
                      int64_t(s) * (int64_t(m) * f.row_tile_cycles + kRangeCycles);
    if (r == 0 || c + c / 32 < best_c) {  // (3 % is as near as the costs are known)
      best = s;
      best_c = c;
    }
  }
  return best;
}
// Row tiles of a piece that hold one of `rows` live rows, m_first row tiles before the piece; at least
// one in all, so that a call with no live row still writes zeros.
__device__ __forceinline__ int live_tiles(int rows, int m_first, int m_tiles) {
  int t = (rows + TM - 1) / TM;
  if (t < 1) t = 1;
  t -= m_first;
  if (t < 0) t = 0;
  return t < m_tiles ? t : m_tiles;
}

// One launch's work.  Tiles are taken in groups of `group` row tiles that sweep all column tiles,
// row tile fastest: the CTA pairs at work share a few column tiles and one group of row tiles,
// which stay in L2.
struct Geo {
  int m_tiles, n_tiles;  // upper bounds (rows_live may lower m_tiles, k_live the k-blocks); set by launch()
  int cols;              // columns of the output
  int width;             // columns of a tile (launch() sets all but the single shape's)
  int arows, stages;     // single shape, B K-major: rows of A's boxes, stages of the ring (launch())
  int per = 1;           // and k-blocks of a stage (launch())
  int nkb;               // k-blocks of the product
  int splits;            // the k-blocks are cut into this many ranges, each a tile of its own
  int seg_kb;            // k-blocks per accumulation segment
  int group;
  int m_first;           // row tiles of rows_live that come before this launch's rows
  const int32_t* rows_live;  // device count of rows of A that matter, or null
  const int32_t* k_live;     // device count of k that matter, or null
  int32_t* status;
  int32_t* abort_flag;
  unsigned long long limit_ns;
  int32_t mark = 1;  // value of the abort flag that means this launch's
  Fit fit;
};

struct Tile {
  int m, n, col0, split;
  int split_row;  // row tiles before this range's, times their rows
  int end;  // column behind the tile's last
  int kb0, kb1;
};

struct Live {
  int m_tiles, nkb, splits, total;
};

template <bool kFits, bool kSingleTile, bool kDeep>
__device__ __forceinline__ Live live_of(const Geo& g) {
  Live v;
  v.m_tiles = g.m_tiles;
  v.nkb = g.nkb;
  if (!kSingleTile && g.rows_live) v.m_tiles = live_tiles(*g.rows_live, g.m_first, g.m_tiles);
  if (!kSingleTile && g.k_live) {
    int t = (*g.k_live + BK - 1) / BK;
    if (t < 1) t = 1;
    if (t < v.nkb) v.nkb = t;
  }
  if (kDeep) v.nkb = (v.nkb + g.per - 1) / g.per;  // (from here on a k-block is all that a stage holds)
  v.splits = kFits ? fit_splits(g.fit, g.splits, g.m_tiles, v.m_tiles) : g.splits;
  v.total = v.m_tiles * g.n_tiles * v.splits;
  return v;
}

__device__ __forceinline__ Tile tile_of(const Geo& g, const Live& v, int it) {
  Tile t;
  const int per_split = v.m_tiles * g.n_tiles;
  t.split = it / per_split;
  int r = it - t.split * per_split;
  const int per_group = g.group * g.n_tiles;
  const int gi = r / per_group;
  r -= gi * per_group;
  const int m0 = gi * g.group;
  const int gm = v.m_tiles - m0 < g.group ? v.m_tiles - m0 : g.group;
  t.n = r / gm;
  t.m = m0 + r - t.n * gm;
  t.col0 = t.n * g.width;
  t.end = t.col0 + g.width < g.cols ? t.col0 + g.width : g.cols;
  t.split_row = t.split * v.m_tiles * TM;
  const int per = (v.nkb + v.splits - 1) / v.splits;
  t.kb0 = t.split * per < v.nkb ? t.split * per : v.nkb;
  t.kb1 = t.kb0 + per < v.nkb ? t.kb0 + per : v.nkb;
  return t;
}

// A call's value of its launches' abort flag, so that the workspace needs no clearing: no earlier call's (nor,
// but for one chance in 2^31, what else lay in the workspace).
inline int32_t call_mark() {
  static std::atomic<uint32_t> calls{0x1b873593u};
  return int32_t(calls.fetch_add(0x9e3779b1u, std::memory_order_relaxed) | 1u);
}

// Byte offset of 16-byte chunk `u` of row `row` in a 128-byte swizzled box.
__device__ __forceinline__ uint32_t box_off(int row, int u) {
  return uint32_t(row) * 128u + (uint32_t(u ^ (row & 7)) << 4);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// Hands a warp's 32 rows x 64 bf16 columns (thread `lane` holds its row's 32 pairs) to the TMA unit as
// one box of a 2-D map at (c0, r0).  The box buffer's previous contents have been read before it is
// written again.
__device__ __forceinline__ void store_box_bf16(uint8_t* box, const CUtensorMap* map, int lane, int c0, int r0,
                                               const uint32_t* w) {
  if (lane == 0) bulk_wait_group_read0();
  __syncwarp();
#pragma unroll
  for (int u = 0; u < 8; ++u)
    *reinterpret_cast<uint4*>(box + box_off(lane, u)) = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    if (LOCA_REQUIRE(c0 >= 0 && r0 >= 0 && c0 % 8 == 0)) tma_store_2d(map, smem_u32(box), c0, r0);
    bulk_commit_group();
  }
}

// Extension of the k axis: for row tile m, entries(m) further stages whose A rows come from the map
// tmAx (row coordinate a_row of the CTA's 128 rows) and whose B rows from tmBx (b_row0 + the tile's
// column, block b_block), ksteps() MMA steps of 16 each.  None here; the adapter projection has one.
struct NoExt {
  static constexpr bool kDeep = false;
  static constexpr bool kOn = false;
  static constexpr bool kSecond = false;
  static constexpr bool kTwin = false;
  static constexpr bool kEarlyA = false;
  __device__ int ksteps() const { return 4; }
  __device__ int entries(int) const { return 0; }
  __device__ void entry(int, int, uint32_t, int&, int&) const {}
};

// The k axis goes on from k-block `first` with a second pair of operands (maps tmAx and tmBx, laid out as the
// first pair): D = A B^T + A2 B2^T as one product.
struct SecondPair : NoExt {
  static constexpr bool kSecond = true;
  int first;
};

// Two products that share A: an accumulator holds the same columns of A B^T and of A B2^T (B2 from tmBx), side
// by side, so that the epilogue has both sums of an element in one thread.  A pair's even CTA loads the rows
// of B and its odd one those of B2, 128 columns of each; the single shape loads `width` of each.  Geo's
// columns and width are those of one product.
struct Twin : NoExt {
  static constexpr bool kTwin = true;
};

// fp32 sums of one k range, stored or added to the sums of earlier launches
// (one writer per element and launch: a fixed order of additions).
struct EpiAcc {
  static constexpr bool kPacks = false;
  static constexpr bool kAhead = false;
  static constexpr bool kFits = true;
  int add;

  __device__ __forceinline__ void operator()(const Tile& t, float (&v)[128], int row, int col0, int lane, uint8_t* box,
                                             const CUtensorMap* out) const {
    const int r0 = t.split_row + row - lane;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (lane == 0) bulk_wait_group_read0();
      __syncwarp();
#pragma unroll
      for (int u = 0; u < 8; ++u)
        *reinterpret_cast<float4*>(box + box_off(lane, u)) =
            make_float4(v[32 * b + 4 * u], v[32 * b + 4 * u + 1], v[32 * b + 4 * u + 2], v[32 * b + 4 * u + 3]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        if (LOCA_REQUIRE(col0 >= 0 && r0 >= 0)) {
          if (add) tma_reduce_add_2d(out, smem_u32(box), col0 + 32 * b, r0);
          else tma_store_2d(out, smem_u32(box), col0 + 32 * b, r0);
        }
        bulk_commit_group();
      }
    }
  }
};

struct NoState {};
template <class Epi, bool kOn>
struct StateOf {
  using type = NoState;
};
template <class Epi>
struct StateOf<Epi, true> {
  using type = typename Epi::State;
};

// Scaled and rounded once.
struct EpiScaled {
  static constexpr bool kPacks = true;
  static constexpr bool kAhead = false;
  static constexpr bool kFits = false;
  static constexpr bool kSums = false;
  float scale;

  struct Row {};
  __device__ __forceinline__ Row row_of(int) const { return Row{}; }
  __device__ __forceinline__ float value(const Row&, int, float v) const { return scale * v; }
};

// Single shape: A is the caller's too, and only the epilogue needs the launch before (which lets this one start
// after all launches before it have completed): the producer waits for it at its own end.
struct CallersA : NoExt {
  static constexpr bool kEarlyA = true;
};

// Single shape, B K-major: two or four k-blocks to a stage (Geo::per).  A kernel of its own: the choice at run time took one
// token 2 us more of 51 at 2048 x 49152, where a stage holds one.
template <class Ext>
struct Deep : Ext {
  static constexpr bool kDeep = true;
};

// What becomes of a finished tile.  An output in bf16 is given value by value (kPacks): Row row_of(row)
// reads what a row needs, before its sums are complete; value(Row, column, sum) is the output.  kSums (not
// in the wide shape): Row adds something up over the values, which finish(Row, half tile, row) gets.  Other
// uses take the sums themselves:  void operator()(const Tile&, float (&v)[128], int row, int col0, int lane,
//                                   uint8_t* box, const CUtensorMap* out) const
// called once per finished accumulator by every epilogue thread, with the sums of row `row`, columns
// col0 .. col0 + 127.  With twin products:  Row before(int row, int col0), called before the sums are complete,
// and operator()(const Tile&, float (&v)[128], Row&, int row, int col0, int lane, uint8_t* box, out, out2) with 64
// columns of the first product in v[0 .. 63] and the same of the second behind them; out2 is tmAx.  The single shape,
// whose tiles are no whole boxes, calls store8(float (&v)[16], int row, int col) for 8 columns of both, in warps that
// hold one of the epilogue's `rows`.
// kAhead (narrow and single): what an epilogue has to look up for a tile is on its way while the sums are not
// complete: a State for each thread; start(State, row of the first tile), ahead(State, row, half tile, row of the next
// tile) before the sums; the state goes to operator().  With kPacks  void all(float (&v)[128], State, int row, int col0,
// int half tile) puts the values in the sums' place in the narrow shape; in the single shape, whose one tile waits for
// each instruction's first fetch, the state goes to row_of(), which also gets the first column, bool simple(Row) chooses
// for a warp between value1() and value(), where low_row is not 0, store_parts(float (&)[32], row, column) takes the values
// of the rows before it, and finish(Row::others, half tile, row) what the values add up to.
// kFits: the number of k ranges is the device's choice (Fit).
template <int kShape, bool kAmn, bool kBmn, class Epi, class Ext>
__global__ void __cluster_dims__(Shape<kShape>::kCtas, 1, 1) __launch_bounds__(THREADS, 1)
    k_gemm_pair(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                const __grid_constant__ CUtensorMap tmAx, const __grid_constant__ CUtensorMap tmBx,
                const __grid_constant__ CUtensorMap tmO, const __grid_constant__ Geo g,
                const __grid_constant__ Epi epi, const __grid_constant__ Ext ext) {
  using S = Shape<kShape>;
  constexpr bool kPair = S::kCtas == 2;
  static_assert(kPair || !Ext::kOn, "an extended k axis takes pairs");
  static_assert(!Ext::kTwin || (!kAmn && !kBmn), "twin products are of K-major operands");
  constexpr int MOST = S::kMostStages, BARS = S::kBars;
  constexpr bool kSlim = kShape == kSingle && !kBmn;  // tiles of `width` columns: two boxes of width / 2 rows
  const int STAGES = kSlim ? g.stages : S::kStages;
  const uint32_t a_bytes = kSlim ? uint32_t(g.arows) * 128u : uint32_t(OPB);
  const uint32_t b_cols = kSlim ? uint32_t(g.width) * (Ext::kTwin ? 2u : 1u) : uint32_t(TN);  // of an accumulator
  constexpr bool kDeep = Ext::kDeep;
  const int per = kDeep ? g.per : 1, seg_kb = kDeep ? g.seg_kb / g.per : g.seg_kb;
  const uint32_t STAGE_BYTES = kSlim ? uint32_t(per) * (a_bytes + b_cols * 128u) : uint32_t(S::kStageBytes);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* boxes = smem + 12 * OPB;
  uint64_t* bars = reinterpret_cast<uint64_t*>(boxes + EPI_WARPS * BOX);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + BARS);
  uint32_t* odd_issued = tmem_slot + 1;
  const uint32_t smem_base = smem_u32(smem);
  const uint32_t bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (MOST + s); };
  auto acc_full = [&](uint32_t b) { return bar_base + 8u * (2 * MOST + b); };
  auto acc_empty = [&](uint32_t b) { return bar_base + 8u * (2 * MOST + 2 + b); };
  const uint32_t drain_bar = bar_base + 8u * (2 * MOST + 4);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int cid = int(cluster_id_x());
  const int ncl = int(ncluster_x());
  const WaitCtl wc{g.status, g.abort_flag, g.limit_ns, g.mark};

  if (threadIdx.x == 0) {
    for (int s = 0; s < MOST; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(acc_full(b), 1);
      mbar_init(acc_empty(b), S::kCtas * EPI_WARPS);  // lane 0 of the epilogue warps
    }
    mbar_init(drain_bar, 1);
    *odd_issued = 0;
    mbar_init_fence();
    prefetch_tensormap(&tmA);
    prefetch_tensormap(&tmB);
    prefetch_tensormap(&tmO);
    if (Ext::kOn || Ext::kSecond || Ext::kTwin) {
      prefetch_tensormap(&tmAx);
      prefetch_tensormap(&tmBx);
    }
  }
  if (warp == 1) {
    if (kPair) tmem_alloc_pair(smem_u32(tmem_slot), 512);
    else tmem_alloc(smem_u32(tmem_slot), 512);
  }
  fence_before();
  cluster_sync();
  fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // The launch before has completed (the prologue above ran beside its end).  With an extended k axis
  // only the extension is that launch's work, which let this one start after all launches before it had
  // completed: the producer waits when it comes to the extension.  In the single shape B is the caller's
  // (the launch before makes A and lets this one start only after all before it): the producer fills the
  // ring with B first.  (Twin products come first in their call: B may be the work of the launch before.)
  constexpr bool kEarlyB = kShape == kSingle && !Ext::kTwin;
  if (!Ext::kOn && !(kEarlyB && warp == 0)) wait_for_previous();
  if (!(kEarlyB && warp == 0)) launch_dependents();
  const Live lv = live_of<Epi::kFits, kShape == kSingle, Ext::kDeep>(g);
  uint32_t iters_done = 0;

  if (warp == 0) {
    if (lane == 0) {
      // ---------------- TMA producer (both CTAs)
      int stage = 0;
      uint32_t phase = 0;
      uint32_t iter = 0;
      bool ok = true, waited = !Ext::kOn && !(kEarlyB && Ext::kEarlyA);
      auto load = [&](uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
        if constexpr (kPair) tma_load_2d_pair(dst, map, bar, c0, c1);
        else tma_load_2d(dst, map, bar, c0, c1);
      };
      // k-block kb: of the second pair from `first` on
      auto second = [&](int& kb) {
        if constexpr (Ext::kSecond) {
          if (kb >= ext.first) {
            kb -= ext.first;
            return true;
          }
        }
        return false;
      };
      auto load_a = [&](const Tile& t, int s, int kb, uint32_t fb) {
        const uint32_t a = smem_base + uint32_t(s) * STAGE_BYTES;
        const int m0 = t.m * TM + int(rank) * HALF;
        const CUtensorMap* map = second(kb) ? &tmAx : &tmA;
        const int k0 = kb * BK;
        if (kAmn) {
          load(a, map, fb, m0, k0);
          load(a + SUB, map, fb, m0 + 64, k0);
        } else {
          load(a, map, fb, per * k0, m0);
          if constexpr (kDeep) {
#pragma unroll
            for (int i = 1; i < kMostPer; ++i)
              if (i < per) load(a + i * a_bytes, map, fb, per * k0 + i * BK, m0);
          }
        }
      };
      // 128 rows of B per operand: this CTA's half of each accumulator, or (single) both halves
      auto load_b = [&](const Tile& t, int s, int kb, uint32_t fb) {
        const uint32_t b = smem_base + uint32_t(s) * STAGE_BYTES + uint32_t(per) * a_bytes;
        const CUtensorMap* map = second(kb) ? &tmBx : &tmB;
        const int k0 = kb * per * BK;
#pragma unroll
        for (int c = 0; c < S::kOpsB; ++c) {
          if constexpr (Ext::kTwin) {
            if constexpr (kSlim) {
              const uint32_t at = b + c * uint32_t(g.width) * 128u;
              load(at, c ? &tmBx : &tmB, fb, k0, t.col0);
              if constexpr (kDeep) {
#pragma unroll
                for (int i = 1; i < kMostPer; ++i)
                  if (i < per) load(at + i * b_cols * 128u, c ? &tmBx : &tmB, fb, k0 + i * BK, t.col0);
              }
            } else {
              load(b + c * OPB, rank ? &tmBx : &tmB, fb, k0, t.col0 + c * HALF);
            }
            continue;
          }
          const int n = t.col0 + int(rank) * HALF + c * (kPair ? TN : kSlim ? g.width / 2 : HALF);
          if (kSlim) {
            const uint32_t at = b + c * uint32_t(g.width * BK);
            load(at, map, fb, k0, n);
            if constexpr (kDeep) {
#pragma unroll
              for (int i = 1; i < kMostPer; ++i)
                if (i < per) load(at + i * b_cols * 128u, map, fb, k0 + i * BK, n);
            }
          } else if (kBmn) {
            load(b + c * OPB, map, fb, n, k0);
            load(b + c * OPB + SUB, map, fb, n + 64, k0);
          } else {
            load(b + c * OPB, map, fb, k0, n);
          }
        }
      };
      uint32_t early = 0;
      if constexpr (kEarlyB) {
        if (cid < lv.total) {
          const Tile t = tile_of(g, lv, cid);
          for (; int(early) < STAGES && int(early) < t.kb1 - t.kb0; ++early) {
            mbar_arrive_expect_tx(full_bar(int(early)), STAGE_BYTES);
            load_b(t, int(early), t.kb0 + int(early), full_bar(int(early)));
          }
        }
        if constexpr (!Ext::kEarlyA) wait_for_previous();
      }
      for (int it = cid; it < lv.total && ok; it += ncl) {
        const Tile t = tile_of(g, lv, it);
        const int nx = Ext::kOn ? ext.entries(t.m) : 0;
        const int nb = t.kb1 - t.kb0;
        for (int j = 0; j < nb + nx; ++j) {
          const bool ahead = kEarlyB && iter < early;
          if (!ahead && !mbar_try_wait_cluster(empty_bar(stage), phase ^ 1u) &&
              !mbar_wait_cluster(empty_bar(stage), phase ^ 1u, wc)) {
            ok = false;
            break;
          }
          if (leader && !ahead) mbar_arrive_expect_tx(full_bar(stage), uint32_t(S::kCtas) * STAGE_BYTES);
          const uint32_t fb = kPair ? mapa_shared(full_bar(stage), 0) : full_bar(stage);
          if (!Ext::kOn || j < nb) {
            load_a(t, stage, t.kb0 + j, fb);
            if (!ahead) load_b(t, stage, t.kb0 + j, fb);
          } else {
            if (!waited) {
              wait_for_previous();
              waited = true;
            }
            int a_row, at;
            ext.entry(t.m, j - nb, rank, a_row, at);
            const uint32_t a = smem_base + uint32_t(stage) * STAGE_BYTES, b = a + a_bytes;
            tma_load_2d_pair(a, &tmAx, fb, 0, a_row);
#pragma unroll
            for (int c = 0; c < S::kAcc; ++c)
              tma_load_3d_pair(b + c * OPB, &tmBx, fb, 0, t.col0 + int(rank) * HALF + c * TN, at);
          }
          ++iter;
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
      if (!waited) wait_for_previous();  // this launch ends after the one before it
      if (!leader) st_shared_cluster_u32(mapa_shared(smem_u32(odd_issued), 0), iter);
      iters_done = iter;
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && leader) {
      // ---------------- MMA issuer (even CTA)
      int stage = 0;
      uint32_t phase = 0, seg = 0;
      bool ok = true, issued = false;
      constexpr uint32_t kKLbo = 16u;  // K-major with the 128-byte swizzle: leading offset unused
      const uint64_t a_kmaj = sdesc(smem_base, kKLbo, 1024u, kSwizzle128B);
      const uint64_t a0 = kAmn ? sdesc(smem_base, SUB, 1024u, kSwizzle128B) : a_kmaj;
      const uint64_t b_kmaj = sdesc(smem_base + uint32_t(per) * a_bytes, kKLbo, 1024u, kSwizzle128B);
      const uint64_t b0 = kBmn ? sdesc(smem_base + a_bytes, SUB, 1024u, kSwizzle128B) : b_kmaj;
      constexpr uint64_t kAStep = kAmn ? 2048 >> 4 : 32 >> 4, kBStep = kBmn ? 2048 >> 4 : 32 >> 4;
      const uint32_t id = tc::idesc(1, 1, kAmn ? 1 : 0, kBmn ? 1 : 0, S::kCtas * HALF, b_cols);
      constexpr uint32_t kIdX = tc::idesc(1, 1, 0, 0, TM, TN);
      // the MMAs of one k-block into accumulator c
      auto block = [&](int s, uint32_t d, int c, bool from_ext, bool first) {
        const uint64_t so = uint64_t(s) * uint64_t(STAGE_BYTES >> 4), bo = so + uint64_t(c) * uint64_t(OPB >> 4);
        if (!Ext::kOn || !from_ext) {
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk)
            if constexpr (kPair)
              mma_f16_pair(d, a0 + so + kk * kAStep, b0 + bo + kk * kBStep, id, !first || kk != 0 ? 1u : 0u);
            else
              mma_f16(d, a0 + so + kk * kAStep, b0 + bo + kk * kBStep, id, !first || kk != 0 ? 1u : 0u);
          if constexpr (kDeep) {
#pragma unroll
            for (int i = 1; i < kMostPer; ++i)
              if (i < per) {
#pragma unroll
                for (int kk = 0; kk < BK / 16; ++kk)
                  mma_f16(d, a0 + so + i * (a_bytes >> 4) + kk * kAStep, b0 + bo + i * (b_cols * 128u >> 4) + kk * kBStep, id, 1u);
              }
          }
        } else {
          for (int kk = 0; kk < ext.ksteps(); ++kk)
            mma_f16_pair(d, a_kmaj + so + kk * 2, b_kmaj + bo + kk * 2, kIdX, !first || kk != 0 ? 1u : 0u);
        }
      };
      auto commit = [&](uint32_t bar) {
        if constexpr (kPair) mma_commit_pair_mc(bar, 0x3);
        else mma_commit(bar);
      };
      auto wait_full = [&](int s, uint32_t ph) {
        if (!mbar_try_wait_cluster(full_bar(s), ph) && !mbar_wait_cluster(full_bar(s), ph, wc)) return false;
        fence_after();
        return true;
      };
      auto wait_acc = [&](uint32_t b, uint32_t ph) {
        if (!mbar_try_wait_cluster(acc_empty(b), ph) && !mbar_wait_cluster(acc_empty(b), ph, wc)) return false;
        fence_after();
        return true;
      };
      for (int it = cid; it < lv.total && ok; it += ncl) {
        const Tile t = tile_of(g, lv, it);
        const int nb = t.kb1 - t.kb0;
        const int all = nb + (Ext::kOn ? ext.entries(t.m) : 0);
        if constexpr (kShape == kWide) {
          if (all == 0) continue;
          const bool two = g.cols - t.col0 > (Ext::kTwin ? HALF : TN);  // the second accumulator holds columns of the output
          const int head = all < STAGES ? all : STAGES;
          const int stage0 = stage;
          ok = wait_acc(0, (seg & 1u) ^ 1u);
          for (int j = 0; ok && j < head; ++j) {
            if (!(ok = wait_full(stage, phase))) break;
            block(stage, tmem_base, 0, j >= nb, j == 0);
            issued = true;
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          }
          // (waited for without a second accumulator too: acc_full(1) must not complete twice unseen)
          if (!ok || !(ok = wait_acc(1, (seg & 1u) ^ 1u))) break;
          if (all == head) commit(acc_full(0));
          for (int j = 0, s = stage0; j < head; ++j) {
            if (two) block(s, tmem_base + uint32_t(TN), 1, j >= nb, j == 0);
            commit(empty_bar(s));
            if (++s == STAGES) s = 0;
          }
          for (int j = head; j < all; ++j) {
            if (!(ok = wait_full(stage, phase))) break;
            block(stage, tmem_base, 0, j >= nb, false);
            if (j == all - 1) commit(acc_full(0));
            if (two) block(stage, tmem_base + uint32_t(TN), 1, j >= nb, false);
            commit(empty_bar(stage));
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          }
          if (!ok) break;
          // (a tile without a second accumulator completes that barrier all the same: one phase a tile)
          commit(acc_full(1));
          ++seg;
        } else {
          uint32_t d = 0;
          for (int j = 0, in_seg = 0; j < all; ++j) {
            if (in_seg == 0) {
              const uint32_t b = seg & 1u;
              if (!(ok = wait_acc(b, ((seg >> 1) & 1u) ^ 1u))) break;
              d = tmem_base + b * uint32_t(TN);
            }
            if (!(ok = wait_full(stage, phase))) break;
            block(stage, d, 0, j >= nb, in_seg == 0);
            issued = true;
            commit(empty_bar(stage));
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            if (++in_seg == seg_kb || j == all - 1) {
              commit(acc_full(seg & 1u));
              ++seg;
              in_seg = 0;
            }
          }
        }
      }
      if (issued) {
        if (kPair) mma_commit_pair(drain_bar);
        else mma_commit(drain_bar);
        mbar_drain(drain_bar, 0, kDrainLimitNs);
      }
    }
    __syncwarp();
  } else {
    // ---------------- epilogue: warps 2..9; TMEM lane quarter = warp % 4, column half = (warp - 2) / 4
    const int q = warp & 3;
    const int h = (warp - 2) >> 2;
    uint8_t* box = boxes + (warp - 2) * BOX;
    uint32_t seg = 0;
    bool go = true;
    typename StateOf<Epi, Epi::kAhead>::type state;
    if constexpr (Epi::kAhead)
      if (cid < lv.total) epi.start(state, tile_of(g, lv, cid).m * TM + int(rank) * HALF + q * 32 + lane);
    for (int it = cid; it < lv.total && go; it += ncl) {
      const Tile t = tile_of(g, lv, it);
      const int all = t.kb1 - t.kb0 + (Ext::kOn ? ext.entries(t.m) : 0);
      const int row = t.m * TM + int(rank) * HALF + q * 32 + lane;
      auto wait_sums = [&](uint32_t b, uint32_t par) {
        const bool ok = mbar_wait_cluster(acc_full(b), par, wc);
        const bool every = __all_sync(0xffffffffu, ok);
        fence_after();
        return every;
      };
      auto release = [&](uint32_t b) {  // this warp has read the accumulator
        fence_before();
        __syncwarp();
        if (lane == 0) {
          if (leader) mbar_arrive(acc_empty(b));
          else mbar_arrive_remote(mapa_shared(acc_empty(b), 0));
        }
      };
      const int r0 = row - lane;
      if constexpr (Ext::kTwin && kSlim) {
        // Half of the tile's columns (in units of 8) of the first product, and the same of the second `width` columns
        // behind.  One sum per tile (launch()), and code that runs once: a loop over 8 columns straight from
        // tensor memory, whose instructions need not all be fetched for one tile (64 columns from registers at a
        // time: one token at 3584 x 14336 46.7 us, so 37.5).  Warps without a row do nothing.
        const int half = (g.width / 2 + 7) / 8 * 8, col0 = t.col0 + h * half, end = col0 + half < t.end ? col0 + half : t.end;
        const uint32_t b = seg & 1u;
        if (!(go = wait_sums(b, (seg >> 1) & 1u))) break;
        const uint32_t ta = tmem_base + (uint32_t(q * 32) << 16) + b * uint32_t(TN) + uint32_t(h * half);
        if (r0 < epi.rows)
#pragma unroll 1
          for (int c = 0; col0 + c < end; c += 8) {
            float v[16];
            tmem_ld8x2(ta + uint32_t(c), uint32_t(g.width), v);
            epi.store8(v, row, col0 + c);
          }
        release(b);
        ++seg;
      } else if constexpr (Ext::kTwin) {
        // 64 columns of the first product and the same of the second, for every accumulator
        const int nseg = kShape == kWide ? 1 : (all + seg_kb - 1) / seg_kb;
#pragma unroll 1
        for (uint32_t a = 0; a < uint32_t(S::kAcc); ++a) {
          const int col0 = t.col0 + int(a) * HALF + h * 64;
          auto pre = epi.before(row, col0);
          float v[128];
          for (int s = 0; s < nseg; ++s) {
            const uint32_t n = kShape == kWide ? seg : (seg + uint32_t(s)) >> 1;
            const uint32_t b = kShape == kWide ? a : (seg + uint32_t(s)) & 1u;
            if (!(go = wait_sums(b, n & 1u))) break;
            const uint32_t ta = tmem_base + (uint32_t(q * 32) << 16) + b * uint32_t(TN) + uint32_t(h * 64);
            if (s == 0) {
#pragma unroll
              for (int c = 0; c < 4; ++c) tmem_ld32(ta + (c & 1) * 32 + (c >> 1) * HALF, v + c * 32);
            } else {
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                float u[32];
                tmem_ld32(ta + (c & 1) * 32 + (c >> 1) * HALF, u);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[c * 32 + i] += u[i];
              }
            }
            release(b);
          }
          if (!go) break;
          if (col0 < t.end) epi(t, v, pre, row, col0, lane, box, &tmO, &tmAx);
        }
        if (!go) break;
        seg += uint32_t(nseg);
      } else if constexpr (kShape == kWide && Epi::kPacks) {
        // both accumulators are in registers, rounded and packed, before the stores that the MMAs need
        // not wait for: 64 words of the first, of which a box (32) leaves before the second is read
        const auto pre = epi.row_of(row);
        const int col0 = t.col0 + h * HALF, col1 = col0 + TN;
        const uint32_t ta = tmem_base + (uint32_t(q * 32) << 16) + uint32_t(h * HALF);
        auto take = [&](uint32_t a, int col, uint32_t* w) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float v[32];
            tmem_ld32(ta + a * uint32_t(TN) + c * 32, v);
#pragma unroll
            for (int i = 0; i < 16; ++i)
              w[c * 16 + i] = pack_bf16(epi.value(pre, col + c * 32 + 2 * i, all > 0 ? v[2 * i] : 0.f),
                                        epi.value(pre, col + c * 32 + 2 * i + 1, all > 0 ? v[2 * i + 1] : 0.f));
          }
        };
        uint32_t w0[64], w1[64];
        if (all > 0 && !(go = wait_sums(0, seg & 1u))) break;
        take(0, col0, w0);
        if (all > 0) release(0);
        if (col0 < g.cols) store_box_bf16(box, &tmO, lane, col0, r0, w0);
        if (all > 0 && !(go = wait_sums(1, seg & 1u))) break;
        take(1, col1, w1);
        if (all > 0) release(1);
        if (col0 + 64 < g.cols) store_box_bf16(box, &tmO, lane, col0 + 64, r0, w0 + 32);
        if (col1 < g.cols) store_box_bf16(box, &tmO, lane, col1, r0, w1);
        if (col1 + 64 < g.cols) store_box_bf16(box, &tmO, lane, col1 + 64, r0, w1 + 32);
        if (all > 0) ++seg;
      } else if constexpr (kShape == kWide) {
#pragma unroll 1
        for (uint32_t a = 0; a < 2; ++a) {
          if (all > 0 && !(go = wait_sums(a, seg & 1u))) break;
          const uint32_t ta = tmem_base + (uint32_t(q * 32) << 16) + a * uint32_t(TN) + uint32_t(h * HALF);
          float v[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32(ta + c * 32, v + c * 32);
          if (all > 0) release(a);
          if (all == 0) {  // no k: the sums are zero
#pragma unroll
            for (int i = 0; i < 128; ++i) v[i] = 0.f;
          }
          const int col0 = t.col0 + int(a) * TN + h * HALF;
          if (col0 < g.cols) epi(t, v, row, col0, lane, box, &tmO);
        }
        if (!go) break;
        if (all > 0) ++seg;
      } else {
        if constexpr (Epi::kAhead) {
          const int after = it + ncl < lv.total ? tile_of(g, lv, it + ncl).m - t.m : 0;
          epi.ahead(state, row, 2 * t.n + h, row + after * TM);
        }
        const int nseg = (all + seg_kb - 1) / seg_kb;
        float v[128];
        if (nseg == 0) {
#pragma unroll
          for (int i = 0; i < 128; ++i) v[i] = 0.f;
        }
        for (int s = 0; s < nseg; ++s, ++seg) {
          const uint32_t b = seg & 1u;
          if (!(go = wait_sums(b, (seg >> 1) & 1u))) break;
          const uint32_t ta = tmem_base + (uint32_t(q * 32) << 16) + b * uint32_t(TN) + uint32_t(h * HALF);
          if (s == 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(ta + c * 32, v + c * 32);
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              float u[32];
              tmem_ld32(ta + c * 32, u);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[c * 32 + i] += u[i];
            }
          }
          release(b);
        }
        if (!go) break;
        const int col0 = t.col0 + h * HALF;
        if constexpr (Epi::kPacks) {
          const auto store = [&](auto value) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              if (col0 + 64 * b >= (kSlim ? t.end : g.cols)) continue;
              uint32_t w[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float lo = value(64 * b + 2 * i), hi = value(64 * b + 2 * i + 1);
                w[i] = pack_bf16(lo, hi);
              }
              store_box_bf16(box, &tmO, lane, col0 + 64 * b, r0, w);
            }
          };
          if constexpr (Epi::kAhead && kShape == kSingle) {
            auto pre = epi.row_of(row, state, col0);
            const bool simple = epi.simple(pre);
            if (epi.low_row > 0) {  // rows below low_row are given in two parts, the second low_row rows behind
              if (q * 32 >= epi.low_row) continue;
#pragma unroll 1
              for (int b = 0; b < 4; ++b) {
                if (col0 + 64 * (b >> 1) >= t.end) break;  // (whole k-blocks of what reads them)
                float f[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  f[i] = v[i];
#pragma unroll
                  for (int c = 1; c < 4; ++c) f[i] = c == b ? v[32 * c + i] : f[i];
                }
                if (simple) {
#pragma unroll
                  for (int i = 0; i < 32; ++i) f[i] = epi.value1(pre, col0 + 32 * b + i, f[i]);
                } else {
#pragma unroll
                  for (int i = 0; i < 32; ++i) f[i] = epi.value(pre, col0 + 32 * b + i, f[i]);
                }
                epi.store_parts(f, row, col0 + 32 * b);
              }
              epi.finish(pre.others, 2 * t.n + h, row);
              continue;
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              if (col0 + 64 * b >= (kSlim ? t.end : g.cols)) continue;
              uint32_t w[32];
              if (simple) {
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const float lo = epi.value1(pre, col0 + 64 * b + 2 * i, v[64 * b + 2 * i]);
                  const float hi = epi.value1(pre, col0 + 64 * b + 2 * i + 1, v[64 * b + 2 * i + 1]);
                  w[i] = pack_bf16(lo, hi);
                }
              } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const float lo = epi.value(pre, col0 + 64 * b + 2 * i, v[64 * b + 2 * i]);
                  const float hi = epi.value(pre, col0 + 64 * b + 2 * i + 1, v[64 * b + 2 * i + 1]);
                  w[i] = pack_bf16(lo, hi);
                }
              }
              store_box_bf16(box, &tmO, lane, col0 + 64 * b, r0, w);
            }
            epi.finish(pre.others, 2 * t.n + h, row);
          } else if constexpr (Epi::kAhead) {
            epi.all(v, state, row, col0, 2 * t.n + h);
            store([&](int i) { return v[i]; });
          } else {
            auto pre = epi.row_of(row);
            store([&](int i) { return epi.value(pre, col0 + i, v[i]); });
            if constexpr (Epi::kSums) epi.finish(pre, 2 * t.n + h, row);
          }
        } else if constexpr (Epi::kAhead) {
          epi(t, v, state, row, col0, lane, box, &tmO);
        } else {
          epi(t, v, row, col0, lane, box, &tmO);
        }
      }
    }
    if (lane == 0) bulk_wait_group0();  // every box written before the CTA can leave
    __syncwarp();
  }

  fence_before();
  cluster_sync();  // every role has stopped; the odd CTA's issue count is visible
  fence_after();
  if (warp == 0 && lane == 0 && leader) {
    // Copies in flight when a role gave up: every stage carries the same bytes.  An iteration the
    // odd CTA never issued gets its bytes settled, one only the odd CTA issued gets armed, and each
    // of the last STAGES iterations is waited for (the earlier ones have landed).
    const uint32_t n_even = iters_done;
    const uint32_t n_odd = kPair ? *reinterpret_cast<volatile uint32_t*>(odd_issued) : n_even;
    const uint32_t hi = n_even > n_odd ? n_even : n_odd;
    const uint32_t lo = hi > uint32_t(STAGES) ? hi - uint32_t(STAGES) : 0u;
    for (uint32_t i = lo; i < hi; ++i) {
      const int s = int(i % STAGES);
      if (i >= n_odd && i < n_even) mbar_complete_tx(full_bar(s), STAGE_BYTES);
      else if (i >= n_even && i < n_odd) mbar_arrive_expect_tx(full_bar(s), STAGE_BYTES);
      mbar_drain(full_bar(s), (i / STAGES) & 1u, kDrainLimitNs);
    }
  }
  fence_before();
  cluster_sync();
  fence_after();
  if (warp == 1) {
    if (kPair) tmem_dealloc_pair(tmem_base, 512);
    else tmem_dealloc(tmem_base, 512);
  }
}

// ------------------------------------------------------------------ host side
// 2-D map of a row-major matrix: `cols` contiguous elements, `rows` rows, pitch in elements.
inline bool map_2d(CUtensorMap* m, CUtensorMapDataType type, int esize, const void* base, int64_t cols, int64_t rows,
                   int64_t pitch, int box_cols, int box_rows) {
  auto fn = tensor_map_encoder();
  if (!fn) return false;
  cuuint64_t dims[2] = {cuuint64_t(cols), cuuint64_t(rows)};
  cuuint64_t strides[1] = {cuuint64_t(pitch) * esize};
  cuuint32_t box[2] = {cuuint32_t(box_cols), cuuint32_t(box_rows)};
  cuuint32_t estr[2] = {1, 1};
  return fn(m, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
inline bool map_3d(CUtensorMap* m, CUtensorMapDataType type, int esize, const void* base, int64_t cols, int64_t rows,
                   int64_t blocks, int64_t pitch, int64_t block_pitch, int box_cols, int box_rows) {
  auto fn = tensor_map_encoder();
  if (!fn) return false;
  cuuint64_t dims[3] = {cuuint64_t(cols), cuuint64_t(rows), cuuint64_t(blocks)};
  cuuint64_t strides[2] = {cuuint64_t(pitch) * esize, cuuint64_t(block_pitch) * esize};
  cuuint32_t box[3] = {cuuint32_t(box_cols), cuuint32_t(box_rows), 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, type, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// An operand whose k is contiguous: boxes of 64 k x 128 rows.
inline bool map_kmajor(CUtensorMap* m, const void* base, int64_t k, int64_t rows, int64_t pitch) {
  return map_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, k, rows, pitch, BK, HALF);
}
// An operand whose rows (m or n) are contiguous: boxes of 64 rows x 64 k.
inline bool map_mnmajor(CUtensorMap* m, const void* base, int64_t rows, int64_t k, int64_t pitch) {
  return map_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, rows, k, pitch, 64, BK);
}
// A bf16 output written in boxes of 64 columns x 32 rows.
inline bool map_out_bf16(CUtensorMap* m, void* base, int64_t cols, int64_t rows, int64_t pitch) {
  return map_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, cols, rows, pitch, 64, 32);
}

// Lets a kernel have `bytes` of dynamic shared memory, asked for once on each device (`done`: a bit for each, of that
// kernel alone), which saves 0.45 us of the host's time for a launch.
inline cudaError_t allow_smem(std::atomic<uint64_t>& done, const void* kernel, int bytes) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// Small kernels between those with 200 KB of shared memory ask for the same split of L1: changing it
// drains the SM (64 single tokens through an adapted projection: 27.1 us with the change, 23.4 without).
template <class K>
inline cudaError_t keep_carveout(K kernel) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
}

// A launch whose prologue may run beside the end of the launch before it; the kernel calls
// wait_for_previous() before it touches what that launch reads or writes.
template <class... P, class... A>
inline cudaError_t launch_early(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (smem == 0) {
    const cudaError_t e = keep_carveout(kernel);
    if (e != cudaSuccess) return e;
  }
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Which shape: rounds of the pairs times a tile's cycles.  Measured on 1024 x 19456 outputs (4 narrow, 2
// wide rounds) at k = 512 .. 8192: narrow 672 cycles a k-block and 3000 a tile, wide 1030 and 9000 (both
// with a share of the launch and of the last tiles' stores); at k = 8192 204 and 170 us (1.60 and 1.92
// PFLOP/s), at k = 512 25 us each.  (The k-blocks of an extended k axis are not counted: the device alone
// knows them.)
inline double kb_cycles(int shape) { return shape == kWide ? 1030.0 : 672.0; }
inline double tile_cycles(int shape) { return shape == kWide ? 9000.0 : 3000.0; }
inline double cycles(int shape, int64_t m_tiles, int64_t cols, int64_t nkb, int splits) {
  const int64_t n = shape == kWide ? (cols + 2 * TN - 1) / (2 * TN) : (cols + TN - 1) / TN;
  const int64_t at_once = shape == kSingle ? sm_count() : sm_count() / 2;
  const double rounds = double((m_tiles * n * splits + at_once - 1) / at_once);
  const double kb = double((nkb + splits - 1) / splits);
  return rounds * (kb_cycles(shape) * kb + tile_cycles(shape));
}
// rows: those of A, where 128 or fewer may take the single shape (0: they may not).  wide_k: the longest k range
// that the wide shape may sum.
inline int pick_shape(int64_t rows, int64_t m_tiles, int64_t cols, int64_t nkb, int splits, int64_t wide_k = kWideK) {
  if (rows > 0 && rows <= HALF) return kSingle;
  const bool wide = cycles(kWide, m_tiles, cols, nkb, splits) < cycles(kNarrow, m_tiles, cols, nkb, splits);
  return wide && nkb <= wide_k / BK * splits ? kWide : kNarrow;
}

// Width of the single shape's tiles: as few rounds of the CTAs as 256 columns would take, in equal parts
// of whole units of 16 columns (64 where they are stored in boxes).
inline int slim_width(int64_t cols, int unit = 16) {
  const int64_t at_once = sm_count();
  const int64_t rounds = (cols + TN * at_once - 1) / (TN * at_once);
  const int64_t w = (cols + rounds * at_once - 1) / (rounds * at_once);
  return int((w + unit - 1) / unit * unit);
}

// (static: a kernel of the same name is another one in each source file, with an `allowed` of its own.)
template <int kShape, bool kAmn, bool kBmn, class Epi, class Ext>
static cudaError_t launch(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& ax, const CUtensorMap& bx,
                          const CUtensorMap& o, Geo g, const Epi& epi, const Ext& ext, cudaStream_t stream) {
  auto kernel = k_gemm_pair<kShape, kAmn, kBmn, Epi, Ext>;
  constexpr int kCtas = Shape<kShape>::kCtas;
  if (kShape != kSingle || kBmn || g.width == 0) g.width = Shape<kShape>::kCols / (Ext::kTwin ? 2 : 1);
  if (kShape == kSingle && !kBmn) {
    if (g.arows == 0) g.arows = HALF;
    const int s = 12 * OPB / ((g.arows + g.width * (Ext::kTwin ? 2 : 1)) * 128);
    // Waiting and signalling cost a stage 0.28 us whatever its size, so two or four k-blocks share one where four such
    // stages fit (gated products: 64 tokens 2048 to 8192 19.0 us with one, 17.2 with two; 7 tokens 4376 to 752 28.1, 22.1
    // and 19.2 with one, two and four).
    g.per = g.splits > 1 ? 1 : s >= 16 && g.seg_kb % 4 == 0 ? 4 : s >= 8 && g.seg_kb % 2 == 0 ? 2 : 1;
    if constexpr (!Ext::kDeep && kShape == kSingle && !kBmn)
      if (g.per > 1) return launch<kShape, kAmn, kBmn, Epi, Deep<Ext>>(a, b, ax, bx, o, g, epi, Deep<Ext>{ext}, stream);
    g.stages = s / g.per < Shape<kSingle>::kMostStages ? s / g.per : Shape<kSingle>::kMostStages;
    if (Ext::kTwin) g.seg_kb = g.nkb + g.per - 1;
  }
  g.n_tiles = (g.cols + g.width - 1) / g.width;
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(allowed, reinterpret_cast<const void*>(kernel), SMEM);
  if (e != cudaSuccess) return e;
  const int64_t total = int64_t(g.m_tiles) * g.n_tiles * g.splits;
  if (total < 1) return cudaSuccess;
  const int at_once = sm_count() / kCtas;  // pairs (76 on 152 SMs) or CTAs at work at once
  const int n = total < at_once && g.fit.room == 0 ? int(total) : at_once;
  return launch_early(kernel, dim3(unsigned(kCtas * n)), dim3(THREADS), SMEM, stream, a, b, ax, bx, o, g, epi, ext);
}

template <bool kAmn, bool kBmn, class Epi, class Ext>
inline cudaError_t launch_shape(int shape, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& ax,
                                const CUtensorMap& bx, const CUtensorMap& o, const Geo& g, const Epi& epi, const Ext& ext,
                                cudaStream_t s) {
  if constexpr (!Ext::kOn && !Ext::kTwin && !kAmn)
    if (shape == kSingle) return launch<kSingle, kAmn, kBmn, Epi, Ext>(a, b, ax, bx, o, g, epi, ext, s);
  return shape == kWide ? launch<kWide, kAmn, kBmn, Epi, Ext>(a, b, ax, bx, o, g, epi, ext, s)
                        : launch<kNarrow, kAmn, kBmn, Epi, Ext>(a, b, ax, bx, o, g, epi, ext, s);
}

// In the pair shape that pick_shape() names.
template <bool kAmn, bool kBmn, class Epi, class Ext>
inline cudaError_t launch_either(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& ax, const CUtensorMap& bx,
                                 const CUtensorMap& o, const Geo& g, const Epi& epi, const Ext& ext, cudaStream_t s) {
  return launch_shape<kAmn, kBmn>(pick_shape(0, g.m_tiles, g.cols, g.nkb, g.splits), a, b, ax, bx, o, g, epi, ext, s);
}

}  // namespace gp
}  // namespace loca
