// Low-rank adapters of many requests beside a shared projection, forward and backward.
//   U = X A_a,  Y = X W^T + s_a U B_a^T                       (Eq. 1 with a frozen W; a = ids[n])
//   T = s_a dY B_a,  dX = dY W + T A_a^T,  dA_a = X_a^T T_a,  dB_a = s_a dY_a^T U_a
// X is N x d_in, W d_out x d_in, A_a d_in x k, B_a d_out x k; a token without an adapter (id outside
// [0, n)) gets X W^T alone.
//
// Adapters as extra k.  For a tile of tokens, X W^T and the low-rank term are one product over a
// longer k axis: behind the d_in columns of [X | U] and [W | s B] come, for each adapter that the
// tile's tokens use, the k columns of U (rows of tokens with another adapter zero) against that
// adapter's k columns of s B.  Eight requests in a tile of 256 cost eight more k-blocks; a decode
// batch of 64 adapters costs 64 steps of k = 16.  The plan finds each tile's adapters on the device;
// a (tile of 128 tokens, adapter) pair is a slot.
//
//   k_plan_*          slots of the token tiles, slots of each adapter (one plan serves every
//                     projection of a step)
//   k_adapter_pack    A and s B as three bf16 parts (hi + mid + lo = the fp32 value to 2^-26)
//   k_adapter_shrink  U (or T) of every slot: tokens x k sums over d.  Bound: the read of X
//   k_adapter_tokens  U of single tokens, where most have an adapter of their own.  Bound: the read of
//                     the adapters
//   k_gemm_pair       the extended product in 256 x 256 or 256 x 512 tiles (many tokens).  Bound: the
//                     tensor cores (8192 tokens of 8 requests at d_in = d_out = 2048, k = 32: 61 us for
//                     the call, 1.15 PFLOP/s)
//   k_adapter_few     the extended product with the roles of the operands exchanged, W's rows as M,
//                     the tokens as N, k split over a cluster (few tokens).  Bound: the read of W, and
//                     with more than 128 tokens what one SM can fetch from L2
//   k_adapter_grad    dA and dB: channels x k sums over an adapter's tokens.  Bound: the read of X, dY
//   k_adapter_join    sums the token ranges of dA, dB in a fixed order, scales, rounds once
// Rounding.  The low-rank term of a bf16 output uses the first part of U and of s B: its relative
// error 2^-8 is of a term that is itself rounded to bf16 with the sum.  fp32 gradients dA and dB take U
// and T summed from all three parts of the adapters and pass them on in three parts; bf16 gradients
// two (2^-17, next to their own rounding of 2^-9).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>

#include "gemm_pair.cuh"

namespace loca {
namespace {

using namespace tc;

constexpr int kTile = 128;       // tokens of a plan tile (one slot: 128 x 64 values of U)
constexpr int kMaxK = 64;
constexpr int kParts = 3;
constexpr int kSlotRows = 128;
constexpr size_t kSlotElems = size_t(kSlotRows) * kMaxK;

// Rows of the packed adapters: whole MMA steps of 16 (TMA moves boxes of 16-byte rows at half the pace
// of 32-byte ones: k = 8 took 51 us in k_adapter_shrink at d = 3584 where k = 16 took 33).
__host__ __device__ inline int k_padded(int k) { return (k + 15) / 16 * 16; }

// ------------------------------------------------------------------ plan
// Five launches of some 5 us that wait for one another: 21 us a step, on the GPU, from one token to 16384 and
// up to 500 adapters.  k_plan_adapters reads every slot for each adapter (2 n slots x 4 bytes from L2).
// Offsets in int32 from the start of the plan.
struct PlanLay {
  int64_t tiles, pairs, smax;
  int64_t tok_slot, tok_adapter, tile_base, adapter, tile, mask, pair_count, pair_ad, pair_s0, pair_s1, ad_off, ad_slots, ad_tile, ad_adapter, ad_mask, total;
};
PlanLay plan_lay(int64_t N, int n) {
  PlanLay p{};
  p.tiles = (N + kTile - 1) / kTile;
  p.pairs = (p.tiles + 1) / 2;
  const int64_t per = n < kTile ? n : kTile;
  p.smax = p.tiles * per < N ? p.tiles * per : N;
  int64_t at = 0;
  auto take = [&](int64_t c) {
    const int64_t o = at;
    at += (c + 63) / 64 * 64;
    return o;
  };
  p.tok_slot = take(N);
  p.tok_adapter = take(N);
  p.tile_base = take(p.tiles + 2);
  p.adapter = take(p.smax);
  p.tile = take(p.smax);
  p.pair_count = take(p.pairs);
  p.pair_ad = take(p.smax);
  p.pair_s0 = take(p.smax);
  p.pair_s1 = take(p.smax);
  p.ad_off = take(n + 1);
  p.ad_slots = take(p.smax);
  p.ad_tile = take(p.smax);
  p.ad_adapter = take(p.smax);
  p.mask = take(4 * p.smax);
  p.ad_mask = take(4 * p.smax);
  p.total = at;
  return p;
}

// A tile's distinct adapters in the order of their first tokens.  fill 0: counts them into
// tile_base[tile + 1]; fill 1: writes the tile's slots at tile_base[tile].
__global__ void __launch_bounds__(kTile) k_plan_tiles(const int32_t* __restrict__ ids, int64_t N, int n, int32_t* plan,
                                                      PlanLay p, int fill) {
  __shared__ int32_t id[kTile];
  __shared__ int32_t warp_sum[4];
  __shared__ int32_t rank[kTile];
  const int j = threadIdx.x, lane = j & 31, warp = j >> 5;
  const int64_t tile = blockIdx.x, tok = tile * kTile + j;
  int a = tok < N ? ids[tok] : -1;
  if (a >= n) a = -1;
  id[j] = a;
  __syncthreads();
  int first = a >= 0 ? j : -1;
  uint32_t rows[kTile / 32] = {};  // the tile's tokens with this token's adapter
  if (a >= 0)
#pragma unroll
    for (int w = 0; w < kTile / 32; ++w)
      for (int i = 0; i < 32; ++i)
        if (id[32 * w + i] == a) {
          if (32 * w + i < first) first = 32 * w + i;
          rows[w] |= 1u << i;
        }
  const bool mine = first == j;
  const unsigned all = __ballot_sync(0xffffffffu, mine);
  if (lane == 0) warp_sum[warp] = __popc(all);
  __syncthreads();
  int before = __popc(all & ((1u << lane) - 1u)), total = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < warp) before += warp_sum[w];
    total += warp_sum[w];
  }
  if (!fill) {
    if (j == 0) plan[p.tile_base + tile + 1] = total;
    return;
  }
  const int base = plan[p.tile_base + tile];
  if (mine) {
    rank[j] = before;
    const int s = base + before;
    if (LOCA_CHECK(s, p.smax)) {
      plan[p.adapter + s] = a;
      plan[p.tile + s] = int32_t(tile);
      for (int w = 0; w < kTile / 32; ++w) plan[p.mask + 4 * int64_t(s) + w] = int32_t(rows[w]);
    }
  }
  __syncthreads();
  if (tok < N) {
    plan[p.tok_slot + tok] = a >= 0 ? base + rank[first] : -1;
    plan[p.tok_adapter + tok] = a;
  }
}

// tile_base: counts to offsets (one block; `tiles` entries in runs of 1024).
__global__ void __launch_bounds__(1024) k_plan_scan(int32_t* plan, PlanLay p) {
  __shared__ int32_t sums[32];
  int32_t* base = plan + p.tile_base;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t carry = 0;
  for (int64_t t0 = 0; t0 < p.tiles; t0 += 1024) {
    const int64_t t = t0 + threadIdx.x;
    int32_t x = t < p.tiles ? base[t + 1] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    int32_t off = carry, all = 0;
    for (int w = 0; w < 32; ++w) {
      if (w < warp) off += sums[w];
      all += sums[w];
    }
    if (t < p.tiles) base[t + 1] = off + x;
    carry += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) base[0] = 0;
  // an odd last tile has an empty partner
  if (threadIdx.x == 0) base[p.tiles + 1] = carry;
}

// Adapters of a pair of tiles (256 rows of the CTA-pair product), with each half's slot or -1.
__global__ void __launch_bounds__(kTile) k_plan_pairs(int32_t* plan, PlanLay p) {
  __shared__ int32_t warp_sum[4];
  const int j = threadIdx.x, lane = j & 31, warp = j >> 5;
  const int64_t t0 = 2 * int64_t(blockIdx.x);
  const int b0 = plan[p.tile_base + t0], b1 = plan[p.tile_base + t0 + 1];
  const int b2 = t0 + 1 < p.tiles ? plan[p.tile_base + t0 + 2] : b1;
  const int n0 = b1 - b0, n1 = b2 - b1;
  if (j < n0) {
    const int a = plan[p.adapter + b0 + j];
    int other = -1;
    for (int i = 0; i < n1; ++i)
      if (plan[p.adapter + b1 + i] == a) other = b1 + i;
    plan[p.pair_ad + b0 + j] = a;
    plan[p.pair_s0 + b0 + j] = b0 + j;
    plan[p.pair_s1 + b0 + j] = other;
  }
  bool alone = j < n1;
  int a1 = -1;
  if (j < n1) {
    a1 = plan[p.adapter + b1 + j];
    for (int i = 0; i < n0; ++i)
      if (plan[p.adapter + b0 + i] == a1) alone = false;
  }
  const unsigned all = __ballot_sync(0xffffffffu, alone);
  if (lane == 0) warp_sum[warp] = __popc(all);
  __syncthreads();
  int at = n0 + __popc(all & ((1u << lane) - 1u)), total = n0;
  for (int w = 0; w < 4; ++w) {
    if (w < warp) at += warp_sum[w];
    total += warp_sum[w];
  }
  if (alone && LOCA_CHECK(b0 + at, p.smax)) {
    plan[p.pair_ad + b0 + at] = a1;
    plan[p.pair_s0 + b0 + at] = -1;
    plan[p.pair_s1 + b0 + at] = b1 + j;
  }
  if (j == 0) plan[p.pair_count + blockIdx.x] = total;
}

// Slots of each adapter, in the order of the tiles: block a takes adapter a.
__global__ void __launch_bounds__(256) k_plan_adapters(int32_t* plan, PlanLay p, int n) {
  __shared__ int32_t below, sums[8];
  const int a = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int total = plan[p.tile_base + p.tiles];
  if (threadIdx.x == 0) below = 0;
  __syncthreads();
  int c = 0;
  for (int s = threadIdx.x; s < total; s += 256) c += plan[p.adapter + s] < a ? 1 : 0;
  atomicAdd(&below, c);  // an integer count: the order of the additions does not matter
  __syncthreads();
  int at = below;
  if (threadIdx.x == 0) {
    plan[p.ad_off + a] = at;
    if (a == n - 1) plan[p.ad_off + n] = total;
  }
  for (int s0 = 0; s0 < total; s0 += 256) {
    const int s = s0 + threadIdx.x;
    const bool mine = s < total && plan[p.adapter + s] == a;
    const unsigned all = __ballot_sync(0xffffffffu, mine);
    if (lane == 0) sums[warp] = __popc(all);
    __syncthreads();
    int off = at + __popc(all & ((1u << lane) - 1u)), here = 0;
    for (int w = 0; w < 8; ++w) {
      if (w < warp) off += sums[w];
      here += sums[w];
    }
    if (mine && LOCA_CHECK(off, p.smax)) {
      plan[p.ad_slots + off] = s;
      plan[p.ad_tile + off] = plan[p.tile + s];
      for (int w = 0; w < kTile / 32; ++w) plan[p.ad_mask + 4 * int64_t(off) + w] = plan[p.mask + 4 * int64_t(s) + w];
      plan[p.ad_adapter + off] = a;
    }
    at += here;
    __syncthreads();
  }
}

// ------------------------------------------------------------------ packed adapters
// The first parts of A (n x d_in x kp bf16) and of s B (n x d_out x kp), which serving reads; then all
// parts of both, side by side in a row (n x d x 3 kp: the columns of one MMA operand); then the n scales
// (fp32) and n marks.  In a shared tile an adapter's columns meet the other tokens' zeros, and zero times infinity
// is not zero: values that are not finite are stored as zero and their adapter is marked, and U and
// T of a marked adapter's tokens are NaN.  One request's broken adapter so spoils its own outputs
// (all of them) and nobody else's.
struct PackLay {
  size_t a, b, all_a, all_b, scale, marks, total;
};
PackLay pack_lay(int n, int64_t d_in, int64_t d_out, int k) {
  const size_t kp = size_t(k_padded(k));
  PackLay p{};
  p.a = 0;
  const size_t sa = 2 * size_t(n) * size_t(d_in) * kp, sb = 2 * size_t(n) * size_t(d_out) * kp;
  p.b = p.a + align256(sa);
  p.all_a = p.b + align256(sb);
  p.all_b = p.all_a + align256(kParts * sa);
  p.scale = p.all_b + align256(kParts * sb);
  p.marks = p.scale + align256(4 * size_t(n));
  p.total = p.marks + align256(4 * size_t(n));
  return p;
}

template <class T>
__device__ __forceinline__ float as_float(T x);
template <>
__device__ __forceinline__ float as_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// One thread per 8 columns of a padded row: one 16-byte store for each copy of a part.
template <class T>
__global__ void __launch_bounds__(256)
    k_adapter_pack(const T* __restrict__ A, const T* __restrict__ B, int n, int64_t d_in, int64_t d_out, int k, int kp,
                   const float* __restrict__ scale, __nv_bfloat16* __restrict__ pa, __nv_bfloat16* __restrict__ pb,
                   __nv_bfloat16* __restrict__ all_a, __nv_bfloat16* __restrict__ all_b, float* __restrict__ ps,
                   int32_t* __restrict__ marks) {
  const int per_row = kp / 8;
  const int64_t rows_a = int64_t(n) * d_in, rows_b = int64_t(n) * d_out;
  const int64_t stride = int64_t(gridDim.x) * blockDim.x, first = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  for (int64_t i = first; i < (rows_a + rows_b) * per_row; i += stride) {
    const int64_t flat = i / per_row;
    const int c = int(i - flat * per_row) * 8;
    const bool isb = flat >= rows_a;
    const int64_t row = isb ? flat - rows_a : flat;
    const T* src = (isb ? B : A) + row * k + c;
    const int have = k - c < 8 ? (k - c < 0 ? 0 : k - c) : 8;
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < have ? as_float<T>(src[j]) : 0.f;
    const int64_t a = row / (isb ? d_out : d_in);
    if (isb && scale) {
      const float s = scale[a];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= s;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (!isfinite(__bfloat162float(__float2bfloat16_rn(x[j])))) {
        x[j] = 0.f;
        marks[a] = 1;
      }
    __nv_bfloat16* all = (isb ? all_b : all_a) + row * (kParts * kp) + c;
    __nv_bfloat16* one = (isb ? pb : pa) + row * kp + c;
    if (!LOCA_CHECK_SPAN(row * kp + c, 8, (isb ? rows_b : rows_a) * kp)) continue;
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
      __align__(16) __nv_bfloat16 h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[j] = __float2bfloat16_rn(x[j]);
        x[j] -= __bfloat162float(h[j]);
      }
      const uint4 v = *reinterpret_cast<const uint4*>(h);
      if (q == 0) *reinterpret_cast<uint4*>(one) = v;
      *reinterpret_cast<uint4*>(all + q * kp) = v;
    }
  }
  for (int64_t i = first; i < n; i += stride) ps[i] = scale ? scale[i] : 1.f;
}

// ------------------------------------------------------------------ U and T: tokens x k sums over d
// One item per slot: M = the tile's 128 tokens, N = the adapter's columns (kp per part, the parts side
// by side), K = d.  With few slots the d axis is split over the CTAs of a cluster, which add their sums
// through distributed shared memory in rank order; one CTA alone writes from registers and goes on.
// Rows of other slots are written as zeros.  Measured at 16384 tokens, k = 16, X from HBM: 0.33 us per
// k-block and 128 CTAs (6.3 TB/s) beyond 8 us of start and end.
constexpr int kShrinkThreads = 192;
constexpr int kShrinkSeg = 8;                    // k-blocks per accumulation segment (several parts)
constexpr int kMaxStages = 8;
constexpr int kRedBytes = kSlotRows * kMaxK * 4; // 32 KB of fp32 sums, in the place of the ring
constexpr int kXBytes = 128 * 64 * 2, kPBytes = 64 * 64 * 2;

struct ShrinkOne {
  __nv_bfloat16* out;  // column tile x smax x 128 x 64
  int64_t d;
};
struct ShrinkGeo {
  ShrinkOne one[2];  // a backward pass makes U from X and T from dY in one launch
  int sets;
  int64_t N;
  const int32_t* marks;
  int kp, parts, stages;
  const int32_t* plan;
  PlanLay p;
  int32_t* status;
  int32_t* abort_flag;
  unsigned long long limit_ns;
  int32_t mark;
};
// 64-wide column tiles of `parts` parts
__host__ __device__ inline int col_tiles(int kp, int parts) { return (kp * parts + 63) / 64; }
int shrink_ring(int ctiles, int stages) {
  const int b = stages * (kXBytes + ctiles * kPBytes);
  return b > kRedBytes ? b : kRedBytes;
}
int shrink_smem(int ctiles, int stages) { return shrink_ring(ctiles, stages) + 512 + 1024; }

// Position of (row, col) in the fp32 sums: 16-byte chunks swizzled over the rows (no bank conflicts).
__device__ __forceinline__ int red_at(int row, int col) {
  return row * kMaxK + (((col >> 2) ^ (row & 15)) << 2) + (col & 3);
}

// Eight values of U in `parts` bf16 parts to columns c .. c + 7 of each part.
__device__ __forceinline__ void store_parts(float (&v)[8], __nv_bfloat16* out, int64_t smax, int s, int row, int c, int kp,
                                            int parts) {
#pragma unroll
  for (int q = 0; q < kParts; ++q) {
    if (q < parts) {
      __align__(16) __nv_bfloat16 w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = __float2bfloat16_rn(v[i]);
        v[i] -= __bfloat162float(w[i]);
      }
      const int col = q * kp + c;
      if (LOCA_CHECK(s, smax))
        *reinterpret_cast<uint4*>(out + ((int64_t(col >> 6) * smax + s) * kSlotRows + row) * kMaxK + (col & 63)) =
            *reinterpret_cast<const uint4*>(w);
    }
  }
}

__global__ void __launch_bounds__(kShrinkThreads, 1)
    k_adapter_shrink(const __grid_constant__ CUtensorMap tmX0, const __grid_constant__ CUtensorMap tmP0,
                     const __grid_constant__ CUtensorMap tmX1, const __grid_constant__ CUtensorMap tmP1,
                     const __grid_constant__ ShrinkGeo g) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int ctiles = col_tiles(g.kp, g.parts);
  const int stage_bytes = kXBytes + ctiles * kPBytes;
  const int ring = g.stages * stage_bytes > kRedBytes ? g.stages * stage_bytes : kRedBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + ring);
  const uint32_t bar_base = smem_u32(bars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kMaxStages + 5);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (kMaxStages + s); };
  auto acc_full = [&](uint32_t b) { return bar_base + 8u * (2 * kMaxStages + b); };
  auto acc_empty = [&](uint32_t b) { return bar_base + 8u * (2 * kMaxStages + 2 + b); };
  const uint32_t drain_bar = bar_base + 8u * (2 * kMaxStages + 4);
  float* red = reinterpret_cast<float*>(smem);  // [128][64] sums of this CTA

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem);
  const WaitCtl wc{g.status, g.abort_flag, g.limit_ns, g.mark};
  const int ks = int(cluster_nctarank()), rank = int(cluster_ctarank());
  const int cid = int(cluster_id_x()), ncl = int(ncluster_x());
  const uint32_t acc_cols = uint32_t(64 * ctiles);  // distance of the two accumulators
  const uint32_t cols = ctiles == 1 ? 128u : ctiles == 2 ? 256u : 512u;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(acc_full(b), 1);
      mbar_init(acc_empty(b), 4);
    }
    mbar_init(drain_bar, 1);
    mbar_init_fence();
    prefetch_tensormap(&tmX0);
    prefetch_tensormap(&tmP0);
    if (g.sets > 1) {
      prefetch_tensormap(&tmX1);
      prefetch_tensormap(&tmP1);
    }
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), cols);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem_base = *tmem_slot;
  wait_for_previous();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *g.abort_flag = 0;  // a captured call that gave up may be replayed
    __threadfence();    // the product may start, and read the flag, from the next line on
  }
  launch_dependents();
  const int total = g.plan[g.p.tile_base + g.p.tiles];
  const int seg_kb = g.parts == 1 ? 64 : kShrinkSeg;

  int stage = 0;
  uint32_t phase = 0, iter = 0, seg = 0;
  bool ok = true, issued = false;
  for (int it = cid; it < total * g.sets; it += ncl) {
    const int set = it >= total ? 1 : 0;
    const int s = it - set * total;
    const int nkb = int((g.one[set].d + 63) / 64);
    const int per = (nkb + ks - 1) / ks;
    const int kb0 = rank * per < nkb ? rank * per : nkb;
    const int kb1 = kb0 + per < nkb ? kb0 + per : nkb;
    const int nb = kb1 - kb0;
    const int a = g.plan[g.p.adapter + s];
    const int64_t row0 = int64_t(g.plan[g.p.tile + s]) * kTile;
    if (warp == 0) {
      // ---------------- TMA producer
      if (lane == 0 && ok) {
        const CUtensorMap* mx = set ? &tmX1 : &tmX0;
        const CUtensorMap* mp = set ? &tmP1 : &tmP0;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_try_wait(empty_bar(stage), phase ^ 1u) && !mbar_wait(empty_bar(stage), phase ^ 1u, wc)) {
            ok = false;
            break;
          }
          mbar_arrive_expect_tx(full_bar(stage), uint32_t(stage_bytes));
          const uint32_t dst = smem_base + uint32_t(stage * stage_bytes);
          tma_load_2d(dst, mx, full_bar(stage), kb * 64, int(row0));
          for (int q = 0; q < ctiles; ++q)
            tma_load_3d(dst + kXBytes + q * kPBytes, mp, full_bar(stage), q * 64, kb * 64, a);
          ++iter;
          if (++stage == g.stages) { stage = 0; phase ^= 1u; }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ---------------- MMA issuer: X tile (K-major) x the adapter's rows (MN-major)
      if (lane == 0 && ok) {
        const uint32_t id = tc::idesc(1, 1, 0, 1, 128, uint32_t(g.kp * g.parts));
        for (int j = 0, in_seg = 0; j < nb; ++j) {
          const uint32_t b = seg & 1u;
          if (in_seg == 0 && !mbar_try_wait(acc_empty(b), ((seg >> 1) & 1u) ^ 1u) &&
              !mbar_wait(acc_empty(b), ((seg >> 1) & 1u) ^ 1u, wc)) {
            ok = false;
            break;
          }
          if (!mbar_try_wait(full_bar(stage), phase) && !mbar_wait(full_bar(stage), phase, wc)) {
            ok = false;
            break;
          }
          fence_after();
          const uint32_t st = smem_base + uint32_t(stage * stage_bytes);
          const uint64_t ad = sdesc(st, 16u, 1024u, kSwizzle128B);
          const uint64_t bd = sdesc(st + kXBytes, kPBytes, 1024u, kSwizzle128B);
          const uint32_t d = tmem_base + b * acc_cols;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_f16(d, ad + kk * 2, bd + kk * (2048 >> 4), id, (in_seg | kk) != 0 ? 1u : 0u);
          issued = true;
          mma_commit(empty_bar(stage));
          if (++stage == g.stages) { stage = 0; phase ^= 1u; }
          if (++in_seg == seg_kb || j == nb - 1) {
            mma_commit(acc_full(b));
            ++seg;
            in_seg = 0;
          }
        }
      }
      __syncwarp();
    } else {
      // ---------------- sums of the segments and of the parts
      const int q = warp & 3;
      const int row = q * 32 + lane;
      const bool mine = uint32_t(g.plan[g.p.mask + 4 * int64_t(s) + q]) >> lane & 1u;
      const bool spoiled = g.marks[a] != 0;
      float u[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) u[i] = 0.f;
      const int nseg = (nb + seg_kb - 1) / seg_kb;
      for (int j = 0; j < nseg && ok; ++j) {
        const uint32_t b = seg & 1u;
        const bool got = mbar_wait(acc_full(b), (seg >> 1) & 1u, wc);
        if (!__all_sync(0xffffffffu, got)) {
          ok = false;
          break;
        }
        fence_after();
        const uint32_t ta = tmem_base + (uint32_t(q * 32) << 16) + b * acc_cols;
        for (int p = 0; p < g.parts; ++p) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (c * 16 < g.kp) {
              float v[16];
              tmem_ld16(ta + uint32_t(p * g.kp + c * 16), v);
#pragma unroll
              for (int i = 0; i < 16; ++i) u[c * 16 + i] += v[i];
            }
          }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acc_empty(b));
        ++seg;
      }
#pragma unroll
      for (int i = 0; i < 64; ++i) u[i] = mine ? (spoiled ? __int_as_float(0x7fffffff) : u[i]) : 0.f;
      if (ok && ks == 1) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (c * 8 < g.kp) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = u[8 * c + i];
            store_parts(v, g.one[set].out, g.p.smax, s, row, c * 8, g.kp, g.parts);
          }
      } else if (ok) {
        // after the last segment's MMAs every load of the item has been read: the sums may take the
        // ring's place
#pragma unroll
        for (int c = 0; c < 16; ++c)
          if (c * 4 < g.kp)
            *reinterpret_cast<float4*>(red + red_at(row, 4 * c)) =
                make_float4(u[4 * c], u[4 * c + 1], u[4 * c + 2], u[4 * c + 3]);
      }
    }
    if (ks == 1) continue;  // the roles need not meet
    __syncwarp();
    cluster_sync();  // every CTA's sums are in its shared memory
    const int rows_per = kSlotRows / ks, chunks = g.kp / 8;
    const uint32_t red_s = smem_u32(red);
    for (int e = threadIdx.x; e < rows_per * chunks; e += kShrinkThreads) {
      const int row = rank * rows_per + e / chunks, ch = e % chunks;
      const uint32_t o0 = red_s + 4u * uint32_t(red_at(row, ch * 8));
      const uint32_t o1 = red_s + 4u * uint32_t(red_at(row, ch * 8 + 4));
      float4 x[8], y[8];  // all loads first: one round trip
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < ks) {
          x[j] = ld_shared_cluster_f32x4(mapa_shared(o0, uint32_t(j)));
          y[j] = ld_shared_cluster_f32x4(mapa_shared(o1, uint32_t(j)));
        }
      float v[8] = {};
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < ks) {
          v[0] += x[j].x; v[1] += x[j].y; v[2] += x[j].z; v[3] += x[j].w;
          v[4] += y[j].x; v[5] += y[j].y; v[6] += y[j].z; v[7] += y[j].w;
        }
      store_parts(v, g.one[set].out, g.p.smax, s, row, ch * 8, g.kp, g.parts);
    }
    fence_proxy_async_smem();  // the ring's next loads come after these accesses
    __syncwarp();
    cluster_sync();
  }
  if (warp == 1 && lane == 0 && issued) {
    mma_commit(drain_bar);
    mbar_drain(drain_bar, 0, kDrainLimitNs);
  }
  if (warp == 0 && lane == 0) {  // copies in flight when a role gave up
    const uint32_t n = uint32_t(g.stages);
    for (uint32_t i = iter > n ? iter - n : 0u; i < iter; ++i)
      mbar_drain(full_bar(int(i % n)), (i / n) & 1u, kDrainLimitNs);
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == 1) tmem_dealloc(tmem_base, cols);
}

// ------------------------------------------------------------------ a step's tokens, one by one
// U of single tokens for a decode batch whose tokens mostly have an adapter each: a tile of 128 rows
// per slot would load X 64 times.  One block per (token, range of d), fp32 sums of the adapter's first
// part, left as one partial sum per range; k_adapter_few adds them.  Bound: the read of each token's
// adapter (2 d k bytes; shared adapters come from L2).
constexpr int kTokThreads = 256;
constexpr int kTokAhead = 4;

struct TokGeo {
  const __nv_bfloat16* X;
  int64_t ldx, d, N;
  const __nv_bfloat16* P;  // adapter x d x kp
  const int32_t* marks;
  const int32_t* tok_adapter;
  int kp, ranges;
  float* out;              // ranges x N x kp
  int32_t* abort_flag;
};

__global__ void __launch_bounds__(kTokThreads) k_adapter_tokens(const TokGeo g) {
  __shared__ float part[kTokThreads / 32][kMaxK];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  wait_for_previous();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    *g.abort_flag = 0;
    __threadfence();
  }
  launch_dependents();
  const int64_t n = blockIdx.y;
  const int a = g.tok_adapter[n];
  if (a < 0) return;  // k_adapter_few does not read this token's sums
  const bool spoiled = g.marks[a] != 0;
  const int chunks = g.kp / 8;  // 16-byte chunks of an adapter row: 2, 4, 6 or 8
  const int nc = chunks <= 2 ? 2 : chunks <= 4 ? 4 : 8;
  const int c = threadIdx.x % nc, stride = kTokThreads / nc;
  const int64_t blocks = (g.d + 63) / 64, per = (blocks + g.ranges - 1) / g.ranges * 64;
  const int64_t k0 = int64_t(blockIdx.x) * per;
  const int64_t k1 = k0 + per < g.d ? k0 + per : g.d;
  const __nv_bfloat16* P = g.P + int64_t(a) * g.d * g.kp + c * 8;
  const __nv_bfloat16* x = g.X + n * g.ldx;
  float acc[8] = {};
  if (c < chunks) {
    for (int64_t k = k0 + threadIdx.x / nc; k < k1; k += kTokAhead * stride) {
      uint4 v[kTokAhead];
      float xv[kTokAhead];
#pragma unroll
      for (int j = 0; j < kTokAhead; ++j) {
        const int64_t r = k + j * stride;
        v[j] = r < k1 ? __ldg(reinterpret_cast<const uint4*>(P + r * g.kp)) : make_uint4(0, 0, 0, 0);
        xv[j] = r < k1 ? __bfloat162float(x[r]) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < kTokAhead; ++j) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = __bfloat1622float2(h[i]);
          acc[2 * i] = fmaf(xv[j], f.x, acc[2 * i]);
          acc[2 * i + 1] = fmaf(xv[j], f.y, acc[2 * i + 1]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int o = 2; o < 32; o <<= 1)
      if (o >= nc) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
    if (lane < nc) part[warp][lane * 8 + i] = acc[i];
  }
  __syncthreads();
  if (threadIdx.x < unsigned(g.kp)) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kTokThreads / 32; ++w) s += part[w][threadIdx.x];
    if (LOCA_CHECK((int64_t(blockIdx.x) * g.N + n) * g.kp + threadIdx.x, int64_t(g.ranges) * g.N * g.kp))
      g.out[(int64_t(blockIdx.x) * g.N + n) * g.kp + threadIdx.x] = spoiled ? __int_as_float(0x7fffffff) : s;
  }
}

// ------------------------------------------------------------------ few tokens
// D[o, n] = sum_k W[o, k] X[n, k] with the output channels as M = 128 and up to 128 tokens as N, so
// that a step of 1 to 64 tokens reads W once at full tiles.  The k axis is split over a cluster of up
// to 8 CTAs, which add their sums through distributed shared memory in rank order: d_out / 128 tiles
// alone would keep 28 of 152 SMs busy at d_out = 3584.  The low-rank term comes in one of two ways:
//   slots (batches that share few adapters)  as k blocks behind those of W and X, from U's slots
//   tokens (an adapter for most tokens)      the epilogue warps, idle until the sums are complete,
//                                            multiply U by each token's rows of s B meanwhile: a
//                                            k-block per adapter would cost as much as W itself.  The
//                                            rows of the first `held` tokens come to shared memory
//                                            before U is there (64 adapters of rank 16 at d = 3584: 4
//                                            us less), the others' from L2 when it is
// The loads of W and X do not wait for U; only what follows them does.  Measured: one token at d_in =
// d_out = 3584 9.4 us with k_adapter_tokens, 64 tokens without an adapter 10.2 us (W at 2.5 TB/s: the
// call's two launches and the sums' way through the cluster are two thirds of it), 512 tokens 26 us at
// d = 4096, 0.31 us a k-block and CTA (105 GB/s per SM, 11.7 TB/s from L2 in all).
constexpr int kFewThreads = 192;
constexpr int kWBytes = 128 * 64 * 2;

struct FewGeo {
  int64_t N, d, o;       // tokens, k, output channels
  int nt;                // tokens per tile (a multiple of 16, at most 128)
  int stages;
  int ksteps;            // MMA steps of 16 per slot
  int tokens;            // 1: the low-rank term token by token
  int kp, ranges;        // tokens: U's columns and partial sums
  int held;              // tokens: how many tokens' rows of s B come to shared memory beforehand
  const float* U;        // tokens: ranges x N x kp
  const __nv_bfloat16* B;  // tokens: adapter x o x kp
  const int32_t* plan;
  int64_t tile_base, adapter, tok_adapter;
  __nv_bfloat16* Y;
  int64_t ldy;
  int32_t* status;
  int32_t* abort_flag;
  unsigned long long limit_ns;
  int32_t mark;
};
__host__ __device__ inline int few_ring(int nt, int stages) {
  const int b = stages * (kWBytes + nt * 128);
  return b > nt * 512 ? b : nt * 512;
}
// tokens of a tile that one of ks CTAs finishes
__host__ __device__ inline int few_own(int nt, int ks) { return (nt + ks - 1) / ks; }
__host__ __device__ inline int few_low(int nt, int ks, int kp) { return few_own(nt, ks) * (512 + 4 * kp + 4); }
// bytes of a token's 128 rows of s B
__host__ __device__ inline int few_rows(int kp) { return 256 * kp; }
int few_smem(int nt, int stages, int low, int held, int kp) {
  return few_ring(nt, stages) + 512 + held * few_rows(kp) + low + 1024;
}

__device__ __forceinline__ void epi_bar() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// The sums of up to kSplits CTAs and the low-rank term, for the tokens rank + ks t of this CTA: an
// epilogue warp takes a token, a lane four channels.  kAhead tokens are on the way at once: many where
// a CTA has many and no other's sums to fetch (one channel a lane: 512 tokens by 3584 channels at
// d = 1024 23.4 us, so 12.3), one at a time in a wide cluster, where more only made the code longer (64
// tokens at d = 3584: 0.5 us more with four).
template <int kSplits, int kAhead>
__device__ __forceinline__ void few_out(const FewGeo& g, const float* low, float* red, int own, int ks, int rank,
                                        int64_t n0, int ntok, int o0) {
  const int warp = int(threadIdx.x >> 5) - 2, c = 4 * int(threadIdx.x & 31);
  constexpr int kWarps = 4;
  const uint32_t red_s = smem_u32(red);
  const bool in = o0 + c < g.o;  // d_out is a multiple of 8
  for (int t0 = warp; t0 < own; t0 += kAhead * kWarps) {
    float4 x[kAhead][kSplits];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const int n = rank + ks * (t0 + q * kWarps);
#pragma unroll
      for (int j = 0; j < kSplits; ++j)
        if (j < ks && n < ntok) {
          const int at = n * 128 + c;
          x[q][j] = kSplits == 1 ? *reinterpret_cast<const float4*>(red + at)
                                 : ld_shared_cluster_f32x4(mapa_shared(red_s + 4u * uint32_t(at), uint32_t(j)));
        } else {
          x[q][j] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const int t = t0 + q * kWarps, n = rank + ks * t;
      if (n >= ntok) break;
      float4 y = g.tokens ? *reinterpret_cast<const float4*>(low + t * 128 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int j = 0; j < kSplits; ++j) {
        y.x += x[q][j].x; y.y += x[q][j].y; y.z += x[q][j].z; y.w += x[q][j].w;
      }
      if (in && LOCA_CHECK(n0 + n, g.N)) {
        __nv_bfloat162 h[2] = {__floats2bfloat162_rn(y.x, y.y), __floats2bfloat162_rn(y.z, y.w)};
        *reinterpret_cast<uint2*>(g.Y + (n0 + n) * g.ldy + o0 + c) = *reinterpret_cast<const uint2*>(h);
      }
    }
  }
}

template <bool kWmn>
__global__ void __launch_bounds__(kFewThreads, 1)
    k_adapter_few(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX,
                  const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmU,
                  const __grid_constant__ FewGeo g) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int stage_bytes = kWBytes + g.nt * 128;
  const int ks = int(cluster_nctarank()), rank = int(cluster_ctarank());
  const int own = few_own(g.nt, ks);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + few_ring(g.nt, g.stages));
  const uint32_t bar_base = smem_u32(bars);
  constexpr int kBarStages = 12;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kBarStages + 2);
  uint8_t* rows = smem + few_ring(g.nt, g.stages) + 512;                        // [held][128][kp] bf16 of s B
  float* low = reinterpret_cast<float*>(rows + g.held * few_rows(g.kp));        // [own][128] low-rank term
  float* us = low + own * 128;                                                  // [own][kp] U
  int32_t* ad = reinterpret_cast<int32_t*>(us + own * g.kp);                    // [own] adapters
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (kBarStages + s); };
  const uint32_t acc_full = bar_base + 8u * (2 * kBarStages);
  const uint32_t rows_full = bar_base + 8u * (2 * kBarStages + 1);
  float* red = reinterpret_cast<float*>(smem);  // [token][128 channels], in the ring's place

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem);
  const WaitCtl wc{g.status, g.abort_flag, g.limit_ns, g.mark};
  const int o0 = int(cluster_id_x()) * 128;
  const int64_t tile = blockIdx.y;
  const int64_t n0 = tile * g.nt;
  const int ntok = int(g.N - n0 < g.nt ? g.N - n0 : g.nt);
  const uint32_t cols = g.nt <= 32 ? 32u : g.nt <= 64 ? 64u : 128u;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kBarStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(acc_full, 1);
    mbar_init(rows_full, 1);
    mbar_init_fence();
    prefetch_tensormap(&tmW);
    prefetch_tensormap(&tmX);
    prefetch_tensormap(&tmB);
    prefetch_tensormap(&tmU);
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), cols);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem_base = *tmem_slot;
  launch_dependents();
  // the launch that makes U lets this one start only once everything before it has completed: X, W,
  // the packed adapters and the plan may be read now, U only after wait_for_previous()
  const int nkb = int((g.d + 63) / 64);
  const int slot0 = g.tokens ? 0 : g.plan[g.tile_base + tile];
  const int steps = nkb + (g.tokens ? 0 : g.plan[g.tile_base + tile + 1] - slot0);
  const int per = (steps + ks - 1) / ks;
  const int j0 = rank * per < steps ? rank * per : steps;
  const int j1 = j0 + per < steps ? j0 + per : steps;
  uint32_t iter = 0;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool waited = false;
      for (int j = j0; j < j1; ++j) {
        if (!mbar_try_wait(empty_bar(stage), phase ^ 1u) && !mbar_wait(empty_bar(stage), phase ^ 1u, wc)) break;
        mbar_arrive_expect_tx(full_bar(stage), uint32_t(stage_bytes));
        const uint32_t a = smem_base + uint32_t(stage * stage_bytes), b = a + kWBytes;
        if (j < nkb) {
          if (kWmn) {
            tma_load_2d(a, &tmW, full_bar(stage), o0, j * 64);
            tma_load_2d(a + kWBytes / 2, &tmW, full_bar(stage), o0 + 64, j * 64);
          } else {
            tma_load_2d(a, &tmW, full_bar(stage), j * 64, o0);
          }
          tma_load_2d(b, &tmX, full_bar(stage), j * 64, int(n0));
        } else {
          if (!waited) {
            wait_for_previous();  // U
            waited = true;
          }
          const int s = slot0 + j - nkb;
          tma_load_3d(a, &tmB, full_bar(stage), 0, o0, g.plan[g.adapter + s]);
          tma_load_2d(b, &tmU, full_bar(stage), 0, s * kSlotRows);
        }
        ++iter;
        if (++stage == g.stages) { stage = 0; phase ^= 1u; }
      }
      if (!waited) wait_for_previous();
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      const uint32_t id = tc::idesc(1, 1, kWmn ? 1 : 0, 0, 128, uint32_t(g.nt));
      const uint32_t idx = tc::idesc(1, 1, 0, 0, 128, uint32_t(g.nt));
      for (int j = j0; j < j1; ++j) {
        if (!mbar_try_wait(full_bar(stage), phase) && !mbar_wait(full_bar(stage), phase, wc)) break;
        fence_after();
        const uint32_t st = smem_base + uint32_t(stage * stage_bytes);
        const uint64_t ak = sdesc(st, 16u, 1024u, kSwizzle128B);
        const uint64_t bk = sdesc(st + kWBytes, 16u, 1024u, kSwizzle128B);
        if (j < nkb) {
          const uint64_t ad0 = kWmn ? sdesc(st, kWBytes / 2, 1024u, kSwizzle128B) : ak;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_f16(tmem_base, ad0 + kk * (kWmn ? 2048 >> 4 : 2), bk + kk * 2, id, j > j0 || kk > 0 ? 1u : 0u);
        } else {
          for (int kk = 0; kk < g.ksteps; ++kk)
            mma_f16(tmem_base, ak + kk * 2, bk + kk * 2, idx, j > j0 || kk > 0 ? 1u : 0u);
        }
        mma_commit(empty_bar(stage));
        if (++stage == g.stages) { stage = 0; phase ^= 1u; }
      }
      // completes once every MMA issued above has; the epilogue and the end of the kernel wait for it
      mma_commit(acc_full);
    }
    __syncwarp();
  } else {
    const int i = (warp - 2) * 32 + lane;
    if (g.tokens) {
      // this CTA's tokens n0 + rank + ks t: U's partial sums in order, then a row of s B per thread
      for (int t = i; t < own; t += 128) ad[t] = rank + ks * t < ntok ? g.plan[g.tok_adapter + n0 + rank + ks * t] : -1;
      epi_bar();
      const int64_t o = o0 + i;
      if (warp == 2) {
        const int64_t left = g.o - o0;
        const uint32_t bytes = uint32_t(left < 128 ? left : 128) * 2u * uint32_t(g.kp);
        uint32_t n = 0;
        for (int t = 0; t < g.held; ++t) n += ad[t] >= 0 ? 1u : 0u;
        if (lane == 0) mbar_arrive_expect_tx(rows_full, n * bytes);
        __syncwarp();
        for (int t = lane; t < g.held; t += 32)
          if (ad[t] >= 0)
            bulk_load(smem_u32(rows + t * few_rows(g.kp)), g.B + (int64_t(ad[t]) * g.o + o0) * g.kp, bytes, rows_full);
      }
      if (o < g.o)
        for (int t = g.held; t < own; ++t)
          if (ad[t] >= 0) {
            const __nv_bfloat16* p = g.B + (int64_t(ad[t]) * g.o + o) * g.kp;
            for (int c = 0; c < g.kp; c += 16) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + c));
          }
      wait_for_previous();
      for (int e = i; e < own * (g.kp / 4); e += 128) {
        const int t = e / (g.kp / 4), c = 4 * (e - t * (g.kp / 4));
        float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
        if (ad[t] >= 0) {
          const float* p = g.U + (n0 + rank + ks * t) * g.kp + c;
          float4 x[8];
#pragma unroll
          for (int r = 0; r < 8; ++r)
            x[r] = r < g.ranges ? *reinterpret_cast<const float4*>(p + r * g.N * g.kp) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            u.x += x[r].x; u.y += x[r].y; u.z += x[r].z; u.w += x[r].w;
          }
        }
        *reinterpret_cast<float4*>(us + 4 * e) = u;
      }
      epi_bar();
      if (g.held > 0) {
        mbar_wait(rows_full, 0, wc);
        // 16-byte chunks of a row in an order of the thread's own: no bank conflicts
        const int nc = g.kp / 8, c0 = (i * nc / 8) % nc;
        for (int t0 = 0; t0 < g.held; t0 += 4) {
          float y[4] = {};
          for (int q = 0, c = c0; q < nc; ++q, c = c + 1 < nc ? c + 1 : 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int t = t0 + j < g.held ? t0 + j : t0;
              const uint4 v = *reinterpret_cast<const uint4*>(rows + t * few_rows(g.kp) + i * 2 * g.kp + 16 * c);
              const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
              const float4* u = reinterpret_cast<const float4*>(us + t * g.kp + 8 * c);
              const float4 ua = u[0], ub = u[1];
              const float2 f0 = __bfloat1622float2(h[0]), f1 = __bfloat1622float2(h[1]);
              const float2 f2 = __bfloat1622float2(h[2]), f3 = __bfloat1622float2(h[3]);
              y[j] = fmaf(ua.x, f0.x, y[j]); y[j] = fmaf(ua.y, f0.y, y[j]);
              y[j] = fmaf(ua.z, f1.x, y[j]); y[j] = fmaf(ua.w, f1.y, y[j]);
              y[j] = fmaf(ub.x, f2.x, y[j]); y[j] = fmaf(ub.y, f2.y, y[j]);
              y[j] = fmaf(ub.z, f3.x, y[j]); y[j] = fmaf(ub.w, f3.y, y[j]);
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j)  // (without an adapter, or past d_out, nothing has come to the row)
            if (t0 + j < g.held) low[(t0 + j) * 128 + i] = ad[t0 + j] >= 0 && o < g.o ? y[j] : 0.f;
        }
      }
      for (int t0 = g.held; t0 < own; t0 += 4) {  // four tokens' rows in flight
        float y[4] = {};
        for (int c = 0; c < g.kp; c += 16) {
          uint4 v[4][2];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int a = t0 + t < own ? ad[t0 + t] : -1;
            if (a >= 0 && o < g.o) {
              const uint4* p = reinterpret_cast<const uint4*>(g.B + (int64_t(a) * g.o + o) * g.kp + c);
              v[t][0] = __ldg(p);
              v[t][1] = __ldg(p + 1);
            } else {
              v[t][0] = v[t][1] = make_uint4(0, 0, 0, 0);
            }
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            if (t0 + t < own) {
              const float* u = us + (t0 + t) * g.kp + c;
              const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v[t][0]);
#pragma unroll
              for (int q = 0; q < 8; ++q) {
                const float2 f = __bfloat1622float2(h[q]);
                y[t] = fmaf(u[2 * q], f.x, y[t]);
                y[t] = fmaf(u[2 * q + 1], f.y, y[t]);
              }
            }
          }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (t0 + t < own) low[(t0 + t) * 128 + i] = y[t];
      }
    }
    const int q = warp & 3;
    const bool got = j1 > j0 && mbar_wait(acc_full, 0, wc);
    const bool all = __all_sync(0xffffffffu, got);
    fence_after();
    for (int c = 0; c < g.nt / 16; ++c) {
      float v[16];
      if (all) {
        tmem_ld16(tmem_base + (uint32_t(q * 32) << 16) + uint32_t(c * 16), v);
      } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) v[x] = 0.f;
      }
#pragma unroll
      for (int x = 0; x < 16; ++x) red[(c * 16 + x) * 128 + q * 32 + lane] = v[x];
    }
    fence_before();
    __syncwarp();
  }
  cluster_sync();
  fence_after();
  if (warp >= 2) {
    if (ks == 1) few_out<1, 8>(g, low, red, own, 1, 0, n0, ntok, o0);
    else if (ks <= 4) few_out<4, 2>(g, low, red, own, ks, rank, n0, ntok, o0);
    else few_out<8, 1>(g, low, red, own, ks, rank, n0, ntok, o0);
  }
  if (warp == 0 && lane == 0) {
    const uint32_t n = uint32_t(g.stages);
    for (uint32_t i = iter > n ? iter - n : 0u; i < iter; ++i)
      mbar_drain(full_bar(int(i % n)), (i / n) & 1u, kDrainLimitNs);
  }
  if (warp == 1 && lane == 0) mbar_drain(acc_full, 0, kDrainLimitNs);
  if (warp == 2 && lane == 0 && g.tokens) mbar_drain(rows_full, 0, kDrainLimitNs);
  __syncwarp();
  fence_before();
  cluster_sync();  // no CTA leaves while its peers read its sums
  fence_after();
  if (warp == 1) tmem_dealloc(tmem_base, cols);
}

// ------------------------------------------------------------------ many tokens
struct AdapterExt {
  static constexpr bool kDeep = false;
  static constexpr bool kOn = true;
  static constexpr bool kSecond = false;
  static constexpr bool kTwin = false;
  static constexpr bool kEarlyA = false;
  const int32_t* plan;
  int64_t tile_base, pair_count, pair_ad, pair_s0, pair_s1;
  int none_row;  // past the last slot: the loads fill zeros
  int nsteps;

  __device__ int ksteps() const { return nsteps; }
  __device__ int entries(int m) const { return plan[pair_count + m]; }
  __device__ void entry(int m, int j, uint32_t rank, int& a_row, int& block) const {
    const int at = plan[tile_base + 2 * int64_t(m)] + j;
    const int s = plan[(rank ? pair_s1 : pair_s0) + at];
    a_row = s < 0 ? none_row : s * kSlotRows;
    block = plan[pair_ad + at];
  }
};

struct EpiRows {
  static constexpr bool kPacks = true;
  static constexpr bool kAhead = false;
  static constexpr bool kFits = false;
  static constexpr bool kSums = false;
  struct Row {};
  __device__ __forceinline__ Row row_of(int) const { return Row{}; }
  __device__ __forceinline__ float value(const Row&, int, float v) const { return v; }
};

// ------------------------------------------------------------------ dA and dB: channels x k sums over tokens
// The slots, in the order of their adapters, are cut into equal ranges; one item per (128 channels,
// range).  M = channels, N = the columns of U or T (kp per part, side by side), K = the slots' 128 tokens
// in two stages, both operands MN-major as they lie in memory.  A range that crosses from one adapter to
// the next writes a partial sum for each: range r's of adapter a is number r + a (each step of the list
// raises r or a, so no two share a number).  The segments (512 tokens) are added in registers.  A slot
// whose tile also holds other tokens has those rows of X (or dY) zeroed in shared memory first: their U
// is zero, but a product with whatever else stands there (infinities, NaN) need not be.  Measured, X and
// dY from HBM: 16384 tokens x 2 x 896 channels 18 us, 8192 x 2 x 3584 31 us; twice the tokens take 11 and 17
// us more (5.8 and 7.0 TB/s), so 8 to 13 us of a launch are its beginning and end.
constexpr int kGradThreads = 224;
constexpr int kGradMaxStages = 8;
constexpr int kGradSeg = 8;

struct GradOne {
  int64_t d;        // channels
  int ctiles, ranges, items;
  float* part;      // (ranges + n) x d x kp
};
struct GradGeo {
  GradOne one[2];
  int64_t N;
  int n, kp, parts, stages, items;  // items of both
  const int32_t* plan;
  PlanLay p;
  int32_t* status;
  int32_t* abort_flag;
  unsigned long long limit_ns;
  int32_t mark;
};
int grad_smem(int utiles, int stages) { return stages * (kXBytes + utiles * kPBytes) + 512 + 1024; }

__global__ void __launch_bounds__(kGradThreads, 1)
    k_adapter_grad(const __grid_constant__ CUtensorMap tmS0, const __grid_constant__ CUtensorMap tmU0,
                   const __grid_constant__ CUtensorMap tmS1, const __grid_constant__ CUtensorMap tmU1,
                   const __grid_constant__ GradGeo g) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int utiles = col_tiles(g.kp, g.parts);
  const int stage_bytes = kXBytes + utiles * kPBytes;
  const int stages = g.stages;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + stages * stage_bytes);
  const uint32_t bar_base = smem_u32(bars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 3 * kGradMaxStages + 5);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (kGradMaxStages + s); };
  auto ready_bar = [&](int s) { return bar_base + 8u * (2 * kGradMaxStages + s); };
  auto acc_full = [&](uint32_t b) { return bar_base + 8u * (3 * kGradMaxStages + b); };
  auto acc_empty = [&](uint32_t b) { return bar_base + 8u * (3 * kGradMaxStages + 2 + b); };
  const uint32_t drain_bar = bar_base + 8u * (3 * kGradMaxStages + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem);
  const WaitCtl wc{g.status, g.abort_flag, g.limit_ns, g.mark};
  const uint32_t acc_cols = uint32_t(64 * utiles);
  const uint32_t cols = utiles == 1 ? 128u : utiles == 2 ? 256u : 512u;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kGradMaxStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 2);  // the MMAs that read the stage, and the warp that zeroes rows
      mbar_init(ready_bar(s), 1);  // stages of mixed slots only
    }
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(acc_full(b), 1);
      mbar_init(acc_empty(b), 4);
    }
    mbar_init(drain_bar, 1);
    mbar_init_fence();
    prefetch_tensormap(&tmS0);
    prefetch_tensormap(&tmU0);
    if (g.one[1].items) {
      prefetch_tensormap(&tmS1);
      prefetch_tensormap(&tmU1);
    }
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), cols);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem_base = *tmem_slot;
  wait_for_previous();
  launch_dependents();
  const int items = g.items;
  uint32_t iter = 0;
  struct Item {
    int set, ct, range, s0, s1;  // s0 .. s1: places in the list of slots by adapter
  };
  const int all_slots = g.plan[g.p.tile_base + g.p.tiles];
  auto item_of = [&](int it) {
    Item w;
    w.set = it >= g.one[0].items ? 1 : 0;
    const GradOne& o = g.one[w.set];
    if (w.set) it -= g.one[0].items;
    w.range = it / o.ctiles;  // channel tiles fastest: CTAs at work share a range's U or T
    w.ct = it - w.range * o.ctiles;
    const int per = (all_slots + o.ranges - 1) / o.ranges;
    w.s0 = w.range * per < all_slots ? w.range * per : all_slots;
    w.s1 = w.s0 + per < all_slots ? w.s0 + per : all_slots;
    return w;
  };
  // place l's tokens among its tile's, and whether the tile also holds tokens of others
  auto mask_of = [&](int l) { return *reinterpret_cast<const uint4*>(g.plan + g.p.ad_mask + 4 * int64_t(l)); };
  auto is_mixed = [&](const uint4& m, int64_t row) {
    return __popc(m.x) + __popc(m.y) + __popc(m.z) + __popc(m.w) < int(g.N - row < kTile ? g.N - row : kTile);
  };
  // end of the run of slots of one adapter that starts at place l
  auto run_end = [&](int l, const Item& w, int& a) {
    a = g.plan[g.p.ad_adapter + l];
    const int e = g.plan[g.p.ad_off + a + 1];
    return e < w.s1 ? e : w.s1;
  };

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
        const Item w = item_of(it);
        const CUtensorMap* ms = w.set ? &tmS1 : &tmS0;
        const CUtensorMap* mu = w.set ? &tmU1 : &tmU0;
        int s = 0, tile = 0;
        if (w.s0 < w.s1) {
          s = g.plan[g.p.ad_slots + w.s0];
          tile = g.plan[g.p.ad_tile + w.s0];
        }
        for (int l = w.s0; l < w.s1 && ok; ++l) {
          const int ln = l + 1 < w.s1 ? l + 1 : l;  // the next slot's entries are under way meanwhile
          const int s_next = g.plan[g.p.ad_slots + ln], tile_next = g.plan[g.p.ad_tile + ln];
          const int row = tile * kTile;
          for (int h = 0; h < 2; ++h) {
            if (!mbar_try_wait(empty_bar(stage), phase ^ 1u) && !mbar_wait(empty_bar(stage), phase ^ 1u, wc)) {
              ok = false;
              break;
            }
            mbar_arrive_expect_tx(full_bar(stage), uint32_t(stage_bytes));
            const uint32_t dst = smem_base + uint32_t(stage * stage_bytes);
            tma_load_2d(dst, ms, full_bar(stage), w.ct * 128, row + 64 * h);
            tma_load_2d(dst + kXBytes / 2, ms, full_bar(stage), w.ct * 128 + 64, row + 64 * h);
            for (int q = 0; q < utiles; ++q)
              tma_load_3d(dst + kXBytes + q * kPBytes, mu, full_bar(stage), 0, s * kSlotRows + 64 * h, q);
            ++iter;
            if (++stage == stages) { stage = 0; phase ^= 1u; }
          }
          s = s_next;
          tile = tile_next;
        }
      }
    }
    __syncwarp();
  } else if (warp == 6) {
    // ---------------- rows of other tokens: zero.  Every stage is waited for in turn (a phase must not
    // pass unseen), but the MMAs wait for this warp only where there is something to zero
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
      const Item w = item_of(it);
      uint4 m = make_uint4(0, 0, 0, 0), m_next = m;
      int tile = 0, tile_next = 0;
      if (w.s0 < w.s1) {
        m_next = mask_of(w.s0);
        tile_next = g.plan[g.p.ad_tile + w.s0];
      }
      for (int l = w.s0; l < w.s1 && ok; ++l) {
        m = m_next;
        tile = tile_next;
        const int ln = l + 1 < w.s1 ? l + 1 : l;
        m_next = mask_of(ln);
        tile_next = g.plan[g.p.ad_tile + ln];
        const bool mixed = is_mixed(m, int64_t(tile) * kTile);
        for (int h = 0; h < 2; ++h) {
          const bool got = mbar_try_wait(full_bar(stage), phase) || mbar_wait(full_bar(stage), phase, wc);
          if (!__all_sync(0xffffffffu, got)) {
            ok = false;
            break;
          }
          if (mixed) {
            uint8_t* box = smem + stage * stage_bytes;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const uint32_t rows = h == 0 ? (r == 0 ? m.x : m.y) : (r == 0 ? m.z : m.w);
              if (!(rows >> lane & 1u)) {  // (rows past the last token are zero already)
                uint8_t* to = box + (32 * r + lane) * 128;
#pragma unroll
                for (int u = 0; u < 8; ++u) {  // each lane begins at another 16 bytes: no bank conflicts
                  *reinterpret_cast<uint4*>(to + ((u + lane) & 7) * 16) = make_uint4(0, 0, 0, 0);
                  *reinterpret_cast<uint4*>(to + kXBytes / 2 + ((u + lane) & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
              }
            }
            fence_proxy_async_smem();
          }
          __syncwarp();
          if (lane == 0) {
            if (mixed) mbar_arrive(ready_bar(stage));
            mbar_arrive(empty_bar(stage));
          }
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0, seg = 0, ready_phase = 0;  // bit s: parity of the next use of ready_bar(s)
      bool ok = true, issued = false;
      const uint32_t id = tc::idesc(1, 1, 1, 1, 128, uint32_t(g.kp * g.parts));
      for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
        const Item w = item_of(it);
        int end = w.s0, a = 0;
        uint4 m_next = make_uint4(0, 0, 0, 0);
        int tile_next = 0;
        bool mixed = false;
        if (w.s0 < w.s1) {
          m_next = mask_of(w.s0);
          tile_next = g.plan[g.p.ad_tile + w.s0];
        }
        const int nb = 2 * (w.s1 - w.s0);
        for (int j = 0, in_seg = 0; j < nb; ++j) {
          const int l = w.s0 + j / 2;
          if ((j & 1) == 0) {
            if (l == end) end = run_end(end, w, a);
            mixed = is_mixed(m_next, int64_t(tile_next) * kTile);
            const int ln = l + 1 < w.s1 ? l + 1 : l;  // the next slot's entries are under way meanwhile
            m_next = mask_of(ln);
            tile_next = g.plan[g.p.ad_tile + ln];
          }
          const uint32_t b = seg & 1u;
          if (in_seg == 0 && !mbar_try_wait(acc_empty(b), ((seg >> 1) & 1u) ^ 1u) &&
              !mbar_wait(acc_empty(b), ((seg >> 1) & 1u) ^ 1u, wc)) {
            ok = false;
            break;
          }
          if (!mbar_try_wait(full_bar(stage), phase) && !mbar_wait(full_bar(stage), phase, wc)) {
            ok = false;
            break;
          }
          if (mixed) {
            const uint32_t par = ready_phase >> stage & 1u;
            if (!mbar_try_wait(ready_bar(stage), par) && !mbar_wait(ready_bar(stage), par, wc)) {
              ok = false;
              break;
            }
            ready_phase ^= 1u << stage;
          }
          fence_after();
          const uint32_t st = smem_base + uint32_t(stage * stage_bytes);
          const uint64_t ad = sdesc(st, kXBytes / 2, 1024u, kSwizzle128B);
          const uint64_t bd = sdesc(st + kXBytes, kPBytes, 1024u, kSwizzle128B);
          const uint32_t d = tmem_base + b * acc_cols;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_f16(d, ad + kk * (2048 >> 4), bd + kk * (2048 >> 4), id, (in_seg | kk) != 0 ? 1u : 0u);
          issued = true;
          mma_commit(empty_bar(stage));
          if (++stage == stages) { stage = 0; phase ^= 1u; }
          if (++in_seg == kGradSeg || j == 2 * (end - w.s0) - 1) {  // full, or the adapter's last slot here
            mma_commit(acc_full(b));
            ++seg;
            in_seg = 0;
          }
        }
      }
      if (issued) {
        mma_commit(drain_bar);
        mbar_drain(drain_bar, 0, kDrainLimitNs);
      }
    }
    __syncwarp();
  } else {
    const int q = warp & 3;
    uint32_t seg = 0;
    bool ok = true;
    for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
      const Item w = item_of(it);
      const GradOne& o = g.one[w.set];
      const int64_t ch = int64_t(w.ct) * 128 + q * 32 + lane;
      for (int l = w.s0; l < w.s1 && ok;) {
        int a;
        const int end = run_end(l, w, a);
        const int nseg = (2 * (end - l) + kGradSeg - 1) / kGradSeg;
        float u[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) u[i] = 0.f;
        for (int j = 0; j < nseg; ++j) {
          const uint32_t b = seg & 1u;
          const bool got = mbar_try_wait(acc_full(b), (seg >> 1) & 1u) || mbar_wait(acc_full(b), (seg >> 1) & 1u, wc);
          if (!__all_sync(0xffffffffu, got)) {
            ok = false;
            break;
          }
          fence_after();
          const uint32_t ta = tmem_base + (uint32_t(q * 32) << 16) + b * acc_cols;
          for (int p = 0; p < g.parts; ++p) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if (c * 16 < g.kp) {
                float v[16];
                tmem_ld16(ta + uint32_t(p * g.kp + c * 16), v);
#pragma unroll
                for (int i = 0; i < 16; ++i) u[c * 16 + i] += v[i];
              }
            }
          }
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(acc_empty(b));
          ++seg;
        }
        if (!ok) break;
        if (ch < o.d && LOCA_CHECK(w.range + a, o.ranges + g.n)) {
          float* to = o.part + (int64_t(w.range + a) * o.d + ch) * g.kp;
#pragma unroll
          for (int c = 0; c < 16; ++c)
            if (4 * c < g.kp)
              *reinterpret_cast<float4*>(to + 4 * c) = make_float4(u[4 * c], u[4 * c + 1], u[4 * c + 2], u[4 * c + 3]);
        }
        l = end;
      }
    }
  }
  if (warp == 0 && lane == 0) {
    const uint32_t n = uint32_t(stages);
    for (uint32_t i = iter > n ? iter - n : 0u; i < iter; ++i)
      mbar_drain(full_bar(int(i % n)), (i / n) & 1u, kDrainLimitNs);
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == 1) tmem_dealloc(tmem_base, cols);
}

struct JoinOne {
  const float* part;
  const float* scale;  // per adapter, or null
  void* out;
  int64_t d;           // n d rows of k values
  int ranges;
};
// One adapter's gradient per (y, z) of the grid.  kLanes lanes share the ranges of four neighbouring
// columns of a channel; their sums meet in a fixed order.  Four where the sums were cut into many ranges
// (16384 tokens of one adapter over 2 x 896 channels: ten, 5 us), one where they were not: 7 adapters of
// rank 64 over 5120 channels in two ranges took 26 us with four and takes 10 with one.
template <class T, int kLanes>
__global__ void __launch_bounds__(256)
    k_adapter_join(const JoinOne j0, const JoinOne j1, int k, int kp, const int32_t* __restrict__ plan,
                   const __grid_constant__ PlanLay pl) {
  wait_for_previous();
  launch_dependents();
  const JoinOne& j = blockIdx.z ? j1 : j0;
  const int a = int(blockIdx.y);
  const int per_row = kp / 4;
  const int lane = threadIdx.x % kLanes;
  const int gi = int(blockIdx.x) * (256 / kLanes) + int(threadIdx.x) / kLanes;
  const bool on = gi < int(j.d) * per_row;
  const int channel = on ? gi / per_row : 0;
  const int c = on ? 4 * (gi - channel * per_row) : 0;
  const int64_t row = int64_t(a) * j.d + channel;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  const int s0 = plan[pl.ad_off + a], s1 = plan[pl.ad_off + a + 1];
  if (on && s0 < s1) {  // the ranges that hold slots of this adapter
    const int per = (plan[pl.tile_base + pl.tiles] + j.ranges - 1) / j.ranges;
    const int r1 = (s1 - 1) / per;
    const float* p = j.part + row * kp + c;  // number r + a: row is a d + channel
    const int64_t pitch = j.d * kp;
#pragma unroll 4
    for (int r = s0 / per + lane; r <= r1; r += kLanes) {
      const float4 x = *reinterpret_cast<const float4*>(p + r * pitch);
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
  }
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    v.z += __shfl_xor_sync(0xffffffffu, v.z, o);
    v.w += __shfl_xor_sync(0xffffffffu, v.w, o);
  }
  if (!on || !LOCA_CHECK_SPAN(row * k, k, int64_t(gridDim.y) * j.d * k)) return;
  T* out = static_cast<T*>(j.out) + row * k;
  const float scale = j.scale ? j.scale[a] : 1.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = scale * (i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
    if (i % kLanes == lane && c + i < k) {
      if constexpr (sizeof(T) == 4) out[c + i] = x;
      else out[c + i] = __float2bfloat16_rn(x);
    }
  }
}

// ------------------------------------------------------------------ host side
// Token by token, or by slots.  A token costs the read of its adapter whoever else has it, a slot a
// tile of X.  At d_in = 3584, d_out = 2048: 9 us + 0.0039 N kp (64 tokens 12 us with k = 16, 25 with 64;
// 400 tokens 33 and 113) against 12 us + 0.23 a slot whatever k (64 tokens 12 us in one slot, 20 in 32,
// 27 in 64; 400 tokens 22 us in 4, 65 in 200).  The host does not know the slots: half of what they may
// come to is the guess.  Measured up to 512 tokens.
bool by_token(int64_t N, int n, int k) { return N <= 512 && N * k_padded(k) < 768 + 30 * plan_lay(N, n).smax; }
// Ranges of d for the token kernel: about four blocks per SM.
int tok_ranges(int64_t N, int64_t d) {
  int64_t r = 4 * int64_t(sm_count()) / (N < 1 ? 1 : N);
  const int64_t most = (d + 255) / 256;
  if (r > most) r = most;
  if (r > 8) r = 8;
  return int(r < 1 ? 1 : r);
}

struct AdapterWs {
  size_t u, t, part_in, part_out, total;
  int ranges;
};
// Ranges of the slots: whole rounds of the SMs over the items of both gradients (`ctiles` channel tiles in all),
// against two slots' time to begin and end an item.
int grad_ranges(int64_t ctiles, int64_t tiles) {
  int best = 1;
  int64_t best_c = 0;
  for (int64_t r = 1; r <= 64 && r <= tiles; ++r) {
    const int64_t rounds = (ctiles * r + sm_count() - 1) / sm_count();
    const int64_t c = rounds * ((tiles + r - 1) / r + 2);
    if (r == 1 || c < best_c) {
      best = int(r);
      best_c = c;
    }
  }
  return best;
}
AdapterWs adapter_ws(int64_t N, int64_t d_in, int64_t d_out, int k, int n, bool backward) {
  AdapterWs w{};
  const PlanLay p = plan_lay(N, n);
  const size_t one = align256(2 * kSlotElems * size_t(p.smax < 1 ? 1 : p.smax) *
                              size_t(col_tiles(k_padded(k), backward ? kParts : 1)));
  size_t at = 256;  // the launches' abort flag
  // U: the slots' tiles, or the tokens' partial sums
  const size_t tok = align256(4 * 8 * size_t(N) * size_t(k_padded(k)));
  const size_t need = by_token(N, n, k) && tok > one ? tok : one;
  w.u = at; at += need;
  if (backward) {
    w.t = at; at += need;
    w.ranges = grad_ranges((d_in + 127) / 128 + (d_out + 127) / 128, p.tiles);
    const size_t parts = size_t(w.ranges) + size_t(n), kp = size_t(k_padded(k));
    w.part_in = at; at += align256(4 * parts * size_t(d_in) * kp);
    w.part_out = at; at += align256(4 * parts * size_t(d_out) * kp);
  }
  w.total = at;
  return w;
}

struct Call {
  int64_t N;
  int n, k, kp;
  PlanLay p;
  const int32_t* plan;
  int32_t* status;
  int32_t* abort_flag;
  int32_t mark;  // this call's value of the abort flag: the workspace needs no clearing
  cudaStream_t s;
};

// The limit on dynamic shared memory that every launch of a kernel sets: the limit belongs to the kernel, not
// to the launch, so a size of the call's own could be replaced by another thread's before the launch.
constexpr int kMostSmem = 232448;

// Every launch may start while the one before it ends (its prologue runs early; wait_for_previous()
// holds back what depends on it).
template <class... P, class... A>
cudaError_t launch_cluster(void (*kernel)(P...), dim3 grid, int threads, int smem, int cluster, cudaStream_t s,
                           A... args) {
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
  else e = gp::keep_carveout(kernel);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = size_t(smem);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = unsigned(cluster);
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Clusters of ks CTAs with an SM each that run at once: less than sm_count() / ks where a cluster does
// not fill what is left of a group of SMs (of 152 SMs: 46 of three, 36 of four, 28 of five, 15 of eight).
int clusters_at_once(int ks) {
  constexpr int kDevices = 64;
  static std::atomic<int> cache[kDevices][9] = {};
  if (ks == 1) return sm_count();
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return sm_count() / ks;
  int n = cache[dev][ks].load(std::memory_order_relaxed);
  if (n > 0) return n;
  const int smem = 200 * 1024;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(ks));
  cfg.blockDim = dim3(kFewThreads);
  cfg.dynamicSmemBytes = size_t(smem);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = unsigned(ks);
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaFuncSetAttribute(k_adapter_few<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, k_adapter_few<false>, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();
    n = sm_count() / ks;
  }
  cache[dev][ks].store(n, std::memory_order_relaxed);
  return n;
}

// The same on SMs that come free one by one: clusters of three and more then do not pack as tightly as on
// an idle chip (64 adapters at d_in = d_out = 3584: of 28 clusters of five the last began when the first
// had ended, 20.0 us; 28 of four, where 36 fit, 14.2; 200 tokens of 8 requests at 2048 x 2048 14.9 and
// 13.5 us; forward and gradients of 780 tokens, 1792 x 4088, with U's clusters planned so 92 and 86 us; in
// some sizes the smaller split costs up to 6 %).
int clusters_at_once(int ks, bool crowded) {
  const int n = clusters_at_once(ks);
  return crowded && ks > 2 && n > 1 ? n * 7 / 8 : n;
}

// CTAs that share the k axis of an item: whole rounds of the clusters that run at once, each of a CTA's
// k-blocks and `fixed` more for its beginning and end.
int cluster_split(int64_t items, int64_t blocks, int64_t fixed, bool powers, bool crowded) {
  int best = 1;
  int64_t best_c = 0;
  for (int ks = 1; ks <= 8 && (ks == 1 || blocks >= 2 * ks); ks = powers ? 2 * ks : ks + 1) {
    const int at_once = clusters_at_once(ks, crowded);
    const int64_t rounds = (items + at_once - 1) / at_once;
    const int64_t c = rounds * ((blocks + ks - 1) / ks + fixed);
    if (ks == 1 || c < best_c) {
      best = ks;
      best_c = c;
    }
  }
  return best;
}

// U and / or T of every slot: rows X (N x d) against the packed operand P, `sets` of them in one launch.
struct Shrink {
  const void* X;
  int64_t ldx, d;
  const __nv_bfloat16* P;
  void* out;
};
cudaError_t shrink(const Call& c, const Shrink* set, int sets, const int32_t* marks, int parts) {
  CUtensorMap mx[2], mp[2];
  ShrinkGeo g{};
  int64_t dmin = 0;
  for (int i = 0; i < sets; ++i) {
    const Shrink& v = set[i];
    const int64_t pitch = parts == 1 ? c.kp : kParts * c.kp;  // the first parts alone, or all side by side
    if (!gp::map_kmajor(&mx[i], v.X, v.d, c.N, v.ldx) ||
        !gp::map_3d(&mp[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, v.P, parts * c.kp, v.d, c.n, pitch, v.d * pitch, 64, 64))
      return cudaErrorInvalidValue;
    g.one[i].d = v.d;
    g.one[i].out = static_cast<__nv_bfloat16*>(v.out);
    if (i == 0 || v.d < dmin) dmin = v.d;
  }
  g.sets = sets;
  g.N = c.N;
  g.marks = marks;
  g.kp = c.kp;
  g.parts = parts;
  // few tokens: a small ring, so that k_adapter_few's CTAs fit beside these
  const int ctiles = col_tiles(c.kp, parts);
  g.stages = parts == 1 && c.N <= kTile ? 3 : 200 * 1024 / (kXBytes + ctiles * kPBytes);
  if (g.stages > kMaxStages) g.stages = kMaxStages;
  g.plan = c.plan;
  g.p = c.p;
  g.status = c.status;
  g.abort_flag = c.abort_flag;
  g.limit_ns = wait_limit_ns();
  g.mark = c.mark;
  // slots are known to the device only: between one per tile and smax.  An item's beginning and end
  // cost about as much as six k-blocks (2 us)
  int64_t guess = c.p.tiles > c.n ? c.p.tiles : c.n;
  if (guess > c.p.smax) guess = c.p.smax;
  const int ks = cluster_split(guess * sets, (dmin + 63) / 64, 6, true, true);
  int64_t clusters = clusters_at_once(ks, true);
  if (clusters > c.p.smax * sets) clusters = c.p.smax * sets;
  const int second = sets - 1;
  return launch_cluster(k_adapter_shrink, dim3(unsigned(clusters * ks)), kShrinkThreads, shrink_smem(ctiles, g.stages),
                        ks, c.s, mx[0], mp[0], mx[second], mp[second], g);
}

// U of every token, in partial sums (ranges x N x kp fp32 at `out`).
cudaError_t tokens(const Call& c, const void* X, int64_t ldx, int64_t d, const __nv_bfloat16* P, const int32_t* marks,
                   void* out) {
  TokGeo g{};
  g.X = static_cast<const __nv_bfloat16*>(X);
  g.ldx = ldx;
  g.d = d;
  g.N = c.N;
  g.P = P;
  g.marks = marks;
  g.tok_adapter = c.plan + c.p.tok_adapter;
  g.kp = c.kp;
  g.ranges = tok_ranges(c.N, d);
  g.out = static_cast<float*>(out);
  g.abort_flag = c.abort_flag;
  return launch_cluster(k_adapter_tokens, dim3(unsigned(g.ranges), unsigned(c.N)), kTokThreads, 0, 1, c.s, g);
}

// Y = X W^T + U (packed B)^T (kWmn false: W is o x d) or dX = dY W + T (packed A)^T (true: W is d x o);
// U as slots, or as the tokens' partial sums.
template <bool kWmn>
cudaError_t project(const Call& c, const void* X, int64_t ldx, int64_t d, const void* W, int64_t o,
                    const __nv_bfloat16* P, const void* U, bool token_sums, void* Y, int64_t ldy) {
  const int64_t slots = c.p.smax;
  const int64_t tiles = ((c.N + gp::TM - 1) / gp::TM) * ((o + gp::TN - 1) / gp::TN);
  // Tiles of 128 x 128 by single CTAs fetch twice the bytes per product that a pair's 256 x 256 do, but
  // four times as many fill the SMs.  With 32 pair tiles (1024 tokens x 2048 channels) they take 11.9 us
  // at d = 1024 and 26 at 4096; one round of pairs takes 15 and 32 whatever it holds up to 76.
  const bool few = token_sums || c.N <= kTile || 2 * tiles < sm_count() / 2;
  CUtensorMap mw, mx, mb, mu;
  if (kWmn ? !gp::map_mnmajor(&mw, W, o, d, o) : !gp::map_kmajor(&mw, W, d, o, d)) return cudaErrorInvalidValue;
  if (token_sums) mb = mw;  // (not loaded from)
  else if (!gp::map_3d(&mb, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, P, c.kp, o, c.n, c.kp, o * c.kp, 64, 128))
    return cudaErrorInvalidValue;
  if (few) {
    FewGeo g{};
    g.N = c.N;
    g.d = d;
    g.o = o;
    g.nt = c.N >= kTile ? kTile : int((c.N + 15) / 16 * 16);
    g.ksteps = (c.k + 15) / 16;
    g.tokens = token_sums ? 1 : 0;
    g.kp = c.kp;
    g.ranges = tok_ranges(c.N, d);
    g.U = static_cast<const float*>(U);
    g.B = P;
    g.plan = c.plan;
    g.tile_base = c.p.tile_base;
    g.adapter = c.p.adapter;
    g.tok_adapter = c.p.tok_adapter;
    g.Y = static_cast<__nv_bfloat16*>(Y);
    g.ldy = ldy;
    g.status = c.status;
    g.abort_flag = c.abort_flag;
    g.limit_ns = wait_limit_ns();
    g.mark = c.mark;
    if (!gp::map_2d(&mx, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, X, d, c.N, ldx, 64, g.nt)) return cudaErrorInvalidValue;
    mu = mx;
    if (!token_sums &&
        !gp::map_2d(&mu, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, U, kMaxK, slots * kSlotRows, kMaxK, 64, g.nt))
      return cudaErrorInvalidValue;
    const int64_t ot = (o + 127) / 128, nt = (c.N + g.nt - 1) / g.nt;
    // (5 us of beginning and end are worth 16 k-blocks of 128 tokens; they keep 56 tiles in one round of
    // two CTAs each where five each would take two: 28 us against 35 at d = 8192)
    // by k_adapter_shrink's CTAs, or by two and more blocks of k_adapter_tokens on an SM
    const bool crowded = !token_sums || c.N * g.ranges > 2 * sm_count();
    const int ks = cluster_split(ot * nt, (d + 63) / 64, 16, false, crowded);
    // slots of one tile: a ring that fits beside a CTA of k_adapter_shrink with its small one
    const int stage = kWBytes + g.nt * 128;
    const int low = token_sums ? few_low(g.nt, ks, c.kp) : 0;
    // (with 222 KB no block of k_adapter_tokens fits beside it: one token 10.0 us, with 206 KB 9.4)
    const int room = (token_sums || c.N > kTile ? 206 : 110) * 1024 - low;
    if (token_sums) {  // rows of s B, beside at least three stages (low is at most 98 KB)
      const int most = room - 3 * stage < 72 * 1024 ? room - 3 * stage : 72 * 1024;
      g.held = few_own(g.nt, ks) < most / few_rows(c.kp) ? few_own(g.nt, ks) : most / few_rows(c.kp);
    }
    g.stages = (room - g.held * few_rows(c.kp)) / stage;
    if (g.stages > 12) g.stages = 12;
    return launch_cluster(k_adapter_few<kWmn>, dim3(unsigned(ot * ks), unsigned(nt)), kFewThreads,
                          few_smem(g.nt, g.stages, low, g.held, c.kp), ks, c.s, mw, mx, mb, mu, g);
  }
  CUtensorMap mo;
  if (!gp::map_kmajor(&mx, X, d, c.N, ldx) || !gp::map_out_bf16(&mo, Y, o, c.N, ldy) ||
      !gp::map_2d(&mu, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, U, kMaxK, slots * kSlotRows, kMaxK, 64, 128))
    return cudaErrorInvalidValue;
  gp::Geo g{};
  g.m_tiles = int((c.N + gp::TM - 1) / gp::TM);
  g.cols = int(o);
  g.nkb = int((d + gp::BK - 1) / gp::BK);
  g.splits = 1;
  g.seg_kb = 64;
  g.group = 16;
  g.status = c.status;
  g.abort_flag = c.abort_flag;
  g.limit_ns = wait_limit_ns();
  g.mark = c.mark;
  const AdapterExt ext{c.plan, c.p.tile_base, c.p.pair_count, c.p.pair_ad, c.p.pair_s0, c.p.pair_s1,
                       int(slots * kSlotRows), (c.k + 15) / 16};
  return gp::launch_either<false, kWmn>(mx, mw, mu, mb, mo, g, EpiRows{}, ext, c.s);
}

// dA from X and T, and / or dB from dY and U.
struct Grad {
  const void* S;
  int64_t lds, d;
  const void* U;
  int ranges;
  float* part;
  const float* scale;
  void* out;
};
cudaError_t grad(const Call& c, const Grad* set, int sets, int parts, int dtype) {
  CUtensorMap ms[2], mu[2];
  GradGeo g{};
  JoinOne j[2] = {};
  int64_t dmax = 0;
  const int utiles = col_tiles(c.kp, parts);
  for (int i = 0; i < sets; ++i) {
    const Grad& v = set[i];
    if (!gp::map_mnmajor(&ms[i], v.S, v.d, c.N, v.lds) ||
        !gp::map_3d(&mu[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, v.U, kMaxK, c.p.smax * kSlotRows, utiles, kMaxK,
                    c.p.smax * int64_t(kSlotElems), 64, 64))
      return cudaErrorInvalidValue;
    g.one[i].d = v.d;
    g.one[i].ctiles = int((v.d + 127) / 128);
    g.one[i].ranges = v.ranges;
    g.one[i].items = g.one[i].ctiles * v.ranges;
    g.one[i].part = v.part;
    g.items += g.one[i].items;
    j[i].part = v.part;
    j[i].scale = v.scale;
    j[i].out = v.out;
    j[i].d = v.d;
    j[i].ranges = v.ranges;
    if (v.d > dmax) dmax = v.d;
  }
  g.N = c.N;
  g.n = c.n;
  g.kp = c.kp;
  g.parts = parts;
  g.stages = 200 * 1024 / (kXBytes + utiles * kPBytes);
  if (g.stages > kGradMaxStages) g.stages = kGradMaxStages;
  g.plan = c.plan;
  g.p = c.p;
  g.status = c.status;
  g.abort_flag = c.abort_flag;
  g.limit_ns = wait_limit_ns();
  g.mark = c.mark;
  const int second = sets - 1;
  const unsigned blocks = unsigned(g.items < sm_count() ? g.items : sm_count());
  const cudaError_t e = launch_cluster(k_adapter_grad, dim3(blocks), kGradThreads, grad_smem(utiles, g.stages), 1, c.s, ms[0], mu[0],
                                       ms[second], mu[second], g);
  if (e != cudaSuccess) return e;
  const bool wide = set[0].ranges >= 8;
  const int64_t groups = dmax * (c.kp / 4), per = wide ? 64 : 256;
  auto join = dtype == LOCA_F32 ? (wide ? k_adapter_join<float, 4> : k_adapter_join<float, 1>)
                                : (wide ? k_adapter_join<__nv_bfloat16, 4> : k_adapter_join<__nv_bfloat16, 1>);
  return launch_cluster(join, dim3(unsigned((groups + per - 1) / per), unsigned(c.n), unsigned(sets)), 256, 0, 1, c.s,
                        j[0], j[1], c.k, c.kp, c.plan, c.p);
}

Call call_of(int64_t N, int n, int k, const void* plan, void* workspace, int32_t* status, cudaStream_t s) {
  Call c{};
  c.N = N;
  c.n = n;
  c.k = k;
  c.kp = k_padded(k);
  c.p = plan_lay(N, n);
  c.plan = static_cast<const int32_t*>(plan);
  c.status = status;
  c.abort_flag = static_cast<int32_t*>(workspace);
  // no earlier call's mark (nor, but for one chance in 2^31, what else lay in the workspace)
  static std::atomic<uint32_t> calls{0x2545f491u};
  c.mark = int32_t(calls.fetch_add(0x9e3779b1u, std::memory_order_relaxed) | 1u);
  c.s = s;
  return c;
}

}  // namespace

int adapter_max_k() { return kMaxK; }
size_t adapter_packed_bytes(int n, int64_t d_in, int64_t d_out, int k) { return pack_lay(n, d_in, d_out, k).total; }
size_t adapter_plan_bytes(int64_t N, int n) { return 4 * size_t(plan_lay(N, n).total); }
size_t adapter_workspace_bytes(int64_t N, int64_t d_in, int64_t d_out, int k, int n, bool backward) {
  return adapter_ws(N, d_in, d_out, k, n, backward).total;
}

cudaError_t launch_adapter_pack(const void* A, const void* B, int dtype, int n, int64_t d_in, int64_t d_out, int k,
                                const float* scale, void* packed, cudaStream_t s) {
  const PackLay p = pack_lay(n, d_in, d_out, k);
  uint8_t* b = static_cast<uint8_t*>(packed);
  __nv_bfloat16* pa = reinterpret_cast<__nv_bfloat16*>(b + p.a);
  __nv_bfloat16* pb = reinterpret_cast<__nv_bfloat16*>(b + p.b);
  __nv_bfloat16* all_a = reinterpret_cast<__nv_bfloat16*>(b + p.all_a);
  __nv_bfloat16* all_b = reinterpret_cast<__nv_bfloat16*>(b + p.all_b);
  float* ps = reinterpret_cast<float*>(b + p.scale);
  int32_t* marks = reinterpret_cast<int32_t*>(b + p.marks);
  const cudaError_t e = cudaMemsetAsync(marks, 0, 4 * size_t(n), s);
  if (e != cudaSuccess) return e;
  const int kp = k_padded(k);
  const int64_t values = int64_t(n) * (d_in + d_out) * (kp / 8);
  const unsigned blocks = unsigned(values / 256 + 1 < 8 * sm_count() ? values / 256 + 1 : 8 * sm_count());
  if (dtype == LOCA_F32)
    k_adapter_pack<float><<<blocks, 256, 0, s>>>(static_cast<const float*>(A), static_cast<const float*>(B), n, d_in,
                                                 d_out, k, kp, scale, pa, pb, all_a, all_b, ps, marks);
  else
    k_adapter_pack<__nv_bfloat16><<<blocks, 256, 0, s>>>(static_cast<const __nv_bfloat16*>(A),
                                                         static_cast<const __nv_bfloat16*>(B), n, d_in, d_out, k, kp,
                                                         scale, pa, pb, all_a, all_b, ps, marks);
  return cudaGetLastError();
}

cudaError_t launch_adapter_plan(const int32_t* ids, int64_t N, int n, void* plan, cudaStream_t s) {
  const PlanLay p = plan_lay(N, n);
  int32_t* pl = static_cast<int32_t*>(plan);
  const unsigned tiles = unsigned(p.tiles);
  k_plan_tiles<<<tiles, kTile, 0, s>>>(ids, N, n, pl, p, 0);
  k_plan_scan<<<1, 1024, 0, s>>>(pl, p);
  k_plan_tiles<<<tiles, kTile, 0, s>>>(ids, N, n, pl, p, 1);
  k_plan_pairs<<<unsigned(p.pairs), kTile, 0, s>>>(pl, p);
  k_plan_adapters<<<unsigned(n), 256, 0, s>>>(pl, p, n);
  return cudaGetLastError();
}

cudaError_t launch_adapter_apply(const void* X, int64_t ldx, int64_t N, int64_t d_in, const void* W, int64_t d_out,
                                 const void* packed, int n, int k, const void* plan, void* Y, int64_t ldy,
                                 void* workspace, int32_t* status, cudaStream_t s) {
  const Call c = call_of(N, n, k, plan, workspace, status, s);
  const AdapterWs w = adapter_ws(N, d_in, d_out, k, n, false);
  const PackLay pk = pack_lay(n, d_in, d_out, k);
  const uint8_t* pb = static_cast<const uint8_t*>(packed);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const __nv_bfloat16* pa = reinterpret_cast<const __nv_bfloat16*>(pb + pk.a);
  const int32_t* marks = reinterpret_cast<const int32_t*>(pb + pk.marks);
  const bool tok = by_token(N, n, k);
  const Shrink u{X, ldx, d_in, pa, ws + w.u};
  const cudaError_t e = tok ? tokens(c, X, ldx, d_in, pa, marks, ws + w.u) : shrink(c, &u, 1, marks, 1);
  if (e != cudaSuccess) return e;
  return project<false>(c, X, ldx, d_in, W, d_out, reinterpret_cast<const __nv_bfloat16*>(pb + pk.b), ws + w.u, tok, Y,
                        ldy);
}

size_t adapter_tokens_workspace_bytes(int64_t N, int64_t d_in, int k) {
  return 256 + align256(4 * size_t(tok_ranges(N, d_in)) * size_t(N) * size_t(k_padded(k)));
}
cudaError_t launch_adapter_tokens(const void* X, int64_t ldx, int64_t N, int64_t d_in, int64_t d_out, const void* packed,
                                  int n, int k, const void* plan, void* workspace, AdapterTokens* out, cudaStream_t s) {
  const Call c = call_of(N, n, k, plan, workspace, nullptr, s);
  const PackLay pk = pack_lay(n, d_in, d_out, k);
  const uint8_t* pb = static_cast<const uint8_t*>(packed);
  uint8_t* u = static_cast<uint8_t*>(workspace) + 256;
  *out = AdapterTokens{reinterpret_cast<const float*>(u), reinterpret_cast<const __nv_bfloat16*>(pb + pk.b),
                       c.plan + c.p.tok_adapter, c.kp, tok_ranges(N, d_in)};
  return tokens(c, X, ldx, d_in, reinterpret_cast<const __nv_bfloat16*>(pb + pk.a),
                reinterpret_cast<const int32_t*>(pb + pk.marks), u);
}

cudaError_t launch_adapter_backward(const void* X, int64_t ldx, const void* dY, int64_t lddy, int64_t N, int64_t d_in,
                                    const void* W, int64_t d_out, const void* packed, int n, int k, const void* plan,
                                    void* dX, int64_t lddx, void* dA, void* dB, int grad_dtype, void* workspace,
                                    int32_t* status, cudaStream_t s) {
  const Call c = call_of(N, n, k, plan, workspace, status, s);
  const AdapterWs w = adapter_ws(N, d_in, d_out, k, n, true);
  const PackLay pk = pack_lay(n, d_in, d_out, k);
  const uint8_t* pb = static_cast<const uint8_t*>(packed);
  const __nv_bfloat16* pa = reinterpret_cast<const __nv_bfloat16*>(pb + pk.a);
  const int32_t* marks = reinterpret_cast<const int32_t*>(pb + pk.marks);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  // gradients in fp32 take three parts of U, T and the adapters, in bf16 two (2^-17), dX alone one
  const int parts = !dA && !dB ? 1 : grad_dtype == LOCA_F32 ? kParts : 2;
  const __nv_bfloat16* sa = reinterpret_cast<const __nv_bfloat16*>(pb + (parts == 1 ? pk.a : pk.all_a));
  const __nv_bfloat16* sb = reinterpret_cast<const __nv_bfloat16*>(pb + (parts == 1 ? pk.b : pk.all_b));
  const Shrink u{X, ldx, d_in, sa, ws + w.u}, t{dY, lddy, d_out, sb, ws + w.t};
  Shrink set[2] = {t, t};
  int sets = 0;
  if (dA || dX) set[sets++] = t;
  if (dB) set[sets++] = u;
  cudaError_t e = shrink(c, set, sets, marks, parts);
  if (e != cudaSuccess) return e;
  if (dX) {
    e = project<true>(c, dY, lddy, d_out, W, d_in, pa, ws + w.t, false, dX, lddx);
    if (e != cudaSuccess) return e;
  }
  const Grad ga{X, ldx, d_in, ws + w.t, w.ranges, reinterpret_cast<float*>(ws + w.part_in), nullptr, dA};
  const Grad gb{dY, lddy, d_out, ws + w.u, w.ranges, reinterpret_cast<float*>(ws + w.part_out),
                reinterpret_cast<const float*>(pb + pk.scale), dB};
  Grad grads[2] = {ga, ga};
  int ng = 0;
  if (dA) grads[ng++] = ga;
  if (dB) grads[ng++] = gb;
  return ng ? grad(c, grads, ng, parts, grad_dtype) : cudaSuccess;
}

}  // namespace loca
