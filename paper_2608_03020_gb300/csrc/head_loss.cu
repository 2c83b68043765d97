// Head loss over a large vocabulary without the logits in memory, and its gradients.
//   z = H W^T,  lse_n = log sum_v exp z_nv,  loss_n = w_n (lse_n - z_{n, y_n})      (masked: 0)
//   E[n, c] = w_n (exp(z_{n, l_c} - lse_n) - [y_n = l_c])      the label-column error of Eq. 4
//   dZ = g_n w_n (exp(z - lse) - [v = y_n]),  dH = scale dZ W,  dW = scale dZ^T H
// dH is the d-wide top error W_u^T eps of the one-shot calibration (Eq. 5).
//
// k_head_rows    the rows whose label is in range, one after the other (their hidden states copied,
//                zero rows up to the next tile): masked rows cost no product, and whatever stands
//                in them (infinities, NaN) reaches neither another row nor dW
// k_gemm_pair    logit tiles (256 x 256) on the tensor cores.  Forward: each epilogue thread has 128
//                logits of one row in registers and writes their maximum and sum of exponentials,
//                plus the target's and the label words' logits where its columns hold them.
//                Backward: the same tiles again, summed in the same segments (p = exp(z - lse) is only
//                as good as z and lse agree: with one accumulator over d = 5120 the gradient of a
//                position with 1 - p = 1e-5 came out 50 times too large), turned into
//                dZ = g w (p - onehot), rounded to bf16 as the operand of the two gradient products, for
//                one piece of the rows or of the vocabulary at a time.  That rounding moves the gradients
//                about as much as their own (0.0024 from the 64-bit value in norm, 0.0017 without it); a
//                second part would cost both products again.  `scale` is applied to the fp32 sums, so it
//                rounds nothing
// k_head_target  the target's p - 1 as minus the sum of the others' p.  Where a dW over many rows cuts the
//                vocabulary into pieces (N V > 2^31) the sum over all of them comes first, from a pass
//                over the logits of its own
// k_head_join    combines a row's maxima and sums in a fixed order: lse, loss, E
// k_head_dh      sums the k ranges of dH, scales, rounds once and puts each row back in its place
// Computing the logits a second time costs 2 N d V operations; keeping them would cost 4 N V bytes
// (2.5 GB per 4096 tokens at V = 151936).
// Bound: the tensor cores from a few hundred tokens on, the read of W below.  8192 live of 16384 tokens at
// d = 2048, V = 49152: 1.06 ms (1.55 PFLOP/s; the rest is the epilogue's exponentials and the clock under
// load); 37 tokens 48 us (201 MB of W: 4.2 TB/s for the call, 4.8 in k_gemm_pair).  Loss and dH of 1531
// tokens at d = 5120, V = 151936: 4.5 ms for 7.15 TFLOP (1.59 PFLOP/s).  Up to 128 tokens each gradient
// reads W again (8 tokens at d = 4648, V = 70557: 370 us for three reads of 656 MB).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstring>

#include "gemm_pair.cuh"

namespace loca {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;

constexpr int kRowsPerBlock = 8;          // one per warp
constexpr int kPadBlocks = 16;         // blocks of k_head_rows that write the zero rows
constexpr int64_t kFwdRows = 16384;    // rows per forward piece (bounds the partial maxima and sums)
constexpr int64_t kBwdRows = 8192;     // rows per backward piece at most when dW is not wanted
constexpr int64_t kDzBytes = int64_t(1) << 30;  // dZ of a piece of the rows (dH alone)
// dZ of a piece of the vocabulary where dW sums over all rows: two pieces cost the logits once more (16384
// tokens at d = 1024, V = 65536 with dH and dW: 5.9 ms in two pieces of 1 GiB, 4.2 in one of 2)
constexpr int64_t kDzBytesAll = int64_t(4) << 30;
constexpr int kSegKb = 16;             // logits: 1024 k per accumulation segment
// Up to 128 tokens wait for W, and shorter segments cost them 1 % where they cost the pairs 12 %: the
// error of lse comes down from 3e-7 to 8e-8 of it.  That counts for few tokens: E of a token whose target
// is no label word holds small probabilities alone, which follow lse (3.3e-6 off at worst before, 1.3e-6
// now, of which lse's own rounding to fp32 is 5e-7).
constexpr int kSegKbFew = 4;
constexpr int kSegKbGrad = 64;         // gradients (rounded to bf16): 4096 k per segment

// e^(a - b).  The difference is taken first, so that a probability of one comes out as one and large
// logits lose nothing to the scaling.
__device__ __forceinline__ float exp_diff(float a, float b) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"((a - b) * kLog2e));
  return y;
}

struct Rows {
  int32_t* abort_flag;
  int32_t* count;   // rows with a label in [0, V)
  int32_t* idx;     // their places in the call's order
  int32_t* y;       // their labels (-1 in the padding)
  float* w;         // their weights (0 in the padding)
  float* lse;       // backward: their normalisers
  __nv_bfloat16* H; // their hidden states, then zero rows up to a multiple of 256
};

__device__ __forceinline__ bool live_label(int32_t y, int64_t V) { return y >= 0 && y < V; }

// Live labels among y[0 .. n), counted by the whole block.
__device__ int count_live(const int32_t* __restrict__ y, int64_t n, int64_t V, int* scratch) {
  int c = 0;
  constexpr int kAhead = 8;
  for (int64_t i0 = threadIdx.x; i0 < n; i0 += kAhead * blockDim.x) {
    int32_t v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) v[j] = i0 + j * int64_t(blockDim.x) < n ? __ldg(y + i0 + j * int64_t(blockDim.x)) : -1;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) c += live_label(v[j], V) ? 1 : 0;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = c;
  __syncthreads();
  int sum = 0;
  for (int i = 0; i < int(blockDim.x >> 5); ++i) sum += scratch[i];
  return sum;
}

// Blocks 0 .. nb - 1 take kRowsPerBlock source rows each: the live ones move to their place among the
// live rows, the others' outputs are zeroed.  The last kPadBlocks blocks write the zero rows behind.
// Bound: reads and writes 2 N d bytes each way; every block counts the labels before its own rows
// (4 N bytes from L2), which keeps the pass one launch without a scan.
__global__ void __launch_bounds__(256)
    k_head_rows(const __nv_bfloat16* __restrict__ H, int64_t ldh, int64_t N, int64_t d, int64_t V,
                const int32_t* __restrict__ y, const float* __restrict__ w, const float* __restrict__ dloss,
                const float* __restrict__ lse, Rows out, int64_t npad, int nb, float* loss0, float* lse0, float* E0,
                int C, __nv_bfloat16* dH0, int64_t lddh) {
  __shared__ int scratch[8];
  __shared__ int place[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t dv = d / 8;  // 16-byte vectors of a row
  wait_for_previous();
  launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0) *out.abort_flag = 0;
  if (int(blockIdx.x) >= nb) {
    const int64_t total = count_live(y, N, V, scratch);
    if (int(blockIdx.x) == nb && threadIdx.x == 0) *out.count = int32_t(total);
    int64_t end = (total + gp::TM - 1) / gp::TM * gp::TM;
    if (end < gp::TM) end = gp::TM;
    for (int64_t r = total + (blockIdx.x - nb) * 8 + warp; r < end; r += kPadBlocks * 8) {
      if (!LOCA_CHECK(r, npad)) break;
      uint4* dst = reinterpret_cast<uint4*>(out.H + r * d);
      for (int64_t i = lane; i < dv; i += 32) dst[i] = make_uint4(0, 0, 0, 0);
      if (lane == 0) {
        out.idx[r] = -1;
        out.y[r] = -1;
        out.w[r] = 0.f;
        if (lse) out.lse[r] = 0.f;
      }
    }
    return;
  }
  const int64_t r0 = int64_t(blockIdx.x) * kRowsPerBlock;
  const int base = count_live(y, r0, V, scratch);
  if (warp == 0) {
    const int64_t n = r0 + lane;
    const int32_t yn = lane < kRowsPerBlock && n < N ? y[n] : -1;
    const bool live = live_label(yn, V);
    const unsigned all = __ballot_sync(0xffffffffu, live);
    const int p = live ? base + __popc(all & ((1u << lane) - 1u)) : -1;
    place[lane] = p;
    if (live && LOCA_CHECK(p, npad)) {
      out.idx[p] = int32_t(n);
      out.y[p] = yn;
      out.w[p] = (w ? w[n] : 1.f) * (dloss ? dloss[n] : 1.f);
      if (lse) out.lse[p] = lse[n];
    }
  }
  __syncthreads();
  for (int i = warp; i < kRowsPerBlock; i += 8) {
    const int64_t n = r0 + i;
    if (n >= N) break;
    const int p = place[i];
    if (p >= 0) {
      if (!LOCA_CHECK_SPAN(int64_t(p) * d, d, npad * d)) break;
      const uint4* src = reinterpret_cast<const uint4*>(H + n * ldh);
      uint4* dst = reinterpret_cast<uint4*>(out.H + int64_t(p) * d);
#pragma unroll 8
      for (int64_t j = lane; j < dv; j += 32) dst[j] = __ldg(src + j);
    } else {
      if (lane == 0 && loss0) loss0[n] = 0.f;
      if (lane == 0 && lse0) lse0[n] = 0.f;
      if (E0)
        for (int c = lane; c < C; c += 32) E0[n * C + c] = 0.f;
      if (dH0) {
        uint4* z = reinterpret_cast<uint4*>(dH0 + n * lddh);
        for (int64_t j = lane; j < dv; j += 32) z[j] = make_uint4(0, 0, 0, 0);
      }
    }
  }
}

// ------------------------------------------------------------------ epilogues of the logit tiles
// Forward: maximum and sum of exponentials of 128 logits of a row.
struct EpiStats {
  static constexpr bool kPacks = false;
  static constexpr bool kFits = false;
  float2* part;        // (2 column tiles) x pitch
  int64_t pitch;       // rows of a piece
  const int32_t* y;    // this piece's rows
  float* zy;           // the target's logit
  const int32_t* cols; // label words
  int C;
  float* zc;           // C x pitch: the label words' logits

  __device__ __forceinline__ void operator()(const gp::Tile& t, float (&v)[128], int row, int col0, int lane, uint8_t*,
                                             const CUtensorMap*) const {
    if (!LOCA_CHECK(row, pitch)) return;
    const int left = t.end - col0 < 128 ? t.end - col0 : 128;  // columns of the vocabulary among these
    if (left < 128) {
#pragma unroll
      for (int i = 0; i < 128; ++i)
        if (i >= left) v[i] = -INFINITY;
    }
    float m0 = v[0], m1 = v[1], m2 = v[2], m3 = v[3];
#pragma unroll
    for (int i = 4; i < 128; i += 4) {
      m0 = fmaxf(m0, v[i]);
      m1 = fmaxf(m1, v[i + 1]);
      m2 = fmaxf(m2, v[i + 2]);
      m3 = fmaxf(m3, v[i + 3]);
    }
    const float m = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
    // (a maximum passes over NaN, also where it finds nothing else: the sum of exponentials keeps it)
    const float base = m == -INFINITY ? 0.f : m;
    float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
    for (int i = 0; i < 128; i += 4) {
      s0 += exp_diff(v[i], base);
      s1 += exp_diff(v[i + 1], base);
      s2 += exp_diff(v[i + 2], base);
      s3 += exp_diff(v[i + 3], base);
    }
    part[int64_t(2 * t.n + (col0 > t.col0 ? 1 : 0)) * pitch + row] = make_float2(m, (s0 + s1) + (s2 + s3));
    const int at = y[row] - col0;
    const bool here_y = at >= 0 && at < left;  // (a label past this tile's end is the next tile's)
    if (__any_sync(0xffffffffu, here_y)) {
#pragma unroll
      for (int i = 0; i < 128; ++i)
        if (here_y && i == at) zy[row] = v[i];
    }
    for (int c0 = 0; c0 < C; c0 += 32) {
      const int col = c0 + lane < C ? cols[c0 + lane] - col0 : -1;
      unsigned here = __ballot_sync(0xffffffffu, col >= 0 && col < left);
      while (here) {
        const int b = __ffs(here) - 1;
        here &= here - 1;
        const int j = __shfl_sync(0xffffffffu, col, b);
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < 128; ++i)
          if (i == j) z = v[i];
        zc[int64_t(c0 + b) * pitch + row] = z;
      }
    }
  }
};

// Backward: dZ = g w p of the same tile, bf16, for the gradient products.  Columns past the vocabulary
// and rows past the live ones are zero; the target's entry waits for k_head_target, which gets the sum of
// the other columns' p.
struct EpiDz {
  static constexpr bool kPacks = true;
  static constexpr bool kFits = false;
  static constexpr bool kSums = true;
  const float* lse;
  const float* w;      // w_n dloss_n
  const int32_t* y;
  const int32_t* count;
  int64_t row_first;   // this piece's first row among the live rows
  int64_t v_first;     // this piece's first vocabulary column
  int v_cols;          // its columns of the vocabulary
  float* others;       // (2 column tiles) x pitch
  int64_t pitch;       // rows of a piece

  struct Row {
    float lse, g, others;
    int at, end;  // the target's column and the columns that count (none in rows past the live ones)
  };
  __device__ __forceinline__ Row row_of(int row) const {
    Row r;
    const bool live = row_first + row < *count;
    r.lse = lse[row];
    r.g = w[row];
    r.others = 0.f;
    const int64_t at = int64_t(y[row]) - v_first;
    r.at = at >= 0 && at < v_cols ? int(at) : -1;
    r.end = live ? v_cols : 0;
    return r;
  }
  __device__ __forceinline__ float value(Row& r, int col, float z) const {
    const float p = col < r.end && col != r.at ? exp_diff(z, r.lse) : 0.f;
    r.others += p;
    return col < r.end ? r.g * p : 0.f;
  }
  __device__ __forceinline__ void finish(const Row& r, int part, int row) const {
    if (LOCA_CHECK(row, pitch)) others[int64_t(part) * pitch + row] = r.others;
  }
};

// dH: fp32 sums of one k range, stored or added to the sums of the earlier pieces of the vocabulary
// (one writer per element and launch: a fixed order of additions).
struct EpiAcc {
  static constexpr bool kPacks = false;
  static constexpr bool kFits = true;
  int add;

  __device__ __forceinline__ void operator()(const gp::Tile& t, float (&v)[128], int row, int col0, int lane, uint8_t* box,
                                             const CUtensorMap* out) const {
    const int r0 = t.split_row + row - lane;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (lane == 0) bulk_wait_group_read0();
      __syncwarp();
#pragma unroll
      for (int u = 0; u < 8; ++u)
        *reinterpret_cast<float4*>(box + gp::box_off(lane, u)) =
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

// dW: scaled and rounded once.
struct EpiScaled {
  static constexpr bool kPacks = true;
  static constexpr bool kFits = false;
  static constexpr bool kSums = false;
  float scale;

  struct Row {};
  __device__ __forceinline__ Row row_of(int) const { return Row{}; }
  __device__ __forceinline__ float value(const Row&, int, float v) const { return scale * v; }
};

// ------------------------------------------------------------------ joins
// 32 rows per block, `blockDim.y` groups of partial maxima and sums.
__global__ void __launch_bounds__(1024)
    k_head_join(const float2* __restrict__ part, int64_t pitch, int nparts, Rows in, int64_t row_first,
                const float* __restrict__ zy, const float* __restrict__ zc, const int32_t* __restrict__ cols, int C,
                float* __restrict__ loss, float* __restrict__ lse, float* __restrict__ E) {
  __shared__ float2 sh[32][33];
  wait_for_previous();
  launch_dependents();
  const int64_t row = int64_t(blockIdx.x) * 32 + threadIdx.x;
  const bool live = row_first + row < *in.count;
  float m = -INFINITY, s = 0.f;
  if (live && LOCA_CHECK(row, pitch)) {
    constexpr int kAhead = 8;
    for (int p0 = threadIdx.y; p0 < nparts; p0 += kAhead * int(blockDim.y)) {
      float2 q[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int p = p0 + i * int(blockDim.y);
        q[i] = p < nparts ? part[int64_t(p) * pitch + row] : make_float2(-INFINITY, 0.f);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const float mm = fmaxf(m, q[i].x);
        if (mm != -INFINITY) s = s * exp_diff(m, mm) + q[i].y * exp_diff(q[i].x, mm);
        else s += q[i].y;  // keeps a NaN
        m = mm;
      }
    }
  }
  sh[threadIdx.y][threadIdx.x] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.y != 0 || !live) return;
  for (int j = 1; j < int(blockDim.y); ++j) {
    const float2 q = sh[j][threadIdx.x];
    const float mm = fmaxf(m, q.x);
    if (mm != -INFINITY) s = s * exp_diff(m, mm) + q.y * exp_diff(q.x, mm);
    else s += q.y;
    m = mm;
  }
  const float l = m + logf(s);
  const int64_t k = row_first + row;
  const int32_t n = in.idx[k];
  const float w = in.w[k];
  loss[n] = w * (l - zy[row]);
  if (lse) lse[n] = l;
  if (E) {
    const int32_t y = in.y[k];
    for (int c = 0; c < C; ++c)
      E[int64_t(n) * C + c] = w * (exp_diff(zc[int64_t(c) * pitch + row], l) - (cols[c] == y ? 1.f : 0.f));
  }
}

// The target's entry of dZ: p - 1 = -(sum of the others' p).  As a difference it would be no better than
// lse's rounding to fp32: at lse = 40 and 1 - p = 1e-5 a fifth of it.  32 rows per block, `blockDim.y` groups of
// partial sums.  add: the sum goes on from `sum`; keep: it goes there; put: it is complete.
__global__ void __launch_bounds__(1024)
    k_head_target(const float* __restrict__ part, int64_t pitch, int nparts, Rows in, int64_t row_first, float* sum,
                  int add, int keep, int put, int64_t v_first, int64_t v_cols, __nv_bfloat16* dz, int64_t ldz) {
  __shared__ float sh[32][33];
  wait_for_previous();
  launch_dependents();
  const int64_t row = int64_t(blockIdx.x) * 32 + threadIdx.x;
  const bool live = row_first + row < *in.count;
  float s = 0.f;
  if (live && LOCA_CHECK(row, pitch)) {
#pragma unroll 8
    for (int p = threadIdx.y; p < nparts; p += int(blockDim.y)) s += part[int64_t(p) * pitch + row];
  }
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y != 0 || !live) return;
  for (int j = 1; j < int(blockDim.y); ++j) s += sh[j][threadIdx.x];
  if (add) s += sum[row];
  if (keep) sum[row] = s;
  if (!isfinite(in.lse[row_first + row])) s = NAN;  // (also where there is no other column to say so)
  const int64_t at = int64_t(in.y[row_first + row]) - v_first;
  if (put && at >= 0 && at < v_cols && LOCA_CHECK(at, ldz))
    dz[row * ldz + at] = __float2bfloat16_rn(-in.w[row_first + row] * s);
}

// One thread per 8 elements of a row; the k ranges' sums are loaded four at a time and added in order.
__global__ void __launch_bounds__(256)
    k_head_dh(const float* __restrict__ part, int64_t rows, int planned, const gp::Fit fit, int64_t d, Rows in,
              int64_t row_first, float scale, __nv_bfloat16* __restrict__ dH, int64_t lddh) {
  wait_for_previous();
  launch_dependents();
  const int dv = int(d / 8);
  const int64_t live = *in.count - row_first;
  const int64_t total = (live < rows ? live : rows) * dv;
  const int m_tiles = gp::live_tiles(*in.count, int(row_first / gp::TM), int(rows / gp::TM));
  const int splits = gp::fit_splits(fit, planned, int(rows / gp::TM), m_tiles);
  const int64_t pitch = int64_t(m_tiles) * gp::TM * d;  // sums of a k range
  for (int64_t e = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; e < total; e += int64_t(gridDim.x) * blockDim.x) {
    const int64_t row = e / dv;
    const int64_t at = row * d + 8 * (e - row * dv);
    const int64_t n = in.idx[row_first + row];
    float a[8] = {};
    for (int s0 = 0; s0 < splits; s0 += 4) {
      float4 x[4][2];
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s0 + s < splits) {
          const float4* p = reinterpret_cast<const float4*>(part + int64_t(s0 + s) * pitch + at);
          x[s][0] = p[0];
          x[s][1] = p[1];
        }
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s0 + s < splits) {
          a[0] += x[s][0].x; a[1] += x[s][0].y; a[2] += x[s][0].z; a[3] += x[s][0].w;
          a[4] += x[s][1].x; a[5] += x[s][1].y; a[6] += x[s][1].z; a[7] += x[s][1].w;
        }
    }
    uint4 q;
    q.x = gp::pack_bf16(scale * a[0], scale * a[1]);
    q.y = gp::pack_bf16(scale * a[2], scale * a[3]);
    q.z = gp::pack_bf16(scale * a[4], scale * a[5]);
    q.w = gp::pack_bf16(scale * a[6], scale * a[7]);
    *reinterpret_cast<uint4*>(dH + n * lddh + (at - row * d)) = q;
  }
}

// ------------------------------------------------------------------ host side
int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

struct RowsWs {
  size_t flags, idx, y, w, lse, H, total;
};
RowsWs rows_ws(int64_t N, int64_t d) {
  const size_t np = size_t(round_up(N < 1 ? 1 : N, gp::TM));
  RowsWs o{};
  size_t at = 0;
  o.flags = at; at += 256;
  o.idx = at; at += align256(4 * np);
  o.y = at; at += align256(4 * np);
  o.w = at; at += align256(4 * np);
  o.lse = at; at += align256(4 * np);
  o.H = at; at += align256(2 * np * size_t(d));
  o.total = at;
  return o;
}
Rows rows_at(void* ws, const RowsWs& o) {
  uint8_t* b = static_cast<uint8_t*>(ws);
  Rows r;
  r.abort_flag = reinterpret_cast<int32_t*>(b + o.flags);
  r.count = r.abort_flag + 1;
  r.idx = reinterpret_cast<int32_t*>(b + o.idx);
  r.y = reinterpret_cast<int32_t*>(b + o.y);
  r.w = reinterpret_cast<float*>(b + o.w);
  r.lse = reinterpret_cast<float*>(b + o.lse);
  r.H = reinterpret_cast<__nv_bfloat16*>(b + o.H);
  return r;
}

struct FwdWs {
  RowsWs rows;
  int64_t piece;
  size_t part, zy, zc, total;
};
FwdWs fwd_ws(int64_t N, int64_t V, int64_t d, int C) {
  FwdWs o{};
  o.rows = rows_ws(N, d);
  const int64_t np = round_up(N < 1 ? 1 : N, gp::TM);
  o.piece = np < kFwdRows ? np : kFwdRows;
  const int width = N <= gp::HALF ? gp::slim_width(V) : gp::TN;
  const size_t nparts = 2 * size_t((V + width - 1) / width);
  size_t at = o.rows.total;
  o.part = at; at += align256(nparts * size_t(o.piece) * sizeof(float2));
  o.zy = at; at += align256(4 * size_t(o.piece));
  o.zc = at; at += align256(4 * size_t(o.piece) * size_t(C));
  o.total = at;
  return o;
}

struct BwdWs {
  RowsWs rows;
  int64_t piece;  // rows of dZ
  int64_t vc;     // vocabulary columns of dZ (a multiple of 256)
  int splits;     // k ranges of dH
  size_t dz, part, others, sum, total;
};
bool few_rows(int64_t N) { return N > 0 && N <= gp::HALF; }
// Column tiles that cols vocabulary columns take at most (few rows: whole rounds of the CTAs, whatever the
// tiles' width).
int64_t dz_tiles(int64_t N, int64_t cols) {
  const int64_t tiles = (cols + gp::TN - 1) / gp::TN;
  return few_rows(N) ? round_up(tiles, sm_count()) : tiles;
}
// k ranges of the dH product: its tiles (rows / 256 x d / 512) are few, so one range per tile would
// leave the last round of CTA pairs mostly idle.  More ranges fill it and cost 8 bytes per element and
// range (written, then read by k_head_dh).  Both sides of the choice in cycles.
int dh_splits(int64_t n, int64_t rows, int64_t d, int64_t vc) {
  const int64_t m = rows / gp::TM, nkb = vc / gp::BK;
  const bool single = few_rows(n);
  const double range = double(single ? n : rows) * double(d) * 8.0 / 3000.0 + gp::kRangeCycles;
  int best = 1;
  double best_c = 0;
  for (int s = 1; s <= 32; ++s) {
    if (s > 1 && nkb / s < (single ? 4 : 16)) break;
    const double c = gp::cycles(gp::pick_shape(n, m, d, nkb, s), m, d, nkb, s) + double(s) * range;
    if (s == 1 || c < best_c) {
      best = s;
      best_c = c;
    }
  }
  return best;
}
BwdWs bwd_ws(int64_t N, int64_t V, int64_t d, bool dh, bool dw) {
  BwdWs o{};
  o.rows = rows_ws(N, d);
  const int64_t np = round_up(N < 1 ? 1 : N, gp::TM);
  const int64_t vp = round_up(V, gp::TN);
  // dH alone: as many rows at a time as fit with the whole vocabulary.  dW sums over all rows, so there it
  // is the vocabulary that is cut, if anything is
  int64_t most = kDzBytes / (2 * vp) / gp::TM * gp::TM;
  most = most < gp::TM ? gp::TM : most < kBwdRows ? most : kBwdRows;
  const int64_t cuts = dw ? 1 : (np + most - 1) / most;
  o.piece = round_up((np + cuts - 1) / cuts, gp::TM);
  int64_t vc = (dw ? kDzBytesAll : kDzBytes) / (2 * o.piece) / gp::TN * gp::TN;
  if (vc < 4 * gp::TN) vc = 4 * gp::TN;
  if (vc > vp) vc = vp;
  const int64_t chunks = (vp + vc - 1) / vc;
  o.vc = round_up((vp + chunks - 1) / chunks, gp::TN);
  o.splits = dh ? dh_splits(N, o.piece, d, o.vc) : 0;
  size_t at = o.rows.total;
  o.dz = at; at += align256(2 * size_t(o.piece) * size_t(o.vc));
  o.part = at; at += align256(4 * size_t(o.splits) * size_t(o.piece) * size_t(d));
  o.others = at; at += align256(4 * 2 * size_t(dz_tiles(N, o.vc)) * size_t(o.piece));
  o.sum = at; at += align256(4 * size_t(o.piece));
  o.total = at;
  return o;
}

gp::Geo geo(int64_t m_tiles, int64_t cols, int64_t nkb, int seg_kb, const Rows& r, int32_t* status) {
  gp::Geo g{};
  g.m_tiles = int(m_tiles);
  g.cols = int(cols);
  g.nkb = int(nkb);
  g.splits = 1;
  g.seg_kb = seg_kb;
  g.group = 16;
  g.status = status;
  g.abort_flag = r.abort_flag;
  g.limit_ns = wait_limit_ns();
  return g;
}

cudaError_t launch_rows(const void* H, int64_t ldh, int64_t N, int64_t d, int64_t V, const int32_t* y, const float* w,
                        const float* dloss, const float* lse, const Rows& r, float* loss0, float* lse0, float* E0, int C,
                        void* dH0, int64_t lddh, cudaStream_t s) {
  const int64_t nb = (N + kRowsPerBlock - 1) / kRowsPerBlock;
  return gp::launch_early(k_head_rows, dim3(unsigned(nb + kPadBlocks)), dim3(256), 0, s,
                          static_cast<const __nv_bfloat16*>(H), ldh, N, d, V, y, w, dloss, lse, r,
                          round_up(N < 1 ? 1 : N, gp::TM), int(nb), loss0, lse0, E0, C,
                          static_cast<__nv_bfloat16*>(dH0), lddh);
}

}  // namespace

size_t head_loss_workspace_bytes(int64_t N, int64_t V, int64_t d, int C) { return fwd_ws(N, V, d, C).total; }
size_t head_loss_backward_workspace_bytes(int64_t N, int64_t V, int64_t d, bool dh, bool dw) {
  return bwd_ws(N, V, d, dh, dw).total;
}

cudaError_t launch_head_loss(const void* H, int64_t ldh, int64_t N, int64_t d, const void* W, int64_t V,
                             const int32_t* y, const float* w, const int32_t* cols, int C, float* loss, float* lse,
                             float* E, void* workspace, int32_t* status, cudaStream_t s) {
  const FwdWs lay = fwd_ws(N, V, d, C);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const Rows r = rows_at(workspace, lay.rows);
  cudaError_t e = launch_rows(H, ldh, N, d, V, y, w, nullptr, nullptr, r, loss, lse, E, C, nullptr, 0, s);
  if (e != cudaSuccess) return e;
  const int64_t np = round_up(N, gp::TM);
  const bool single = N <= gp::HALF;
  const int width = single ? gp::slim_width(V) : gp::TN;
  const int nparts = int(2 * ((V + width - 1) / width));
  CUtensorMap mb;
  if (single ? !gp::map_2d(&mb, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, W, d, V, d, gp::BK, width / 2)
             : !gp::map_kmajor(&mb, W, d, V, d))
    return cudaErrorInvalidValue;
  float2* part = reinterpret_cast<float2*>(ws + lay.part);
  float* zy = reinterpret_cast<float*>(ws + lay.zy);
  float* zc = reinterpret_cast<float*>(ws + lay.zc);
  for (int64_t p0 = 0; p0 < np; p0 += lay.piece) {
    const int64_t rows = np - p0 < lay.piece ? np - p0 : lay.piece;
    CUtensorMap ma;
    const int arows = single ? int(round_up(N, 8)) : gp::HALF;
    if (!gp::map_2d(&ma, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, r.H + p0 * d, d, rows, d, gp::BK, arows))
      return cudaErrorInvalidValue;
    gp::Geo g = geo(rows / gp::TM, V, (d + gp::BK - 1) / gp::BK, single ? kSegKbFew : kSegKb, r, status);
    g.rows_live = r.count;
    g.m_first = int(p0 / gp::TM);
    EpiStats epi{part, lay.piece, r.y + p0, zy, cols, E ? C : 0, zc};
    g.width = width;
    g.arows = arows;
    e = single ? gp::launch<gp::kSingle, false, false>(ma, mb, ma, mb, ma, g, epi, gp::NoExt{}, s)
                      : gp::launch<gp::kNarrow, false, false>(ma, mb, ma, mb, ma, g, epi, gp::NoExt{}, s);
    if (e != cudaSuccess) return e;
    e = gp::launch_early(k_head_join, dim3(unsigned(rows / 32)), dim3(32, nparts >= 128 ? 32 : 8), 0, s, part, lay.piece,
                         nparts, r, p0, zy, zc, cols, C, loss, lse, E);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_head_loss_backward(const void* H, int64_t ldh, int64_t N, int64_t d, const void* W, int64_t V,
                                      const int32_t* y, const float* w, const float* lse, const float* dloss,
                                      float scale, void* dH, int64_t lddh, void* dW, void* workspace, int32_t* status,
                                      cudaStream_t s) {
  const BwdWs lay = bwd_ws(N, V, d, dH != nullptr, dW != nullptr);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const Rows r = rows_at(workspace, lay.rows);
  cudaError_t e = launch_rows(H, ldh, N, d, V, y, w, dloss, lse, r, nullptr, nullptr, nullptr, 0, dH, lddh, s);
  if (e != cudaSuccess) return e;
  const int64_t np = round_up(N < 1 ? 1 : N, gp::TM);
  const __nv_bfloat16* Wb = static_cast<const __nv_bfloat16*>(W);
  __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(ws + lay.dz);
  float* part = reinterpret_cast<float*>(ws + lay.part);
  float* others = reinterpret_cast<float*>(ws + lay.others);
  float* sum = reinterpret_cast<float*>(ws + lay.sum);
  for (int64_t p0 = 0; p0 < np; p0 += lay.piece) {
    const int64_t rows = np - p0 < lay.piece ? np - p0 : lay.piece;
    const int64_t kblocks = (lay.vc + gp::BK - 1) / gp::BK;  // of a whole piece of the vocabulary
    const int shape = gp::pick_shape(N, rows / gp::TM, d, kblocks, lay.splits);
    gp::Fit fit{};
    if (dH && shape != gp::kSingle) {
      const int width = shape == gp::kWide ? 2 * gp::TN : gp::TN;
      fit.room = int(lay.splits * (lay.piece / gp::TM));
      fit.at_once = sm_count() / 2;
      fit.n_tiles = int((d + width - 1) / width);
      fit.nkb = int(kblocks);
      fit.kb_cycles = int(gp::kb_cycles(shape));
      fit.tile_cycles = int(gp::tile_cycles(shape));
      fit.row_tile_cycles = int(gp::TM * d * 8 / 3000);
    }
    // dZ of the vocabulary columns v0 .. v0 + vn.  all: they are all there are, so the sum of the others' p that
    // the target's entry takes is whole; done: earlier calls have made it; neither: this call adds to it
    const bool single = few_rows(N);
    auto make_dz = [&](int64_t v0, int64_t vn, bool all, bool done) {
      CUtensorMap mh, mw, mz_out;
      // the forward pass's shape and segments, so that z comes out as it went into lse
      gp::Geo g = geo(rows / gp::TM, vn, (d + gp::BK - 1) / gp::BK, single ? kSegKbFew : kSegKb, r, status);
      g.rows_live = r.count;
      g.m_first = int(p0 / gp::TM);
      g.arows = single ? int(round_up(N, 8)) : gp::HALF;
      g.width = single ? gp::slim_width(vn, 64) : gp::TN;
      if (!gp::map_2d(&mh, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, r.H + p0 * d, d, rows, d, gp::BK, g.arows) ||
          !gp::map_2d(&mw, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, Wb + v0 * d, d, vn, d, gp::BK, g.width / 2) ||
          !gp::map_out_bf16(&mz_out, dz, lay.vc, lay.piece, lay.vc))
        return cudaErrorInvalidValue;
      const EpiDz dzed{r.lse + p0, r.w + p0, r.y + p0, r.count, p0, v0, int(vn), others, lay.piece};
      const cudaError_t e = single ? gp::launch<gp::kSingle, false, false>(mh, mw, mh, mw, mz_out, g, dzed, gp::NoExt{}, s)
                                   : gp::launch<gp::kNarrow, false, false>(mh, mw, mh, mw, mz_out, g, dzed, gp::NoExt{}, s);
      if (e != cudaSuccess) return e;
      const int nparts = done ? 0 : int(2 * ((vn + g.width - 1) / g.width));
      return gp::launch_early(k_head_target, dim3(unsigned(rows / 32)), dim3(32, nparts >= 128 ? 32 : 8), 0, s, others,
                              lay.piece, nparts, r, p0, sum, int(done || v0 > 0), int(!all && !done), int(all || done), v0,
                              vn, dz, lay.vc);
    };
    const bool whole = V <= lay.vc;
    for (int64_t v0 = 0; v0 < V && !whole; v0 += lay.vc)
      if ((e = make_dz(v0, V - v0 < lay.vc ? V - v0 : lay.vc, false, false)) != cudaSuccess) return e;
    for (int64_t v0 = 0; v0 < V; v0 += lay.vc) {
      const int64_t vn = V - v0 < lay.vc ? V - v0 : lay.vc;   // columns of the vocabulary
      const int64_t vtiles = (vn + gp::TN - 1) / gp::TN;
      if ((e = make_dz(v0, vn, whole, !whole)) != cudaSuccess) return e;
      CUtensorMap mz_k, mw_mn;
      if (dH) {
        CUtensorMap mo;
        if (!gp::map_kmajor(&mz_k, dz, lay.vc, lay.piece, lay.vc) || !gp::map_mnmajor(&mw_mn, Wb + v0 * d, d, vn, d) ||
            !gp::map_2d(&mo, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, part, d, lay.piece * lay.splits, d, 32, 32))
          return cudaErrorInvalidValue;
        gp::Geo gh = geo(rows / gp::TM, d, (vn + gp::BK - 1) / gp::BK, kSegKbGrad, r, status);
        gh.rows_live = r.count;
        gh.m_first = int(p0 / gp::TM);
        gh.splits = lay.splits;
        gh.fit = fit;
        e = gp::launch_shape<false, true>(shape, mz_k, mw_mn, mz_k, mw_mn, mo, gh, EpiAcc{v0 > 0 ? 1 : 0}, gp::NoExt{}, s);
        if (e != cudaSuccess) return e;
      }
      if (dW) {
        CUtensorMap mz_mn, mh_mn, mo;
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(dW) + v0 * d;
        if (!gp::map_mnmajor(&mz_mn, dz, lay.vc, lay.piece, lay.vc) || !gp::map_mnmajor(&mh_mn, r.H, d, np, d) ||
            !gp::map_out_bf16(&mo, o, d, vn, d))
          return cudaErrorInvalidValue;
        gp::Geo gw = geo(vtiles, d, np / gp::BK, kSegKbGrad, r, status);
        gw.k_live = r.count;
        e = gp::launch_either<true, true>(mz_mn, mh_mn, mz_mn, mh_mn, mo, gw, EpiScaled{scale}, gp::NoExt{}, s);
        if (e != cudaSuccess) return e;
      }
    }
    if (dH) {
      const int64_t blocks = rows * (d / 8) / 256 + 1;
      const int64_t most = 8 * int64_t(sm_count());
      e = gp::launch_early(k_head_dh, dim3(unsigned(blocks < most ? blocks : most)), dim3(256), 0, s, part, rows,
                           lay.splits, fit, d, r, p0, scale, static_cast<__nv_bfloat16*>(dH), lddh);
      if (e != cudaSuccess) return e;
    }
  }
  return cudaSuccess;
}

}  // namespace loca
