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
// k_head_target  the target's p - 1 as minus the sum of the others' p (with a teacher: p - q of a word with more than
//                half of q as minus the sum of the others' p - q).  Where a dW over many rows cuts the
//                vocabulary into pieces (N V > 2^31) the sum over all of them comes first, from a pass
//                over the logits of its own
// k_head_join    combines a row's maxima and sums in a fixed order: lse, loss, E
// k_head_dh      sums the k ranges of dH, scales, rounds once and puts each row back in its place (k_head_dh_few: of up
//                to 64 positions whose dZ is in two parts)
// Distillation from K teacher logits t of a position, at words i_k:
//   q = softmax(t / tau) over the K,  p = softmax(z / tau) over the vocabulary
//   loss_n = w_n tau^2 sum_k q_k (log q_k - log p_{i_k}),  dZ = g_n w_n tau (p - q)
// k_teacher      each position's words in order, a word that comes twice once with both shares, q and
//                sum q log q, and which word has more than half of q; positions without a word are masked
//                Beside them goes a table of the first word in each row and 128 columns (2 bytes)
// The epilogue of a logit tile reads that table while the sums are not complete and goes on from word to word:
// forward it stores their logits (K of V), backward it takes q off p in fp32, before dZ is rounded, but for a word with
// more than half of q: where p and q are both nearly one their difference is no better than lse's rounding (1 - p = 1e-5
// at lse = 30: 10 % of it), the others' sum is.  (The sum and k_head_target cost 4096 x 2048 x 49152 with both gradients
// 1 %, one position with dH 16 us of 183.)  Bisection in the row's words and a test for each column took 777 tokens at
// d = 896, V = 32003 66 and 75 us where the loss without a teacher takes 37 and 47.
// k_teacher_join as k_head_join, with the sum over the words
// Computing the logits a second time costs 2 N d V operations; keeping them would cost 4 N V bytes
// (2.5 GB per 4096 tokens at V = 151936).
// Bound: the tensor cores from a few hundred tokens on, the read of W below.  8192 live of 16384 tokens at
// d = 2048, V = 49152: 1.06 ms (1.55 PFLOP/s; the rest is the epilogue's exponentials and the clock under
// load); 37 tokens 48 us (201 MB of W: 4.2 TB/s for the call, 4.8 in k_gemm_pair).  Loss and dH of 1531
// tokens at d = 5120, V = 151936: 4.5 ms for 7.15 TFLOP (1.59 PFLOP/s).  Up to 128 tokens each gradient
// reads W again (8 tokens at d = 4648, V = 70557: 370 us for three reads of 656 MB).  Distillation at d = 2048, V = 49152:
// 37 positions 51 us, 4096 of which a quarter is masked, with both gradients, 1.65 to 1.71 ms.
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

// e^((a - b) / tau) with scale = log2(e) / tau
__device__ __forceinline__ float exp_scaled(float a, float b, float scale) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"((a - b) * scale));
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
// dup > 0: the live rows (at most dup of them) come a second time, dup rows behind.
// Bound: reads and writes 2 N d bytes each way; every block counts the labels before its own rows
// (4 N bytes from L2), which keeps the pass one launch without a scan.
__global__ void __launch_bounds__(256)
    k_head_rows(const __nv_bfloat16* __restrict__ H, int64_t ldh, int64_t N, int64_t d, int64_t V,
                const int32_t* __restrict__ y, const float* __restrict__ w, const float* __restrict__ dloss,
                const float* __restrict__ lse, Rows out, int64_t npad, int nb, float* loss0, float* lse0, float* E0,
                int C, __nv_bfloat16* dH0, int64_t lddh, int dup) {
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
      if (dup == 0 || r < dup || r >= dup + total)
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
      if (dup > 0)
        for (int64_t j = lane; j < dv; j += 32) dst[dup * dv + j] = __ldg(src + j);
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
  static constexpr bool kAhead = false;
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
  static constexpr bool kAhead = false;
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

// ------------------------------------------------------------------ a teacher's words
constexpr int kMostWords = 256;
constexpr int kTeacherWarps = 4;  // rows of a block of k_teacher
constexpr int32_t kNoWord = 0x7fffffff;

// Each position's words, ascending and without repetition (kNoWord behind the last), with their shares q.
struct Words {
  int32_t* at;   // N x K
  float* q;      // N x K
  float* ent;    // N: sum q log q over the given entries
  // N: the word with more than half of q, V where there is none, -1 where a position has no word (or no share: all
  // its logits -inf)
  int32_t* main;
  uint16_t* table;  // N x pitch: the first word in a half tile (kNoEntry: none)
  int K;
  int pitch;     // half tiles of a row, to a multiple of 8
  // the half tiles: of tiles of `width` columns, in pieces of the vocabulary of `piece` columns and `of_piece` half tiles
  int width, piece, of_piece;
};
// Column within the half tile | place among the row's words << 7 | whether the next word may be here too << 15.
constexpr uint32_t kNoEntry = 0xffffu;  // (word 255 is the last: none comes after it)
__device__ __forceinline__ int half_of(const Words& t, int32_t v, int& at) {
  const int p = v / t.piece;
  v -= p * t.piece;
  const int n = v / t.width;
  v -= n * t.width;
  at = v & 127;
  return p * t.of_piece + 2 * n + (v >> 7);
}

// One warp a row: the words sorted in shared memory by exchanges whose order the sizes alone fix (bitonic), then
// runs of one word joined from left to right.  Entries outside [0, V) are none.  A NaN among the logits, or +inf,
// makes the row's q NaN.  Bound: latency; 16384 rows of 128 words take 3 waves of the SMs' warps.
__global__ void __launch_bounds__(32 * kTeacherWarps)
    k_teacher(const int32_t* __restrict__ idx, const float* __restrict__ t, int64_t N, int64_t V, float inv_tau, int padded,
              Words out) {
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int32_t* key = reinterpret_cast<int32_t*>(smem_raw) + warp * 2 * padded;
  float* val = reinterpret_cast<float*>(key + padded);
  wait_for_previous();
  launch_dependents();
  const int64_t n = int64_t(blockIdx.x) * kTeacherWarps + warp;
  if (n >= N) return;
  const int K = out.K;
  uint16_t* table = out.table + n * out.pitch;
  for (int i = lane; i < out.pitch / 8; i += 32) reinterpret_cast<uint4*>(table)[i] = make_uint4(~0u, ~0u, ~0u, ~0u);
  for (int i = lane; i < padded; i += 32) {
    const int32_t v = i < K ? __ldg(idx + n * K + i) : -1;
    const bool word = v >= 0 && v < V;
    key[i] = word ? v : kNoWord;
    val[i] = word ? __ldg(t + n * K + i) * inv_tau : -INFINITY;
  }
  __syncwarp();
  for (int span = 2; span <= padded; span <<= 1)
    for (int step = span >> 1; step > 0; step >>= 1) {
      for (int c = lane; c < padded / 2; c += 32) {
        const int i = 2 * c - (c & (step - 1)), j = i + step;
        const int32_t a = key[i], b = key[j];
        if ((a > b) == ((i & span) == 0) && a != b) {
          key[i] = b;
          key[j] = a;
          const float x = val[i];
          val[i] = val[j];
          val[j] = x;
        }
      }
      __syncwarp();
    }
  float m = -INFINITY;
  for (int i = lane; i < padded; i += 32) m = fmaxf(m, val[i]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float base = m == -INFINITY ? 0.f : m;  // (a maximum passes over NaN: the mass keeps it)
  float mass = 0.f;
  for (int i = lane; i < padded; i += 32) mass += expf(val[i] - base);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
  const float log_mass = logf(mass);
  float ent = 0.f;
  int count = 0, main = -1;
  for (int i0 = 0; i0 < padded; i0 += 32) {
    const int i = i0 + lane;
    const int32_t w = i < padded ? key[i] : kNoWord;
    const bool word = w != kNoWord;
    const bool first = word && (i == 0 || key[i - 1] != w);
    float q = 0.f;
    if (word) {
      const float l = val[i] - base - log_mass;
      const float share = expf(l);
      if (!(share == 0.f)) ent += share * l;
    }
    int end = i;  // of the word's run
    if (first)
      for (; end < padded && key[end] == w; ++end) q += expf(val[end] - base - log_mass);
    const unsigned all = __ballot_sync(0xffffffffu, first);
    const int at = count + __popc(all & ((1u << lane) - 1u));
    if (first && LOCA_CHECK(n * K + at, N * K)) {
      out.at[n * K + at] = w;
      out.q[n * K + at] = q;
      if (q > 0.5f) main = w;
      int col, other;
      const int half = half_of(out, w, col);
      const bool more = end < padded && key[end] != kNoWord && half_of(out, key[end], other) == half;
      if ((i == 0 || half_of(out, key[i - 1], other) != half) && LOCA_CHECK(half, out.pitch))
        table[half] = uint16_t(col | at << 7 | (more ? 1 << 15 : 0));
    }
    count += __popc(all);
  }
  for (int i = count + lane; i < K; i += 32) {
    out.at[n * K + i] = kNoWord;
    out.q[n * K + i] = 0.f;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ent += __shfl_xor_sync(0xffffffffu, ent, o);
  main = __reduce_max_sync(0xffffffffu, main);  // (one lane's at most)
  if (lane == 0) {
    out.ent[n] = ent;
    out.main[n] = mass == 0.f ? -1 : main >= 0 ? main : int32_t(V);  // (NaN lives, without such a word)
  }
}

// A thread's look-ups: its row's place in the call's order, a tile ahead, and what the table has for this tile.
struct WordState {
  int32_t n, next_n;
  uint32_t entry;
};
// idx: the rows' places in the call's order, or null where they stand in it (`rows` of them).
__device__ __forceinline__ int32_t place_of(const int32_t* idx, int rows, int row) {
  return idx ? idx[row] : row < rows ? row : -1;
}
__device__ __forceinline__ void words_ahead(const Words& t, const int32_t* idx, int rows, WordState& s, int half,
                                            int next_row) {
  s.n = s.next_n;
  s.entry = kNoEntry;
  if (s.n >= 0 && LOCA_CHECK(half, t.pitch)) s.entry = __ldg(t.table + int64_t(s.n) * t.pitch + half);
  s.next_n = place_of(idx, rows, next_row);
}

// v[i] for an i that differs from thread to thread: halves chosen bit by bit.
__device__ __forceinline__ float pick(const float (&v)[128], int i) {
  float a[64];
#pragma unroll
  for (int k = 0; k < 64; ++k) a[k] = i & 64 ? v[64 + k] : v[k];
#pragma unroll
  for (int w = 32; w > 0; w >>= 1)
#pragma unroll
    for (int k = 0; k < w; ++k) a[k] = i & w ? a[w + k] : a[k];
  return a[0];
}

// Forward: maximum and sum of exponentials of 128 logits of a row, and the logits of its words.
struct EpiTeacher {
  static constexpr bool kPacks = false;
  static constexpr bool kFits = false;
  static constexpr bool kAhead = true;
  using State = WordState;
  float2* part;        // (2 column tiles) x pitch
  int64_t pitch;       // rows of a piece
  const int32_t* idx;  // this piece's rows: their places in the call's order (null: `rows` of them in it)
  int rows;
  Words words;
  float* zk;           // pitch x K
  float scale;         // log2(e) / tau

  __device__ __forceinline__ void start(State& s, int row) const { s.next_n = place_of(idx, rows, row); }
  __device__ __forceinline__ void ahead(State& s, int row, int half, int next_row) const {
    words_ahead(words, idx, rows, s, half, next_row);
  }
  __device__ __forceinline__ void operator()(const gp::Tile& t, float (&v)[128], const State& st, int row, int col0, int lane,
                                             uint8_t*, const CUtensorMap*) const {
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
    const float base = m == -INFINITY ? 0.f : m;  // (as EpiStats)
    float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
    for (int i = 0; i < 128; i += 4) {
      s0 += exp_scaled(v[i], base, scale);
      s1 += exp_scaled(v[i + 1], base, scale);
      s2 += exp_scaled(v[i + 2], base, scale);
      s3 += exp_scaled(v[i + 3], base, scale);
    }
    part[int64_t(2 * t.n + (col0 > t.col0 ? 1 : 0)) * pitch + row] = make_float2(m, (s0 + s1) + (s2 + s3));
    bool here = st.entry != kNoEntry;
    int at = st.entry & 127, k = st.entry >> 7 & 255;
    bool more = st.entry >> 15 & 1;
    while (__any_sync(0xffffffffu, here)) {
      const bool on = here && more && k + 1 < words.K;
      const int32_t next = on ? __ldg(words.at + int64_t(st.n) * words.K + k + 1) : kNoWord;  // (back before pick() is)
      const float z = pick(v, at);
      if (here && LOCA_CHECK(k, words.K)) zk[int64_t(row) * words.K + k] = z;
      here = on && next < col0 + left;
      at = next - col0;
      ++k;
    }
  }
};

// Backward: dZ = g tau (p - q) of the same tile, bf16, for the gradient products.  Columns past the vocabulary and
// rows past the live ones are zero.  The entry of a word with more than half of q waits for k_head_target, which gets the
// sum of the other columns' p - q.
struct EpiDzTeacher {
  static constexpr bool kPacks = true;
  static constexpr bool kFits = false;
  static constexpr bool kAhead = true;
  using State = WordState;
  const float* lse;    // this piece's rows
  const float* w;      // w_n dloss_n
  const int32_t* y;    // the word with more than half of q, or none of [0, V)
  const int32_t* idx;
  Words words;
  float tau, inv_tau;
  const int32_t* count;
  int64_t row_first;   // this piece's first row among the live rows
  int64_t v_first;     // this piece's first vocabulary column
  int v_cols;          // its columns of the vocabulary
  int half_first;      // its first half tile
  float* others;       // (2 column tiles) x pitch
  int64_t pitch;       // rows of a piece
  // Few rows: dZ in two bf16 parts (2^-17), the second low_row rows behind the first, where the tile of 128 rows has
  // room for it, so that it costs no product.  The gradient of a row of few words is as good as its largest entries.
  int low_row;
  __nv_bfloat16* dz;
  int64_t ldz;

  __device__ __forceinline__ void store_parts(const float (&f)[32], int row, int col) const {
    if (row >= low_row) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = f[8 * j + 2 * i], b = f[8 * j + 2 * i + 1];
        hi[i] = gp::pack_bf16(a, b);
        const float2 r = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&hi[i]));
        lo[i] = gp::pack_bf16(a - r.x, b - r.y);
      }
      if (col + 8 * j >= int(ldz) || !LOCA_CHECK_SPAN(col + 8 * j, 8, ldz)) continue;
      *reinterpret_cast<uint4*>(dz + row * ldz + col + 8 * j) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(dz + (row + low_row) * ldz + col + 8 * j) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  }

  struct Row {
    float lse, g, others;
    float keep, q;  // what becomes of the next word's p: p - q, or 0
    int end;   // the columns that count (none in rows past the live ones)
    int main;  // the column of the word with more than half of q
    int next;  // the next word's column, its place and whether another may follow
    int k;
    bool more;
    int64_t from;  // of the row's words
  };
  __device__ __forceinline__ void start(State& s, int row) const { s.next_n = idx[row]; }
  __device__ __forceinline__ void ahead(State& s, int row, int half, int next_row) const {
    words_ahead(words, idx, 0, s, half_first + half, next_row);
  }
  __device__ __forceinline__ Row row_of(int row, const State& st, int col0) const {
    Row r;
    const bool here = st.entry != kNoEntry;  // (the table has nothing for rows past the live ones)
    r.end = row_first + row < *count ? v_cols : 0;
    r.main = int(y[row] - v_first);
    r.others = 0.f;
    r.k = st.entry >> 7 & 255;
    r.from = int64_t(st.n) * words.K;
    r.next = here ? col0 + int(st.entry & 127) : kNoWord;
    r.keep = r.next != r.main ? 1.f : 0.f;
    r.q = here && r.next != r.main ? __ldg(words.q + r.from + r.k) : 0.f;
    r.more = here && (st.entry >> 15 & 1);
    r.lse = lse[row];
    r.g = w[row] * tau;
    return r;
  }
  __device__ __forceinline__ bool simple(const Row& r) const { return !__any_sync(0xffffffffu, r.more); }
  __device__ __forceinline__ float value1(Row& r, int col, float z) const {
    float p = exp_diff(fmaf(z, inv_tau, -r.lse), 0.f);
    if (col == r.next) p = fmaf(p, r.keep, -r.q);
    p = col < r.end ? p : 0.f;
    r.others += p;
    return r.g * p;
  }
  __device__ __forceinline__ float value(Row& r, int col, float z) const {
    if (col >= r.end) return 0.f;
    float p = exp_diff(fmaf(z, inv_tau, -r.lse), 0.f);
    if (col == r.next) {
      p = fmaf(p, r.keep, -r.q);
      r.next = kNoWord;
      if (++r.k < words.K) {
        const int32_t v = __ldg(words.at + r.from + r.k);
        r.q = __ldg(words.q + r.from + r.k);  // (with it, not behind it: behind the last word nobody takes it)
        if (v != kNoWord) r.next = int(v - v_first);
        r.keep = r.next != r.main ? 1.f : 0.f;
        if (r.next == r.main) r.q = 0.f;
      }
    }
    r.others += p;
    return r.g * p;
  }
  __device__ __forceinline__ void finish(float sum, int part, int row) const {
    if (LOCA_CHECK(row, pitch)) others[int64_t(part) * pitch + row] = sum;
  }
  // p of every column, then q off it, then the factor.  The first words of the warp's rows go one by one, each against
  // all columns (260 instructions); where a row has more than kOneByOne, the rest column by column, where a lane that
  // meets its word waits for the next.  (Loss and dH, one by one alone, column by column alone, and both: 4217 positions with
  // 96 words at d = 744, V = 48060 1102, 1700 and 1034 us; 192 with 87 words at V = 4839 163, 125 and 125.)
  static constexpr int kOneByOne = 8;
  __device__ __forceinline__ void all(float (&v)[128], const State& st, int row, int col0, int part) const {
    const float row_lse = lse[row], g = w[row] * tau;
    const int end = row_first + row < *count ? v_cols - col0 : 0;  // the columns that count (none in rows past the live ones)
    const bool here = st.entry != kNoEntry;  // (the table has nothing for rows past the live ones)
    const int32_t first = int32_t(v_first) + col0;
    const int64_t from = int64_t(st.n) * words.K;
    int k = st.entry >> 7 & 255;
    int last = here ? st.entry >> 15 & 1 ? words.K - 1 : k : -1;  // no word here behind it
    int at = here ? int(st.entry & 127) : -1;
    const int main = int(y[row] - first);
    // what becomes of the word's p: p - q, or 0
    float q = here && at != main ? __ldg(words.q + from + k) : 0.f, keep = at != main ? 1.f : 0.f;
    int32_t next = kNoWord;  // the word behind, and its share
    float next_q = 0.f;
    auto fetch = [&] {
      next = kNoWord;
      if (++k <= last) {
        next = __ldg(words.at + from + k);
        next_q = __ldg(words.q + from + k);
      }
    };
    auto advance = [&] {  // (a column below 0 or from 128 on is none of these)
      at = next < first + 128 ? next - first : -1;
      keep = at != main ? 1.f : 0.f;
      q = at != main ? next_q : 0.f;
      fetch();
    };
    fetch();
#pragma unroll
    for (int i = 0; i < 128; ++i) v[i] = exp_diff(fmaf(v[i], inv_tau, -row_lse), 0.f);
    int n = 0;
    for (; n < kOneByOne && __any_sync(0xffffffffu, at >= 0); ++n) {
#pragma unroll
      for (int i = 0; i < 128; ++i)
        if (i == at) v[i] = fmaf(v[i], keep, -q);
      advance();
    }
    if (n == kOneByOne && __any_sync(0xffffffffu, at >= 0)) {
#pragma unroll
      for (int i = 0; i < 128; ++i)
        if (i == at) {
          v[i] = fmaf(v[i], keep, -q);
          advance();
        }
    }
    float s[4] = {};
#pragma unroll
    for (int i = 0; i < 128; ++i) {
      v[i] = i < end ? v[i] : 0.f;
      s[i & 3] += v[i];
      v[i] *= g;
    }
    finish((s[0] + s[1]) + (s[2] + s[3]), part, row);
  }
};

// ------------------------------------------------------------------ joins
// A row's maximum and sum of exponentials from `blockDim.y` groups of partial ones, 32 rows per block; complete in
// the threads of group 0.  exp: e^(difference).
template <class Exp>
__device__ __forceinline__ float2 join_parts(const float2* __restrict__ part, int64_t pitch, int nparts, int64_t row,
                                             bool live, float2 (&sh)[32][33], const Exp& exp) {
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
        if (mm != -INFINITY) s = s * exp(m, mm) + q[i].y * exp(q[i].x, mm);
        else s += q[i].y;  // keeps a NaN
        m = mm;
      }
    }
  }
  sh[threadIdx.y][threadIdx.x] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.y == 0 && live)
    for (int j = 1; j < int(blockDim.y); ++j) {
      const float2 q = sh[j][threadIdx.x];
      const float mm = fmaxf(m, q.x);
      if (mm != -INFINITY) s = s * exp(m, mm) + q.y * exp(q.x, mm);
      else s += q.y;
      m = mm;
    }
  return make_float2(m, s);
}

__global__ void __launch_bounds__(1024)
    k_head_join(const float2* __restrict__ part, int64_t pitch, int nparts, Rows in, int64_t row_first,
                const float* __restrict__ zy, const float* __restrict__ zc, const int32_t* __restrict__ cols, int C,
                float* __restrict__ loss, float* __restrict__ lse, float* __restrict__ E) {
  __shared__ float2 sh[32][33];
  wait_for_previous();
  launch_dependents();
  const int64_t row = int64_t(blockIdx.x) * 32 + threadIdx.x;
  const bool live = row_first + row < *in.count;
  const float2 ms = join_parts(part, pitch, nparts, row, live, sh, [](float a, float b) { return exp_diff(a, b); });
  if (threadIdx.y != 0 || !live) return;
  const float m = ms.x, s = ms.y;
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

// lse, and the loss from the words' logits: a warp per row, in the order of the words within a lane.
__global__ void __launch_bounds__(1024)
    k_teacher_join(const float2* __restrict__ part, int64_t pitch, int nparts, Rows in, int64_t row_first,
                   const float* __restrict__ zk, Words words, float tau, float inv_tau, float* __restrict__ loss,
                   float* __restrict__ lse) {
  __shared__ float2 sh[32][33];
  wait_for_previous();
  launch_dependents();
  const int64_t row = int64_t(blockIdx.x) * 32 + threadIdx.x;
  const bool live = row_first + row < *in.count;
  const float scale = kLog2e * inv_tau;
  const float2 ms =
      join_parts(part, pitch, nparts, row, live, sh, [scale](float a, float b) { return exp_scaled(a, b, scale); });
  __syncthreads();
  if (threadIdx.y == 0) sh[0][threadIdx.x] = make_float2(ms.x, logf(ms.y));
  __syncthreads();
  for (int r = threadIdx.y; r < 32; r += int(blockDim.y)) {
    const int64_t k = row_first + int64_t(blockIdx.x) * 32 + r;
    if (k >= *in.count) break;
    const float m = sh[0][r].x, log_s = sh[0][r].y;
    const int32_t n = in.idx[k];
    const int64_t at = int64_t(n) * words.K, from = (k - row_first) * words.K;
    float sum = 0.f;
    for (int j = threadIdx.x; j < words.K; j += 32) {
      const float q = words.q[at + j];
      if (words.at[at + j] != kNoWord && !(q == 0.f)) sum += q * ((zk[from + j] - m) * inv_tau - log_s);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x == 0) {
      loss[n] = in.w[k] * tau * tau * (words.ent[n] - sum);
      if (lse) lse[n] = m * inv_tau + log_s;
    }
  }
}

// The same for few rows that stand in the call's order: a block per row.
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads)
    k_teacher_join_few(const float2* __restrict__ part, int64_t pitch, int nparts, const float* __restrict__ zk, Words words,
                       const float* __restrict__ w, float tau, float inv_tau, float* __restrict__ loss,
                       float* __restrict__ lse) {
  __shared__ float2 sh[kJoinThreads / 32];
  __shared__ float sums[kJoinThreads / 32];
  wait_for_previous();
  launch_dependents();
  const int n = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (words.main[n] < 0) {
    if (threadIdx.x == 0) {
      loss[n] = 0.f;
      if (lse) lse[n] = 0.f;
    }
    return;
  }
  const float scale = kLog2e * inv_tau;
  float m = -INFINITY, s = 0.f;
  auto add = [&](float m2, float s2) {
    const float mm = fmaxf(m, m2);
    if (mm != -INFINITY) s = s * exp_scaled(m, mm, scale) + s2 * exp_scaled(m2, mm, scale);
    else s += s2;  // keeps a NaN
    m = mm;
  };
  constexpr int kMore = 4;
  for (int p0 = threadIdx.x; p0 < nparts; p0 += kMore * kJoinThreads) {
    float2 q[kMore];
#pragma unroll
    for (int i = 0; i < kMore; ++i)
      q[i] = p0 + i * kJoinThreads < nparts ? part[int64_t(p0 + i * kJoinThreads) * pitch + n] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int i = 0; i < kMore; ++i) add(q[i].x, q[i].y);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m2 = __shfl_down_sync(0xffffffffu, m, o), s2 = __shfl_down_sync(0xffffffffu, s, o);
    add(m2, s2);
  }
  if (lane == 0) sh[warp] = make_float2(m, s);
  __syncthreads();
  m = sh[0].x;
  s = sh[0].y;
  for (int i = 1; i < kJoinThreads / 32; ++i) add(sh[i].x, sh[i].y);
  const float log_s = logf(s);
  float sum = 0.f;
  static_assert(kMostWords <= kJoinThreads, "a word a thread");
  if (int(threadIdx.x) < words.K) {
    const int64_t at = int64_t(n) * words.K + threadIdx.x;
    const float q = words.q[at];
    if (words.at[at] != kNoWord && !(q == 0.f)) sum = q * ((zk[at] - m) * inv_tau - log_s);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sums[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = sums[0];
    for (int i = 1; i < kJoinThreads / 32; ++i) sum += sums[i];
    loss[n] = (w ? w[n] : 1.f) * tau * tau * (words.ent[n] - sum);
    if (lse) lse[n] = m * inv_tau + log_s;
  }
}

// The target's entry of dZ: p - 1 = -(sum of the others' p).  As a difference it would be no better than
// lse's rounding to fp32: at lse = 40 and 1 - p = 1e-5 a fifth of it.  With a teacher p - q = -(sum of the others' p - q)
// where one word has more than half of q: the others' p, which carry lse's rounding too, then have less of the error than
// the word's own.  32 rows per block, `blockDim.y` groups of partial sums.  add: the sum goes on from `sum`; keep: it goes
// there; put: it is complete.  low_row > 0: the second part of the entry comes so many rows behind.
__global__ void __launch_bounds__(1024)
    k_head_target(const float* __restrict__ part, int64_t pitch, int nparts, Rows in, int64_t row_first, float* sum,
                  int add, int keep, int put, int64_t v_first, int64_t v_cols, float factor, int low_row,
                  __nv_bfloat16* dz, int64_t ldz) {
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
  if (put && at >= 0 && at < v_cols && LOCA_CHECK(at, ldz)) {
    const float v = -(in.w[row_first + row] * factor) * s;
    const __nv_bfloat16 hi = __float2bfloat16_rn(v);
    dz[row * ldz + at] = hi;
    if (low_row > 0 && LOCA_CHECK(row, low_row)) dz[(row + low_row) * ldz + at] = __float2bfloat16_rn(v - __bfloat162float(hi));
  }
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

// Few rows, dZ in two parts: eight warps share an output's ranges (both parts' sums of each), and meet in order.  In one
// thread they took 10 us more (one row, d = 2048, 19 ranges).
__global__ void __launch_bounds__(256) k_head_dh_few(const float* __restrict__ part, int splits, int64_t d, Rows in, float scale,
                                                     int low_row, __nv_bfloat16* __restrict__ dH, int64_t lddh) {
  __shared__ float sums[8][32][9];
  wait_for_previous();
  launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, dv = int(d / 8);
  const int total = *in.count * dv, e = int(blockIdx.x) * 32 + lane;
  const int row = e / dv, col = 8 * (e - row * dv);
  float a[8] = {};
  if (e < total)
#pragma unroll 2
    for (int s = warp; s < splits; s += 8)
#pragma unroll
      for (int lo = 0; lo < 2; ++lo) {
        const float4* p = reinterpret_cast<const float4*>(part + (int64_t(s) * gp::TM + row + lo * low_row) * d + col);
        const float4 x = p[0], y = p[1];
        a[0] += x.x; a[1] += x.y; a[2] += x.z; a[3] += x.w;
        a[4] += y.x; a[5] += y.y; a[6] += y.z; a[7] += y.w;
      }
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[warp][lane][i] = a[i];
  __syncthreads();
  if (warp > 0 || e >= total) return;
  for (int w = 1; w < 8; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] += sums[w][lane][i];
  uint4 q;
  q.x = gp::pack_bf16(scale * a[0], scale * a[1]);
  q.y = gp::pack_bf16(scale * a[2], scale * a[3]);
  q.z = gp::pack_bf16(scale * a[4], scale * a[5]);
  q.w = gp::pack_bf16(scale * a[6], scale * a[7]);
  *reinterpret_cast<uint4*>(dH + int64_t(in.idx[row]) * lddh + col) = q;
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

int fwd_width(int64_t N, int64_t V) { return N <= gp::HALF ? gp::slim_width(V) : gp::TN; }

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
  const int width = fwd_width(N, V);
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
  int room;       // row tiles x ranges that the sums' memory holds
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
// fill: room for as many ranges of the live rows as fill four rounds of the pairs (fit_splits(); without it 3081 live of 4096
// tokens at d = 2048, V = 49152 are three rounds of 256 k-blocks, with it three of 192: dH of distillation 952 and 855 us).
BwdWs bwd_ws(int64_t N, int64_t V, int64_t d, bool dh, bool dw, bool fill) {
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
  const int64_t m = o.piece / gp::TM;
  o.room = int(o.splits * m);
  if (fill && dh && !few_rows(N)) {
    const int64_t ranges = o.vc / gp::BK / 16 < 32 ? o.vc / gp::BK / 16 : 32;  // (at most: as fit_splits())
    int64_t room = 4 * (sm_count() / 2) / ((d + 2 * gp::TN - 1) / (2 * gp::TN));
    if (room > m * ranges) room = m * ranges;
    if (room > o.room) o.room = int(room);
  }
  size_t at = o.rows.total;
  o.dz = at; at += align256(2 * size_t(o.piece) * size_t(o.vc));
  o.part = at; at += align256(4 * size_t(o.room) * gp::TM * size_t(d));
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
                        void* dH0, int64_t lddh, cudaStream_t s, int dup = 0) {
  const int64_t nb = (N + kRowsPerBlock - 1) / kRowsPerBlock;
  return gp::launch_early(k_head_rows, dim3(unsigned(nb + kPadBlocks)), dim3(256), 0, s,
                          static_cast<const __nv_bfloat16*>(H), ldh, N, d, V, y, w, dloss, lse, r,
                          round_up(N < 1 ? 1 : N, gp::TM), int(nb), loss0, lse0, E0, C,
                          static_cast<__nv_bfloat16*>(dH0), lddh, dup);
}

// The logit tiles of a forward piece; width: columns of a tile.
template <class Epi>
cudaError_t forward_tiles(const Rows& r, int64_t N, int64_t p0, int64_t rows, int64_t d, const void* W, int64_t V,
                          const Epi& epi, int32_t* status, int width, cudaStream_t s) {
  const bool single = N <= gp::HALF;
  const int arows = single ? int(round_up(N, 8)) : gp::HALF;
  CUtensorMap ma, mb;
  if ((single ? !gp::map_2d(&mb, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, W, d, V, d, gp::BK, width / 2)
              : !gp::map_kmajor(&mb, W, d, V, d)) ||
      !gp::map_2d(&ma, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, r.H + p0 * d, d, rows, d, gp::BK, arows))
    return cudaErrorInvalidValue;
  gp::Geo g = geo(rows / gp::TM, V, (d + gp::BK - 1) / gp::BK, single ? kSegKbFew : kSegKb, r, status);
  g.rows_live = r.count;
  g.m_first = int(p0 / gp::TM);
  g.width = width;
  g.arows = arows;
  return single ? gp::launch<gp::kSingle, false, false>(ma, mb, ma, mb, ma, g, epi, gp::NoExt{}, s)
                : gp::launch<gp::kNarrow, false, false>(ma, mb, ma, mb, ma, g, epi, gp::NoExt{}, s);
}

// Columns of the backward pass's logit tiles.
int back_width(int64_t N, int64_t cols) { return few_rows(N) ? gp::slim_width(cols, 64) : gp::TN; }

struct Backward {
  BwdWs lay;
  Rows r;
  uint8_t* ws;
  int64_t N, d;
  const __nv_bfloat16* W;
  int64_t V;
  float scale;
  __nv_bfloat16* dH;
  int64_t lddh;
  __nv_bfloat16* dW;
  int32_t* status;
  cudaStream_t s;
  int low_row = 0;  // dZ has a second part so many rows behind the first (0: none)
};

// The logits of a piece once more, into dZ, in the forward pass's shape and segments, so that z comes out as it went
// into lse; width: columns of a tile.
template <class Epi>
cudaError_t logit_tiles(const Backward& b, int64_t p0, int64_t rows, int64_t v0, int64_t vn, const Epi& epi, int width) {
  const bool single = few_rows(b.N);
  CUtensorMap mh, mw, mz_out;
  gp::Geo g = geo(rows / gp::TM, vn, (b.d + gp::BK - 1) / gp::BK, single ? kSegKbFew : kSegKb, b.r, b.status);
  g.rows_live = b.r.count;
  g.m_first = int(p0 / gp::TM);
  g.arows = single ? int(round_up(b.N, 8)) : gp::HALF;
  g.width = width;
  if (!gp::map_2d(&mh, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, b.r.H + p0 * b.d, b.d, rows, b.d, gp::BK, g.arows) ||
      !gp::map_2d(&mw, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, b.W + v0 * b.d, b.d, vn, b.d, gp::BK, g.width / 2) ||
      !gp::map_out_bf16(&mz_out, b.ws + b.lay.dz, b.lay.vc, b.lay.piece, b.lay.vc))
    return cudaErrorInvalidValue;
  return single ? gp::launch<gp::kSingle, false, false>(mh, mw, mh, mw, mz_out, g, epi, gp::NoExt{}, b.s)
                : gp::launch<gp::kNarrow, false, false>(mh, mw, mh, mw, mz_out, g, epi, gp::NoExt{}, b.s);
}

// dH and dW in pieces of the rows and of the vocabulary.  before(p0, rows) comes ahead of a piece of rows;
// make_dz(p0, rows, v0, vn) leaves its dZ of vn vocabulary columns in the workspace.
template <class Before, class MakeDz>
cudaError_t backward_pieces(const Backward& b, const Before& before, const MakeDz& make_dz) {
  const BwdWs& lay = b.lay;
  const Rows& r = b.r;
  const int64_t N = b.N, d = b.d, V = b.V, lddh = b.lddh;
  __nv_bfloat16 *dH = b.dH, *dW = b.dW;
  const int64_t np = round_up(N < 1 ? 1 : N, gp::TM);
  __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(b.ws + lay.dz);
  float* part = reinterpret_cast<float*>(b.ws + lay.part);
  cudaError_t e = cudaSuccess;
  for (int64_t p0 = 0; p0 < np; p0 += lay.piece) {
    const int64_t rows = np - p0 < lay.piece ? np - p0 : lay.piece;
    const int64_t kblocks = (lay.vc + gp::BK - 1) / gp::BK;  // of a whole piece of the vocabulary
    const int shape = gp::pick_shape(N, rows / gp::TM, d, kblocks, lay.splits);
    gp::Fit fit{};
    if (dH && shape != gp::kSingle) {
      const int width = shape == gp::kWide ? 2 * gp::TN : gp::TN;
      fit.room = lay.room;
      fit.at_once = sm_count() / 2;
      fit.n_tiles = int((d + width - 1) / width);
      fit.nkb = int(kblocks);
      fit.kb_cycles = int(gp::kb_cycles(shape));
      fit.tile_cycles = int(gp::tile_cycles(shape));
      fit.row_tile_cycles = int(gp::TM * d * 8 / 3000);
    }
    if ((e = before(p0, rows)) != cudaSuccess) return e;
    for (int64_t v0 = 0; v0 < V; v0 += lay.vc) {
      const int64_t vn = V - v0 < lay.vc ? V - v0 : lay.vc;   // columns of the vocabulary
      const int64_t vtiles = (vn + gp::TN - 1) / gp::TN;
      if ((e = make_dz(p0, rows, v0, vn)) != cudaSuccess) return e;
      CUtensorMap mz_k, mw_mn;
      if (dH) {
        CUtensorMap mo;
        if (!gp::map_kmajor(&mz_k, dz, lay.vc, lay.piece, lay.vc) || !gp::map_mnmajor(&mw_mn, b.W + v0 * d, d, vn, d) ||
            !gp::map_2d(&mo, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, part, d, int64_t(lay.room) * gp::TM, d, 32, 32))
          return cudaErrorInvalidValue;
        gp::Geo gh = geo(rows / gp::TM, d, (vn + gp::BK - 1) / gp::BK, kSegKbGrad, r, b.status);
        gh.rows_live = r.count;
        gh.m_first = int(p0 / gp::TM);
        gh.splits = lay.splits;
        gh.fit = fit;
        e = gp::launch_shape<false, true>(shape, mz_k, mw_mn, mz_k, mw_mn, mo, gh, gp::EpiAcc{v0 > 0 ? 1 : 0}, gp::NoExt{},
                                          b.s);
        if (e != cudaSuccess) return e;
      }
      if (dW) {
        CUtensorMap mz_mn, mh_mn, mo;
        if (!gp::map_mnmajor(&mz_mn, dz, lay.vc, lay.piece, lay.vc) || !gp::map_mnmajor(&mh_mn, r.H, d, np, d) ||
            !gp::map_out_bf16(&mo, dW + v0 * d, d, vn, d))
          return cudaErrorInvalidValue;
        gp::Geo gw = geo(vtiles, d, np / gp::BK, kSegKbGrad, r, b.status);
        if (b.low_row > 0) gw.nkb = 2 * b.low_row / gp::BK;  // both parts of dZ, against H twice
        else gw.k_live = r.count;
        e = gp::launch_either<true, true>(mz_mn, mh_mn, mz_mn, mh_mn, mo, gw, gp::EpiScaled{b.scale}, gp::NoExt{}, b.s);
        if (e != cudaSuccess) return e;
      }
    }
    if (dH) {
      const int64_t blocks = rows * (d / 8) / 256 + 1;
      const int64_t most = 8 * int64_t(sm_count());
      e = b.low_row > 0
              ? gp::launch_early(k_head_dh_few, dim3(unsigned((N * (d / 8) + 31) / 32)), dim3(256), 0, b.s,
                                 static_cast<const float*>(part), lay.splits, d, r, b.scale, b.low_row, dH, lddh)
              : gp::launch_early(k_head_dh, dim3(unsigned(blocks < most ? blocks : most)), dim3(256), 0, b.s,
                                 static_cast<const float*>(part), rows, lay.splits, fit, d, r, p0, b.scale, dH, lddh);
      if (e != cudaSuccess) return e;
    }
  }
  return cudaSuccess;
}

// backward_pieces() of a dZ whose entries at the rows' words `y` are minus the sum of the others (k_head_target), times
// `factor`.  tiles(p0, rows, v0, vn, width, others) leaves the other entries in the workspace and the sums of tiles of
// width(vn) columns in `others`.
template <class Width, class Tiles>
cudaError_t backward_with_target(const Backward& b, float factor, const Width& width_of, const Tiles& tiles) {
  const BwdWs& lay = b.lay;
  float* others = reinterpret_cast<float*>(b.ws + lay.others);
  float* sum = reinterpret_cast<float*>(b.ws + lay.sum);
  const int64_t V = b.V;
  // dZ of the vocabulary columns v0 .. v0 + vn.  all: they are all there are, so the sum of the others that
  // the target's entry takes is whole; done: earlier calls have made it; neither: this call adds to it
  auto make_dz = [&](int64_t p0, int64_t rows, int64_t v0, int64_t vn, bool all, bool done) {
    const int width = width_of(vn);
    const cudaError_t e = tiles(p0, rows, v0, vn, width, others);
    if (e != cudaSuccess) return e;
    const int nparts = done ? 0 : int(2 * ((vn + width - 1) / width));
    return gp::launch_early(k_head_target, dim3(unsigned(rows / 32)), dim3(32, nparts >= 128 ? 32 : 8), 0, b.s, others,
                            lay.piece, nparts, b.r, p0, sum, int(done || v0 > 0), int(!all && !done), int(all || done), v0,
                            vn, factor, b.low_row, reinterpret_cast<__nv_bfloat16*>(b.ws + lay.dz), lay.vc);
  };
  const bool whole = V <= lay.vc;
  return backward_pieces(
      b,
      [&](int64_t p0, int64_t rows) {
        for (int64_t v0 = 0; v0 < V && !whole; v0 += lay.vc) {
          const cudaError_t e = make_dz(p0, rows, v0, V - v0 < lay.vc ? V - v0 : lay.vc, false, false);
          if (e != cudaSuccess) return e;
        }
        return cudaSuccess;
      },
      [&](int64_t p0, int64_t rows, int64_t v0, int64_t vn) { return make_dz(p0, rows, v0, vn, whole, !whole); });
}

}  // namespace

size_t head_loss_workspace_bytes(int64_t N, int64_t V, int64_t d, int C) { return fwd_ws(N, V, d, C).total; }
size_t head_loss_backward_workspace_bytes(int64_t N, int64_t V, int64_t d, bool dh, bool dw) {
  return bwd_ws(N, V, d, dh, dw, false).total;
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
  float2* part = reinterpret_cast<float2*>(ws + lay.part);
  float* zy = reinterpret_cast<float*>(ws + lay.zy);
  float* zc = reinterpret_cast<float*>(ws + lay.zc);
  for (int64_t p0 = 0; p0 < np; p0 += lay.piece) {
    const int64_t rows = np - p0 < lay.piece ? np - p0 : lay.piece;
    const int width = fwd_width(N, V);
    e = forward_tiles(r, N, p0, rows, d, W, V, EpiStats{part, lay.piece, r.y + p0, zy, cols, E ? C : 0, zc}, status, width,
                      s);
    if (e != cudaSuccess) return e;
    const int nparts = int(2 * ((V + width - 1) / width));
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
  const BwdWs lay = bwd_ws(N, V, d, dH != nullptr, dW != nullptr, false);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const Rows r = rows_at(workspace, lay.rows);
  cudaError_t e = launch_rows(H, ldh, N, d, V, y, w, dloss, lse, r, nullptr, nullptr, nullptr, 0, dH, lddh, s);
  if (e != cudaSuccess) return e;
  const Backward b{lay, r, ws, N, d, static_cast<const __nv_bfloat16*>(W), V, scale, static_cast<__nv_bfloat16*>(dH), lddh,
                   static_cast<__nv_bfloat16*>(dW), status, s};
  return backward_with_target(
      b, 1.f, [&](int64_t cols) { return back_width(N, cols); },
      [&](int64_t p0, int64_t rows, int64_t v0, int64_t vn, int width, float* others) {
        return logit_tiles(b, p0, rows, v0, vn,
                           EpiDz{r.lse + p0, r.w + p0, r.y + p0, r.count, p0, v0, int(vn), others, lay.piece}, width);
      });
}

// ------------------------------------------------------------------ distillation
namespace {

struct WordsWs {
  int width, piece, of_piece, pitch;
  size_t at, q, ent, main, table, total;
};
WordsWs words_ws(int64_t N, int64_t V, int K, int width, int64_t piece, size_t from) {
  WordsWs o{};
  o.width = width;
  o.piece = int(piece);
  o.of_piece = int(2 * ((piece + width - 1) / width));
  o.pitch = int(round_up((V + piece - 1) / piece * o.of_piece, 8));
  o.at = from; from += align256(4 * size_t(N) * size_t(K));
  o.q = from; from += align256(4 * size_t(N) * size_t(K));
  o.ent = from; from += align256(4 * size_t(N));
  o.main = from; from += align256(4 * size_t(N));
  o.table = from; from += align256(2 * size_t(N) * size_t(o.pitch));
  o.total = from;
  return o;
}
struct DistillWs {
  FwdWs fwd;
  WordsWs words;
  size_t zk, total;
};
DistillWs distill_ws(int64_t N, int64_t V, int64_t d, int K) {
  DistillWs o{};
  o.fwd = fwd_ws(N, V, d, 0);
  o.words = words_ws(N, V, K, fwd_width(N, V), V, o.fwd.total);
  o.zk = o.words.total;
  o.total = o.zk + align256(4 * size_t(o.fwd.piece) * size_t(K));
  return o;
}

cudaError_t launch_teacher(const int32_t* idx, const float* t, int64_t N, int64_t V, int K, float tau, uint8_t* ws,
                           const WordsWs& lay, Words* out, cudaStream_t s) {
  *out = Words{reinterpret_cast<int32_t*>(ws + lay.at), reinterpret_cast<float*>(ws + lay.q),
               reinterpret_cast<float*>(ws + lay.ent), reinterpret_cast<int32_t*>(ws + lay.main),
               reinterpret_cast<uint16_t*>(ws + lay.table), K, lay.pitch, lay.width, lay.piece, lay.of_piece};
  int padded = 32;
  while (padded < K) padded *= 2;
  const cudaError_t e = gp::keep_carveout(k_teacher);
  if (e != cudaSuccess) return e;
  return gp::launch_early(k_teacher, dim3(unsigned((N + kTeacherWarps - 1) / kTeacherWarps)), dim3(32 * kTeacherWarps),
                          size_t(kTeacherWarps) * 8 * size_t(padded), s, idx, t, N, V, 1.f / tau, padded, *out);
}

WordsWs back_words(int64_t N, int64_t V, int K, const BwdWs& lay) {
  const int64_t piece = V < lay.vc ? V : lay.vc;
  return words_ws(N, V, K, back_width(N, piece), piece, lay.total);
}

}  // namespace

int head_distill_max_words() { return kMostWords; }
size_t head_distill_workspace_bytes(int64_t N, int64_t V, int64_t d, int K) { return distill_ws(N, V, d, K).total; }
size_t head_distill_backward_workspace_bytes(int64_t N, int64_t V, int64_t d, int K, bool dh, bool dw) {
  return back_words(N, V, K, bwd_ws(N, V, d, dh, dw, true)).total;
}

cudaError_t launch_head_distill(const void* H, int64_t ldh, int64_t N, int64_t d, const void* W, int64_t V,
                                const int32_t* idx, const float* t, int K, float tau, const float* w, float* loss,
                                float* lse, void* workspace, int32_t* status, cudaStream_t s) {
  const DistillWs lay = distill_ws(N, V, d, K);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  Words words;
  cudaError_t e = launch_teacher(idx, t, N, V, K, tau, ws, lay.words, &words, s);
  if (e != cudaSuccess) return e;
  const Rows r = rows_at(workspace, lay.fwd.rows);
  float2* part = reinterpret_cast<float2*>(ws + lay.fwd.part);
  float* zk = reinterpret_cast<float*>(ws + lay.zk);
  if (N <= gp::HALF) {
    // Few rows cost the same with the masked ones among them (a row's sums are its own): nothing is gathered, and
    // the product reads hidden states and head while k_teacher runs.  37 tokens at 2048 x 49152: 56.5 us with
    // the gathering, 51 without.
    const int width = lay.words.width, arows = int(round_up(N, 8));
    CUtensorMap ma, mb;
    if (!gp::map_2d(&mb, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, W, d, V, d, gp::BK, width / 2) ||
        !gp::map_2d(&ma, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, H, d, N, ldh, gp::BK, arows))
      return cudaErrorInvalidValue;
    gp::Geo g = geo(1, V, (d + gp::BK - 1) / gp::BK, kSegKbFew, r, status);
    g.width = width;
    g.arows = arows;
    g.mark = gp::call_mark();
    e = gp::launch<gp::kSingle, false, false>(
        ma, mb, ma, mb, ma, g, EpiTeacher{part, lay.fwd.piece, nullptr, int(N), words, zk, kLog2e / tau}, gp::CallersA{}, s);
    if (e != cudaSuccess) return e;
    return gp::launch_early(k_teacher_join_few, dim3(unsigned(N)), dim3(kJoinThreads), 0, s,
                            static_cast<const float2*>(part), lay.fwd.piece, lay.words.of_piece, static_cast<const float*>(zk),
                            words, w, tau, 1.f / tau, loss, lse);
  }
  e = launch_rows(H, ldh, N, d, V + 1, words.main, w, nullptr, nullptr, r, loss, lse, nullptr, 0, nullptr, 0, s);
  if (e != cudaSuccess) return e;
  const int64_t np = round_up(N, gp::TM);
  for (int64_t p0 = 0; p0 < np; p0 += lay.fwd.piece) {
    const int64_t rows = np - p0 < lay.fwd.piece ? np - p0 : lay.fwd.piece;
    e = forward_tiles(r, N, p0, rows, d, W, V, EpiTeacher{part, lay.fwd.piece, r.idx + p0, 0, words, zk, kLog2e / tau}, status,
                      lay.words.width, s);
    if (e != cudaSuccess) return e;
    const int nparts = lay.words.of_piece;
    e = gp::launch_early(k_teacher_join, dim3(unsigned(rows / 32)), dim3(32, nparts >= 128 ? 32 : 8), 0, s, part,
                         lay.fwd.piece, nparts, r, p0, zk, words, tau, 1.f / tau, loss, lse);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_head_distill_backward(const void* H, int64_t ldh, int64_t N, int64_t d, const void* W, int64_t V,
                                         const int32_t* idx, const float* t, int K, float tau, const float* w,
                                         const float* lse, const float* dloss, float scale, void* dH, int64_t lddh,
                                         void* dW, void* workspace, int32_t* status, cudaStream_t s) {
  const BwdWs lay = bwd_ws(N, V, d, dH != nullptr, dW != nullptr, true);
  const WordsWs wlay = back_words(N, V, K, lay);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  Words words;
  cudaError_t e = launch_teacher(idx, t, N, V, K, tau, ws, wlay, &words, s);
  if (e != cudaSuccess) return e;
  const Rows r = rows_at(workspace, lay.rows);
  const int low_row = N <= gp::HALF / 2 ? gp::HALF / 2 : 0;
  e = launch_rows(H, ldh, N, d, V + 1, words.main, w, dloss, lse, r, nullptr, nullptr, nullptr, 0, dH, lddh, s, low_row);
  if (e != cudaSuccess) return e;
  const Backward b{lay, r, ws, N, d, static_cast<const __nv_bfloat16*>(W), V, scale, static_cast<__nv_bfloat16*>(dH), lddh,
                   static_cast<__nv_bfloat16*>(dW), status, s, low_row};
  return backward_with_target(
      b, tau, [&](int64_t) { return wlay.width; },
      [&](int64_t p0, int64_t rows, int64_t v0, int64_t vn, int width, float* others) {
        return logit_tiles(b, p0, rows, v0, vn,
                           EpiDzTeacher{r.lse + p0, r.w + p0, r.y + p0, r.idx + p0, words, tau, 1.f / tau, r.count, p0, v0,
                                        int(vn), int(v0 / wlay.piece) * wlay.of_piece, others, lay.piece, b.low_row,
                                        reinterpret_cast<__nv_bfloat16*>(ws + lay.dz), lay.vc},
                           width);
      });
}

}  // namespace loca
