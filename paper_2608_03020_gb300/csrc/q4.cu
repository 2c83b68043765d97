// A frozen projection in 4 bits with group scales, for a few tokens, with each token's adapter beside it.
//   W[o, k] = s[o, k / group] (q[o, k] - z[o, k / group]),   Y = X W^T + s_a (X A_a) B_a^T
//
// Exact products.  q - z is an integer of at most 15, exact in bf16, as X is: the tensor cores sum x (q - z) over the
// k of one group in fp32, and the sum is scaled by s and added in fp32.  So W is never rounded.
//
// Up to 16 tokens m16n8k16 MMAs with W's rows as M and the tokens as N (mma.sync: a code becomes an operand in
// registers, one shift and mask and one subtraction for two of them; tcgen05 wants the 16-bit operand written to
// shared memory first, four bytes for each byte read); for more tokens tcgen05, which reads that operand once
// for all of them.
//
//   k_q4_pack   codes in the order of the MMAs' fragments: 512 bytes are 16 rows x 64 k, of which each lane's 16
//               are what it multiplies; the order of k within 64 is chosen so that a lane's part of X is two runs
//               of 16 bytes and that 32 k of one group stay together.  Rows and k are padded to 32 and 128
//   k_q4        a warp takes 16 rows and a range of k in spans of 128, three of which are on the way to its part of
//               shared memory (each lane copies and reads its own 16 bytes, so that it waits for nothing else);
//               ks warps' sums meet in shared memory, in order, with the low-rank term of each token's adapter
//               (U in fp32 from k_adapter_tokens); one rounding
//   k_q4_tiles  more than 16 tokens: see there
// Bound of k_q4, next to the read of the codes and scales: with one token, or groups of 32, the instructions that make
// operands of codes (44 of some 80 for 64 k of 16 rows; 65 and 73 % of the issue slots); with more tokens nothing alone (8 at
// 20480 x 5120: 52 % of the issue slots, 58 % of L1's data path, which a warp's X takes 2 KB a span for 1 KB of codes; two
// fifths of the warps wait for loads).  One token at 28672 x 8192 25.6 us (4.7 TB/s), 3 tokens at 151931 x 2048 with groups
// of 32 45.5 us (4.4 TB/s), 8 at 20480 x 5120 with groups of 64 18.7 us (3.0 TB/s), with adapters of rank 32 23.7; 16
// tokens at 14336 x 3584 14.4 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "gemm_pair.cuh"

namespace loca {
namespace {

using namespace tc;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxSmem = 98304;
constexpr int kTokensByWarps = 16;  // (above: 20 tokens with adapters of rank 16 at 3584 x 3584 14.4 us by warps, 10.8 in tiles)

__host__ __device__ inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of 16 rows (an even number of them) x chunks of 64 k.
struct PackLay {
  int64_t tiles, chunks, groups;
  size_t scales, zeros, total;
};
__host__ __device__ inline size_t up256(size_t n) { return (n + 255) & ~size_t(255); }
PackLay pack_lay(int64_t o, int64_t d, int group, int dtype, bool zeros) {
  PackLay p{};
  p.tiles = div_up(o, 32) * 2;
  p.chunks = div_up(d, 128) * 2;
  p.groups = p.chunks * 64 / group;  // (those behind the last have scales of 0)
  p.scales = up256(size_t(p.tiles) * size_t(p.chunks) * 512);
  p.zeros = p.scales + up256(size_t(p.tiles) * size_t(p.groups) * 16 * (dtype == LOCA_F32 ? 4 : 2));
  p.total = p.zeros + (zeros ? up256(size_t(p.tiles) * size_t(p.groups) * 8) : 0);
  return p;
}

// Position of k within its 64: step of 16, lane of the quad, place among the lane's four of the step.
// The lane's places 0, 1 are the fragment's first register pair, 2, 3 its second.
__device__ __forceinline__ int k_of(int step, int t, int place) { return 32 * (step >> 1) + 8 * t + 4 * (step & 1) + place; }

// One thread per 16 bytes of the packed codes; then the scales and zeros, in pairs of rows g and g + 8.
__global__ void __launch_bounds__(256)
    k_q4_pack(const uint8_t* __restrict__ codes, const void* __restrict__ scales, int f32, const uint8_t* __restrict__ zeros,
              int64_t o, int64_t d, PackLay p, int group, uint8_t* __restrict__ packed) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x, first = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  for (int64_t i = first; i < p.tiles * p.chunks * 32; i += stride) {
    const int lane = int(i & 31);
    const int64_t chunk = (i >> 5) % p.chunks, tile = (i >> 5) / p.chunks;
    const int g = lane >> 2, t = lane & 3;
    uint32_t w[4] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // row g, row g + 8
        const int64_t row = tile * 16 + g + 8 * h;
        const int64_t k = chunk * 64 + k_of(j, t, 0);
        uint32_t four = 0;
        if (row < o && k < d && LOCA_CHECK(row * (d / 2) + k / 2 + 1, o * (d / 2)))
          four = uint32_t(codes[row * (d / 2) + k / 2]) | uint32_t(codes[row * (d / 2) + k / 2 + 1]) << 8;
        // nibbles n and n + 4 of a word become the two halves of a register: (row, first or second pair)
        w[j] |= (four & 15) << (4 * h) | (four >> 4 & 15) << (16 + 4 * h) | (four >> 8 & 15) << (8 + 4 * h) |
                (four >> 12 & 15) << (24 + 4 * h);
      }
    *reinterpret_cast<uint4*>(packed + i * 16) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  for (int64_t i = first; i < p.tiles * p.groups * 8; i += stride) {
    const int g = int(i & 7);
    const int64_t q = (i >> 3) % p.groups, tile = (i >> 3) / p.groups;
    uint32_t both = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t row = tile * 16 + g + 8 * h;
      const int64_t at = row * (d / group) + q;
      const bool in = row < o && q < d / group;
      if (f32)
        reinterpret_cast<float*>(packed + p.scales)[2 * i + h] = in ? static_cast<const float*>(scales)[at] : 0.f;
      else
        reinterpret_cast<uint16_t*>(packed + p.scales)[2 * i + h] = in ? static_cast<const uint16_t*>(scales)[at] : uint16_t(0);
      if (zeros && in) both |= uint32_t(zeros[at] & 15) << (4 * h);
    }
    if (zeros) packed[p.zeros + i] = uint8_t(both);
  }
}

struct Q4Geo {
  const uint4* codes;
  const uint8_t* scales;
  const uint8_t* zeros;  // or null: 8
  int f32;
  int64_t o, d;
  int64_t tiles;
  int spans, groups;
  int ks, per_warp;      // warps that share rows, their spans
  const __nv_bfloat16* X;
  int64_t ldx, N;
  AdapterTokens low;     // U null: none
  __nv_bfloat16* Y;
  int64_t ldy;
};

__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two codes (bits s .. s + 3 of both halves of w) less their row's zero, by the published way of turning small integers into
// floating point through the bit pattern: 128 + q has q in the last bits of its bf16 pattern 0x4300 | q, and so has
// 128 + z; their difference is exact.
template <int kShift>
__device__ __forceinline__ uint32_t two_codes(uint32_t w, __nv_bfloat162 zero) {
  uint32_t q;  // (codes & mask) | pattern in one instruction (one token at 28672 x 8192 31 us in two, 25.8 in one)
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(q) : "r"(w >> kShift), "n"(0x000f000f), "r"(0x43004300u));
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&q), zero);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Blocks of a SM (registers decide).
constexpr int resident(int nt) { return nt == 1 ? 3 : 2; }
constexpr int kMetaBytes = 32 * 8 + 32;  // of four groups: 32 pairs of scales, 32 bytes of zeros
// A warp's shared memory: four spans of 128 k on the way, the scales and zeros of two rounds of four spans.
__host__ __device__ constexpr int warp_bytes(int groups) { return 4 * 1024 + 2 * groups * kMetaBytes; }

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

// U[n, r], the sum over the ranges of k in order, eight of them on the way at a time.
__device__ __forceinline__ float low_sum(const Q4Geo& g, int64_t n, int r) {
  const float* u = g.low.U + n * g.low.kp + r;
  const int64_t pitch = g.N * g.low.kp;
  float sum = 0.f;
  for (int c = 0; c < g.low.ranges; c += 8) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = c + i < g.low.ranges ? u[(c + i) * pitch] : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += x[i];
  }
  return sum;
}

// kGroups: of 128 k (1, 2 or 4).
template <int NT, int kGroups>
__global__ void __launch_bounds__(kThreads, resident(NT)) k_q4(const __grid_constant__ Q4Geo g) {
  extern __shared__ float smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int gr = lane >> 2, t = lane & 3;
  const int per_block = kWarps / g.ks;  // tiles of a block
  const int kw = warp % g.ks;
  const int64_t tile = int64_t(blockIdx.x) * per_block + warp / g.ks;
  constexpr int R = 16, T = 8 * NT;
  // With adapters the launch before is k_adapter_tokens, which let this one start only after all launches before
  // it had completed: what it writes is needed at the end.
  if (!g.low.U) wait_for_previous();
  launch_dependents();
  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
  const int tokens = int(g.N);  // (8 NT at most)
  const int rows = per_block * R;
  const int64_t row0 = int64_t(blockIdx.x) * rows;
  // the adapters' rows that this thread multiplies at the end, to L2 meanwhile
  auto prefetch_rows = [&]() {
    for (int i = threadIdx.x; i < rows * tokens; i += kThreads) {
      const int n = i / rows, r = i - n * rows;
      const int a = g.low.tok_adapter[n];
      if (a >= 0 && row0 + r < g.o)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(g.low.B + (int64_t(a) * g.o + row0 + r) * g.low.kp));
    }
  };
  const int c0 = kw * g.per_warp, c1 = c0 + g.per_warp < g.spans ? c0 + g.per_warp : g.spans;
  if (tile < g.tiles && c0 < c1) {
    uint8_t* mine = reinterpret_cast<uint8_t*>(smem) + warp * warp_bytes(kGroups);
    const uint8_t* slots = mine + lane * 16;  // span i of a round: at 1024 i, in two halves
    const uint32_t slots_s = smem_u32(slots), metas_s = smem_u32(mine) + 4096;
    const uint8_t* metas = mine + 4096;
    const uint4* codes = g.codes + (tile * g.spans + c0) * 64 + lane;
    // scales and zeros of the four spans from c on, into half `to` of theirs
    const int meta_end = g.groups * 8;  // pairs of rows and groups of a tile
    auto fetch_meta = [&](int c, uint32_t to) {
      if (c >= c1) return;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const int e = (c * kGroups + 4 * i) * 8;
        const int64_t at = tile * meta_end + e;
        const uint32_t dst = metas_s + to + uint32_t(i * kMetaBytes);
        if (e + lane < meta_end && LOCA_CHECK(at + lane, g.tiles * meta_end)) {
          if (g.f32) copy8(dst + lane * 8, g.scales + (at + lane) * 8);
          else copy4(dst + lane * 8, g.scales + (at + lane) * 4);
        }
        if (g.zeros && lane < 8 && e + 4 * lane < meta_end) copy4(dst + 256 + lane * 4, g.zeros + at + 4 * lane);
      }
    };
    // span i of this round (i >= 4: of the next) where it is there
    auto fetch = [&](int i, int left) {
      if (i < left && LOCA_CHECK(codes + i * 64 - g.codes, g.tiles * g.spans * 64)) {
        copy16(slots_s + uint32_t((i & 3) * 1024), codes + i * 64);
        copy16(slots_s + uint32_t((i & 3) * 1024 + 512), codes + i * 64 + 32);
      }
      copy_commit();
    };
    fetch_meta(c0, 0);
#pragma unroll
    for (int i = 0; i < 3; ++i) fetch(i, c1 - c0);
    if (g.low.U) prefetch_rows();
    // (columns of tokens that are not there hold the last token's and are not stored)
    const __nv_bfloat16* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int tok = 8 * n + gr < tokens ? 8 * n + gr : tokens - 1;
      x[n] = g.X + int64_t(tok) * g.ldx + 128 * c0 + 8 * t;
    }
    uint32_t half = 0;
    for (int left = c1 - c0, k_left = int(g.d) - 128 * c0; left > 0; left -= 4, k_left -= 512) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= left) break;
        copy_wait<2>();
        if (i == 0) {
          __syncwarp();  // the round's scales and zeros are everyone's, and those of the last round have been read
          fetch_meta(c1 - left + 4, half ^ uint32_t(kGroups * kMetaBytes));
        }
        const uint4 w[2] = {*reinterpret_cast<const uint4*>(slots + i * 1024),
                            *reinterpret_cast<const uint4*>(slots + i * 1024 + 512)};
        fetch(i + 3, left);
        uint4 xv[4][NT];
        const bool full = 128 * (i + 1) <= k_left;  // (else the last span of rows that are no multiple of 128)
        auto load_x = [&](int q) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
            xv[q][n] = (full || 128 * i + 32 * q < k_left) && LOCA_CHECK_SPAN(x[n] + 128 * i + 32 * q - g.X, 8, (g.N - 1) * g.ldx + g.d)
                           ? __ldg(reinterpret_cast<const uint4*>(x[n] + 128 * i) + 4 * q)
                           : make_uint4(0, 0, 0, 0);
        };
        // (twice the same: without a condition at each load 18.7 us where one loop for both took 19.1, 8 tokens at 20480 x
        // 5120, and 41.6 us for 43.1, one at 151931 x 2048)
        if (full) {
#pragma unroll
          for (int q = 0; q < 4; ++q) load_x(q);
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) load_x(q);
        }
        float part[NT][4];
        float s0 = 0.f, s1 = 0.f;
        __nv_bfloat162 zero0, zero1;
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // 32 k
          if (q % (4 / kGroups) == 0) {
            const int group = i * kGroups + q * kGroups / 4;  // of the round
            const uint8_t* meta = metas + half + (group >> 2) * kMetaBytes;
            const int e = (group & 3) * 8 + gr;
            if (g.f32) {
              const float2 s = *reinterpret_cast<const float2*>(meta + e * 8);
              s0 = s.x;
              s1 = s.y;
            } else {
              const uint32_t s = *reinterpret_cast<const uint32_t*>(meta + e * 8);
              s0 = __uint_as_float(s << 16);
              s1 = __uint_as_float(s & 0xffff0000u);
            }
            uint32_t z0 = 0x43084308u, z1 = 0x43084308u;
            if (g.zeros) {
              const uint32_t z = meta[256 + e];
              z0 = (z & 15u) * 0x10001u + 0x43004300u;
              z1 = (z >> 4) * 0x10001u + 0x43004300u;
            }
            zero0 = *reinterpret_cast<const __nv_bfloat162*>(&z0);
            zero1 = *reinterpret_cast<const __nv_bfloat162*>(&z1);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int f = 0; f < 4; ++f) part[n][f] = 0.f;
          }
#pragma unroll
          for (int s = 0; s < 2; ++s) {  // 16 k
            const uint32_t word = reinterpret_cast<const uint32_t*>(&w[q >> 1])[2 * (q & 1) + s];
            const uint32_t a[4] = {two_codes<0>(word, zero0), two_codes<4>(word, zero1), two_codes<8>(word, zero0),
                                   two_codes<12>(word, zero1)};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint32_t* b = reinterpret_cast<const uint32_t*>(&xv[q][n]) + 2 * s;
              mma_16816(part[n], a, b[0], b[1]);
            }
          }
          if ((q + 1) % (4 / kGroups) == 0) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              acc[n][0] = fmaf(s0, part[n][0], acc[n][0]);
              acc[n][1] = fmaf(s0, part[n][1], acc[n][1]);
              acc[n][2] = fmaf(s1, part[n][2], acc[n][2]);
              acc[n][3] = fmaf(s1, part[n][3], acc[n][3]);
            }
          }
        }
      }
      codes += 256;
      half ^= uint32_t(kGroups * kMetaBytes);
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n] += 512;
    }
    copy_wait<0>();
  }
  __syncthreads();  // the sums take the rings' place
  if (g.low.U) wait_for_previous();
  // sums of the warps: [warp][token][row]
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) smem[(warp * T + 8 * n + 2 * t + (i & 1)) * R + gr + 8 * (i >> 1)] = acc[n][i];
  float* u = smem + kWarps * T * R;
  if (g.low.U)
    for (int i = threadIdx.x; i < tokens * g.low.kp; i += kThreads) {
      const int n = i / g.low.kp, r = i - n * g.low.kp;
      u[i] = g.low.tok_adapter[n] >= 0 && LOCA_CHECK(n, g.N) ? low_sum(g, n, r) : 0.f;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * tokens; i += kThreads) {
    const int n = i / rows, r = i - n * rows;
    const int64_t row = row0 + r;
    if (row >= g.o) continue;
    const float* at = smem + (int64_t(r / R) * g.ks * T + n) * R + r % R;
    float y = 0.f;
    for (int q = 0; q < g.ks; ++q) y += at[q * T * R];
    if (g.low.U) {
      const int a = g.low.tok_adapter[n];
      if (a >= 0) {
        const uint4* b = reinterpret_cast<const uint4*>(g.low.B + (int64_t(a) * g.o + row) * g.low.kp);
        float s = 0.f;
        for (int c = 0; c < g.low.kp / 8; ++c) {
          const uint4 v = __ldg(b + c);
          const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 f = __bfloat1622float2(h[k]);
            s = fmaf(u[n * g.low.kp + 8 * c + 2 * k], f.x, s);
            s = fmaf(u[n * g.low.kp + 8 * c + 2 * k + 1], f.y, s);
          }
        }
        y += s;
      }
    }
    if (LOCA_CHECK(n * g.ldy + row, (g.N - 1) * g.ldy + g.o)) g.Y[n * g.ldy + row] = __float2bfloat16_rn(y);
  }
}

// Warps on the same rows: more of them shorten a warp's way through k, and add a block's start and end (about 2 us, and
// 0.4 for each that shares the SM) for each of its fewer spans.  A span takes a lone block's warps 0.62 us; eight warps'
// worth of a span keeps an SM busy for 0.44, whatever shares the SM.  20480 x 5120, 8 tokens: 28.6 us with one warp, 21.0 with
// two, 20.0 with four, 20.2 with eight; 3584 x 3584, one token: 7.2, 4.7 and 3.9 with two, four and eight.
template <int NT>
void share_rows(Q4Geo& g) {
  auto round = [](int64_t blocks, int64_t spans) {
    const double each = blocks * 0.44;
    return blocks > 0 ? double(spans) * (each > 0.62 ? each : 0.62) + 2.0 + 0.4 * blocks : 0.0;
  };
  double best = 0;
  for (int ks = 1; ks <= kWarps; ks *= 2) {
    const int64_t per = div_up(g.spans, ks), blocks = div_up(div_up(g.tiles, kWarps / ks), sm_count());
    const double c = double(blocks / resident(NT)) * round(resident(NT), per) + round(blocks % resident(NT), per);
    if (ks == 1 || c < best) {
      best = c;
      g.ks = ks;
      g.per_warp = int(per);
    }
  }
}

template <int NT, int kGroups>
cudaError_t launch_one(Q4Geo g, cudaStream_t s) {
  share_rows<NT>(g);
  const int sums = 4 * (kWarps * 8 * NT * 16 + (g.low.U ? 8 * NT * g.low.kp : 0)), rings = kWarps * warp_bytes(kGroups);
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = gp::allow_smem(allowed, reinterpret_cast<const void*>(k_q4<NT, kGroups>), kMaxSmem);
  if (e != cudaSuccess) return e;
  return gp::launch_early(k_q4<NT, kGroups>, dim3(unsigned(div_up(g.tiles, kWarps / g.ks))), dim3(kThreads),
                          size_t(sums > rings ? sums : rings), s, g);
}

template <int kGroups>
cudaError_t launch_tokens(const Q4Geo& g, cudaStream_t s) {
  return g.N <= 8 ? launch_one<1, kGroups>(g, s) : launch_one<2, kGroups>(g, s);
}

// ------------------------------------------------------------------ more tokens
// The same product on tcgen05, D[row, token] with 128 rows of W as M and 32, 64 or 128 tokens as N.  A group's products
// go to an accumulator of their own in tensor memory; four lanes' warps read it, a row per lane, and add it
// times the row's scale to the row's sums: W is not rounded here either.
//   warp 0        TMA producer: X, a span (128 k) of the tile's tokens a stage
//   warp 1        one thread issues the MMAs, eight a span, and one commit
//   warps 2..9    codes into bf16 integers in the stage's operand (K-major, 128-byte swizzle), 32 rows of every other span
//   warps 10..17  a row per lane, half of the tokens each: sums of the groups
// The k axis is split over a cluster of up to 8 CTAs, which add their sums through distributed shared memory, in rank
// order.  Bound: the way from warp to warp.  A span takes 0.45 us, 0.35 with neither codes unpacked nor products
// read, so everything that waits or signals does so once a span (64 k a stage, a barrier for each accumulator and a
// commit for each ring: 0.8 us), and a warp unpacks 32 rows of a span at a wait rather than 16 (64 tokens at 14336 x
// 3584: 31.7 us so, 23.5 with whole spans, 21.8 with 32 rows).  Times at 14336 x 3584: 32 tokens 20.7 us (k_q4, built for
// as many: 25.3), 64 21.8 (42.2), 128 26.9, 512 with groups of 64 139; 64 at 151931 x 2048 118 (246); 24 at 20480 x 5120
// with groups of 64 50.0 (48.7: 160 tiles are two rounds of the SMs).
// A token's adapter is multiplied at the end, a row a lane: 25 tokens of rank 24 at 55544 x 6016 125 us, 99 without
// (their rows brought to L2 meanwhile, as k_q4 does, took 2 us more; all of a row's loads at once 8).
// Every wait is bounded; the failure path is that of the adapters' kernels.
constexpr int kTileThreads = 576;
constexpr int kDequantWarps = 8, kSumWarps = 8;
constexpr int kBoxW = 128 * 128;  // bytes of 128 rows x 64 k
constexpr int kTileSmem = 232448;
// On the way from memory: eight spans of codes and zeros for each warp that unpacks them, the scales of eight groups or
// more for each warp that sums.
constexpr int kRaw = 8;
// NT tokens and kGroups groups of a span.
template <int NT, int kGroups>
struct Tiling {
  static constexpr int kStages = NT <= 64 && NT * kGroups <= 128 ? 3 : 2;
  static constexpr int kBoxX = NT * 128, kStage = 2 * (kBoxW + kBoxX);
  static constexpr int kRawSlot = 1024 + (kGroups <= 2 ? 16 : 32), kScales = kGroups <= 2 ? 8 : 16;
  static constexpr int kAside = kDequantWarps * kRaw * kRawSlot + kSumWarps * kScales * 128;
  static constexpr int kSmem = kStages * kStage + kAside + 1024 + 256;
  static constexpr int kCols = NT * kGroups;  // of tensor memory, in a stage
  static_assert(kSmem <= kTileSmem && kStages * kCols <= 512, "shared and tensor memory");
};

struct TileGeo {
  Q4Geo q;
  int per_cta;     // spans of a CTA
  int32_t* status;
  int32_t* abort_flag;
  unsigned long long limit_ns;
  int32_t mark;
};
// kHalf: half of the tile's tokens.
template <int kHalf, int kGroups>
__global__ void __launch_bounds__(kTileThreads, 1)
    k_q4_tiles(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ TileGeo g) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int NT = 2 * kHalf;
  using T = Tiling<NT, kGroups>;
  constexpr int kStages = T::kStages, kRawSlot = T::kRawSlot, kScales = T::kScales;
  constexpr uint32_t kAlloc = kStages * T::kCols <= 128 ? 128u : kStages * T::kCols <= 256 ? 256u : 512u;
  const Q4Geo& p = g.q;
  const int ks = int(cluster_nctarank()), rank = int(cluster_ctarank());
  uint8_t* raw = smem + kStages * T::kStage;
  uint64_t* bars = reinterpret_cast<uint64_t*>(raw + T::kAside);
  const uint32_t bar_base = smem_u32(bars), smem_base = smem_u32(smem);
  auto x_full = [&](int s) { return bar_base + 8u * s; };
  auto w_full = [&](int s) { return bar_base + 8u * (kStages + s); };
  auto done = [&](int s) { return bar_base + 8u * (2 * kStages + s); };   // operands read, products in tensor memory
  auto taken = [&](int s) { return bar_base + 8u * (3 * kStages + s); };  // products read
  constexpr int kBars = 4 * kStages + 1;
  const uint32_t drain_bar = bar_base + 8u * (kBars - 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kBars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WaitCtl wc{g.status, g.abort_flag, g.limit_ns, g.mark};
  const int64_t o0 = int64_t(cluster_id_x()) * 128;
  const int64_t n0 = int64_t(blockIdx.y) * NT;
  const int c0 = rank * g.per_cta < p.spans ? rank * g.per_cta : p.spans;
  const int c1 = c0 + g.per_cta < p.spans ? c0 + g.per_cta : p.spans;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(x_full(s), 1);
      mbar_init(w_full(s), kDequantWarps / 2);
      mbar_init(done(s), 1);
      mbar_init(taken(s), kSumWarps);
    }
    mbar_init(drain_bar, 1);
    mbar_init_fence();
    prefetch_tensormap(&tmX);
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), kAlloc);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // (with adapters the launch before is k_adapter_tokens: see k_q4)
  if (!p.low.U) wait_for_previous();
  launch_dependents();
  auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_try_wait(bar, parity) || mbar_wait(bar, parity, wc); };
  const int spans = c1 - c0;
  int stage = 0;  // every role goes around the stages, a span each
  uint32_t phase = 0, issued = 0;
  auto next = [&] {
    if (++stage == kStages) { stage = 0; phase ^= 1u; }
  };

  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < spans; ++i, next()) {
        // (the stage's products too have been read: the MMAs that follow X need not ask)
        if (!wait(done(stage), phase ^ 1u) || !wait(taken(stage), phase ^ 1u)) break;
        mbar_arrive_expect_tx(x_full(stage), uint32_t(2 * T::kBoxX));
        const uint32_t st = smem_base + uint32_t(stage * T::kStage + 2 * kBoxW);
        tma_load_2d(st, &tmX, x_full(stage), 128 * (c0 + i), int(n0));
        tma_load_2d(st + T::kBoxX, &tmX, x_full(stage), 128 * (c0 + i) + 64, int(n0));
        ++issued;
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t id = tc::idesc(1, 1, 0, 0, 128, uint32_t(NT));
      bool mma = false;
      for (int i = 0; i < spans; ++i, next()) {
        if (!wait(w_full(stage), phase) || !wait(x_full(stage), phase)) break;
        fence_after();
        const uint32_t st = smem_base + uint32_t(stage * T::kStage);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          constexpr int kSteps = 8 / kGroups;  // of 16 k in a group
          const uint64_t a = sdesc(st + uint32_t(kk / 4 * kBoxW), 16u, 1024u, kSwizzle128B) + kk % 4 * 2;
          const uint64_t b = sdesc(st + uint32_t(2 * kBoxW + kk / 4 * T::kBoxX), 16u, 1024u, kSwizzle128B) + kk % 4 * 2;
          mma_f16(tmem_base + uint32_t(stage * T::kCols + kk / kSteps * NT), a, b, id, kk % kSteps != 0 ? 1u : 0u);
        }
        mma_commit(done(stage));
        mma = true;
      }
      if (mma) {
        mma_commit(drain_bar);
        mbar_drain(drain_bar, 0, kDrainLimitNs);
      }
    }
    __syncwarp();
  } else if (warp < 2 + kDequantWarps) {
    // ---------------- codes: 32 rows of every other span; lane (r, t) has rows r and r + 8 of 16, k 8 t .. 8 t + 7 and 32
    // more
    const int w = warp - 2, gr = lane >> 2, t = lane & 3, rows = w & 3, odd = w >> 2;
    const int64_t tile = o0 / 16 + 2 * rows;
    const bool here = tile < p.tiles;  // (of whole pairs)
    uint8_t* slots = raw + w * (kRaw * kRawSlot);
    const uint32_t slots_s = smem_u32(slots);
    const uint4* codes = p.codes + ((here ? tile : 0) * p.spans + c0) * 64 + lane;
    const int64_t next_tile = int64_t(p.spans) * 64;
    const int zt = lane / (2 * kGroups);  // whose zeros the lane copies, if below 2
    const uint8_t* zeros = p.zeros + (((here ? tile : 0) + (zt & 1)) * p.groups + int64_t(c0) * kGroups) * 8 + lane % (2 * kGroups) * 4;
    auto fetch = [&](int i) {  // span i, into one of kRaw / 2 slots
      if (here && i < spans && LOCA_CHECK(codes + next_tile + i * 64 - p.codes, p.tiles * p.spans * 64)) {
        const uint32_t dst = slots_s + uint32_t((i >> 1 & (kRaw / 2 - 1)) * 2 * kRawSlot);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          copy16(dst + x * kRawSlot + lane * 16, codes + x * next_tile + i * 64);
          copy16(dst + x * kRawSlot + lane * 16 + 512, codes + x * next_tile + i * 64 + 32);
        }
        if (p.zeros && zt < 2) copy4(dst + zt * kRawSlot + 1024 + lane % (2 * kGroups) * 4, zeros + i * kGroups * 8);
      }
      copy_commit();
    };
#pragma unroll
    for (int i = 0; i < kRaw / 2 - 1; ++i) fetch(odd + 2 * i);
    if (odd) next();
    for (int i = odd; i < spans; i += 2, next(), next()) {
      copy_wait<kRaw / 2 - 2>();
      __syncwarp();  // the span's zeros are everyone's, and the slot that comes next has been read
      const uint8_t* slot = slots + (i >> 1 & (kRaw / 2 - 1)) * 2 * kRawSlot;
      uint4 code[2][2];
      uint32_t z[2][kGroups];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        code[x][0] = *reinterpret_cast<const uint4*>(slot + x * kRawSlot + lane * 16);
        code[x][1] = *reinterpret_cast<const uint4*>(slot + x * kRawSlot + lane * 16 + 512);
#pragma unroll
        for (int q = 0; q < kGroups; ++q) z[x][q] = p.zeros ? slot[x * kRawSlot + 1024 + q * 8 + gr] : 0x88u;
      }
      fetch(i + kRaw - 2);
      if (!__all_sync(0xffffffffu, wait(done(stage), phase ^ 1u))) break;
      if (here) {
#pragma unroll
        for (int y = 0; y < 8; ++y) {  // 8 k of both rows
          const int x = y >> 2, h = y >> 1 & 1, run = y & 1;
          uint8_t* st = smem + stage * T::kStage + h * kBoxW;
          const uint32_t zz = z[x][kGroups == 1 ? 0 : kGroups == 2 ? h : 2 * h + run];
          const uint32_t z0 = (zz & 15u) * 0x10001u + 0x43004300u, z1 = (zz >> 4) * 0x10001u + 0x43004300u;
          const __nv_bfloat162 zero0 = *reinterpret_cast<const __nv_bfloat162*>(&z0);
          const __nv_bfloat162 zero1 = *reinterpret_cast<const __nv_bfloat162*>(&z1);
          const uint32_t w0 = run ? code[x][h].z : code[x][h].x, w1 = run ? code[x][h].w : code[x][h].y;
          const uint4 lo = make_uint4(two_codes<0>(w0, zero0), two_codes<8>(w0, zero0), two_codes<0>(w1, zero0),
                                      two_codes<8>(w1, zero0));
          const uint4 hi = make_uint4(two_codes<4>(w0, zero1), two_codes<12>(w0, zero1), two_codes<4>(w1, zero1),
                                      two_codes<12>(w1, zero1));
          const int row = 32 * rows + 16 * x + gr;
          *reinterpret_cast<uint4*>(st + gp::box_off(row, 4 * run + t)) = lo;
          *reinterpret_cast<uint4*>(st + gp::box_off(row + 8, 4 * run + t)) = hi;
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(w_full(stage));
    }
    copy_wait<0>();
  } else {
    // ---------------- sums of a row over the groups
    const int q = warp & 3, h = (warp - 2 - kDequantWarps) >> 2;
    const int row = q * 32 + lane;
    const int64_t tile = o0 / 16 + row / 16 < p.tiles ? o0 / 16 + row / 16 : p.tiles - 1;
    const int64_t scale0 = (tile * p.groups + int64_t(c0) * kGroups) * 16 + 2 * (row & 7) + (row >> 3 & 1);
    const int groups = spans * kGroups;
    // a lane's own scales, 4 bytes each: fp32, or the bf16 pair that holds it
    uint8_t* ring = raw + kDequantWarps * (kRaw * kRawSlot) + (warp - 2 - kDequantWarps) * (kScales * 128) + lane * 4;
    const uint32_t ring_s = smem_u32(ring);
    const uint8_t* from = p.scales + (p.f32 ? scale0 * 4 : (scale0 & ~int64_t(1)) * 2);
    const int step = p.f32 ? 64 : 32;
    auto fetch = [&](int i) {
      if (i < groups && LOCA_CHECK(scale0 + 16 * i, p.tiles * p.groups * 16))
        copy4(ring_s + uint32_t((i & (kScales - 1)) * 128), from + int64_t(i) * step);
      copy_commit();
    };
#pragma unroll 1
    for (int i = 0; i < kScales - 1; ++i) fetch(i);
    constexpr int kRead = kHalf == 32 ? 32 : 16;  // (32 at once of 64 spill)
    float acc[kHalf];
#pragma unroll
    for (int i = 0; i < kHalf; ++i) acc[i] = 0.f;
    for (int j = 0; j < spans; ++j, next()) {
      if (!__all_sync(0xffffffffu, wait(done(stage), phase))) break;
      fence_after();
#pragma unroll
      for (int x = 0; x < kGroups; ++x) {
        const int i = j * kGroups + x;
        copy_wait<kScales - 2>();
        const uint32_t bits = *reinterpret_cast<const uint32_t*>(ring + (i & (kScales - 1)) * 128);
        const float s = __uint_as_float(p.f32 ? bits : scale0 & 1 ? bits & 0xffff0000u : bits << 16);
        fetch(i + kScales - 1);
        const uint32_t ta = tmem_base + (uint32_t(q * 32) << 16) + uint32_t(stage * T::kCols + x * NT + h * kHalf);
#pragma unroll
        for (int c = 0; c < kHalf; c += kRead) {
          float v[kRead];
          if constexpr (kRead == 16) tmem_ld16(ta + c, v);
          else tmem_ld32(ta + c, v);
          if (x == kGroups - 1 && c + kRead >= kHalf) {
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(taken(stage));
          }
#pragma unroll
          for (int e = 0; e < kRead; ++e) acc[c + e] = fmaf(s, v[e], acc[c + e]);
        }
      }
    }
    copy_wait<0>();
    // after the last group's MMAs every stage has been read: the sums take the ring's place, [token][row]
    float* red = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int i = 0; i < kHalf; ++i) red[(h * kHalf + i) * 128 + row] = acc[i];
  }
  cluster_sync();
  fence_after();
  if (p.low.U) wait_for_previous();
  // the tokens rank + ks t of this CTA, a warp each; a lane's rows are 32 apart
  const int tokens = p.N - n0 < NT ? int(p.N - n0) : NT;
  float* us = reinterpret_cast<float*>(smem) + NT * 128;  // [warp][kp]
  const uint32_t red_s = smem_base;
  for (int t = warp; rank + ks * t < tokens; t += kTileThreads / 32) {
    const int n = rank + ks * t;
    float y[4] = {};
    for (int r = 0; r < ks; ++r) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t at = red_s + 4u * uint32_t(n * 128 + 32 * j + lane);
        float v;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(mapa_shared(at, uint32_t(r))) : "memory");
        y[j] += v;
      }
    }
    const int a = p.low.U ? p.low.tok_adapter[n0 + n] : -1;
    if (a >= 0) {
      float* u = us + warp * p.low.kp;
      __syncwarp();
      for (int r = lane; r < p.low.kp; r += 32) u[r] = low_sum(p, n0 + n, r);
      __syncwarp();
      float low[4] = {};
      const __nv_bfloat16* b = p.low.B + (int64_t(a) * p.o + o0 + lane) * p.low.kp;
#pragma unroll 1
      for (int c = 0; c < p.low.kp; c += 8) {
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          v[j] = o0 + 32 * j + lane < p.o ? __ldg(reinterpret_cast<const uint4*>(b + 32 * j * p.low.kp + c)) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const __nv_bfloat162* hh = reinterpret_cast<const __nv_bfloat162*>(&v[j]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 f = __bfloat1622float2(hh[k]);
            low[j] = fmaf(u[c + 2 * k], f.x, low[j]);
            low[j] = fmaf(u[c + 2 * k + 1], f.y, low[j]);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] += low[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t row = o0 + 32 * j + lane;
      if (row < p.o && LOCA_CHECK((n0 + n) * p.ldy + row, (p.N - 1) * p.ldy + p.o))
        p.Y[(n0 + n) * p.ldy + row] = __float2bfloat16_rn(y[j]);
    }
  }
  if (warp == 0 && lane == 0) {  // copies in flight when a role gave up
    const uint32_t n = uint32_t(kStages);
    for (uint32_t i = issued > n ? issued - n : 0u; i < issued; ++i)
      mbar_drain(x_full(int(i % n)), (i / n) & 1u, kDrainLimitNs);
  }
  __syncwarp();
  fence_before();
  cluster_sync();  // no CTA leaves while its peers read its sums
  fence_after();
  if (warp == 1) tmem_dealloc(tmem_base, kAlloc);
}

template <int kHalf, int kGroups>
cudaError_t launch_tiles(const Q4Geo& q, void* flag, int32_t* status, cudaStream_t s) {
  constexpr int NT = 2 * kHalf;
  TileGeo g{};
  g.q = q;
  g.status = status;
  g.abort_flag = static_cast<int32_t*>(flag);
  g.limit_ns = wait_limit_ns();
  g.mark = gp::call_mark();
  CUtensorMap mx;
  if (!gp::map_2d(&mx, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, q.X, q.d, q.N, q.ldx, 64, NT)) return cudaErrorInvalidValue;
  const int64_t rows = div_up(q.o, 128), sets = div_up(q.N, NT);
  // CTAs of a cluster: rounds of the SMs times a CTA's way, about 0.4 us a span and 7 us to begin and end.  (Of four
  // 36 fit at once, of eight 15: the SMs of a processing cluster are no multiple of them.)
  int ks = 1;
  double best = 0;
  for (int k = 1; k <= 8; k *= 2) {
    const int at_once = k == 1 ? sm_count() : k == 2 ? sm_count() / 2 : k == 4 ? sm_count() * 36 / 152 : sm_count() * 15 / 152;
    const double c = double(div_up(rows * sets, at_once < 1 ? 1 : at_once)) * (0.4 * double(div_up(q.spans, k)) + 7.0);
    if (k == 1 || c < best) {
      best = c;
      ks = k;
    }
  }
  g.per_cta = int(div_up(q.spans, ks));
  auto kernel = k_q4_tiles<kHalf, kGroups>;
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = gp::allow_smem(allowed, reinterpret_cast<const void*>(kernel), kTileSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(rows * ks), unsigned(sets));
  cfg.blockDim = dim3(kTileThreads);
  cfg.dynamicSmemBytes = size_t(Tiling<NT, kGroups>::kSmem);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = unsigned(ks);
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, mx, g);
}

// Tiles of 128 tokens where a span has one group: with more, their products would need half of the tensor memory or more
// for a stage (512 tokens at 14336 x 3584 with groups of 64: 182 us in tiles of 128, 139 in tiles of 64).
template <int kGroups>
cudaError_t launch_many(const Q4Geo& g, void* flag, int32_t* status, cudaStream_t s) {
  if (g.N <= 32) return launch_tiles<16, kGroups>(g, flag, status, s);
  if (g.N <= 64) return launch_tiles<32, kGroups>(g, flag, status, s);
  if constexpr (kGroups > 1) return launch_tiles<32, kGroups>(g, flag, status, s);
  else return launch_tiles<64, kGroups>(g, flag, status, s);
}

}  // namespace

// U's sums of single tokens come behind 256 bytes of flags.
size_t q4_workspace_bytes(int64_t N, int64_t d, int k) { return k > 0 && N > 0 ? adapter_tokens_workspace_bytes(N, d, k) : 256; }

size_t q4_packed_bytes(int64_t o, int64_t d, int group, int scale_dtype, bool zeros) {
  return pack_lay(o, d, group, scale_dtype, zeros).total;
}

cudaError_t launch_q4_pack(const void* codes, const void* scales, int scale_dtype, const void* zeros, int64_t o, int64_t d,
                           int group, void* packed, cudaStream_t s) {
  const PackLay p = pack_lay(o, d, group, scale_dtype, zeros != nullptr);
  const int64_t most = 16 * int64_t(sm_count()), blocks = div_up(p.tiles * p.chunks * 32, 256);
  k_q4_pack<<<unsigned(blocks < most ? blocks : most), 256, 0, s>>>(
      static_cast<const uint8_t*>(codes), scales, scale_dtype == LOCA_F32, static_cast<const uint8_t*>(zeros), o, d, p, group,
      static_cast<uint8_t*>(packed));
  return cudaGetLastError();
}

cudaError_t launch_q4_apply(const void* X, int64_t ldx, int64_t N, int64_t d, const void* packed, int64_t o, int group,
                            int scale_dtype, bool zeros, const void* adapters, int n, int k, const void* plan, void* Y,
                            int64_t ldy, void* workspace, int32_t* status, cudaStream_t s) {
  const PackLay p = pack_lay(o, d, group, scale_dtype, zeros);
  const uint8_t* b = static_cast<const uint8_t*>(packed);
  Q4Geo g{};
  g.codes = reinterpret_cast<const uint4*>(b);
  g.scales = b + p.scales;
  g.zeros = zeros ? b + p.zeros : nullptr;
  g.f32 = scale_dtype == LOCA_F32;
  g.o = o;
  g.d = d;
  g.tiles = p.tiles;
  g.spans = int(p.chunks / 2);
  g.groups = int(p.groups);
  g.X = static_cast<const __nv_bfloat16*>(X);
  g.ldx = ldx;
  g.N = N;
  g.Y = static_cast<__nv_bfloat16*>(Y);
  g.ldy = ldy;
  if (adapters) {
    const cudaError_t e = launch_adapter_tokens(X, ldx, N, d, o, adapters, n, k, plan, workspace, &g.low, s);
    if (e != cudaSuccess) return e;
  }
  if (N > kTokensByWarps) {
    void* flag = static_cast<uint8_t*>(workspace) + 128;
    switch (128 / group) {
      case 1: return launch_many<1>(g, flag, status, s);
      case 2: return launch_many<2>(g, flag, status, s);
      default: return launch_many<4>(g, flag, status, s);
    }
  }
  switch (128 / group) {
    case 1: return launch_tokens<1>(g, s);
    case 2: return launch_tokens<2>(g, s);
    default: return launch_tokens<4>(g, s);
  }
}

}  // namespace loca
