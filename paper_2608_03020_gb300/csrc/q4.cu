// A frozen projection in 4 bits with group scales, for a few tokens, with each token's adapter beside it.
//   W[o, k] = s[o, k / group] (q[o, k] - z[o, k / group]),   Y = X W^T + s_a (X A_a) B_a^T
//
// Exact products.  q - z is an integer of at most 15, exact in bf16, as X is: the tensor cores sum x (q - z) over
// up to 64 k of one group in fp32, and the sum is scaled by s and added in fp32.  So W is never rounded.
//
// m16n8k16 MMAs with W's rows as M and the tokens as N (mma.sync: a code becomes an operand in registers, one
// shift and mask and one subtraction for two of them; tcgen05 would want the 16-bit operand written to
// shared memory first, four bytes for each byte read, and its 128 rows of tokens filled to an eighth).
//
//   k_q4_pack   codes in the order of the MMAs' fragments: 512 bytes are 16 rows x 64 k, of which each lane's 16
//               are what it multiplies; the order of k within 64 is chosen so that a lane's part of X is two runs
//               of 16 bytes and that 32 k of one group stay together.  Rows and k are padded to 32 and 128
//   k_q4        a warp takes 16 rows and a range of k in spans of 128, three of which are on the way to its part of
//               shared memory (each lane copies and reads its own 16 bytes, so that it waits for nothing else);
//               ks warps' sums meet in shared memory, in order, with the low-rank term of each token's adapter
//               (U in fp32 from k_adapter_tokens); one rounding
// Bound: up to 16 tokens the instructions that make operands of codes (44 of some 80 for 64 k of 16 rows; 60 to 70 % of
// the issue slots), next to the read of the codes and scales; above, X's way from L2 for every 16 rows, and
// the legacy MMAs' rate (1024 products a cycle and SM).  One token at 28672 x 8192 25.8 us (4.7 TB/s), 3 tokens at
// 151931 x 2048 with groups of 32 48 us (4.2 TB/s), at 20480 x 5120 16.5 us for one token and 20 for eight (2.7 TB/s),
// 16, 32 and 64 tokens at 14336 x 3584 14.4, 25 and 42 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "gemm_pair.cuh"

namespace loca {
namespace {

using namespace tc;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxSmem = 98304;

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
  int shift;             // log2(group)
  int64_t o, d;
  int64_t tiles;
  int spans, groups;
  int ks, per_warp;      // warps that share rows, their spans
  int row_blocks;        // blocks of rows
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

// Two codes (bits s .. s + 3 of both halves of w) less their row's zero: 128 + q has q in the last bits of its
// bf16 pattern 0x4300 | q, and so has 128 + z; their difference is exact.
template <int kShift>
__device__ __forceinline__ uint32_t two_codes(uint32_t w, __nv_bfloat162 zero) {
  uint32_t q;  // (codes & mask) | pattern: one instruction, where the compiler made two (36 instead of 52 of the integer pipe for 64 k)
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(q) : "r"(w >> kShift), "n"(0x000f000f), "r"(0x43004300u));
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&q), zero);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Blocks of a SM (registers decide).
constexpr int resident(int nt) { return nt == 1 ? 3 : nt <= 4 ? 2 : 1; }
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

// kGroups: of 128 k (1, 2 or 4).
template <int NT, int kGroups>
__global__ void __launch_bounds__(kThreads, resident(NT)) k_q4(const __grid_constant__ Q4Geo g) {
  extern __shared__ float smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int gr = lane >> 2, t = lane & 3;
  const int rb = int(blockIdx.x) % g.row_blocks;
  const int n0 = int(blockIdx.x) / g.row_blocks * (8 * NT);
  const int per_block = kWarps / g.ks;  // tiles of a block
  const int kw = warp % g.ks;
  const int64_t tile = int64_t(rb) * per_block + warp / g.ks;
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
  const int tokens = int(g.N) - n0 < T ? int(g.N) - n0 : T;
  const int rows = per_block * R;
  const int64_t row0 = int64_t(rb) * rows;
  // the adapters' rows that this thread multiplies at the end, to L2 meanwhile
  auto prefetch_rows = [&]() {
    for (int i = threadIdx.x; i < rows * tokens; i += kThreads) {
      const int n = i / rows, r = i - n * rows;
      const int a = g.low.tok_adapter[n0 + n];
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
      const int tok = n0 + 8 * n + gr < int(g.N) ? n0 + 8 * n + gr : int(g.N) - 1;
      x[n] = g.X + int64_t(tok) * g.ldx + 128 * c0 + 8 * t;
    }
    uint32_t half = 0;
    for (int left = c1 - c0, k_left = int(g.d) - 128 * c0; left > 0; left -= 4, k_left -= 512) {
      constexpr int kUnroll = NT <= 2 ? 4 : 1;  // (long bodies: 64 tokens 46.3 us unrolled, 43.0 not)
#pragma unroll kUnroll
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
        // X: the whole span where it fits in registers, else 32 k at a time, 32 ahead
        constexpr int kQ = NT <= 2 ? 4 : 2;
        uint4 xv[kQ][NT];
        auto load_x = [&](int q, bool full) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
            xv[q & (kQ - 1)][n] = (full || 128 * i + 32 * q < k_left) &&
                                          LOCA_CHECK_SPAN(x[n] + 128 * i + 32 * q - g.X, 8, (g.N - 1) * g.ldx + g.d)
                                      ? __ldg(reinterpret_cast<const uint4*>(x[n] + 128 * i) + 4 * q)
                                      : make_uint4(0, 0, 0, 0);
        };
        const bool full = 128 * (i + 1) <= k_left;  // (else the last span of rows that are no multiple of 128)
        if (kQ == 4) {
          if (full) {
#pragma unroll
            for (int q = 0; q < 4; ++q) load_x(q, true);
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) load_x(q, false);
          }
        } else {
          load_x(0, false);
        }
        float part[NT][4];
        float s0 = 0.f, s1 = 0.f;
        __nv_bfloat162 zero0, zero1;
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // 32 k
          if (kQ == 2 && q < 3) load_x(q + 1, false);
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
              const uint32_t* b = reinterpret_cast<const uint32_t*>(&xv[q & (kQ - 1)][n]) + 2 * s;
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
      float s = 0.f;
      if (g.low.tok_adapter[n0 + n] >= 0 && LOCA_CHECK(n0 + n, g.N))
        for (int q = 0; q < g.low.ranges; ++q) s += g.low.U[(int64_t(q) * g.N + n0 + n) * g.low.kp + r];
      u[i] = s;
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
      const int a = g.low.tok_adapter[n0 + n];
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
    if (LOCA_CHECK((n0 + n) * g.ldy + row, (g.N - 1) * g.ldy + g.o)) g.Y[(n0 + n) * g.ldy + row] = __float2bfloat16_rn(y);
  }
}

// Warps on the same rows: more of them shorten a warp's way through k, and add a block's start and end (about
// 2 us, and 0.4 for each that shares the SM) for each of its fewer spans.  A span takes a lone block's warps 0.62 us; eight warps' worth of a span
// keeps an SM busy for `busy` of it, whatever shares the SM.  20480 x 5120, 8 tokens: 28.6 us with one warp, 21.0 with
// two, 20.0 with four, 20.2 with eight; 3584 x 3584, one token: 7.2, 4.7 and 3.9 with two, four and eight.
template <int NT>
void share_rows(Q4Geo& g, int64_t sets) {
  constexpr double busy = NT <= 2 ? 0.44 : NT == 4 ? 0.8 : 1.2;
  auto round = [](int64_t blocks, int64_t spans) {
    const double each = blocks * busy;
    return blocks > 0 ? double(spans) * (each > 0.62 ? each : 0.62) + 2.0 + 0.4 * blocks : 0.0;
  };
  double best = 0;
  for (int ks = 1; ks <= kWarps; ks *= 2) {
    const int64_t per = div_up(g.spans, ks), blocks = div_up(div_up(g.tiles, kWarps / ks) * sets, sm_count());
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
  const int64_t sets = div_up(g.N, 8 * NT);
  share_rows<NT>(g, sets);
  g.row_blocks = int(div_up(g.tiles, kWarps / g.ks));
  const int sums = 4 * (kWarps * 8 * NT * 16 + (g.low.U ? 8 * NT * g.low.kp : 0)), rings = kWarps * warp_bytes(kGroups);
  const cudaError_t e = cudaFuncSetAttribute(k_q4<NT, kGroups>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  if (e != cudaSuccess) return e;
  return gp::launch_early(k_q4<NT, kGroups>, dim3(unsigned(g.row_blocks * sets)), dim3(kThreads),
                          size_t(sums > rings ? sums : rings), s, g);
}

template <int kGroups>
cudaError_t launch_tokens(const Q4Geo& g, cudaStream_t s) {
  if (g.N <= 8) return launch_one<1, kGroups>(g, s);
  if (g.N <= 16) return launch_one<2, kGroups>(g, s);
  if (g.N <= 32) return launch_one<4, kGroups>(g, s);
  return launch_one<8, kGroups>(g, s);
}

}  // namespace

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
                            int64_t ldy, void* workspace, cudaStream_t s) {
  const PackLay p = pack_lay(o, d, group, scale_dtype, zeros);
  const uint8_t* b = static_cast<const uint8_t*>(packed);
  Q4Geo g{};
  g.codes = reinterpret_cast<const uint4*>(b);
  g.scales = b + p.scales;
  g.zeros = zeros ? b + p.zeros : nullptr;
  g.f32 = scale_dtype == LOCA_F32;
  g.shift = group == 32 ? 5 : group == 64 ? 6 : 7;
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
  switch (128 / group) {
    case 1: return launch_tokens<1>(g, s);
    case 2: return launch_tokens<2>(g, s);
    default: return launch_tokens<4>(g, s);
  }
}

}  // namespace loca
