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
//   k_q4_pack   codes in the order of the MMAs' fragments: a warp's load of 512 bytes is 16 rows x 64 k, of
//               which each lane gets what it multiplies; the order of k within 64 is chosen so that a lane's
//               part of X is two runs of 16 bytes and that 32 k of one group stay together
//   k_q4        a warp takes 16 or 32 rows and every ks-th 64 k; ks warps' sums meet in shared memory, in order,
//               with the low-rank term of each token's adapter (U in fp32 from k_adapter_tokens); one rounding
// Bound: the read of the codes and scales.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "gemm_pair.cuh"

namespace loca {
namespace {

using namespace tc;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kAhead = 4;    // chunks of 64 k that a warp has on the way
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
  p.chunks = div_up(d, 64);
  p.groups = d / group;
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
      const int64_t at = row * p.groups + q;
      const bool in = row < o;
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
  int chunks, groups;
  int ks;                // warps that share rows
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
  const uint32_t q = ((w >> kShift) & 0x000f000fu) | 0x43004300u;
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&q), zero);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int NT, int MT>
__global__ void __launch_bounds__(kThreads) k_q4(const __grid_constant__ Q4Geo g) {
  extern __shared__ float smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int gr = lane >> 2, t = lane & 3;
  const int rb = int(blockIdx.x) % g.row_blocks;
  const int64_t n0 = int64_t(int(blockIdx.x) / g.row_blocks) * (8 * NT);
  const int per_block = kWarps / g.ks;  // row groups of a block
  const int kw = warp % g.ks;
  const int64_t tile0 = (int64_t(rb) * per_block + warp / g.ks) * MT;
  constexpr int R = 16 * MT, T = 8 * NT;
  // With adapters the launch before is k_adapter_tokens, which let this one start only after all launches before
  // it had completed: what it writes is needed at the end.
  if (!g.low.U) wait_for_previous();
  launch_dependents();
  float acc[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;
  if (tile0 < g.tiles) {
    const uint4* codes = g.codes + tile0 * g.chunks * 32 + lane;
    const __nv_bfloat16* x = g.X + (n0 + gr) * g.ldx + 8 * t;
    for (int c0 = kw; c0 < g.chunks; c0 += kAhead * g.ks) {
      uint4 w[kAhead][MT];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int c = c0 + j * g.ks;
#pragma unroll
        for (int m = 0; m < MT; ++m)
          w[j][m] = c < g.chunks && LOCA_CHECK((tile0 + m) * g.chunks + c, g.tiles * g.chunks)
                        ? __ldg(codes + (int64_t(m) * g.chunks + c) * 32)
                        : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int c = c0 + j * g.ks;
        if (c >= g.chunks) break;
        const bool second = 64 * c + 32 < g.d;  // (a last half chunk, with groups of 32)
        uint4 xv[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const bool in = n0 + 8 * n + gr < g.N && LOCA_CHECK_SPAN(64 * c + 8 * t + (second ? 32 : 0), 8, g.d);
          const uint4* p = reinterpret_cast<const uint4*>(x + 8 * n * g.ldx + 64 * c);
          xv[n][0] = in ? __ldg(p) : make_uint4(0, 0, 0, 0);
          xv[n][1] = in && second ? __ldg(p + 4) : make_uint4(0, 0, 0, 0);
        }
        const int q0 = (64 * c) >> g.shift, q1 = second ? (64 * c + 32) >> g.shift : q0;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          float part[NT][4];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int64_t at = ((tile0 + m) * g.groups + (half ? q1 : q0)) * 8 + gr;
            uint32_t z = 0x88u;
            if (!LOCA_CHECK(at, g.tiles * g.groups * 8)) continue;
            if (g.zeros) z = __ldg(g.zeros + at);
            const uint32_t z0 = (z & 15u) | 0x4300u, z1 = (z >> 4) | 0x4300u;
            const uint32_t zz0 = z0 | z0 << 16, zz1 = z1 | z1 << 16;
            const __nv_bfloat162 zero0 = *reinterpret_cast<const __nv_bfloat162*>(&zz0);
            const __nv_bfloat162 zero1 = *reinterpret_cast<const __nv_bfloat162*>(&zz1);
            if (half == 0 || q1 != q0) {
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) part[n][i] = 0.f;
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const uint32_t word = reinterpret_cast<const uint32_t*>(&w[j][m])[2 * half + s];
              const uint32_t a[4] = {two_codes<0>(word, zero0), two_codes<4>(word, zero1), two_codes<8>(word, zero0),
                                     two_codes<12>(word, zero1)};
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                const uint32_t* b = reinterpret_cast<const uint32_t*>(&xv[n][half]) + 2 * s;
                mma_16816(part[n], a, b[0], b[1]);
              }
            }
            if (half == 1 || q1 != q0) {
              float s0, s1;
              if (g.f32) {
                const float2 s = __ldg(reinterpret_cast<const float2*>(g.scales) + at);
                s0 = s.x;
                s1 = s.y;
              } else {
                const uint32_t s = __ldg(reinterpret_cast<const uint32_t*>(g.scales) + at);
                s0 = __uint_as_float(s << 16);
                s1 = __uint_as_float(s & 0xffff0000u);
              }
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                acc[m][n][0] = fmaf(s0, part[n][0], acc[m][n][0]);
                acc[m][n][1] = fmaf(s0, part[n][1], acc[m][n][1]);
                acc[m][n][2] = fmaf(s1, part[n][2], acc[m][n][2]);
                acc[m][n][3] = fmaf(s1, part[n][3], acc[m][n][3]);
              }
            }
          }
        }
      }
    }
  }
  if (g.low.U) wait_for_previous();
  // sums of the warps: [warp][token][row]
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        smem[(warp * T + 8 * n + 2 * t + (i & 1)) * R + 16 * m + gr + 8 * (i >> 1)] = acc[m][n][i];
  float* u = smem + kWarps * T * R;
  const int tokens = g.N - n0 < T ? int(g.N - n0) : T;
  if (g.low.U)
    for (int i = threadIdx.x; i < tokens * g.low.kp; i += kThreads) {
      const int n = i / g.low.kp, r = i - n * g.low.kp;
      float s = 0.f;
      if (g.low.tok_adapter[n0 + n] >= 0)
        for (int q = 0; q < g.low.ranges; ++q) s += g.low.U[(int64_t(q) * g.N + n0 + n) * g.low.kp + r];
      u[i] = s;
    }
  __syncthreads();
  const int rows = per_block * R;
  const int64_t row0 = int64_t(rb) * rows;
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

template <int NT, int MT>
cudaError_t launch_one(Q4Geo g, cudaStream_t s) {
  // as many warps on the same rows as it takes to give every SM two blocks
  const int64_t groups = g.tiles / MT;
  g.ks = 1;
  while (g.ks < kWarps && div_up(groups, kWarps / g.ks) < 2 * sm_count() && g.chunks >= 2 * kAhead * g.ks) g.ks *= 2;
  const int per_block = kWarps / g.ks;
  g.row_blocks = int(div_up(groups, per_block));
  const int64_t blocks = int64_t(g.row_blocks) * div_up(g.N, 8 * NT);
  const int smem = 4 * (kWarps * 8 * NT * 16 * MT + (g.low.U ? 8 * NT * g.low.kp : 0));
  cudaError_t e = cudaFuncSetAttribute(k_q4<NT, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  if (e != cudaSuccess) return e;
  return gp::launch_early(k_q4<NT, MT>, dim3(unsigned(blocks)), dim3(kThreads), size_t(smem), s, g);
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
  g.chunks = int(p.chunks);
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
  if (N <= 8) return launch_one<1, 2>(g, s);
  if (N <= 16) return launch_one<2, 2>(g, s);
  if (N <= 32) return launch_one<4, 2>(g, s);
  return launch_one<8, 2>(g, s);
}

}  // namespace loca
