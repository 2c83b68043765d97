// Gated feed-forward of a block and its gradients.
//   G = X Wg^T,  U = X Wu^T,  H = act(G) U                       (X N x d, Wg and Wu f x d, H N x f)
//   dG = dH U act'(G),  dU = dH act(G)
//   dX = dG Wg + dU Wu,  dWg = dG^T X,  dWu = dU^T X
// Both activations are g times a sigmoid of an odd polynomial,
//   act(g) = g s,  s = 1 / (1 + exp(-(a g + b g^3))),  act'(g) = s + g s (1 - s) (a + 3 b g^2),
// with a = 1, b = 0 for SiLU and a = 2 c, b = 2 c 0.044715, c = sqrt(2 / pi), for the tanh form of GELU
// (0.5 (1 + tanh y) = 1 / (1 + exp(-2 y))).
//
// k_gemm_pair, twin   both products in one launch: a tile holds the same columns of G and of U side by side in
//                     tensor memory, an epilogue thread has 64 of each of one row in registers.  Forward:
//                     H leaves, G and U never do.  Backward: the same tiles again, turned into dG and dU
//                     with the row's dH, rounded to bf16 as the operand of the gradient products.  That rounding
//                     moves the gradients about as much as their own (0.0024 of them in norm, 0.0017 without
//                     it); G and U themselves stay in fp32, which is why they are computed again instead of
//                     kept in bf16 (0.003).  Kept in fp32 they would cost 8 N f bytes of memory, and
//                     20 N f bytes of traffic against the 4 N d f operations of computing them: equal at
//                     d = 1400, a fifth of a training step at d = 5120
// k_gemm_pair, joined dX as one product over 2 f: dG against Wg, then dU against Wu, into the same sums
// k_gemm_pair         dWg and dWu
// k_gated_join        sums the k ranges of dX where its tiles alone would not fill the SMs
// Bound: the tensor cores from a few hundred tokens on, the read of Wg and Wu below.  8192 tokens at d = 3584,
// f = 14336: 856 us cold, 935 to 948 under load (1.97 and 1.79 PFLOP/s); one token there 37.5 us (206 MB: 5.5 TB/s); 64
// tokens at d = 2048, f = 8192 17.0 us (3.9 TB/s); forward and backward of 4096 tokens there 700 us (1.57 PFLOP/s with
// the products computed again).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "gemm_pair.cuh"

namespace loca {
namespace {

using namespace tc;

constexpr int kSegKb = 64;             // 4096 k per accumulation segment: outputs are rounded to bf16
// dX sums 2 f terms, and a wide tile has one running sum: up to 2048 steps that lose at most 2^-22 of it each, 2^-11 in
// all, where a rounding to bf16 moves the value by up to 2^-8 of it.  1531 x 5120 over k = 27312: one round of 60 wide tiles without ranges, against five
// ranges and their join (dX after dG and dU 250 us, 265 with ranges).
constexpr int64_t kLongK = 32768;
constexpr int64_t kRowBytes = int64_t(1) << 30;  // dG and dU of a piece of the rows (dX alone)
constexpr int64_t kAllBytes = int64_t(4) << 30;  // of a piece of the columns (dWg and dWu sum over all rows)

struct Act {
  float a, b;   // of the sigmoid's argument, times -log2(e)
  float da, db; // of its derivative
  float lim;    // beyond it the sigmoid is 0 or 1 to fp32; powers of g stay finite
};
Act act_of(int code) {
  constexpr float kLog2e = 1.4426950408889634f;
  constexpr float c2 = 1.5957691216057308f;  // 2 sqrt(2 / pi)
  constexpr float k3 = 0.044715f;
  if (code == 0) return Act{-kLog2e, 0.f, 1.f, 0.f, 200.f};
  return Act{-kLog2e * c2, -kLog2e * c2 * k3, c2, 3.f * c2 * k3, 16.f};
}

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float clamped(const Act& p, float g) { return fminf(fmaxf(g, -p.lim), p.lim); }
// The sigmoid of the activation at x = clamped(g).
__device__ __forceinline__ float gate_of(const Act& p, float x) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * fmaf(p.b, x * x, p.a)));
  return rcp_approx(1.f + e);
}

// 8 columns of a row at `at`.
__device__ __forceinline__ void put8(__nv_bfloat16* at, const uint32_t* w) {
  *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
}

struct EpiGate {
  static constexpr bool kFits = false;
  static constexpr bool kAhead = false;
  Act p;
  __nv_bfloat16* H;
  int64_t pitch;
  int rows;

  struct Row {};
  __device__ __forceinline__ Row before(int, int) const { return Row{}; }
  __device__ __forceinline__ float value(float g, float u) const { return g * gate_of(p, clamped(p, g)) * u; }
  __device__ __forceinline__ void operator()(const gp::Tile&, float (&v)[128], Row&, int row, int col0, int lane,
                                             uint8_t* box, const CUtensorMap* out, const CUtensorMap*) const {
    uint32_t w[32];
#pragma unroll
    for (int i = 0; i < 32; ++i)
      w[i] = gp::pack_bf16(value(v[2 * i], v[64 + 2 * i]), value(v[2 * i + 1], v[64 + 2 * i + 1]));
    gp::store_box_bf16(box, out, lane, col0, row - lane, w);
  }
  __device__ __forceinline__ void store8(float (&v)[16], int row, int col) const {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = gp::pack_bf16(value(v[2 * i], v[8 + 2 * i]), value(v[2 * i + 1], v[8 + 2 * i + 1]));
    if (row < rows && LOCA_CHECK_SPAN(col, 8, pitch)) put8(H + int64_t(row) * pitch + col, w);
  }
};

struct EpiGateBack {
  static constexpr bool kFits = false;
  static constexpr bool kAhead = false;
  Act p;
  const __nv_bfloat16* dH;  // this piece's rows and columns
  int64_t pitch;
  int rows, cols;           // of the piece
  __nv_bfloat16* D;         // its dG; dU is fc columns behind
  int64_t fc;

  struct Row {};
  // dH is on its way to L2 while the sums are not complete (its place in registers is the sums').
  __device__ __forceinline__ Row before(int row, int col0) const {
    if (row < rows && col0 < cols) {
      const __nv_bfloat16* at = dH + int64_t(row) * pitch + col0;
      asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
      if (col0 + 56 < cols) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + 56));
    }
    return Row{};
  }
  __device__ __forceinline__ void one(float g, float u, float dh, float& dg, float& du) const {
    const float x = clamped(p, g);
    const float s = gate_of(p, x);
    float d = fmaf(x * s, (1.f - s) * fmaf(p.db, x * x, p.da), s);
    if (g != g) d = g;  // (the clamp lets no NaN through)
    dg = dh * u * d;
    du = dh * (g * s);
  }
  // 8 columns: dG in wg, dU in wu
  __device__ __forceinline__ void eight(const float* g, const float* u, const uint4& dh, uint32_t* wg, uint32_t* wu) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = reinterpret_cast<const uint32_t*>(&dh)[i];
      const float2 h = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&two));
      float g0, g1, u0, u1;
      one(g[2 * i], u[2 * i], h.x, g0, u0);
      one(g[2 * i + 1], u[2 * i + 1], h.y, g1, u1);
      wg[i] = gp::pack_bf16(g0, g1);
      wu[i] = gp::pack_bf16(u0, u1);
    }
  }
  __device__ __forceinline__ uint4 dh8(int row, int col) const {
    return row < rows && col < cols ? __ldg(reinterpret_cast<const uint4*>(dH + int64_t(row) * pitch + col))
                                    : make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void operator()(const gp::Tile&, float (&v)[128], Row&, int row, int col0, int lane,
                                             uint8_t* box, const CUtensorMap* out, const CUtensorMap* out2) const {
    uint32_t wu[32];
    if (lane == 0) bulk_wait_group_read0();
    __syncwarp();
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      uint4 dh[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) dh[j] = dh8(row, col0 + 32 * b + 8 * j);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = 32 * b + 8 * j;
        uint32_t wg[4];
        eight(v + at, v + 64 + at, dh[j], wg, wu + at / 2);
        *reinterpret_cast<uint4*>(box + gp::box_off(lane, at / 8)) = make_uint4(wg[0], wg[1], wg[2], wg[3]);
      }
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      if (LOCA_REQUIRE(col0 >= 0 && row >= 0 && col0 % 8 == 0)) tma_store_2d(out, smem_u32(box), col0, row);
      bulk_commit_group();
    }
    gp::store_box_bf16(box, out2, lane, col0, row - lane, wu);
  }
  __device__ __forceinline__ void store8(float (&v)[16], int row, int col) const {
    uint32_t wg[4], wu[4];
    eight(v, v + 8, dh8(row, col), wg, wu);
    if (row >= rows || !LOCA_CHECK_SPAN(col, 8, fc)) return;
    put8(D + int64_t(row) * 2 * fc + col, wg);
    put8(D + int64_t(row) * 2 * fc + fc + col, wu);
  }
};

// Sums the k ranges of dX in order and rounds once.  One thread per 8 elements of a row.
__global__ void __launch_bounds__(256) k_gated_join(const float* __restrict__ part, int splits, int64_t range, int64_t rows,
                                                    int64_t d, __nv_bfloat16* __restrict__ dX, int64_t lddx) {
  wait_for_previous();
  launch_dependents();
  const int dv = int(d / 8);
  const int64_t total = rows * dv;
  for (int64_t e = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; e < total; e += int64_t(gridDim.x) * blockDim.x) {
    const int64_t row = e / dv, at = row * d + 8 * (e - row * dv);
    float a[8] = {};
    for (int s0 = 0; s0 < splits; s0 += 4) {
      float4 x[4][2];
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s0 + s < splits && LOCA_CHECK_SPAN(int64_t(s0 + s) * range + at, 8, int64_t(splits) * range)) {
          const float4* p = reinterpret_cast<const float4*>(part + int64_t(s0 + s) * range + at);
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
    q.x = gp::pack_bf16(a[0], a[1]);
    q.y = gp::pack_bf16(a[2], a[3]);
    q.z = gp::pack_bf16(a[4], a[5]);
    q.w = gp::pack_bf16(a[6], a[7]);
    *reinterpret_cast<uint4*>(dX + row * lddx + (at - row * d)) = q;
  }
}

// ------------------------------------------------------------------ host side
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

gp::Geo geo(int64_t rows, int64_t cols, int64_t nkb, int32_t* status, void* workspace, int32_t mark) {
  gp::Geo g{};
  g.m_tiles = int(ceil_div(rows, gp::TM));
  g.cols = int(cols);
  g.nkb = int(nkb);
  g.splits = 1;
  g.seg_kb = kSegKb;
  g.group = 16;
  g.status = status;
  g.abort_flag = static_cast<int32_t*>(workspace);
  g.limit_ns = wait_limit_ns();
  g.mark = mark;
  return g;
}

// Columns of the single shape's tiles, a multiple of 8 up to 128: what counts is how many rows of both operands
// a CTA fetches in all.  3584 x 14336 takes 150 tiles of 96.
int twin_width(int64_t rows, int64_t cols) {
  const int64_t a = ceil_div(rows, 8) * 8;
  int64_t best = 0;
  int width = 0;
  for (int w = 32; w <= 128; w += 8) {
    const int64_t c = ceil_div(ceil_div(cols, w), sm_count()) * (a + 2 * w);
    if (width == 0 || c < best) {
      best = c;
      width = w;
    }
  }
  return width;
}

// Both products of a piece: rows of X against cols rows of Wg and of Wu.
template <class Epi>
cudaError_t launch_twin(const void* X, int64_t ldx, int64_t rows, int64_t d, const __nv_bfloat16* Wg,
                        const __nv_bfloat16* Wu, int64_t cols, const CUtensorMap& out, const CUtensorMap& out2, gp::Geo g,
                        const Epi& epi, cudaStream_t s) {
  CUtensorMap mx, mg, mu;
  const int64_t nkb = ceil_div(d, gp::BK);
  const bool single = rows <= gp::HALF && d <= gp::kWideK;  // (one sum per tile there)
  g.arows = single ? int(ceil_div(rows, 8) * 8) : gp::HALF;
  g.width = single ? twin_width(rows, cols) : 0;
  const int brows = single ? g.width : gp::HALF;
  if (!gp::map_2d(&mx, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, X, d, rows, ldx, gp::BK, g.arows) ||
      !gp::map_2d(&mg, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, Wg, d, cols, d, gp::BK, brows) ||
      !gp::map_2d(&mu, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, Wu, d, cols, d, gp::BK, brows))
    return cudaErrorInvalidValue;
  if (single) return gp::launch<gp::kSingle, false, false>(mx, mg, out2, mu, out, g, epi, gp::Twin{}, s);
  // (2 cols accumulator columns in all, whatever a tile makes of them)
  if (gp::pick_shape(0, g.m_tiles, 2 * cols, nkb, 1) == gp::kWide)
    return gp::launch<gp::kWide, false, false>(mx, mg, out2, mu, out, g, epi, gp::Twin{}, s);
  return gp::launch<gp::kNarrow, false, false>(mx, mg, out2, mu, out, g, epi, gp::Twin{}, s);
}

struct BwdWs {
  int64_t piece, fc;  // rows and columns of dG and dU
  int splits;         // k ranges of dX
  bool sums;          // dX goes through fp32 sums in memory
  size_t d, part, total;
};
// k ranges of dX: its tiles are few, so ranges fill the SMs; a range costs 8 bytes an element (written, then read
// by the join).  Both sides in cycles (as for the head's gradient).
int dx_splits(int64_t rows, int64_t d, int64_t nkb) {
  const int64_t m = ceil_div(rows, gp::TM);
  const bool single = rows <= gp::HALF;
  int best = 1;
  double best_c = 0;
  for (int s = 1; s <= 32; ++s) {
    if (s > 1 && nkb / s < (single ? 4 : 16)) break;
    const double join = s > 1 ? double(s) * (double(single ? rows : m * gp::TM) * double(d) * 8.0 / 3000.0 + gp::kRangeCycles) + 3000.0 : 0.0;
    const double c = gp::cycles(gp::pick_shape(rows, m, d, nkb, s, kLongK), m, d, nkb, s) + join;
    if (s == 1 || c < best_c) {
      best = s;
      best_c = c;
    }
  }
  return best;
}
BwdWs bwd_ws(int64_t N, int64_t d, int64_t f, bool dx, bool dw) {
  BwdWs o{};
  const int64_t n = N < 1 ? 1 : N;
  o.piece = n;
  o.fc = f;
  if (dw) {
    int64_t most = kAllBytes / (4 * n) / gp::TN * gp::TN;
    if (most < gp::TN) most = gp::TN;
    if (f > most) o.fc = ceil_div(ceil_div(f, ceil_div(f, most)), gp::TN) * gp::TN;
  } else {
    int64_t most = kRowBytes / (4 * f) / gp::TM * gp::TM;
    if (most < gp::TM) most = gp::TM;
    if (n > most) o.piece = ceil_div(ceil_div(n, ceil_div(n, most)), gp::TM) * gp::TM;
  }
  const int64_t nkb = 2 * ceil_div(o.fc, gp::BK);
  o.splits = dx ? dx_splits(o.piece, d, nkb) : 1;
  o.sums = dx && (o.splits > 1 || o.fc < f);
  size_t at = 256;
  o.d = at; at += align256(4 * size_t(o.piece) * size_t(o.fc));
  o.part = at; at += o.sums ? align256(4 * size_t(o.splits) * size_t(ceil_div(o.piece, gp::TM) * gp::TM) * size_t(d)) : 0;
  o.total = at;
  return o;
}

}  // namespace

size_t gated_workspace_bytes() { return 256; }
size_t gated_backward_workspace_bytes(int64_t N, int64_t d, int64_t f, bool dx, bool dw) {
  return bwd_ws(N, d, f, dx, dw).total;
}

cudaError_t launch_gated(const void* X, int64_t ldx, int64_t N, int64_t d, const void* Wg, const void* Wu, int64_t f,
                         int act, void* H, int64_t ldh, void* workspace, int32_t* status, cudaStream_t s) {
  CUtensorMap mo;
  if (!gp::map_out_bf16(&mo, H, f, N, ldh)) return cudaErrorInvalidValue;
  const gp::Geo g = geo(N, f, ceil_div(d, gp::BK), status, workspace, gp::call_mark());
  return launch_twin(X, ldx, N, d, static_cast<const __nv_bfloat16*>(Wg), static_cast<const __nv_bfloat16*>(Wu), f, mo, mo,
                     g, EpiGate{act_of(act), static_cast<__nv_bfloat16*>(H), ldh, int(N)}, s);
}

cudaError_t launch_gated_backward(const void* X, int64_t ldx, int64_t N, int64_t d, const void* Wg, const void* Wu,
                                  int64_t f, int act, const void* dH, int64_t lddh, void* dX, int64_t lddx, void* dWg,
                                  void* dWu, void* workspace, int32_t* status, cudaStream_t s) {
  const bool dw = dWg != nullptr || dWu != nullptr;
  const BwdWs lay = bwd_ws(N, d, f, dX != nullptr, dw);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  __nv_bfloat16* D = reinterpret_cast<__nv_bfloat16*>(ws + lay.d);
  float* part = reinterpret_cast<float*>(ws + lay.part);
  const __nv_bfloat16* Xb = static_cast<const __nv_bfloat16*>(X);
  const __nv_bfloat16* Wgb = static_cast<const __nv_bfloat16*>(Wg);
  const __nv_bfloat16* Wub = static_cast<const __nv_bfloat16*>(Wu);
  const __nv_bfloat16* dHb = static_cast<const __nv_bfloat16*>(dH);
  const int32_t mark = gp::call_mark();
  cudaError_t e = cudaSuccess;
  for (int64_t p0 = 0; p0 < N; p0 += lay.piece) {
    const int64_t rows = N - p0 < lay.piece ? N - p0 : lay.piece;
    const __nv_bfloat16* Xp = Xb + p0 * ldx;
    const int64_t range = ceil_div(rows, gp::TM) * gp::TM * d;  // sums of a k range
    const int shape = gp::pick_shape(rows, ceil_div(rows, gp::TM), d, 2 * ceil_div(lay.fc, gp::BK), lay.splits, kLongK);
    for (int64_t v0 = 0; v0 < f; v0 += lay.fc) {
      const int64_t vn = f - v0 < lay.fc ? f - v0 : lay.fc;
      const int64_t pitch = 2 * lay.fc;  // a row's dG, then its dU
      CUtensorMap og, ou;
      if (!gp::map_out_bf16(&og, D, vn, rows, pitch) || !gp::map_out_bf16(&ou, D + lay.fc, vn, rows, pitch))
        return cudaErrorInvalidValue;
      const EpiGateBack epi{act_of(act), dHb + p0 * lddh + v0, lddh, int(rows), int(vn), D, lay.fc};
      e = launch_twin(Xp, ldx, rows, d, Wgb + v0 * d, Wub + v0 * d, vn, og, ou,
                      geo(rows, vn, ceil_div(d, gp::BK), status, workspace, mark), epi, s);
      if (e != cudaSuccess) return e;
      for (int i = 0; i < 2; ++i) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(i ? dWu : dWg);
        if (!o) continue;
        CUtensorMap ma, mb, mo;
        if (!gp::map_mnmajor(&ma, D + i * lay.fc, vn, rows, pitch) || !gp::map_mnmajor(&mb, Xp, d, rows, ldx) ||
            !gp::map_out_bf16(&mo, o + v0 * d, d, vn, d))
          return cudaErrorInvalidValue;
        e = gp::launch_either<true, true>(ma, mb, ma, mb, mo, geo(vn, d, ceil_div(rows, gp::BK), status, workspace, mark),
                                          gp::EpiScaled{1.f}, gp::NoExt{}, s);
        if (e != cudaSuccess) return e;
      }
      if (!dX) continue;
      CUtensorMap ma, mb, ma2, mb2, mo;
      if (!gp::map_kmajor(&ma, D, vn, rows, pitch) || !gp::map_kmajor(&ma2, D + lay.fc, vn, rows, pitch) ||
          !gp::map_mnmajor(&mb, Wgb + v0 * d, d, vn, d) || !gp::map_mnmajor(&mb2, Wub + v0 * d, d, vn, d))
        return cudaErrorInvalidValue;
      const int64_t half = ceil_div(vn, gp::BK);
      gp::Geo g = geo(rows, d, 2 * half, status, workspace, mark);
      g.splits = lay.splits;
      gp::SecondPair second;
      second.first = int(half);
      if (lay.sums) {
        if (!gp::map_2d(&mo, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, part, d, lay.splits * (range / d), d, 32, 32))
          return cudaErrorInvalidValue;
        e = gp::launch_shape<false, true>(shape, ma, mb, ma2, mb2, mo, g, gp::EpiAcc{v0 > 0 ? 1 : 0}, second, s);
      } else {
        if (!gp::map_out_bf16(&mo, static_cast<__nv_bfloat16*>(dX) + p0 * lddx, d, rows, lddx)) return cudaErrorInvalidValue;
        e = gp::launch_shape<false, true>(shape, ma, mb, ma2, mb2, mo, g, gp::EpiScaled{1.f}, second, s);
      }
      if (e != cudaSuccess) return e;
    }
    if (lay.sums) {
      const int64_t blocks = rows * (d / 8) / 256 + 1;
      const int64_t most = 8 * int64_t(sm_count());
      e = gp::launch_early(k_gated_join, dim3(unsigned(blocks < most ? blocks : most)), dim3(256), 0, s,
                           static_cast<const float*>(part), lay.splits, range, rows, d,
                           static_cast<__nv_bfloat16*>(dX) + p0 * lddx, lddx);
      if (e != cudaSuccess) return e;
    }
  }
  return cudaSuccess;
}

}  // namespace loca
