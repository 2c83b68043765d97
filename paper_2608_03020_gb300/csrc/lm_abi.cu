// C ABI entry points of the operators around the pass (head loss, adapted projection, gradient
// clipping): host-side validation and dispatch.  See include/loca.h for the contract of each.
#include <cuda_runtime.h>

#include <cmath>

#include "loca_internal.h"

using namespace loca;

namespace {

template <class... A>
int fail(int code, const char* fmt, A... a) {
  return set_error_message(code, fmt, a...);
}
int clear() { return set_error_message(LOCA_OK, "%s", ""); }
int cuda_fail(cudaError_t e, const char* where) { return fail(LOCA_ERR_CUDA, "%s: %s", where, cudaGetErrorString(e)); }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_ws(const void* workspace, size_t have, size_t need) {
  if (have < need || (need > 0 && !workspace))
    return fail(LOCA_ERR_WORKSPACE, "workspace too small: need %zu bytes, got %zu", need, workspace ? have : size_t(0));
  if (!aligned(workspace, 256)) return fail(LOCA_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
  return LOCA_OK;
}

int check_head(int64_t N, int64_t V, int64_t d) {
  if (N < 0 || N > (int64_t(1) << 24)) return fail(LOCA_ERR_SHAPE, "need 0 <= N <= 2^24, got %lld", (long long)N);
  if (V < 1 || V > (int64_t(1) << 24)) return fail(LOCA_ERR_SHAPE, "need 1 <= V <= 2^24, got %lld", (long long)V);
  if (d < 8 || d > 65536 || d % 8 != 0)
    return fail(LOCA_ERR_SHAPE, "need 8 <= d <= 65536, a multiple of 8, got %lld", (long long)d);
  return LOCA_OK;
}

int check_adapter(int64_t N, int64_t d_in, int64_t d_out, int32_t k, int32_t n) {
  if (N < 0 || N > (int64_t(1) << 22)) return fail(LOCA_ERR_SHAPE, "need 0 <= N <= 2^22, got %lld", (long long)N);
  if (d_in < 8 || d_in > 65536 || d_in % 8 != 0 || d_out < 8 || d_out > 65536 || d_out % 8 != 0)
    return fail(LOCA_ERR_SHAPE, "need 8 <= d_in, d_out <= 65536, multiples of 8, got %lld, %lld", (long long)d_in,
                (long long)d_out);
  if (k < 1 || k > adapter_max_k()) return fail(LOCA_ERR_SHAPE, "need 1 <= k <= %d, got %d", adapter_max_k(), k);
  if (n < 1 || n > 65535) return fail(LOCA_ERR_SHAPE, "need 1 <= n <= 65535 adapters, got %d", n);
  return LOCA_OK;
}

// A bf16 matrix that TMA reads or writes: pitch at least its columns, 16-byte rows.
int check_rows(const void* p, int64_t pitch, int64_t cols, const char* name) {
  if (pitch < cols)
    return fail(LOCA_ERR_SHAPE, "row pitch of %s %lld is below its %lld columns", name, (long long)pitch, (long long)cols);
  if (pitch % 8 != 0 || !aligned(p, 16))
    return fail(LOCA_ERR_ALIGNMENT, "%s needs 16-byte alignment and a row pitch that is a multiple of 8", name);
  return LOCA_OK;
}

// Whether rows of `wide` bytes, `pitch` bytes apart, share a byte with the rows of another such matrix
// (columns of one buffer side by side do not).
struct Block {
  const void* p;
  int64_t pitch, wide;
};
bool overlap(const Block& x, const Block& y, int64_t rows) {
  const int64_t a = reinterpret_cast<int64_t>(x.p), b = reinterpret_cast<int64_t>(y.p);
  if (!x.p || !y.p || a + (rows - 1) * x.pitch + x.wide <= b || b + (rows - 1) * y.pitch + y.wide <= a) return false;
  if (x.pitch == y.pitch) {  // row i of y begins `at` bytes behind the begin of row i + q of x
    int64_t q = (b - a) / x.pitch, at = (b - a) % x.pitch;
    if (at < 0) {
      --q;
      at += x.pitch;
    }
    return (at < x.wide && q > -rows && q < rows) || (at + y.wide > x.pitch && q + 1 > -rows && q + 1 < rows);
  }
  for (int64_t i = 0; i < rows; ++i) {
    const int64_t begin = a + i * x.pitch, end = begin + x.wide;
    int64_t j = begin - y.wide - b < 0 ? 0 : (begin - y.wide - b) / y.pitch + 1;  // first row that ends behind begin
    if (j < rows && b + j * y.pitch < end) return true;
  }
  return false;
}

}  // namespace

extern "C" {

int loca_head_loss_workspace_size(int64_t N, int64_t V, int64_t d, int32_t C, size_t* bytes) {
  clear();
  if (!bytes) return fail(LOCA_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = check_head(N, V, d);
  if (rc != LOCA_OK) return rc;
  if (C < 0 || C > 1024) return fail(LOCA_ERR_SHAPE, "need 0 <= C <= 1024, got %d", C);
  *bytes = head_loss_workspace_bytes(N, V, d, C);
  return LOCA_OK;
}

int loca_head_loss(const void* H, int64_t ldh, int64_t N, int64_t d, const void* W, int64_t V, const int32_t* y,
                   const float* w, const int32_t* label_cols, int32_t C, float* loss, float* lse, float* E,
                   void* workspace, size_t workspace_bytes, void* stream) {
  clear();
  int rc = check_head(N, V, d);
  if (rc != LOCA_OK) return rc;
  if (C < 0 || C > 1024 || (E && C < 1)) return fail(LOCA_ERR_SHAPE, "E needs 1 <= C <= 1024 label columns, got %d", C);
  if (N == 0) return LOCA_OK;
  if (!H || !W || !y || !loss) return fail(LOCA_ERR_INVALID_ARG, "H, W, y and loss are required");
  if (E && !label_cols) return fail(LOCA_ERR_INVALID_ARG, "E needs label_cols");
  if (ldh < d) return fail(LOCA_ERR_SHAPE, "row pitch of H %lld is below d = %lld", (long long)ldh, (long long)d);
  if (ldh % 8 != 0 || !aligned(H, 16) || !aligned(W, 16))
    return fail(LOCA_ERR_ALIGNMENT, "H and W need 16-byte alignment and a row pitch that is a multiple of 8");
  if (!aligned(y, 4) || !aligned(w, 4) || !aligned(label_cols, 4) || !aligned(loss, 4) || !aligned(lse, 4) ||
      !aligned(E, 4))
    return fail(LOCA_ERR_ALIGNMENT, "y, w, label_cols, loss, lse and E need 4-byte alignment");
  rc = check_ws(workspace, workspace_bytes, head_loss_workspace_bytes(N, V, d, C));
  if (rc != LOCA_OK) return rc;
  int32_t* status = device_status_word();
  if (!status) return fail(LOCA_ERR_CUDA, "cannot resolve the device status word");
  const cudaError_t e = launch_head_loss(H, ldh, N, d, W, V, y, w, label_cols, C, loss, lse, E, workspace, status,
                                         static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "loca_head_loss launch");
  return LOCA_OK;
}

int loca_head_loss_backward_workspace_size(int64_t N, int64_t V, int64_t d, int want_dH, int want_dW, size_t* bytes) {
  clear();
  if (!bytes) return fail(LOCA_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = check_head(N, V, d);
  if (rc != LOCA_OK) return rc;
  *bytes = head_loss_backward_workspace_bytes(N, V, d, want_dH != 0, want_dW != 0);
  return LOCA_OK;
}

int loca_head_loss_backward(const void* H, int64_t ldh, int64_t N, int64_t d, const void* W, int64_t V,
                            const int32_t* y, const float* w, const float* lse, const float* dloss, float grad_scale,
                            void* dH, int64_t lddh, void* dW, void* workspace, size_t workspace_bytes, void* stream) {
  clear();
  int rc = check_head(N, V, d);
  if (rc != LOCA_OK) return rc;
  if (!dH && !dW) return fail(LOCA_ERR_INVALID_ARG, "dH or dW is required");
  if (N == 0 && !dW) return LOCA_OK;
  if (!W || (N > 0 && (!H || !y || !lse))) return fail(LOCA_ERR_INVALID_ARG, "H, W, y and lse are required");
  if (N > 0 && (ldh < d || (dH && lddh < d)))
    return fail(LOCA_ERR_SHAPE, "row pitch of H %lld or dH %lld is below d = %lld", (long long)ldh, (long long)lddh,
                (long long)d);
  if ((N > 0 && (ldh % 8 != 0 || (dH && lddh % 8 != 0))) || !aligned(H, 16) || !aligned(W, 16) || !aligned(dH, 16) ||
      !aligned(dW, 16))
    return fail(LOCA_ERR_ALIGNMENT, "H, W, dH and dW need 16-byte alignment and row pitches that are multiples of 8");
  if (!aligned(y, 4) || !aligned(w, 4) || !aligned(lse, 4) || !aligned(dloss, 4))
    return fail(LOCA_ERR_ALIGNMENT, "y, w, lse and dloss need 4-byte alignment");
  if (!std::isfinite(grad_scale)) return fail(LOCA_ERR_INVALID_ARG, "grad_scale must be finite");
  rc = check_ws(workspace, workspace_bytes, head_loss_backward_workspace_bytes(N, V, d, dH != nullptr, dW != nullptr));
  if (rc != LOCA_OK) return rc;
  if (N > 0 && (dH != H || lddh != ldh) && overlap({H, 2 * ldh, 2 * d}, {dH, 2 * lddh, 2 * d}, N))
    return fail(LOCA_ERR_INVALID_ARG, "dH must be H itself or not overlap it");
  int32_t* status = device_status_word();
  if (!status) return fail(LOCA_ERR_CUDA, "cannot resolve the device status word");
  const cudaError_t e = launch_head_loss_backward(H, ldh, N, d, W, V, y, w, lse, dloss, grad_scale, N > 0 ? dH : nullptr,
                                                  lddh, dW, workspace, status, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "loca_head_loss_backward launch");
  return LOCA_OK;
}

int loca_adapter_packed_size(int32_t n, int64_t d_in, int64_t d_out, int32_t k, size_t* bytes) {
  clear();
  if (!bytes) return fail(LOCA_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = check_adapter(0, d_in, d_out, k, n);
  if (rc != LOCA_OK) return rc;
  *bytes = adapter_packed_bytes(n, d_in, d_out, k);
  return LOCA_OK;
}

int loca_adapter_pack(const void* A, const void* B, int dtype, int32_t n, int64_t d_in, int64_t d_out, int32_t k,
                      const float* scale, void* packed, void* stream) {
  clear();
  if (dtype != LOCA_F32 && dtype != LOCA_BF16) return fail(LOCA_ERR_UNSUPPORTED_DTYPE, "unknown dtype code %d", dtype);
  const int rc = check_adapter(0, d_in, d_out, k, n);
  if (rc != LOCA_OK) return rc;
  if (!A || !B || !packed) return fail(LOCA_ERR_INVALID_ARG, "A, B and packed are required");
  const size_t es = dtype == LOCA_F32 ? 4 : 2;
  if (!aligned(A, es) || !aligned(B, es) || !aligned(scale, 4) || !aligned(packed, 256))
    return fail(LOCA_ERR_ALIGNMENT, "A, B and scale need the alignment of their elements, packed 256 bytes");
  const cudaError_t e =
      launch_adapter_pack(A, B, dtype, n, d_in, d_out, k, scale, packed, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "loca_adapter_pack launch");
  return LOCA_OK;
}

int loca_adapter_plan_size(int64_t N, int32_t n, size_t* bytes) {
  clear();
  if (!bytes) return fail(LOCA_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = check_adapter(N, 8, 8, 1, n);
  if (rc != LOCA_OK) return rc;
  *bytes = adapter_plan_bytes(N, n);
  return LOCA_OK;
}

int loca_adapter_plan(const int32_t* ids, int64_t N, int32_t n, void* plan, void* stream) {
  clear();
  const int rc = check_adapter(N, 8, 8, 1, n);
  if (rc != LOCA_OK) return rc;
  if (N == 0) return LOCA_OK;
  if (!ids || !plan) return fail(LOCA_ERR_INVALID_ARG, "ids and plan are required");
  if (!aligned(ids, 4) || !aligned(plan, 256))
    return fail(LOCA_ERR_ALIGNMENT, "ids needs 4-byte, plan 256-byte alignment");
  const cudaError_t e = launch_adapter_plan(ids, N, n, plan, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "loca_adapter_plan launch");
  return LOCA_OK;
}

int loca_adapter_workspace_size(int64_t N, int64_t d_in, int64_t d_out, int32_t k, int32_t n, int backward,
                                size_t* bytes) {
  clear();
  if (!bytes) return fail(LOCA_ERR_INVALID_ARG, "bytes is NULL");
  const int rc = check_adapter(N, d_in, d_out, k, n);
  if (rc != LOCA_OK) return rc;
  *bytes = adapter_workspace_bytes(N, d_in, d_out, k, n, backward != 0);
  return LOCA_OK;
}

int loca_adapter_apply(const void* X, int64_t ldx, int64_t N, int64_t d_in, const void* W, int64_t d_out,
                       const void* packed, int32_t n, int32_t k, const void* plan, void* Y, int64_t ldy,
                       void* workspace, size_t workspace_bytes, void* stream) {
  clear();
  int rc = check_adapter(N, d_in, d_out, k, n);
  if (rc != LOCA_OK) return rc;
  if (N == 0) return LOCA_OK;
  if (!X || !W || !packed || !plan || !Y) return fail(LOCA_ERR_INVALID_ARG, "X, W, packed, plan and Y are required");
  if ((rc = check_rows(X, ldx, d_in, "X")) != LOCA_OK || (rc = check_rows(Y, ldy, d_out, "Y")) != LOCA_OK ||
      (rc = check_rows(W, d_in, d_in, "W")) != LOCA_OK)
    return rc;
  if (!aligned(packed, 256) || !aligned(plan, 256))
    return fail(LOCA_ERR_ALIGNMENT, "packed and plan need 256-byte alignment");
  rc = check_ws(workspace, workspace_bytes, adapter_workspace_bytes(N, d_in, d_out, k, n, false));
  if (rc != LOCA_OK) return rc;
  if (overlap({X, 2 * ldx, 2 * d_in}, {Y, 2 * ldy, 2 * d_out}, N))
    return fail(LOCA_ERR_INVALID_ARG, "Y must not overlap X");
  int32_t* status = device_status_word();
  if (!status) return fail(LOCA_ERR_CUDA, "cannot resolve the device status word");
  const cudaError_t e = launch_adapter_apply(X, ldx, N, d_in, W, d_out, packed, n, k, plan, Y, ldy, workspace, status,
                                             static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "loca_adapter_apply launch");
  return LOCA_OK;
}

int loca_adapter_backward(const void* X, int64_t ldx, const void* dY, int64_t lddy, int64_t N, int64_t d_in,
                          const void* W, int64_t d_out, const void* packed, int32_t n, int32_t k, const void* plan,
                          void* dX, int64_t lddx, void* dA, void* dB, int grad_dtype, void* workspace,
                          size_t workspace_bytes, void* stream) {
  clear();
  int rc = check_adapter(N, d_in, d_out, k, n);
  if (rc != LOCA_OK) return rc;
  if (grad_dtype != LOCA_F32 && grad_dtype != LOCA_BF16)
    return fail(LOCA_ERR_UNSUPPORTED_DTYPE, "unknown dtype code %d", grad_dtype);
  if (!dX && !dA && !dB) return fail(LOCA_ERR_INVALID_ARG, "one of dX, dA and dB is required");
  const size_t es = grad_dtype == LOCA_F32 ? 4 : 2;
  if (!aligned(dA, es) || !aligned(dB, es))
    return fail(LOCA_ERR_ALIGNMENT, "dA and dB need the alignment of their elements");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (N == 0) {  // sums over no token
    cudaError_t e = dA ? cudaMemsetAsync(dA, 0, es * size_t(n) * size_t(d_in) * size_t(k), s) : cudaSuccess;
    if (e == cudaSuccess && dB) e = cudaMemsetAsync(dB, 0, es * size_t(n) * size_t(d_out) * size_t(k), s);
    return e == cudaSuccess ? int(LOCA_OK) : cuda_fail(e, "loca_adapter_backward memset");
  }
  if (!X || !dY || !W || !packed || !plan) return fail(LOCA_ERR_INVALID_ARG, "X, dY, W, packed and plan are required");
  if ((rc = check_rows(X, ldx, d_in, "X")) != LOCA_OK || (rc = check_rows(dY, lddy, d_out, "dY")) != LOCA_OK ||
      (rc = check_rows(W, d_in, d_in, "W")) != LOCA_OK || (dX && (rc = check_rows(dX, lddx, d_in, "dX")) != LOCA_OK))
    return rc;
  if (!aligned(packed, 256) || !aligned(plan, 256))
    return fail(LOCA_ERR_ALIGNMENT, "packed and plan need 256-byte alignment");
  rc = check_ws(workspace, workspace_bytes, adapter_workspace_bytes(N, d_in, d_out, k, n, true));
  if (rc != LOCA_OK) return rc;
  if (dX && (overlap({dY, 2 * lddy, 2 * d_out}, {dX, 2 * lddx, 2 * d_in}, N) ||
             ((dA || dB) && overlap({X, 2 * ldx, 2 * d_in}, {dX, 2 * lddx, 2 * d_in}, N))))
    return fail(LOCA_ERR_INVALID_ARG, "dX must not overlap dY, nor X where dA or dB is wanted");
  int32_t* status = device_status_word();
  if (!status) return fail(LOCA_ERR_CUDA, "cannot resolve the device status word");
  const cudaError_t e = launch_adapter_backward(X, ldx, dY, lddy, N, d_in, W, d_out, packed, n, k, plan, dX, lddx, dA, dB,
                                                grad_dtype, workspace, status, s);
  if (e != cudaSuccess) return cuda_fail(e, "loca_adapter_backward launch");
  return LOCA_OK;
}

int loca_grad_clip_workspace_size(int32_t n, size_t* bytes) {
  clear();
  if (!bytes) return fail(LOCA_ERR_INVALID_ARG, "bytes is NULL");
  if (n < 0 || n > 100000) return fail(LOCA_ERR_SHAPE, "need 0 <= n <= 100000 tensors, got %d", n);
  *bytes = grad_clip_workspace_bytes(n);
  return LOCA_OK;
}

int loca_grad_clip(const void* const* grads, void* const* out, const int64_t* numel, const int32_t* dtype, int32_t n,
                   float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  clear();
  if (n < 0 || n > 100000) return fail(LOCA_ERR_SHAPE, "need 0 <= n <= 100000 tensors, got %d", n);
  if (!(max_norm > 0.f)) return fail(LOCA_ERR_INVALID_ARG, "max_norm must be positive");
  if (!norm || (n > 0 && (!grads || !numel || !dtype)))
    return fail(LOCA_ERR_INVALID_ARG, "grads, numel, dtype and norm are required");
  if (!aligned(norm, 4)) return fail(LOCA_ERR_ALIGNMENT, "norm needs 4-byte alignment");
  int64_t total = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (dtype[i] != LOCA_F32 && dtype[i] != LOCA_BF16)
      return fail(LOCA_ERR_UNSUPPORTED_DTYPE, "tensor %d has unknown dtype code %d", i, dtype[i]);
    if (numel[i] < 0 || numel[i] > grad_clip_max_numel() || (total += numel[i]) > grad_clip_max_numel())
      return fail(LOCA_ERR_SHAPE, "tensor %d: element counts must be >= 0 and sum to at most %lld", i,
                  (long long)grad_clip_max_numel());
    const size_t es = dtype[i] == LOCA_F32 ? 4 : 2;
    if (numel[i] > 0 && (!grads[i] || (out && !out[i]))) return fail(LOCA_ERR_INVALID_ARG, "tensor %d is NULL", i);
    if (!aligned(grads[i], es) || (out && !aligned(out[i], es)))
      return fail(LOCA_ERR_ALIGNMENT, "tensor %d needs the alignment of its elements", i);
  }
  const int rc = check_ws(workspace, workspace_bytes, grad_clip_workspace_bytes(n));
  if (rc != LOCA_OK) return rc;
  const cudaError_t e = launch_grad_clip(grads, out, numel, dtype, n, max_norm, norm, workspace,
                                         static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "loca_grad_clip launch");
  return LOCA_OK;
}

}  // extern "C"
