// The C ABI of the operators around the heads: the residual sum and RMS norm
// and their gradient, quantisation to 8 bits, the 8-bit product, and the
// latent layer that has its projections in 8 bits.  As in api.cpp: arguments
// are checked before anything is enqueued, nothing is allocated and nothing
// waits.

#include <cmath>

#include "api_internal.hpp"
#include "scaled_launch.hpp"

using namespace mhl::api;

namespace {

mhlmoe_status check_dtype(mhlmoe_dtype dtype) {
  if (dtype != MHLMOE_F32 && dtype != MHLMOE_BF16)
    return fail(MHLMOE_EINVAL, "unknown dtype %d", (int)dtype);
  return MHLMOE_OK;
}

mhlmoe_status check_norm(int64_t T, int d_model, float eps, mhlmoe_dtype dtype) {
  if (T < 0) return fail(MHLMOE_EINVAL, "T must be >= 0 (got %lld)", (long long)T);
  if (T >= int64_t(1) << 31) return fail(MHLMOE_EUNSUPPORTED, "T must be < 2^31");
  if (d_model < 1 || d_model > 65536)
    return fail(MHLMOE_EUNSUPPORTED, "d_model must be in [1, 65536] (got %d)", d_model);
  if (!std::isfinite(eps) || eps <= 0.0f)
    return fail(MHLMOE_EINVAL, "eps must be finite and > 0");
  return check_dtype(dtype);
}

size_t rmsnorm_bwd_bytes(int64_t T, int d_model, size_t* rows_at) {
  size_t cur = 0;
  bump(cur, sizeof(float) * (size_t)mhl::rmsnorm_bwd_parts(T, d_model) * d_model);
  const size_t at = bump(cur, mhl::rmsnorm_bwd_wide(d_model) ? 2 * sizeof(float) * (size_t)T : 0);
  if (rows_at) *rows_at = at;
  return cur;
}

mhlmoe_status check_workspace(const void* ws, size_t have, size_t need_bytes) {
  if (need_bytes == 0) return MHLMOE_OK;
  if (ws == nullptr) return fail(MHLMOE_EWORKSPACE, "workspace is NULL (need %zu bytes)", need_bytes);
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0)
    return fail(MHLMOE_EINVAL, "workspace is not 256-byte aligned");
  if (have < need_bytes)
    return fail(MHLMOE_EWORKSPACE, "workspace has %zu bytes, need %zu", have, need_bytes);
  return MHLMOE_OK;
}

// Fewer than 2^24 workgroups (a launch's threads are counted in 32 bits); a and b
// below 2^31, so that their product is exact.
bool fits_grid(int64_t a, int64_t b) { return a * b < int64_t(1) << 24; }

mhlmoe_status check_gemm(int64_t M, int64_t N, int64_t K, int b_block_rows) {
  if (M < 0 || N < 0 || K < 0)
    return fail(MHLMOE_EINVAL, "M, N and K must be >= 0 (got %lld, %lld, %lld)", (long long)M,
                (long long)N, (long long)K);
  if (K % 16 != 0) return fail(MHLMOE_EUNSUPPORTED, "K %lld is no multiple of 16", (long long)K);
  if (b_block_rows != 1 && b_block_rows != 128)
    return fail(MHLMOE_EINVAL, "b_block_rows must be 1 or 128 (got %d)", b_block_rows);
  const int64_t most = int64_t(1) << 31;
  if (M >= most || N >= most || K >= (int64_t(1) << 23) ||
      !fits_grid(mhl::ceil_div(M, 128), mhl::ceil_div(N, 128)))
    return fail(MHLMOE_EUNSUPPORTED,
                "product too large: M, N < 2^31, K < 2^23, ceil(M/128) ceil(N/128) < 2^24");
  return MHLMOE_OK;
}

mhlmoe_status run_gemm(const char* name, const void* A, const float* scale_a, const void* B,
                       const float* scale_b, int64_t M, int64_t N, int64_t K, int b_block_rows,
                       mhlmoe_dtype dtype, void* C, hipStream_t stream) {
  if (M == 0 || N == 0) return MHLMOE_OK;
  return run_kernel(name, stream, [&] {
    return mhl::launch_gemm_scaled(A, scale_a, B, scale_b, M, N, K, b_block_rows == 1,
                                   dtype == MHLMOE_F32, C, stream);
  });
}

// The workspace of mhlmoe_latent_layer_scaled: the layer's own first.
struct ScaledLayout {
  size_t layer_bytes = 0, lat_x = 0, lat_r = 0, lat_y = 0, xq = 0, xs = 0, yq = 0, ys = 0, total = 0;
};

mhlmoe_status scaled_layout(int64_t T, int d_model, int n_heads, int d_head, int n_experts,
                            int top_k, int d_ff, mhlmoe_dtype dtype, ScaledLayout* L) {
  if (d_model < 16 || d_model > 65536 || d_model % 16 != 0)
    return fail(MHLMOE_EUNSUPPORTED, "d_model must be a multiple of 16 in [16, 65536] (got %d)",
                d_model);
  MHL_TRY(mhlmoe_workspace_size(MHLMOE_OP_LAYER, T, n_heads, d_head, n_experts, top_k, d_ff, dtype,
                                &L->layer_bytes));
  const int64_t N = (int64_t)n_heads * d_head;
  MHL_TRY(check_gemm(T, N > d_model ? N : d_model, 16, 128));
  size_t cur = 0;
  bump(cur, L->layer_bytes);
  const size_t lat = (dtype == MHLMOE_F32 ? 4 : 2) * (size_t)T * N;
  L->lat_x = bump(cur, lat);
  L->lat_r = bump(cur, lat);
  L->lat_y = bump(cur, lat);
  L->xq = bump(cur, (size_t)T * d_model);
  L->xs = bump(cur, sizeof(float) * (size_t)T * mhl::ceil_div(d_model, 128));
  L->yq = bump(cur, (size_t)T * N);
  L->ys = bump(cur, sizeof(float) * (size_t)T * mhl::ceil_div(N, 128));
  L->total = cur;
  return MHLMOE_OK;
}

}  // namespace

extern "C" {

mhlmoe_status mhlmoe_rmsnorm(const void* x, const void* residual, const float* weight, int64_t T,
                             int d_model, float eps, mhlmoe_dtype dtype, void* sum, void* y,
                             void* q, float* scales, hipStream_t stream) {
  clear_error();
  MHL_TRY(check_norm(T, d_model, eps, dtype));
  MHL_TRY(need_rows(x, "x", T));
  MHL_TRY(maybe(residual, "residual"));
  MHL_TRY(need(weight, "weight"));
  MHL_TRY(maybe(sum, "sum"));
  MHL_TRY(maybe(y, "y"));
  MHL_TRY(maybe(q, "q"));
  MHL_TRY(maybe(scales, "scales"));
  if (T == 0) return MHLMOE_OK;
  if ((residual == nullptr) != (sum == nullptr))
    return fail(MHLMOE_EINVAL, "residual and sum go together: %s is NULL",
                sum == nullptr ? "sum" : "residual");
  if ((q == nullptr) != (scales == nullptr))
    return fail(MHLMOE_EINVAL, "q and scales go together: %s is NULL",
                q == nullptr ? "q" : "scales");
  if (y == nullptr && q == nullptr) return fail(MHLMOE_EINVAL, "y and q are both NULL");
  if (y != nullptr && (y == sum || y == residual))
    return fail(MHLMOE_EINVAL, "y must not be sum or residual");
  if (q != nullptr && d_model % 16 != 0)
    return fail(MHLMOE_EUNSUPPORTED, "8-bit output: d_model %d is no multiple of 16", d_model);
  return run_kernel("rmsnorm", stream, [&] {
    return mhl::launch_rmsnorm(x, residual, weight, T, d_model, eps, dtype == MHLMOE_F32, sum, y, q,
                               scales, stream);
  });
}

mhlmoe_status mhlmoe_rmsnorm_backward_workspace(int64_t T, int d_model, size_t* bytes) {
  clear_error();
  if (bytes == nullptr) return fail(MHLMOE_EINVAL, "bytes is NULL");
  MHL_TRY(check_norm(T, d_model, 1.0f, MHLMOE_F32));
  *bytes = rmsnorm_bwd_bytes(T, d_model, nullptr);
  return MHLMOE_OK;
}

mhlmoe_status mhlmoe_rmsnorm_backward(const void* h, const float* weight, const void* dy,
                                      const void* dsum, int64_t T, int d_model, float eps,
                                      mhlmoe_dtype dtype, void* dx, float* dweight, void* workspace,
                                      size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  MHL_TRY(check_norm(T, d_model, eps, dtype));
  MHL_TRY(need_rows(h, "h", T));
  MHL_TRY(need(weight, "weight"));
  MHL_TRY(need_rows(dy, "dy", T));
  MHL_TRY(maybe(dsum, "dsum"));
  MHL_TRY(need_rows(dx, "dx", T));
  MHL_TRY(need(dweight, "dweight"));
  if (T > 0 && dx == h) return fail(MHLMOE_EINVAL, "dx must not be h");
  size_t rows_at = 0;
  MHL_TRY(check_workspace(workspace, workspace_bytes, rmsnorm_bwd_bytes(T, d_model, &rows_at)));
  float* part = at<float>(workspace, 0);
  if (T > 0)
    MHL_TRY(run_kernel("rmsnorm_bwd", stream, [&] {
      return mhl::launch_rmsnorm_bwd(h, weight, dy, dsum, T, d_model, eps, dtype == MHLMOE_F32, dx,
                                     part, at<float>(workspace, rows_at), stream);
    }));
  return run_kernel("rmsnorm_dw", stream, [&] {
    return mhl::launch_rmsnorm_dw(part, mhl::rmsnorm_bwd_parts(T, d_model), d_model, dweight,
                                  stream);
  });
}

mhlmoe_status mhlmoe_quantize(const void* x, int64_t rows, int64_t cols, mhlmoe_dtype dtype,
                              int block_rows, int transpose, void* q, float* scales,
                              hipStream_t stream) {
  clear_error();
  MHL_TRY(check_dtype(dtype));
  if (rows < 0 || cols < 0)
    return fail(MHLMOE_EINVAL, "rows and cols must be >= 0 (got %lld, %lld)", (long long)rows,
                (long long)cols);
  if (block_rows != 1 && block_rows != 128)
    return fail(MHLMOE_EINVAL, "block_rows must be 1 or 128 (got %d)", block_rows);
  if (transpose != 0 && transpose != 1)
    return fail(MHLMOE_EINVAL, "transpose must be 0 or 1 (got %d)", transpose);
  if (cols % 16 != 0)
    return fail(MHLMOE_EUNSUPPORTED, "cols %lld is no multiple of 16", (long long)cols);
  const int64_t most = int64_t(1) << 31;
  // 1 x 128 blocks of x's rows are counted in 32 bits, tiles as workgroups
  if (rows >= most || cols >= most ||
      !(block_rows == 1 && !transpose
            ? rows * mhl::ceil_div(cols, 128) < int64_t(1) << 32
            : fits_grid(mhl::ceil_div(rows, 128), mhl::ceil_div(cols, 128))))
    return fail(MHLMOE_EUNSUPPORTED, "%lld x %lld is too large", (long long)rows, (long long)cols);
  const int64_t n = rows == 0 || cols == 0 ? 0 : 1;
  MHL_TRY(need_rows(x, "x", n));
  MHL_TRY(need_rows(q, "q", n));
  MHL_TRY(need_rows(scales, "scales", n));
  if (n == 0) return MHLMOE_OK;
  return run_kernel("quantize", stream, [&] {
    return mhl::launch_quantize(x, rows, cols, dtype == MHLMOE_F32, block_rows, transpose != 0, q,
                                scales, stream);
  });
}

mhlmoe_status mhlmoe_gemm_scaled(const void* A, const float* scale_a, const void* B,
                                 const float* scale_b, int64_t M, int64_t N, int64_t K,
                                 int b_block_rows, mhlmoe_dtype out_dtype, void* C,
                                 hipStream_t stream) {
  clear_error();
  MHL_TRY(check_dtype(out_dtype));
  MHL_TRY(check_gemm(M, N, K, b_block_rows));
  MHL_TRY(need_rows(A, "A", M * K));
  MHL_TRY(need_rows(scale_a, "scale_a", M * K));
  MHL_TRY(need_rows(B, "B", N * K));
  MHL_TRY(need_rows(scale_b, "scale_b", N * K));
  MHL_TRY(need_rows(C, "C", M == 0 ? 0 : N));
  return run_gemm("gemm_scaled", A, scale_a, B, scale_b, M, N, K, b_block_rows, out_dtype, C,
                  stream);
}

mhlmoe_status mhlmoe_latent_layer_scaled_workspace(int64_t T, int d_model, int n_heads, int d_head,
                                                   int n_experts, int top_k, int d_ff,
                                                   mhlmoe_dtype dtype, size_t* bytes) {
  clear_error();
  if (bytes == nullptr) return fail(MHLMOE_EINVAL, "bytes is NULL");
  ScaledLayout L;
  MHL_TRY(scaled_layout(T, d_model, n_heads, d_head, n_experts, top_k, d_ff, dtype, &L));
  *bytes = L.total;
  return MHLMOE_OK;
}

mhlmoe_status mhlmoe_latent_layer_scaled(
    const void* x, const void* residual, const float* norm_weight, float eps, const void* W_in,
    const float* scale_in, const void* W_r, const float* scale_r, const float* W_router,
    const float* bias, const void* W1, const void* W3, const void* W2, const void* W_out,
    const float* scale_out, int64_t T, int d_model, int n_heads, int d_head, int n_experts,
    int top_k, int d_ff, mhlmoe_dtype dtype, void* out, void* sum, void* X_lat, void* R_lat,
    void* Y_lat, int32_t* idx, float* gate, int32_t* counts, void* workspace,
    size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  ScaledLayout L;
  MHL_TRY(scaled_layout(T, d_model, n_heads, d_head, n_experts, top_k, d_ff, dtype, &L));
  MHL_TRY(check_norm(T, d_model, eps, dtype));
  MHL_TRY(need_rows(x, "x", T));
  MHL_TRY(maybe(residual, "residual"));
  MHL_TRY(maybe(sum, "sum"));
  if (T > 0 && (residual == nullptr) != (sum == nullptr))
    return fail(MHLMOE_EINVAL, "residual and sum go together: %s is NULL",
                sum == nullptr ? "sum" : "residual");
  MHL_TRY(need(norm_weight, "norm_weight"));
  MHL_TRY(need(W_in, "W_in"));
  MHL_TRY(need(scale_in, "scale_in"));
  MHL_TRY(maybe(W_r, "W_r"));
  if (W_r != nullptr) MHL_TRY(need(scale_r, "scale_r"));
  MHL_TRY(need(W_router, "W_router"));
  MHL_TRY(maybe(bias, "bias"));
  MHL_TRY(need(W1, "W1"));
  MHL_TRY(maybe(W3, "W3"));
  MHL_TRY(need(W2, "W2"));
  MHL_TRY(need(W_out, "W_out"));
  MHL_TRY(need(scale_out, "scale_out"));
  MHL_TRY(need_rows(out, "out", T));
  MHL_TRY(maybe(X_lat, "X_lat"));
  MHL_TRY(maybe(R_lat, "R_lat"));
  MHL_TRY(maybe(Y_lat, "Y_lat"));
  MHL_TRY(maybe(idx, "idx"));
  MHL_TRY(maybe(gate, "gate"));
  MHL_TRY(maybe(counts, "counts"));
  MHL_TRY(check_workspace(workspace, workspace_bytes, L.total));
  const bool f32 = dtype == MHLMOE_F32;
  const int64_t N = (int64_t)n_heads * d_head;
  if (X_lat == nullptr) X_lat = at<void>(workspace, L.lat_x);
  if (R_lat == nullptr) R_lat = at<void>(workspace, L.lat_r);
  if (Y_lat == nullptr) Y_lat = at<void>(workspace, L.lat_y);
  if (W_r == nullptr) R_lat = X_lat;
  void* xq = at<void>(workspace, L.xq);
  float* xs = at<float>(workspace, L.xs);
  void* yq = at<void>(workspace, L.yq);
  float* ys = at<float>(workspace, L.ys);
  if (T > 0)
    MHL_TRY(run_kernel("rmsnorm", stream, [&] {
      return mhl::launch_rmsnorm(x, residual, norm_weight, T, d_model, eps, f32, sum, nullptr, xq,
                                 xs, stream);
    }));
  MHL_TRY(run_gemm("proj_in", xq, xs, W_in, scale_in, T, N, d_model, 128, dtype, X_lat, stream));
  if (W_r != nullptr)
    MHL_TRY(run_gemm("proj_in", xq, xs, W_r, scale_r, T, N, d_model, 128, dtype, R_lat, stream));
  MHL_TRY(mhlmoe_layer_routed(X_lat, R_lat, W_router, bias, W1, W3, W2, T, n_heads, d_head,
                              n_experts, top_k, d_ff, dtype, Y_lat, idx, gate, counts, workspace,
                              L.layer_bytes, stream));
  if (T > 0)
    MHL_TRY(run_kernel("quantize", stream, [&] {
      return mhl::launch_quantize(Y_lat, T, N, f32, 1, false, yq, ys, stream);
    }));
  return run_gemm("proj_out", yq, ys, W_out, scale_out, T, d_model, N, 128, dtype, out, stream);
}

}  // extern "C"
