// The C ABI of what a training step has around the layer: layer norm and its
// gradient, the experts' counts and the balance loss with its gradient, and AdamW.
// As in api.cpp: arguments are checked before anything is enqueued, nothing is
// allocated on the device and nothing waits.

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "api_internal.hpp"
#include "training_launch.hpp"

using namespace mhl::api;

namespace {

mhlmoe_status check_dtype(mhlmoe_dtype dtype, const char* name) {
  if (dtype != MHLMOE_F32 && dtype != MHLMOE_BF16)
    return fail(MHLMOE_EINVAL, "unknown %s %d", name, (int)dtype);
  return MHLMOE_OK;
}

mhlmoe_status check_norm(int64_t T, int d_model, float eps, mhlmoe_dtype dtype) {
  if (T < 0) return fail(MHLMOE_EINVAL, "T must be >= 0 (got %lld)", (long long)T);
  if (T >= int64_t(1) << 31) return fail(MHLMOE_EUNSUPPORTED, "T must be < 2^31");
  if (d_model < 1 || d_model > 65536)
    return fail(MHLMOE_EUNSUPPORTED, "d_model must be in [1, 65536] (got %d)", d_model);
  if (!std::isfinite(eps) || eps <= 0.0f)
    return fail(MHLMOE_EINVAL, "eps must be finite and > 0");
  return check_dtype(dtype, "dtype");
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

size_t layernorm_bwd_bytes(int64_t T, int d_model, size_t* rows_at) {
  size_t cur = 0;
  bump(cur, sizeof(float) * 2 * (size_t)mhl::layernorm_bwd_parts(T, d_model) * d_model);
  const size_t at = bump(cur, mhl::layernorm_bwd_wide(d_model)
                                  ? mhl::kLayernormRowFloats * sizeof(float) * (size_t)T
                                  : 0);
  if (rows_at) *rows_at = at;
  return cur;
}

mhlmoe_status check_heads(int64_t T, int n_heads, int n_experts) {
  if (T < 0) return fail(MHLMOE_EINVAL, "T must be >= 0 (got %lld)", (long long)T);
  if (n_heads < 1) return fail(MHLMOE_EINVAL, "n_heads must be >= 1 (got %d)", n_heads);
  if (n_heads > mhl::kMaxHeadsSupported)
    return fail(MHLMOE_EUNSUPPORTED, "n_heads must be <= %d", mhl::kMaxHeadsSupported);
  if (n_experts < 1) return fail(MHLMOE_EINVAL, "n_experts must be >= 1 (got %d)", n_experts);
  if (n_experts > 1024) return fail(MHLMOE_EUNSUPPORTED, "n_experts %d > 1024", n_experts);
  return MHLMOE_OK;
}

mhlmoe_status check_balance(int64_t T, int n_heads, int d_head, int n_experts) {
  MHL_TRY(check_heads(T, n_heads, n_experts));
  // (also the launches' limit: fewer than 2^24 workgroups of 128 rows)
  if (T > ((int64_t(1) << 31) - 1) / n_heads - 128)
    return fail(MHLMOE_EUNSUPPORTED, "(T + 128) * n_heads must be < 2^31");
  if (d_head != 64 && d_head != 128)
    return fail(MHLMOE_EUNSUPPORTED, "d_head %d not in {64, 128}", d_head);
  return MHLMOE_OK;
}

struct BalanceLayout {
  size_t weights = 0, part = 0, total = 0;
};
BalanceLayout balance_layout(int64_t T, int n_heads, int d_head, int n_experts, bool backward) {
  BalanceLayout L;
  size_t cur = 0;
  L.weights = bump(cur, mhl::balance_weight_bytes(n_heads, d_head, n_experts));
  // dW's partial results (none where there is one: it is dW), or the loss's
  const size_t splits = (size_t)mhl::balance_splits(T, n_heads, d_head, n_experts);
  L.part = bump(cur, backward ? (splits == 1 ? 0
                                             : sizeof(float) * splits * n_heads *
                                                   mhl::balance_blocks(n_experts) * 32 * d_head)
                              : sizeof(double) * (size_t)n_heads *
                                    mhl::balance_token_blocks(T, n_heads, n_experts));
  L.total = cur;
  return L;
}

// Memory that a step writes, or only reads.
struct Range {
  uintptr_t begin, end;
  int tensor;
  bool written;
};

size_t elem_size(mhlmoe_dtype d) { return d == MHLMOE_F32 ? 4 : 2; }

mhlmoe_status check_tensor(const mhlmoe_adamw_tensor& t, int i) {
  if (t.n < 0) return fail(MHLMOE_EINVAL, "tensor %d: n must be >= 0 (got %lld)", i, (long long)t.n);
  if (t.n >= int64_t(1) << 40) return fail(MHLMOE_EUNSUPPORTED, "tensor %d: n must be < 2^40", i);
  MHL_TRY(check_dtype(t.param_dtype, "param_dtype"));
  MHL_TRY(check_dtype(t.grad_dtype, "grad_dtype"));
  if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.0f)
    return fail(MHLMOE_EINVAL, "tensor %d: weight_decay must be finite and >= 0", i);
  MHL_TRY(need_rows(t.param, "param", t.n));
  MHL_TRY(maybe(t.master, "master"));
  MHL_TRY(need_rows(t.grad, "grad", t.n));
  MHL_TRY(need_rows(t.m, "m", t.n));
  MHL_TRY(need_rows(t.v, "v", t.n));
  MHL_TRY(maybe(t.m_scale, "m_scale"));
  MHL_TRY(maybe(t.v_scale, "v_scale"));
  if (t.master != nullptr && t.param_dtype == MHLMOE_F32)
    return fail(MHLMOE_EINVAL, "tensor %d: master goes with a bf16 param only", i);
  if ((t.m_scale == nullptr) != (t.v_scale == nullptr))
    return fail(MHLMOE_EINVAL, "tensor %d: m_scale and v_scale go together: %s is NULL", i,
                t.m_scale == nullptr ? "m_scale" : "v_scale");
  return MHLMOE_OK;
}

// What the step writes is written by one workgroup and read by no other.
mhlmoe_status check_apart(const mhlmoe_adamw_tensor* tensors, int n, const float* grad_scale) {
  std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[(size_t)n * 7 + 1]);
  if (!ranges) return fail(MHLMOE_EHIP, "no host memory for %d tensors", n);
  size_t count = 0;
  auto add = [&](const void* p, size_t bytes, int i, bool written) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    if (p != nullptr && bytes > 0) ranges[count++] = Range{a, a + bytes, i, written};
  };
  for (int i = 0; i < n; ++i) {
    const mhlmoe_adamw_tensor& t = tensors[i];
    const size_t m = (size_t)t.n, state = t.m_scale ? 1 : 4, blocks = 4 * ((m + 127) / 128);
    add(t.param, m * elem_size(t.param_dtype), i, true);
    add(t.master, m * 4, i, true);
    add(t.grad, m * elem_size(t.grad_dtype), i, false);
    add(t.m, m * state, i, true);
    add(t.v, m * state, i, true);
    add(t.m_scale, blocks, i, true);
    add(t.v_scale, blocks, i, true);
  }
  add(grad_scale, 4, -1, false);
  std::sort(ranges.get(), ranges.get() + count,
            [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t end = 0, written_end = 0;  // of the ranges so far
  for (size_t i = 0; i < count; ++i) {
    const Range& r = ranges[i];
    if (r.begin < written_end || (r.written && r.begin < end))
      return fail(MHLMOE_EINVAL, "tensor %d: memory that the step writes overlaps other memory of it",
                  r.tensor < 0 ? 0 : r.tensor);
    end = std::max(end, r.end);
    if (r.written) written_end = std::max(written_end, r.end);
  }
  return MHLMOE_OK;
}

}  // namespace

extern "C" {

mhlmoe_status mhlmoe_layernorm(const void* x, const void* residual, const float* weight,
                               const float* bias, int64_t T, int d_model, float eps,
                               mhlmoe_dtype dtype, void* sum, void* y, void* q, float* scales,
                               hipStream_t stream) {
  clear_error();
  MHL_TRY(check_norm(T, d_model, eps, dtype));
  MHL_TRY(need_rows(x, "x", T));
  MHL_TRY(maybe(residual, "residual"));
  MHL_TRY(need(weight, "weight"));
  MHL_TRY(maybe(bias, "bias"));
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
  return run_kernel("layernorm", stream, [&] {
    return mhl::launch_layernorm(x, residual, weight, bias, T, d_model, eps, dtype == MHLMOE_F32,
                                 sum, y, q, scales, stream);
  });
}

mhlmoe_status mhlmoe_layernorm_backward_workspace(int64_t T, int d_model, size_t* bytes) {
  clear_error();
  if (bytes == nullptr) return fail(MHLMOE_EINVAL, "bytes is NULL");
  MHL_TRY(check_norm(T, d_model, 1.0f, MHLMOE_F32));
  *bytes = layernorm_bwd_bytes(T, d_model, nullptr);
  return MHLMOE_OK;
}

mhlmoe_status mhlmoe_layernorm_backward(const void* h, const float* weight, const void* dy,
                                        const void* dsum, int64_t T, int d_model, float eps,
                                        mhlmoe_dtype dtype, void* dx, float* dweight, float* dbias,
                                        void* workspace, size_t workspace_bytes,
                                        hipStream_t stream) {
  clear_error();
  MHL_TRY(check_norm(T, d_model, eps, dtype));
  MHL_TRY(need_rows(h, "h", T));
  MHL_TRY(need(weight, "weight"));
  MHL_TRY(need_rows(dy, "dy", T));
  MHL_TRY(maybe(dsum, "dsum"));
  MHL_TRY(need_rows(dx, "dx", T));
  MHL_TRY(need(dweight, "dweight"));
  MHL_TRY(maybe(dbias, "dbias"));
  if (dbias == dweight) return fail(MHLMOE_EINVAL, "dbias must not be dweight");
  if (T > 0 && dx == h) return fail(MHLMOE_EINVAL, "dx must not be h");
  size_t rows_at = 0;
  MHL_TRY(check_workspace(workspace, workspace_bytes, layernorm_bwd_bytes(T, d_model, &rows_at)));
  float* part = at<float>(workspace, 0);
  if (T > 0)
    MHL_TRY(run_kernel("layernorm_bwd", stream, [&] {
      return mhl::launch_layernorm_bwd(h, weight, dy, dsum, T, d_model, eps, dtype == MHLMOE_F32,
                                       dx, part, at<float>(workspace, rows_at), stream);
    }));
  return run_kernel("layernorm_dw", stream, [&] {
    return mhl::launch_layernorm_dw(part, mhl::layernorm_bwd_parts(T, d_model), d_model, dweight,
                                    dbias, stream);
  });
}

mhlmoe_status mhlmoe_expert_counts(const int32_t* idx, const uint8_t* mask, int64_t T, int n_heads,
                                   int n_experts, int top_k, int32_t* counts, hipStream_t stream) {
  clear_error();
  MHL_TRY(check_heads(T, n_heads, n_experts));
  if (top_k < 1) return fail(MHLMOE_EINVAL, "top_k must be >= 1 (got %d)", top_k);
  if (top_k > 32) return fail(MHLMOE_EUNSUPPORTED, "top_k %d > 32", top_k);
  if (T > ((int64_t(1) << 31) - 1) / top_k)
    return fail(MHLMOE_EUNSUPPORTED, "T * top_k must be < 2^31");
  MHL_TRY(need_rows(idx, "idx", T));
  MHL_TRY(maybe(mask, "mask"));
  MHL_TRY(need(counts, "counts"));
  return run_kernel("expert_counts", stream, [&] {
    return mhl::launch_expert_counts(idx, mask, T, n_heads, n_experts, top_k, counts, stream);
  });
}

mhlmoe_status mhlmoe_balance_loss_workspace(int64_t T, int n_heads, int d_head, int n_experts,
                                            size_t* bytes) {
  clear_error();
  if (bytes == nullptr) return fail(MHLMOE_EINVAL, "bytes is NULL");
  MHL_TRY(check_balance(T, n_heads, d_head, n_experts));
  *bytes = balance_layout(T, n_heads, d_head, n_experts, false).total;
  return MHLMOE_OK;
}

mhlmoe_status mhlmoe_balance_loss(const void* X, const float* W_router, const int32_t* counts,
                                  const uint8_t* mask, int64_t T, int n_heads, int d_head,
                                  int n_experts, mhlmoe_dtype dtype, float* loss, float* stats,
                                  void* workspace, size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  MHL_TRY(check_balance(T, n_heads, d_head, n_experts));
  MHL_TRY(check_dtype(dtype, "dtype"));
  MHL_TRY(need_rows(X, "X", T));
  MHL_TRY(need(W_router, "W_router"));
  MHL_TRY(need(counts, "counts"));
  MHL_TRY(maybe(mask, "mask"));
  MHL_TRY(need(loss, "loss"));
  MHL_TRY(need(stats, "stats"));
  const BalanceLayout L = balance_layout(T, n_heads, d_head, n_experts, false);
  MHL_TRY(check_workspace(workspace, workspace_bytes, L.total));
  void* weights = at<void>(workspace, L.weights);
  double* part = at<double>(workspace, L.part);
  const bool few = mhl::balance_few(T, n_heads, n_experts);
  if (T > 0 && !few)
    MHL_TRY(run_kernel("balance_weights", stream, [&] {
      return mhl::launch_balance_weights(W_router, counts, n_heads, d_head, n_experts, weights,
                                         stream);
    }));
  if (T > 0)
    MHL_TRY(run_kernel("balance_loss", stream, [&] {
      return mhl::launch_balance_loss(X, W_router, weights, counts, mask, T, n_heads, d_head,
                                      n_experts, dtype == MHLMOE_F32, stats, part, loss, stream);
    }));
  if (mhl::balance_loss_at_once(T, n_heads, n_experts)) return MHLMOE_OK;
  return run_kernel("balance_sum", stream, [&] {
    return mhl::launch_balance_loss_sum(part, counts, mask, T, n_heads, n_experts, loss, stats,
                                        stream);
  });
}

mhlmoe_status mhlmoe_balance_loss_backward_workspace(int64_t T, int n_heads, int d_head,
                                                     int n_experts, size_t* bytes) {
  clear_error();
  if (bytes == nullptr) return fail(MHLMOE_EINVAL, "bytes is NULL");
  MHL_TRY(check_balance(T, n_heads, d_head, n_experts));
  *bytes = balance_layout(T, n_heads, d_head, n_experts, true).total;
  return MHLMOE_OK;
}

mhlmoe_status mhlmoe_balance_loss_backward(
    const void* X, const float* W_router, const int32_t* counts, const float* stats,
    const float* dloss, const uint8_t* mask, const void* dX_add, const float* dW_add, int64_t T,
    int n_heads, int d_head, int n_experts, mhlmoe_dtype dtype, void* dX, float* dW_router,
    void* workspace, size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  MHL_TRY(check_balance(T, n_heads, d_head, n_experts));
  MHL_TRY(check_dtype(dtype, "dtype"));
  MHL_TRY(need_rows(X, "X", T));
  MHL_TRY(need(W_router, "W_router"));
  MHL_TRY(need(counts, "counts"));
  MHL_TRY(need(stats, "stats"));
  MHL_TRY(need(dloss, "dloss"));
  MHL_TRY(maybe(mask, "mask"));
  MHL_TRY(maybe(dX_add, "dX_add"));
  MHL_TRY(maybe(dW_add, "dW_add"));
  MHL_TRY(need_rows(dX, "dX", T));
  MHL_TRY(need(dW_router, "dW_router"));
  if (T > 0 && dX == X) return fail(MHLMOE_EINVAL, "dX must not be X");
  if (dW_router == W_router) return fail(MHLMOE_EINVAL, "dW_router must not be W_router");
  const BalanceLayout L = balance_layout(T, n_heads, d_head, n_experts, true);
  MHL_TRY(check_workspace(workspace, workspace_bytes, L.total));
  void* weights = at<void>(workspace, L.weights);
  float* part = at<float>(workspace, L.part);
  const bool f32 = dtype == MHLMOE_F32;
  if (T > 0 && mhl::balance_few(T, n_heads, n_experts)) {
    MHL_TRY(run_kernel("balance_dx_dw", stream, [&] {
      return mhl::launch_balance_bwd_few(X, W_router, counts, stats, dloss, mask, dX_add, dW_add, T,
                                         n_heads, d_head, n_experts, f32, dX, dW_router, part,
                                         stream);
    }));
  } else if (T > 0) {
    MHL_TRY(run_kernel("balance_weights", stream, [&] {
      return mhl::launch_balance_weights(W_router, counts, n_heads, d_head, n_experts, weights,
                                         stream);
    }));
    if (mhl::balance_together(T, n_heads, d_head, n_experts)) {
      MHL_TRY(run_kernel("balance_dx_dw", stream, [&] {
        return mhl::launch_balance_dw_dx(X, W_router, weights, counts, stats, dloss, mask, dX_add,
                                         dW_add, T, n_heads, d_head, n_experts, f32, dX, dW_router,
                                         part, stream);
      }));
    } else {
      MHL_TRY(run_kernel("balance_dx", stream, [&] {
        return mhl::launch_balance_dx(X, weights, stats, dloss, mask, dX_add, T, n_heads, d_head,
                                      n_experts, f32, dX, stream);
      }));
      MHL_TRY(run_kernel("balance_dw", stream, [&] {
        return mhl::launch_balance_dw(X, W_router, counts, stats, dloss, mask, dW_add, T, n_heads,
                                      d_head, n_experts, f32, dW_router, part, stream);
      }));
    }
  }
  if (mhl::balance_splits(T, n_heads, d_head, n_experts) == 1) return MHLMOE_OK;
  return run_kernel("balance_sum", stream, [&] {
    return mhl::launch_balance_dw_sum(part, stats, dloss, dW_add, T, n_heads, d_head, n_experts,
                                      dW_router, stream);
  });
}

mhlmoe_status mhlmoe_adamw(const mhlmoe_adamw_tensor* tensors, int n_tensors,
                           const mhlmoe_adamw_step* step, hipStream_t stream) {
  clear_error();
  if (n_tensors < 0) return fail(MHLMOE_EINVAL, "n_tensors must be >= 0 (got %d)", n_tensors);
  if (n_tensors > 0 && tensors == nullptr) return fail(MHLMOE_EINVAL, "tensors is NULL");
  if (step == nullptr) return fail(MHLMOE_EINVAL, "step is NULL");
  if (!std::isfinite(step->lr) || step->lr < 0.0)
    return fail(MHLMOE_EINVAL, "lr must be finite and >= 0");
  if (!(step->beta1 >= 0.0 && step->beta1 < 1.0))
    return fail(MHLMOE_EINVAL, "beta1 must be in [0, 1)");
  if (!(step->beta2 >= 0.0 && step->beta2 < 1.0))
    return fail(MHLMOE_EINVAL, "beta2 must be in [0, 1)");
  if (!std::isfinite(step->eps) || (float)step->eps <= 0.0f)
    return fail(MHLMOE_EINVAL, "eps must be finite and > 0");
  if (step->step < 1)
    return fail(MHLMOE_EINVAL, "step must be >= 1 (got %lld)", (long long)step->step);
  if ((reinterpret_cast<uintptr_t>(step->grad_scale) & 3u) != 0)
    return fail(MHLMOE_EINVAL, "grad_scale is not 4-byte aligned");
  for (int i = 0; i < n_tensors; ++i) MHL_TRY(check_tensor(tensors[i], i));
  MHL_TRY(check_apart(tensors, n_tensors, step->grad_scale));
  mhl::AdamLaunch a;
  a.step.beta1 = (float)step->beta1;
  a.step.beta2 = (float)step->beta2;
  a.step.rest1 = (float)(1.0 - step->beta1);
  a.step.rest2 = (float)(1.0 - step->beta2);
  a.step.rate = (float)(step->lr / (1.0 - std::pow(step->beta1, (double)step->step)));
  a.step.root = (float)(1.0 / std::sqrt(1.0 - std::pow(step->beta2, (double)step->step)));
  a.step.eps = (float)step->eps;
  a.step.grad_scale = step->grad_scale;
  for (int i = 0; i < n_tensors;) {
    // the next tensors that are not empty
    int used = 0;
    int64_t workgroups = 0;
    const int begin = i;
    a.chunk = mhl::kAdamChunk;
    for (;;) {
      used = 0, workgroups = 0;
      for (i = begin; i < n_tensors && used < mhl::kAdamTensors; ++i) {
        const mhlmoe_adamw_tensor& t = tensors[i];
        if (t.n == 0) continue;
        a.first[used] = (uint32_t)workgroups;
        a.t[used] = mhl::AdamTensor{t.param, t.master, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.n,
                                    (float)(step->lr * (double)t.weight_decay),
                                    mhl::adam_key(t.seed, step->step),
                                    (uint8_t)(t.param_dtype == MHLMOE_BF16),
                                    (uint8_t)(t.grad_dtype == MHLMOE_BF16)};
        workgroups += mhl::ceil_div(t.n, a.chunk);
        ++used;
      }
      if (workgroups < int64_t(1) << 23) break;  // a launch's threads are counted in 32 bits
      a.chunk *= 2;
    }
    if (used == 0) break;
    for (int j = used; j < mhl::kAdamTensors; ++j) {
      a.first[j] = UINT32_MAX;
      a.t[j] = mhl::AdamTensor{};
    }
    MHL_TRY(run_kernel("adamw", stream,
                       [&] { return mhl::launch_adamw(a, (unsigned)workgroups, stream); }));
  }
  return MHLMOE_OK;
}

}  // extern "C"
