// Launch interface of the training step's operators (api_training.cpp) to their
// kernels: layer norm and its gradient, the experts' counts and balance loss and
// its gradient, and AdamW.  As in launch.hpp, a launcher only enqueues work on its
// stream and gets shapes that the ABI layer has validated.
#pragma once

#include "mhlmoe.h"
#include "scaled_launch.hpp"

namespace mhl {

// As launch_rmsnorm; b may be NULL.
hipError_t launch_layernorm(const void* x, const void* residual, const float* w, const float* b,
                            int64_t T, int d, float eps, bool f32, void* sum, void* y, void* q,
                            float* scales, hipStream_t s);

// Rows are held as the RMS norm's of the next multiple of 8 (NormForm; the wide ones of
// no multiple of 8 column by column).
inline NormForm layernorm_form(int d) { return norm_form((d + 7) / 8 * 8); }
inline bool layernorm_bwd_wide(int d) { return layernorm_form(d) >= NormForm::kLarge8; }

// The gradient: dx, and dw and db as layernorm_bwd_parts partial rows of 2 d floats,
// which launch_layernorm_dw adds in order (db may be NULL).  rows:
// kLayernormRowFloats T floats where layernorm_bwd_wide, else unused.
constexpr int kLayernormRowFloats = 5;
inline int64_t layernorm_bwd_parts(int64_t T, int d) {
  const int padded = (d + 7) / 8 * 8;
  if (!layernorm_bwd_wide(d)) {
    // A workgroup per row: at least two rows to a partial one, four of more than 8192
    // columns (us with one, two, four: 20, 16, 20 at 300 x 8192, 62, 62, 49 at 1000 x 16000).
    const int64_t n = rmsnorm_bwd_parts(T, padded);
    const int64_t most = norm_rows(layernorm_form(d)) > 1 ? n : ceil_div(T, padded > 8192 ? 4 : 2);
    return n < most ? n : most;
  }
  const int64_t fill = (int64_t(1) << (d % 8 == 0 ? 22 : 19)) / d, most = fill > 16 ? fill : 16;
  return ceil_div(T, 8) < most ? ceil_div(T, 8) : most;
}
hipError_t launch_layernorm_bwd(const void* h, const float* w, const void* dy, const void* dsum,
                                int64_t T, int d, float eps, bool f32, void* dx, float* part,
                                float* rows, hipStream_t s);
hipError_t launch_layernorm_dw(const float* part, int64_t n, int d, float* dw, float* db,
                               hipStream_t s);

// AdamW.  A launch takes up to kAdamTensors tensors, as kernel arguments; its
// workgroups take `chunk` elements (a multiple of kAdamChunk) of one tensor each,
// those of tensor i from workgroup first[i] on (2^32 - 1 behind the last).
constexpr int kAdamTensors = 48;
constexpr int kAdamChunk = 2048;
struct AdamTensor {
  void* param;
  float* master;  // NULL: the parameter itself
  const void* grad;
  void *m, *v;               // float, or e4m3 with scales
  float *m_scale, *v_scale;  // NULL: 32-bit states
  int64_t n;
  float decay;   // lr * weight decay
  uint32_t key;  // of the random numbers
  uint8_t param_bf16, grad_bf16;
};
struct AdamStep {
  float beta1, beta2, rest1, rest2;  // rest: 1 - beta
  float rate, root;                  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  float eps;
  const float* grad_scale;  // NULL: 1
};
struct AdamLaunch {
  uint32_t first[kAdamTensors];
  AdamStep step;
  int64_t chunk;
  AdamTensor t[kAdamTensors];
};
static_assert(sizeof(AdamLaunch) <= 4096, "kernel arguments");
// The random numbers' key of (seed, step): a hash of two rounds.
inline uint32_t adam_mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}
inline uint32_t adam_key(uint32_t seed, int64_t step) {
  return adam_mix(adam_mix(seed) + (uint32_t)step);
}
hipError_t launch_adamw(const AdamLaunch& a, unsigned workgroups, hipStream_t s);

// How often each head's experts are in idx [T][Nh][k], over the tokens of mask
// (NULL: all).
hipError_t launch_expert_counts(const int32_t* idx, const uint8_t* mask, int64_t T, int Nh, int Ne,
                                int k, int32_t* counts, hipStream_t s);

// The balance loss and its gradient.  The router's weights are first laid out as two
// fp16 pieces, with a head's other numbers (kBalanceHeadBytes) behind them, for the
// loss and dX.  dW comes from W itself, in balance_splits partial results of Nh x (Ne
// rounded up to 32) x dh floats that launch_balance_dw_sum adds in order, or, where
// there is one, at once.
constexpr size_t kBalanceHeadBytes = 4 * (1024 + 32 + 32);
inline int balance_blocks(int Ne) { return (int)ceil_div(Ne, 32); }
inline size_t balance_operand_bytes(int Nh, int dh, int Ne) {
  return (size_t)Nh * balance_blocks(Ne) * 32 * dh * 2 * 2;
}
inline size_t balance_weight_bytes(int Nh, int dh, int Ne) {
  return balance_operand_bytes(Nh, dh, Ne) + Nh * kBalanceHeadBytes;
}
constexpr int kBalanceTokens = 128;  // per workgroup of the loss and of dX
// Few tokens: no launch in front that lays the weights out (every group of 32 tokens
// splits them itself), and the wavefronts of a workgroup share out the experts, too.
// us at 8 heads, d_h 128, bf16, so / with the weights laid out (a call of the loss and
// the counts, of the gradient):
//   tokens  experts   loss       gradient
//      512    1024   29 / 41     41 / 88
//     1024    1024   31 / 41     70 / 91
//     2048      64   23 / 25     31 / 24
//     2048     256   27 / 24     53 / 48
//     4096      16   24 / 27     35 / 28
//     4096      64   24 / 28     43 / 26
// (the limit is the loss's; the gradient of 2048 tokens and more with few experts would be
// faster with the weights laid out).
constexpr int kBalanceFewWaves = 8;
inline bool balance_few(int64_t T, int Nh, int Ne) {
  const int64_t groups = Nh * ceil_div(T, 32);
  return groups <= 256 || groups * balance_blocks(Ne) <= 1024;
}
// Of so many wavefronts, those that have experts of their own: a power of two.
inline int balance_few_groups(int Ne, int waves) {
  int n = 1;
  while (n < balance_blocks(Ne) && n < waves) n *= 2;
  return n;
}
// Tokens and workgroups per head of the loss.
inline int64_t balance_loss_tokens(int64_t T, int Nh, int Ne) {
  return balance_few(T, Nh, Ne)
             ? 32 * (kBalanceFewWaves / balance_few_groups(Ne, kBalanceFewWaves))
             : kBalanceTokens;
}
inline int64_t balance_token_blocks(int64_t T, int Nh, int Ne) {
  return ceil_div(T, balance_loss_tokens(T, Nh, Ne));
}
// Whether launch_balance_loss writes the loss itself.
inline bool balance_loss_at_once(int64_t T, int Nh, int Ne) {
  return T > 0 && balance_few(T, Nh, Ne) && balance_token_blocks(T, Nh, Ne) == 1;
}
// dW: blocks of experts that a workgroup has, a wavefront each (four wavefronts share
// them out over the tokens where there are fewer than three), and the chunks that the
// tokens are cut into, of at least four tiles, so that there are eight wavefronts per
// CU at once (us of the gradient in bf16 with 512 workgroups of four wavefronts and with
// 1024: 128 and 138 at 16384 x 16 heads x 128 experts, 71 and 87 at 8000).  Eight blocks
// share the splitting of their tokens' X (65536 x 8 x 1024: 1127 us, with four 1207;
// 16384 x 16 x 256 188, 192; d_h 64: 3 us more at 16384 x 16 x 200).
inline int balance_dw_blocks(int64_t T, int Nh, int dh, int Ne) {
  return Ne <= 32 ? 1 : Ne <= 64 ? 2 : Ne <= 128 || dh < 128 || balance_few(T, Nh, Ne) ? 4 : 8;
}
// Where not few tokens: dX and dW in one launch, whose workgroups then fill the card
// together, unless dX loses too much by dW's registers and LDS.  us together / apart in
// bf16 at 16 heads (fp32 alike):
//   d_h   64: 33 / 41 at 3001 tokens x 200 experts, 91 / 97 at 32768 x 64
//   d_h  128: 28 / 38 at 2000 x 100, 124 / 132 at 16384 x 128, 443 / 435 at 65536 x 128;
//             31 / 40 at 2500 x 20, 49 / 46 at 6000 x 16, 115 / 97 at 16384 x 16
inline bool balance_together(int64_t T, int Nh, int dh, int Ne) {
  const int ew = balance_dw_blocks(T, Nh, dh, Ne);
  return ew <= 4 && (dh < 128 || Nh * ceil_div(T, kBalanceTokens) <= (ew == 1 ? 512 : 2048));
}
inline int64_t balance_splits(int64_t T, int Nh, int dh, int Ne) {
  const int ew = balance_dw_blocks(T, Nh, dh, Ne);
  const int64_t groups = Nh * ceil_div(balance_blocks(Ne), ew);
  int64_t want = ceil_div(ew == 8 ? 256 : 512, groups);
  // beside dX's workgroups: what the card then still holds at once (3001 x 16 heads x 200
  // experts, d_h 64, fp32: 38 -> 35 us)
  const int64_t dx = Nh * ceil_div(T, kBalanceTokens), free = 256 * (dh < 128 ? 3 : 2) - dx;
  if (balance_together(T, Nh, dh, Ne) && !balance_few(T, Nh, Ne) && free >= groups)
    want = free / groups;
  const int64_t most = ceil_div(T, 4 * 32 * (ew < 4 ? 4 / ew : 1));
  return want < most ? want : most;
}
hipError_t launch_balance_weights(const float* W, const int32_t* counts, int Nh, int dh, int Ne,
                                  void* out, hipStream_t s);
hipError_t launch_balance_loss(const void* X, const float* W, const void* weights,
                               const int32_t* counts, const uint8_t* mask, int64_t T, int Nh,
                               int dh, int Ne, bool f32, float* stats, double* part, float* loss,
                               hipStream_t s);
hipError_t launch_balance_loss_sum(const double* part, const int32_t* counts, const uint8_t* mask,
                                   int64_t T, int Nh, int Ne, float* loss, float* stats,
                                   hipStream_t s);
hipError_t launch_balance_dx(const void* X, const void* weights, const float* stats,
                             const float* dloss, const uint8_t* mask, const void* dX_add, int64_t T,
                             int Nh, int dh, int Ne, bool f32, void* dX, hipStream_t s);
hipError_t launch_balance_dw(const void* X, const float* W, const int32_t* counts,
                             const float* stats, const float* dloss, const uint8_t* mask,
                             const float* dW_add, int64_t T, int Nh, int dh, int Ne, bool f32,
                             float* dW, float* part, hipStream_t s);
// Both in one launch where balance_together.
hipError_t launch_balance_dw_dx(const void* X, const float* W, const void* weights,
                                const int32_t* counts, const float* stats, const float* dloss,
                                const uint8_t* mask, const void* dX_add, const float* dW_add,
                                int64_t T, int Nh, int dh, int Ne, bool f32, void* dX, float* dW,
                                float* part, hipStream_t s);
// dX and dW where balance_few.
hipError_t launch_balance_bwd_few(const void* X, const float* W, const int32_t* counts,
                                  const float* stats, const float* dloss, const uint8_t* mask,
                                  const void* dX_add, const float* dW_add, int64_t T, int Nh,
                                  int dh, int Ne, bool f32, void* dX, float* dW, float* part,
                                  hipStream_t s);
hipError_t launch_balance_dw_sum(const float* part, const float* stats, const float* dloss,
                                 const float* dW_add, int64_t T, int Nh, int dh, int Ne, float* dW,
                                 hipStream_t s);

}  // namespace mhl
