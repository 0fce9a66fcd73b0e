// Host-side driver of the scaled operators' entry points for the sanitizer
// tier: sizes workspaces over a table of shapes ("norm T d status bytes",
// "latent T dm Nh dh Ne k dff dtype status bytes") and makes calls that must
// be refused at the largest extents ("FAIL ..." lines).  No call reaches a
// kernel: the launchers are stubs that abort.
#include <cstdint>
#include <cstdio>

#include "mhlmoe.h"
#include "scaled_launch.hpp"

namespace {
int g_fail = 0;
void expect(const char* what, mhlmoe_status got, mhlmoe_status want) {
  if (got == want) return;
  std::printf("FAIL %s: %d, expected %d (%s)\n", what, (int)got, (int)want, mhlmoe_last_error());
  ++g_fail;
}
}  // namespace

int main() {
  const int64_t Ts[] = {0, 1, 63, 4096, 65536, (int64_t(1) << 31) - 1, int64_t(1) << 31, -1,
                        INT64_MAX, INT64_MIN};
  const int ds[] = {0, 1, 16, 208, 1001, 4096, 16400, 65536, 65537, INT32_MAX, -16};
  for (int64_t T : Ts)
    for (int d : ds) {
      size_t b = 0;
      mhlmoe_status st = mhlmoe_rmsnorm_backward_workspace(T, d, &b);
      std::printf("norm %lld %d %d %zu\n", (long long)T, d, (int)st, st == MHLMOE_OK ? b : 0);
      st = mhlmoe_latent_layer_scaled_workspace(T, d, 8, 128, 64, 8, 256, MHLMOE_BF16, &b);
      std::printf("latent %lld %d 8 128 64 8 256 1 %d %zu\n", (long long)T, d, (int)st,
                  st == MHLMOE_OK ? b : 0);
      st = mhlmoe_latent_layer_scaled_workspace(T, d, 1024, 64, 1024, 32, 512, MHLMOE_F32, &b);
      std::printf("latent %lld %d 1024 64 1024 32 512 0 %d %zu\n", (long long)T, d, (int)st,
                  st == MHLMOE_OK ? b : 0);
    }
  void* A = reinterpret_cast<void*>(uintptr_t(0x10000));
  float* F = static_cast<float*>(A);
  const int64_t big[] = {INT64_MAX, INT64_MAX - 15, INT64_MIN, int64_t(1) << 31, int64_t(1) << 62};
  for (int64_t v : big) {
    const mhlmoe_status want = v < 0 ? MHLMOE_EINVAL : MHLMOE_EUNSUPPORTED;
    expect("gemm M", mhlmoe_gemm_scaled(A, F, A, F, v, 64, 64, 128, MHLMOE_BF16, A, nullptr), want);
    expect("gemm N", mhlmoe_gemm_scaled(A, F, A, F, 64, v, 64, 1, MHLMOE_BF16, A, nullptr), want);
    expect("gemm K", mhlmoe_gemm_scaled(A, F, A, F, 64, 64, v, 1, MHLMOE_F32, A, nullptr), want);
    expect("quantize rows", mhlmoe_quantize(A, v, 64, MHLMOE_BF16, 1, 0, A, F, nullptr), want);
    expect("quantize tile rows", mhlmoe_quantize(A, v, 64, MHLMOE_BF16, 128, 0, A, F, nullptr), want);
    expect("quantize cols", mhlmoe_quantize(A, 64, v, MHLMOE_BF16, 128, 1, A, F, nullptr), want);
    expect("rmsnorm T", mhlmoe_rmsnorm(A, nullptr, F, v, 64, 1e-6f, MHLMOE_BF16, nullptr, A, nullptr,
                                       nullptr, nullptr), want);
  }
  expect("quantize block_rows", mhlmoe_quantize(A, 64, 64, MHLMOE_BF16, INT32_MIN, 0, A, F, nullptr),
         MHLMOE_EINVAL);
  expect("gemm dtype", mhlmoe_gemm_scaled(A, F, A, F, 1, 64, 64, 128, (mhlmoe_dtype)77, A, nullptr),
         MHLMOE_EINVAL);
  // every product that the ABI takes is a launch of fewer than 2^32 threads
  const int64_t sizes[] = {1, 16, 17, 32, 33, 64, 65, 1000, 4096, 65536, 1 << 20, 1 << 24, 1 << 26,
                           (1 << 26) + 1, 1 << 27, (int64_t(1) << 31) - 1};
  for (int64_t M : sizes)
    for (int64_t N : sizes) {
      if (mhl::ceil_div(M, 128) >= (int64_t(1) << 24) / mhl::ceil_div(N, 128)) continue;
      for (int v = 0; v < 4; ++v) {
        const int f32 = v & 1;
        const int64_t K = v & 2 ? 8192 : 256;
        const mhl::GemmForm f = mhl::gemm_scaled_form(M, N, K, f32 != 0);
        int64_t groups = 0, threads = 0;
        switch (f) {
          case mhl::GemmForm::kFew16:
          case mhl::GemmForm::kFew32: groups = mhl::ceil_div(N, 16), threads = 512; break;
          case mhl::GemmForm::kFew16Wide:
          case mhl::GemmForm::kFew32Wide: groups = mhl::ceil_div(N, 32), threads = 512; break;
          case mhl::GemmForm::kFew32Widest: groups = mhl::ceil_div(N, 64), threads = 512; break;
          case mhl::GemmForm::k64:
            groups = mhl::ceil_div(M, 64) * mhl::ceil_div(N, 64), threads = 512;
            break;
          case mhl::GemmForm::k128Split:
            groups = mhl::ceil_div(M, 128) * mhl::ceil_div(N, 128), threads = 512;
            break;
          case mhl::GemmForm::k128:
            groups = mhl::ceil_div(M, 128) * mhl::ceil_div(N, 128), threads = 256;
            break;
          case mhl::GemmForm::k256:
            groups = mhl::ceil_div(M, 256) * mhl::ceil_div(N, 256), threads = 512;
            break;
        }
        if (groups < 1 || groups * threads >= (int64_t(1) << 32) || (f32 && f == mhl::GemmForm::k256)) {
          std::printf("FAIL form %lld %lld %d\n", (long long)M, (long long)N, f32);
          ++g_fail;
        }
      }
    }
  std::printf("done %d failures\n", g_fail);
  return g_fail == 0 ? 0 : 1;
}
