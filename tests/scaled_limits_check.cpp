// Host-side driver of the extents that mhlmoe_gemm_scaled, mhlmoe_quantize and
// the size query of the scaled layer take: both sides of each documented limit,
// decided from the products themselves, with factors that divide no power of
// two.  The launchers are stubs that only count: no call reaches a GPU.
#include <cstdint>
#include <cstdio>

#include "mhlmoe.h"
#include "scaled_launch.hpp"

extern int g_launches;

namespace {
int g_fail = 0, g_taken = 0, g_refused = 0;

void expect(bool fits, mhlmoe_status got, const char* what, int64_t a, int64_t b) {
  const bool launched = g_launches > 0;
  g_launches = 0;
  (fits ? g_taken : g_refused)++;
  if (got == (fits ? MHLMOE_OK : MHLMOE_EUNSUPPORTED) && launched == fits) return;
  std::printf("FAIL %s %lld x %lld: status %d, %s (%s)\n", what, (long long)a, (long long)b, (int)got,
              fits ? "must be taken" : "must be refused", mhlmoe_last_error());
  ++g_fail;
}

// Every form's launch is counted in 32 bits.
void check_threads(int64_t M, int64_t N) {
  for (int v = 0; v < 4; ++v) {
    const bool f32 = (v & 1) != 0;
    int64_t m = 0, n = 0, threads = 512;
    switch (mhl::gemm_scaled_form(M, N, v & 2 ? 8192 : 256, f32)) {
      case mhl::GemmForm::kFew16:
      case mhl::GemmForm::kFew32: n = 16; break;
      case mhl::GemmForm::kFew16Wide:
      case mhl::GemmForm::kFew32Wide: n = 32; break;
      case mhl::GemmForm::kFew32Widest: n = 64; break;
      case mhl::GemmForm::k64: m = n = 64; break;
      case mhl::GemmForm::k128Split: m = n = 128; break;
      case mhl::GemmForm::k128: m = n = 128, threads = 256; break;
      case mhl::GemmForm::k256: m = n = 256; break;
    }
    const int64_t groups = (m ? mhl::ceil_div(M, m) : 1) * mhl::ceil_div(N, n);
    if (groups * threads < int64_t(1) << 32) continue;
    std::printf("FAIL threads %lld x %lld\n", (long long)M, (long long)N);
    ++g_fail;
  }
}
}  // namespace

int main() {
  void* A = reinterpret_cast<void*>(uintptr_t(0x10000));
  float* F = static_cast<float*>(A);
  const int64_t tiles = int64_t(1) << 24, blocks = int64_t(1) << 32, most = int64_t(1) << 31;
  for (int64_t b : {1, 2, 3, 5, 7, 11, 100, 127, 128, 1000, 4095, 4096, 4097, 65535, 1000003}) {
    // a: as many tiles of 128 as fit beside b of them, one less, one more
    for (int64_t a : {(tiles - 1) / b - 1, (tiles - 1) / b, (tiles - 1) / b + 1}) {
      if (a < 1) continue;
      const bool fits = a * b < tiles;
      // at the tiles' full height and with one row in the last
      for (int64_t rows : {a * 128, a * 128 - 127}) {
        for (int64_t other : {b * 128, b * 128 - 112}) {
          if (rows >= most || other >= most) continue;
          expect(fits, mhlmoe_gemm_scaled(A, F, A, F, rows, other, 64, 128, MHLMOE_BF16, A, nullptr),
                 "gemm", rows, other);
          expect(fits, mhlmoe_gemm_scaled(A, F, A, F, other, rows, 64, 1, MHLMOE_F32, A, nullptr),
                 "gemm", other, rows);
          if (fits) check_threads(rows, other), check_threads(other, rows);
          for (int transpose : {0, 1})
            expect(fits, mhlmoe_quantize(A, rows, other, MHLMOE_BF16, 128, transpose, A, F, nullptr),
                   "quantize tiles", rows, other);
          expect(fits, mhlmoe_quantize(A, rows, other, MHLMOE_F32, 1, 1, A, F, nullptr),
                 "quantize transposed rows", rows, other);
        }
      }
    }
    // rows of x beside b blocks of 1 x 128 each
    for (int64_t rows : {(blocks - 1) / b - 1, (blocks - 1) / b, (blocks - 1) / b + 1}) {
      if (rows >= most) continue;
      for (int64_t cols : {b * 128, b * 128 - 112})
        expect(rows * b < blocks, mhlmoe_quantize(A, rows, cols, MHLMOE_BF16, 1, 0, A, F, nullptr),
               "quantize rows", rows, cols);
    }
  }
  std::printf("done %d failures, %d taken, %d refused\n", g_fail, g_taken, g_refused);
  return g_fail == 0 ? 0 : 1;
}
