// Launch interface of the operators around the heads (api_scaled.cpp) to their
// kernels: the residual sum and RMS norm, quantisation to 8 bits and the 8-bit
// product.  As in launch.hpp, a launcher only enqueues work on its stream and
// gets shapes that the ABI layer has validated.
#pragma once

#include "launch.hpp"

namespace mhl {

// How a row of d columns is held by the norm kernels.  Multiples of 8 by pieces
// of 8 columns: in the registers of 16 or 32 lanes (up to 128 or 256 columns),
// of a wavefront (up to 2048, 1 to 4 pieces per lane; no barrier, four rows per
// workgroup) or of a workgroup (at 16384 rows of 4096 with 8 bits out 46 us, 64 in
// a wavefront's registers) of 256 threads (up to 8192) or 512 (16384; us forward
// and backward at 8192 rows of 16384 with 256 threads and 8 pieces 122 and 190,
// with 512 and 4 97 and 167; forward only, up to 32768: 272 -> 223 at 4096 rows).
// Other widths column by column: 16 lanes (up to 64 columns), a wavefront (512), a
// workgroup (4096).  Wider rows are not held at all.
enum class NormForm {
  kPart16, kPart32, kWave1, kWave2, kWave4, kGroup2, kGroup4, kLarge4,
  kOdd16, kOddWave, kOddGroup, kLarge8, kWide8, kWide1
};
inline NormForm norm_form(int d) {
  if (d % 8 != 0)
    return d <= 64     ? NormForm::kOdd16
           : d <= 512  ? NormForm::kOddWave
           : d <= 4096 ? NormForm::kOddGroup
                       : NormForm::kWide1;
  return d <= 128     ? NormForm::kPart16
         : d <= 256   ? NormForm::kPart32
         : d <= 512   ? NormForm::kWave1
         : d <= 1024  ? NormForm::kWave2
         : d <= 2048  ? NormForm::kWave4
         : d <= 4096  ? NormForm::kGroup2
         : d <= 8192  ? NormForm::kGroup4
         : d <= 16384 ? NormForm::kLarge4
         : d <= 32768 ? NormForm::kLarge8
                      : NormForm::kWide8;
}
// Rows that a workgroup of the register forms has at once.
inline int norm_rows(NormForm f) {
  return f == NormForm::kPart16 || f == NormForm::kOdd16 ? 16
         : f == NormForm::kPart32                        ? 8
         : f == NormForm::kGroup2 || f == NormForm::kGroup4 || f == NormForm::kLarge4 ||
                 f == NormForm::kLarge8 || f == NormForm::kOddGroup
             ? 1
             : 4;
}

// h = round(x + residual) to sum (residual NULL: h = x, sum not written), the
// RMS norm of h to y (NULL: not written) and, in 8 bits with a scale per 128
// columns, to q and scales (NULL: not written; d a multiple of 16).
hipError_t launch_rmsnorm(const void* x, const void* residual, const float* w, int64_t T, int d,
                          float eps, bool f32, void* sum, void* y, void* q, float* scales,
                          hipStream_t s);

// The norm's gradient: dx, and dw as rmsnorm_bwd_parts partial rows of d
// floats, which launch_rmsnorm_dw adds in order.  rows: 2 T floats where
// rmsnorm_bwd_wide, else unused.
inline bool rmsnorm_bwd_wide(int d) {
  return norm_form(d) >= NormForm::kLarge8;  // the last three
}
inline int64_t rmsnorm_bwd_parts(int64_t T, int d) {
  if (rmsnorm_bwd_wide(d)) {  // chunks of rows under each 2048 or 256 columns
    const int64_t fill = (int64_t(1) << (d % 8 == 0 ? 22 : 19)) / d, most = fill > 16 ? fill : 16;
    return ceil_div(T, 8) < most ? ceil_div(T, 8) : most;
  }
  // one per workgroup: two workgroups per CU, four where their rows are short and
  // many (us with 256, 512, 1024, 2048: 61, 56, 58, 62 at 16384 x 2048, 34, 31, 32, 34
  // at 16384 x 1024, 21, 17, 16, 19 at 16384 x 512, 12, 12, 13, 13 at 4096 x 1024)
  const int64_t n = ceil_div(T, norm_rows(norm_form(d)));
  const int64_t most = d <= 512 && T >= 16384 ? 1024 : 512;
  return n < most ? n : most;
}
hipError_t launch_rmsnorm_bwd(const void* h, const float* w, const void* dy, const void* dsum,
                              int64_t T, int d, float eps, bool f32, void* dx, float* part,
                              float* rows, hipStream_t s);
hipError_t launch_rmsnorm_dw(const float* part, int64_t n, int d, float* dw, hipStream_t s);

// x [rows][cols] (cols a multiple of 16) in 8 bits with a scale per block_rows
// (1 or 128) x 128 block, of x or of its transpose (q [cols][rows rounded up
// to 16]).
hipError_t launch_quantize(const void* x, int64_t rows, int64_t cols, bool f32, int block_rows,
                           bool transpose, void* q, float* scales, hipStream_t s);

// How the 8-bit product is cut up.  Few rows of A: B straight into registers, 16,
// 32 or 64 of its rows per workgroup (below).  Else tiles of C: 64 x 64 with the blocks
// along K over four groups of wavefronts (kept while they do not outnumber the
// CUs), 128 x 128 over two groups, 128 x 128 with two workgroups per CU, or 256 x
// 256 (bf16 results; fp32 ones need the registers for widened pieces).  us at
// K = 1024 (2048 at N = 2048, 2048 at 3584, 8192 at 8192), bf16:
//      M     N     64   128 split   128    256
//    128  1024    5.6      7.7      8.0   14.3
//   1024  1024    6.0      8.2      8.4   14.8
//   2048  1024   10.4      8.7      8.8   15.4
//   4096  1024   20.5     10.0     10.0   16.4
//   8192  1024   38       18.4     14.6   18.2
//   2048  2048   28       14.6     15.7   25.7
//   4096  2048   53       27       22     28
//   3584  3584   83       50       37     30
//   8192  8192 1412      754      600    458
// A round of 256 x 256 tiles (one per CU) takes about 9 / 5 of one of 128 x 128
// tiles (two per CU); whichever's rounds take less is chosen.
// fp32 results (no 256 x 256) take the same thresholds, which were not measured
// for them.
//
// Few rows of A, us by rows of B per workgroup, of which more share the reads of
// A (64 x 64 tiles: 22.5 at 64 x 8192 x 8192, 33 with A in registers):
//     M      N     K     16     32     64
//     1   8192  8192   12.3   14.9   19.4
//     1  16384  2048    8.4    7.2
//     1  16384  8192   24.8   28.2
//     1  65536  2048   29.5   25.9   27.0
//    16   4096  4096    7.1    8.7   12.8
//    16   8192  8192   20.5   18.5   23.4
//    16  11264  1024    7.1    5.6
//    16  12288  8192   31.1   32.3
//    16  16384  8192   42.1   34.8
//    16  65536  2048   43.4   32.8   32.1
//    32   8192  8192   32     23.8   31.2
//    32  16384  2048          11.8   10.5
//    32  65536  2048          41.1   33.8
// The rule goes by the workgroups that are left.  Up to 16 rows of A: 32 of B where
// that leaves 320 and K is at most 4096, or 512 and A has more than 4 rows (so 16
// x 8192 x 8192 stays with 16, at 20.5 against 18.5, and 16 x 12288 x 8192 with 31.1
// against 32.3).  Up to 32: 64 or else 32 where that leaves 256.
enum class GemmForm {
  kFew16, kFew16Wide, kFew32, kFew32Wide, kFew32Widest, k64, k128Split, k128, k256
};
inline GemmForm gemm_scaled_form(int64_t M, int64_t N, int64_t K, bool f32) {
  // (the few rows' workgroups of 512 threads must fit a grid of 2^32)
  if (M <= 16 && N < (1 << 26))
    return (N >= 32 * 320 && K <= 4096) || (N >= 32 * 512 && M > 4) ? GemmForm::kFew16Wide
                                                                    : GemmForm::kFew16;
  if (M <= 32 && N < (1 << 26))
    return N >= 64 * 256   ? GemmForm::kFew32Widest
           : N >= 32 * 256 ? GemmForm::kFew32Wide
                           : GemmForm::kFew32;
  if (ceil_div(M, 64) * ceil_div(N, 64) <= 256) return GemmForm::k64;
  const int64_t tiles = ceil_div(M, 128) * ceil_div(N, 128);
  if (tiles <= 256) return GemmForm::k128Split;
  const int64_t rounds = ceil_div(tiles, 512);
  const int64_t rounds256 = ceil_div(ceil_div(M, 256) * ceil_div(N, 256), 256);
  return !f32 && 9 * rounds256 <= 5 * rounds ? GemmForm::k256 : GemmForm::k128;
}

// C[M][N] (bf16, fp32 when f32) of 8-bit A[M][K] and B[N][K] (K a multiple of
// 16) with scales sa[M][ceil(K / 128)] and sb[N or ceil(N / 128)][ceil(K / 128)]
// (b_rows: one per row of B).  K == 0 writes zeros.
hipError_t launch_gemm_scaled(const void* A, const float* sa, const void* B, const float* sb,
                              int64_t M, int64_t N, int64_t K, bool b_rows, bool f32, void* C,
                              hipStream_t s);

}  // namespace mhl
