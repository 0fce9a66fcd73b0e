// Launch interface of the operators around the heads (api_scaled.cpp) to their
// kernels: the residual sum and RMS norm, quantisation to 8 bits and the 8-bit
// product.  As in launch.hpp, a launcher only enqueues work on its stream and
// gets shapes that the ABI layer has validated.
#pragma once

#include "launch.hpp"

namespace mhl {

// How a row of d columns is held by the norm kernels.  Multiples of 8 by pieces
// of 8 columns: in the registers of 16 or 32 lanes (up to 128 or 256 columns),
// of a wavefront (up to 4096, 1 to 8 pieces per lane; no barrier, four rows per
// workgroup) or of a workgroup (up to 16384).  Other widths column by column: 16
// lanes (up to 64 columns), a wavefront (512), a workgroup (4096).  Wider rows
// are not held at all.
enum class NormForm {
  kPart16, kPart32, kWave1, kWave2, kWave4, kWave8, kGroup4, kGroup8,
  kOdd16, kOddWave, kOddGroup, kWide8, kWide1
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
         : d <= 4096  ? NormForm::kWave8
         : d <= 8192  ? NormForm::kGroup4
         : d <= 16384 ? NormForm::kGroup8
                      : NormForm::kWide8;
}
// Rows that a workgroup of the register forms has at once.
inline int norm_rows(NormForm f) {
  return f == NormForm::kPart16 || f == NormForm::kOdd16 ? 16
         : f == NormForm::kPart32                        ? 8
         : f == NormForm::kGroup4 || f == NormForm::kGroup8 || f == NormForm::kOddGroup ? 1
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
  return norm_form(d) == NormForm::kWide8 || norm_form(d) == NormForm::kWide1;
}
inline int64_t rmsnorm_bwd_parts(int64_t T, int d) {
  if (rmsnorm_bwd_wide(d)) {  // chunks of rows under each 256 columns
    const int64_t most = (int64_t(1) << 19) / d > 16 ? (int64_t(1) << 19) / d : 16;
    return ceil_div(T, 8) < most ? ceil_div(T, 8) : most;
  }
  const int64_t n = ceil_div(T, norm_rows(norm_form(d)));  // workgroups, two per CU at most
  return n < 512 ? n : 512;
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

// C[M][N] (bf16, fp32 when f32) of 8-bit A[M][K] and B[N][K] (K a multiple of
// 16) with scales sa[M][ceil(K / 128)] and sb[N or ceil(N / 128)][ceil(K / 128)]
// (b_rows: one per row of B).  K == 0 writes zeros.
hipError_t launch_gemm_scaled(const void* A, const float* sa, const void* B, const float* sb,
                              int64_t M, int64_t N, int64_t K, bool b_rows, bool f32, void* C,
                              hipStream_t s);

}  // namespace mhl
