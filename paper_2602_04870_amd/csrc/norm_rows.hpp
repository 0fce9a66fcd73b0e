// What the kernels of the two norms share: a row of d columns in the registers
// of the lanes that normalise it (NormForm), its sums, and the norm's output in
// the type or in 8 bits.
#pragma once

#include "scaled_common.hpp"
#include "scaled_launch.hpp"

namespace mhl {

constexpr int kNormThreads = 256;
// threads of a workgroup with LANES lanes per row
constexpr int norm_threads(int lanes) { return lanes > kNormThreads ? lanes : kNormThreads; }
constexpr int kNormWaves = 512 / kWave;  // most of a workgroup
constexpr unsigned kNormMaxGrid = 1u << 20;  // workgroups; rows beyond them are looped over

// Sum over the lanes of a row: part of a wavefront, or the workgroup (whose
// wavefronts' sums are added in their order).
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  v = lane_sum<(LANES < kWave ? LANES : kWave)>(v);
  if (LANES <= kWave) return v;
  __syncthreads();  // the readers of the sums before
  if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = lds[0];
#pragma unroll
  for (int w = 1; w < LANES / kWave; ++w) s += lds[w];
  return s;
}

// Writes a lane's columns of y: in the type, and/or (VEC 8) in 8 bits with the
// scale of the 16 lanes' 128 columns.  All 16 lanes take part.
template <bool F32, int VEC>
__device__ __forceinline__ void write_y(const float (&y)[VEC], bool ok, int64_t row, uint32_t col,
                                        int d, void* out, uint8_t* q, float* scales) {
  if (out && ok) {
    Piece<F32, VEC> p;
    p.set(y);
    p.store(from<F32>(out, row * d), col);
  }
  if constexpr (VEC == 8) {
    if (!q) return;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = magnitude(y[i]);
      m = b > m ? b : m;
    }
    float inv;
    const float s = block_scale(max16(ok ? m : 0u), inv);
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = over_scale(y[i], s, inv);
    if (ok) {
      *reinterpret_cast<u32x2*>(q + row * d + col) =
          u32x2{pack_e4m3(z[0], z[1], z[2], z[3]), pack_e4m3(z[4], z[5], z[6], z[7])};
      if ((threadIdx.x & 15) == 0)
        scales[row * ceil_div(d, kScaleBlock) + col / kScaleBlock] = s;
    }
  }
}

// A thread's first row; one number per wavefront where the wavefront has one
// row, so that its addresses are a scalar base and a lane's 32-bit offset.
template <int LANES>
__device__ __forceinline__ int64_t first_row() {
  constexpr int kRows = norm_threads(LANES) / LANES;
  const int r = threadIdx.x / LANES;
  return (int64_t)blockIdx.x * kRows + (LANES >= kWave ? __builtin_amdgcn_readfirstlane(r) : r);
}

template <int VEC>
__device__ __forceinline__ void load_weight(const float* w, uint32_t col, bool ok,
                                            float (&f)[VEC]) {
  Piece<true, VEC> p;
  p.load(w, col, ok);
  p.get(f);
}

inline unsigned norm_grid(int64_t rows, int per_wg, unsigned most) {
  const int64_t n = ceil_div(rows, per_wg);
  return (unsigned)(n < (int64_t)most ? n : (int64_t)most);
}

// The register forms: VEC, LANES, NV of NormForm's members.
#define MHL_NORM_FORMS(F32, KERNEL)                        \
  case NormForm::kPart16: KERNEL(F32, 8, 16, 1); break;    \
  case NormForm::kPart32: KERNEL(F32, 8, 32, 1); break;    \
  case NormForm::kWave1: KERNEL(F32, 8, 64, 1); break;     \
  case NormForm::kWave2: KERNEL(F32, 8, 64, 2); break;     \
  case NormForm::kWave4: KERNEL(F32, 8, 64, 4); break;     \
  case NormForm::kGroup2: KERNEL(F32, 8, 256, 2); break;   \
  case NormForm::kGroup4: KERNEL(F32, 8, 256, 4); break;   \
  case NormForm::kLarge4: KERNEL(F32, 8, 512, 4); break;   \
  case NormForm::kOdd16: KERNEL(F32, 1, 16, 4); break;     \
  case NormForm::kOddWave: KERNEL(F32, 1, 64, 8); break;   \
  case NormForm::kOddGroup: KERNEL(F32, 1, 256, 16); break;

}  // namespace mhl
