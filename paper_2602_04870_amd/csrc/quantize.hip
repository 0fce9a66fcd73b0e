// Quantisation to 8 bits (e4m3) with an fp32 scale per block of 128 values
// along the contraction, for the operands of the 8-bit product:
//
//   scale = max(max |x| over the block / 448, 2^-126),  q = e4m3(x / scale).
//
// A block is 1 x 128 (activations: every row its own scales) or 128 x 128
// (weights).  The transposed forms quantise x^T, whose rows run down x's
// columns, for products that contract over the other axis; their rows are
// padded with zeros to a multiple of 16 bytes.

#include "scaled_common.hpp"
#include "scaled_launch.hpp"

namespace mhl {
namespace {

constexpr int kQuantThreads = 256;
constexpr int kQuantBlocks = 4;  // 1 x 128 blocks per 16 lanes: as many loads in flight
constexpr int kQuantMaxGrid = 1 << 20;

// 1 x 128 blocks of x's rows: 16 lanes of 8 values each; block i is block
// i % G of row i / G.  The 16-lane groups of a workgroup take consecutive blocks.
template <bool F32>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(
    const void* __restrict__ x, uint32_t blocks, uint32_t G, int64_t cols, uint8_t* __restrict__ q,
    float* __restrict__ scales) {
  constexpr uint32_t kGroups = kQuantThreads / 16;
  const uint32_t lane16 = threadIdx.x % 16, group = threadIdx.x / 16;
  constexpr uint32_t kStep = kGroups * kQuantBlocks;
  for (uint64_t first = (uint64_t)blockIdx.x * kStep; first < blocks;
       first += (uint64_t)gridDim.x * kStep) {
    Raw8<F32> raw[kQuantBlocks];
    int64_t at[kQuantBlocks];
    bool ok[kQuantBlocks];
#pragma unroll
    for (int u = 0; u < kQuantBlocks; ++u) {
      const uint64_t i = first + u * kGroups + group;
      const uint32_t row = (uint32_t)i / G;
      const int64_t col = (int64_t)((uint32_t)i - row * G) * kScaleBlock + lane16 * 8;
      ok[u] = i < blocks && col < cols;
      at[u] = row * cols + col;
      raw[u] = load8<F32>(x, at[u], ok[u]);
    }
#pragma unroll
    for (int u = 0; u < kQuantBlocks; ++u) {
      const uint64_t i = first + u * kGroups + group;
      float f[8];
      unpack8<F32>(raw[u], f);
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t b = magnitude(f[e]);
        m = b > m ? b : m;
      }
      float inv;
      const float s = block_scale(max16(m), inv);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = over_scale(f[e], s, inv);
      if (ok[u])
        *reinterpret_cast<u32x2*>(q + at[u]) =
            u32x2{pack_e4m3(f[0], f[1], f[2], f[3]), pack_e4m3(f[4], f[5], f[6], f[7])};
      if (lane16 == 0 && i < blocks) scales[i] = s;
    }
  }
}

// One 128 x 128 tile of x per workgroup: a thread holds the 8 x 8 values of
// rows 8 (tid / 16) .. and columns 8 (tid % 16) ...  TILE: one scale for the
// tile, else (TRANSPOSE only) one per column of x.  TRANSPOSE turns the tile
// through LDS: q[col][ld], ld the rows rounded up to 16.
template <bool F32, bool TILE, bool TRANSPOSE>
__global__ __launch_bounds__(kQuantThreads) void quantize_tile_kernel(
    const void* __restrict__ x, int64_t rows, int64_t cols, int64_t ld, uint8_t* __restrict__ q,
    float* __restrict__ scales) {
  static_assert(TILE || TRANSPOSE, "1 x 128 blocks along x's rows: quantize_rows_kernel");
  __shared__ uint32_t amax[TILE ? 4 : 4 * kScaleBlock];
  __shared__ __align__(16) uint8_t turned[TRANSPOSE ? kScaleBlock * kScaleBlock : 16];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int cg = tid % 16, rg = tid / 16;
  // an accelerator die's workgroups take a contiguous run of tiles, along q's
  // rows: where those are no multiple of 128 bytes apart, two tiles share lines
  const int64_t tiles_r = ceil_div(rows, kScaleBlock), tiles_c = ceil_div(cols, kScaleBlock);
  const uint32_t xcd = blockIdx.x % kXcds, per = gridDim.x / kXcds, rem = gridDim.x % kXcds;
  const uint32_t tile = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / kXcds;
  const int64_t tr = TRANSPOSE ? tile % tiles_r : tile / tiles_c;
  const int64_t tc = TRANSPOSE ? tile / tiles_r : tile % tiles_c;
  const int64_t r0 = tr * kScaleBlock + rg * 8, c0 = tc * kScaleBlock + cg * 8;

  Raw8<F32> raw[8];
#pragma unroll
  for (int p = 0; p < 8; ++p)
    raw[p] = load8<F32>(x, (r0 + p) * cols + c0, r0 + p < rows && c0 < cols);

  float s[TILE ? 1 : 8], inv[TILE ? 1 : 8];
  if (TILE) {
    uint32_t m = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      float f[8];
      unpack8<F32>(raw[p], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t b = magnitude(f[e]);
        m = b > m ? b : m;
      }
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const uint32_t o = __shfl_xor(m, d, kWave);
      m = o > m ? o : m;
    }
    if (lane_id() == 0) amax[wave] = m;
    __syncthreads();
    m = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = amax[w] > m ? amax[w] : m;
    s[0] = block_scale(m, inv[0]);
    if (tid == 0) scales[TRANSPOSE ? tc * tiles_r + tr : tr * tiles_c + tc] = s[0];
  } else {
    uint32_t m[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      float f[8];
      unpack8<F32>(raw[p], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t b = magnitude(f[e]);
        m[e] = b > m[e] ? b : m[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int d = 16; d < kWave; d <<= 1) {
        const uint32_t o = __shfl_xor(m[e], d, kWave);
        m[e] = o > m[e] ? o : m[e];
      }
    }
    if ((tid & 48) == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) amax[wave * kScaleBlock + cg * 8 + e] = m[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t v = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t o = amax[w * kScaleBlock + cg * 8 + e];
        v = o > v ? o : v;
      }
      s[e] = block_scale(v, inv[e]);
    }
    if (rg == 0 && c0 < cols) {
#pragma unroll
      for (int e = 0; e < 8; ++e) scales[(c0 + e) * tiles_r + tr] = s[e];
    }
  }

  if (!TRANSPOSE) {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      float f[8];
      unpack8<F32>(raw[p], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = over_scale(f[e], s[0], inv[0]);
      if (r0 + p < rows && c0 < cols)
        *reinterpret_cast<u32x2*>(q + (r0 + p) * cols + c0) =
            u32x2{pack_e4m3(f[0], f[1], f[2], f[3]), pack_e4m3(f[4], f[5], f[6], f[7])};
    }
    return;
  }
  // rows 8 rg .. + 7 of column 8 cg + e: 8 bytes of q's row, put at byte
  // 8 (rg ^ cg) of it, so that the 16 lanes of a write hit distinct banks
  uint32_t word[8][2];
#pragma unroll
  for (int p = 0; p < 8; p += 2) {
    float a[8], b[8];
    unpack8<F32>(raw[p], a);
    unpack8<F32>(raw[p + 1], b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float se = s[TILE ? 0 : e], ie = inv[TILE ? 0 : e];
      const int old = (p & 2) ? (int)word[e][p >> 2] : 0;
      const float va = over_scale(a[e], se, ie), vb = over_scale(b[e], se, ie);
      word[e][p >> 2] = (uint32_t)((p & 2) ? __builtin_amdgcn_cvt_pk_fp8_f32(va, vb, old, true)
                                           : __builtin_amdgcn_cvt_pk_fp8_f32(va, vb, old, false));
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    *reinterpret_cast<u32x2*>(turned + (cg * 8 + e) * kScaleBlock + 8 * (rg ^ cg)) =
        u32x2{word[e][0], word[e][1]};
  __syncthreads();
  // 8 lanes of 16 bytes per row of q
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int i = u * kQuantThreads + tid;
    const int c = i / 8, piece = i % 8;
    const uint8_t* src = turned + c * kScaleBlock;
    const u32x2 lo = *reinterpret_cast<const u32x2*>(src + 8 * ((2 * piece) ^ (c / 8)));
    const u32x2 hi = *reinterpret_cast<const u32x2*>(src + 8 * ((2 * piece + 1) ^ (c / 8)));
    const int64_t col = tc * kScaleBlock + c, r = tr * kScaleBlock + piece * 16;
    if (col < cols && r < ld)
      *reinterpret_cast<u32x4*>(q + col * ld + r) = u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
}

}  // namespace

hipError_t launch_quantize(const void* x, int64_t rows, int64_t cols, bool f32, int block_rows,
                           bool transpose, void* q, float* scales, hipStream_t s) {
  uint8_t* q8 = static_cast<uint8_t*>(q);
  if (block_rows == 1 && !transpose) {
    const int64_t G = ceil_div(cols, kScaleBlock), blocks = rows * G;
    const int64_t n = ceil_div(blocks, kQuantThreads / 16 * kQuantBlocks);
    const dim3 grid((unsigned)(n < kQuantMaxGrid ? n : kQuantMaxGrid));
    if (f32)
      hipLaunchKernelGGL((quantize_rows_kernel<true>), grid, dim3(kQuantThreads), 0, s, x,
                         (uint32_t)blocks, (uint32_t)G, cols, q8, scales);
    else
      hipLaunchKernelGGL((quantize_rows_kernel<false>), grid, dim3(kQuantThreads), 0, s, x,
                         (uint32_t)blocks, (uint32_t)G, cols, q8, scales);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)(ceil_div(rows, kScaleBlock) * ceil_div(cols, kScaleBlock)));
  const int64_t ld = (rows + 15) & ~int64_t(15);
#define MHL_QUANT(F32, TILE, TRANSPOSE)                                                       \
  hipLaunchKernelGGL((quantize_tile_kernel<F32, TILE, TRANSPOSE>), grid, dim3(kQuantThreads), 0, \
                     s, x, rows, cols, ld, q8, scales)
#define MHL_QUANT_TYPE(F32)              \
  do {                                   \
    if (block_rows == 1)                 \
      MHL_QUANT(F32, false, true);       \
    else if (transpose)                  \
      MHL_QUANT(F32, true, true);        \
    else                                 \
      MHL_QUANT(F32, true, false);       \
  } while (0)
  if (f32)
    MHL_QUANT_TYPE(true);
  else
    MHL_QUANT_TYPE(false);
#undef MHL_QUANT_TYPE
#undef MHL_QUANT
  return hipGetLastError();
}

}  // namespace mhl
