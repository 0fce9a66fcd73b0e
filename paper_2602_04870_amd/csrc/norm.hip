// The residual sum and RMS norm in front of the layer, and their gradient.
//
//   h = round(x + residual);  rs = 1 / sqrt(mean_c h^2 + eps);  y = h rs w
//
// and, for a gradient dy of y and dsum of h (from h's other readers),
//
//   g = dy w;  dx = dsum + rs (g - h rs^2 mean_c(g h));  dw = sum_t dy h rs.
//
// The norm is that of the stored (rounded) h, so the backward, which has only
// h, differentiates what the forward computed.  Sums are in fp32.
//
// Every element is read once: a row stays in the registers of the lanes that
// normalise it, 16 of them to a workgroup (NormForm).  Rows too wide for that
// are walked twice by a workgroup (the second time out of the caches).

#include "scaled_common.hpp"
#include "scaled_launch.hpp"

namespace mhl {
namespace {

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

// LANES lanes per row, each with NV pieces of VEC columns; d a multiple of VEC,
// at most LANES * NV * VEC.  residual == NULL: h is x, and sum is not written.
// sum may be x or residual, y may be x: a lane stores only what it has read.
template <bool F32, int VEC, int LANES, int NV>
__global__ __launch_bounds__(norm_threads(LANES)) void rmsnorm_kernel(
    const void* x, const void* residual, const float* __restrict__ w, int64_t T, int d, float eps,
    void* sum, void* y, uint8_t* q, float* scales) {
  __shared__ float lds[kNormWaves];
  constexpr int kRows = norm_threads(LANES) / LANES;
  const int l = threadIdx.x % LANES;
  for (int64_t row = first_row<LANES>(); row < T; row += (int64_t)gridDim.x * kRows) {
    const void *x_row = from<F32>(x, row * d), *r_row = from<F32>(residual, row * d);
    void* const sum_row = from<F32>(sum, row * d);
    Piece<F32, VEC> hr[NV], rr[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const uint32_t col = (v * LANES + l) * VEC;
      hr[v].load(x_row, col, col < (uint32_t)d);
    }
    if (residual) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const uint32_t col = (v * LANES + l) * VEC;
        rr[v].load(r_row, col, col < (uint32_t)d);
      }
    }
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const uint32_t col = (v * LANES + l) * VEC;
      float h[VEC];
      hr[v].get(h);
      if (residual) {
        float r[VEC];
        rr[v].get(r);
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[i] += r[i];
        hr[v].set(h);
        if (col < (uint32_t)d) hr[v].store(sum_row, col);
        hr[v].get(h);
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) ss = fmaf(h[i], h[i], ss);
    }
    const float rs = 1.0f / sqrtf(row_sum<LANES>(ss, lds) / (float)d + eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const uint32_t col = (v * LANES + l) * VEC;
      float h[VEC], wf[VEC];
      hr[v].get(h);
      load_weight<VEC>(w, col, col < (uint32_t)d, wf);
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[i] = h[i] * rs * wf[i];
      write_y<F32, VEC>(h, col < (uint32_t)d, row, col, d, y, q, scales);
    }
  }
}

// Any width, one workgroup per row, VEC columns at a time (VEC 8: d a multiple
// of 8; VEC 1 writes no 8 bits).
template <bool F32, int VEC>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_wide_kernel(
    const void* x, const void* residual, const float* __restrict__ w, int64_t T, int d, float eps,
    void* sum, void* y, uint8_t* q, float* scales) {
  __shared__ float lds[kNormWaves];
  for (int64_t row = blockIdx.x; row < T; row += gridDim.x) {
    const void* h_src = residual ? sum : x;  // each thread reads back what it wrote itself
    float ss = 0.0f;
    for (int c = threadIdx.x * VEC; c < d; c += kNormThreads * VEC) {
      const int64_t at = row * d + c;
      Piece<F32, VEC> p;
      float h[VEC];
      p.load(x, at, true);
      p.get(h);
      if (residual) {
        float r[VEC];
        p.load(residual, at, true);
        p.get(r);
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[i] += r[i];
        p.set(h);
        p.store(sum, at);
        p.get(h);
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) ss = fmaf(h[i], h[i], ss);
    }
    const float rs = 1.0f / sqrtf(row_sum<kNormThreads>(ss, lds) / (float)d + eps);
    // whole wavefronts to the end: the 8-bit output reduces over 16 lanes
    for (int c0 = 0; c0 < d; c0 += kNormThreads * VEC) {
      const int c = c0 + threadIdx.x * VEC;
      Piece<F32, VEC> p;
      float h[VEC], wf[VEC];
      p.load(h_src, row * d + c, c < d);
      p.get(h);
      load_weight<VEC>(w, c, c < d, wf);
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[i] = h[i] * rs * wf[i];
      write_y<F32, VEC>(h, c < d, row, c, d, y, q, scales);
    }
  }
}

// The gradient, rows as above; a workgroup goes over rows blockIdx.x,
// blockIdx.x + gridDim.x, ... (of kRows rows each) with its columns' dw in
// registers and leaves their sum in part[blockIdx.x][d], its rows' lanes added
// in order.  dx may be dy or dsum.
template <bool F32, int VEC, int LANES, int NV>
__global__ __launch_bounds__(norm_threads(LANES)) void rmsnorm_bwd_kernel(
    const void* h_src, const float* __restrict__ w, const void* dy, const void* dsum, int64_t T,
    int d, float eps, void* dx, float* __restrict__ part) {
  constexpr int kRows = norm_threads(LANES) / LANES;
  __shared__ float lds[2 * kNormWaves];
  __shared__ float add[kRows > 1 ? kNormThreads * VEC : 1];
  const int l = threadIdx.x % LANES;
  // the weights stay in registers, too (62.2 -> 55.8 us at 16384 x 2048: loaded anew
  // for every row they were most of the L1's traffic)
  float wf[NV][VEC];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const uint32_t col = (v * LANES + l) * VEC;
    load_weight<VEC>(w, col, col < (uint32_t)d, wf[v]);
  }
  float dw[NV][VEC];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[v][i] = 0.0f;
  // (fetching the next row ahead of this one's work took registers and time: 62.5
  // -> 64.1 us at 16384 x 2048, 58.4 -> 66.7 at 8192 x 2048 in fp32)
  for (int64_t row = first_row<LANES>(); row < T; row += (int64_t)gridDim.x * kRows) {
    const void *h_row = from<F32>(h_src, row * d), *dy_row = from<F32>(dy, row * d);
    const void* const dsum_row = from<F32>(dsum, row * d);
    void* const dx_row = from<F32>(dx, row * d);
    Piece<F32, VEC> hr[NV], gr[NV], sr[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const uint32_t col = (v * LANES + l) * VEC;
      hr[v].load(h_row, col, col < (uint32_t)d);
      gr[v].load(dy_row, col, col < (uint32_t)d);
    }
    if (dsum) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const uint32_t col = (v * LANES + l) * VEC;
        sr[v].load(dsum_row, col, col < (uint32_t)d);
      }
    }
    float ss = 0.0f, gh = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float h[VEC], g[VEC];
      hr[v].get(h);
      gr[v].get(g);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        ss = fmaf(h[i], h[i], ss);
        gh = fmaf(g[i] * wf[v][i], h[i], gh);
      }
    }
    ss = row_sum<LANES>(ss, lds);
    gh = row_sum<LANES>(gh, lds + kNormWaves);
    const float rs = 1.0f / sqrtf(ss / (float)d + eps);
    const float k = gh / (float)d * rs * rs;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const uint32_t col = (v * LANES + l) * VEC;
      float h[VEC], g[VEC], s[VEC];
      hr[v].get(h);
      gr[v].get(g);
      if (dsum) sr[v].get(s);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        dw[v][i] = fmaf(g[i], h[i] * rs, dw[v][i]);
        const float t = rs * fmaf(-h[i], k, g[i] * wf[v][i]);
        h[i] = dsum ? s[i] + t : t;
      }
      hr[v].set(h);
      if (col < (uint32_t)d) hr[v].store(dx_row, col);
    }
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const uint32_t col = (v * LANES + l) * VEC;
    if (kRows > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < VEC; ++i) add[i * kNormThreads + threadIdx.x] = dw[v][i];
      __syncthreads();
      if (threadIdx.x < LANES) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float t = add[i * kNormThreads + l];
#pragma unroll
          for (int r = 1; r < kRows; ++r) t += add[i * kNormThreads + r * LANES + l];
          dw[v][i] = t;
        }
      }
    }
    if (threadIdx.x < LANES && col < (uint32_t)d) {
      Piece<true, VEC> p;
      p.set(dw[v]);
      p.store(part, (int64_t)blockIdx.x * d + col);
    }
  }
}

// Any width, VEC columns at a time (VEC 8: d a multiple of 8): rs and k of every
// row ...
template <bool F32, int VEC>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_bwd_wide_kernel(
    const void* h_src, const float* __restrict__ w, const void* dy, int64_t T, int d, float eps,
    float* __restrict__ rs_out, float* __restrict__ k_out) {
  __shared__ float lds[2 * kNormWaves];
  for (int64_t row = blockIdx.x; row < T; row += gridDim.x) {
    float ss = 0.0f, gh = 0.0f;
    for (int c = threadIdx.x * VEC; c < d; c += kNormThreads * VEC) {
      Piece<F32, VEC> hr, gr;
      float h[VEC], g[VEC], wf[VEC];
      hr.load(h_src, row * d + c, true);
      gr.load(dy, row * d + c, true);
      load_weight<VEC>(w, c, true, wf);
      hr.get(h);
      gr.get(g);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        ss = fmaf(h[i], h[i], ss);
        gh = fmaf(g[i] * wf[i], h[i], gh);
      }
    }
    ss = row_sum<kNormThreads>(ss, lds);
    gh = row_sum<kNormThreads>(gh, lds + kNormWaves);
    const float rs = 1.0f / sqrtf(ss / (float)d + eps);
    if (threadIdx.x == 0) {
      rs_out[row] = rs;
      k_out[row] = gh / (float)d * rs * rs;
    }
  }
}

// ... and, grid (ceil(d / (256 VEC)), chunks of rows), dx and the chunks' dw: a
// thread goes down VEC columns (8 with 8 times the chunks against 1: 500 -> 334 us at
// 4096 x 32768 in bf16; a row of it in registers of 512 threads spills: 825).
template <bool F32, int VEC>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_bwd_columns_kernel(
    const void* h_src, const float* __restrict__ w, const void* dy, const void* dsum, int64_t T,
    int d, const float* __restrict__ rs_in, const float* __restrict__ k_in, void* dx,
    float* __restrict__ part) {
  const int c = (blockIdx.x * kNormThreads + threadIdx.x) * VEC;
  if (c >= d) return;
  const int64_t t0 = T * blockIdx.y / gridDim.y, t1 = T * (blockIdx.y + 1) / gridDim.y;
  float wf[VEC], dw[VEC];
  load_weight<VEC>(w, c, true, wf);
#pragma unroll
  for (int i = 0; i < VEC; ++i) dw[i] = 0.0f;
#pragma unroll 4
  for (int64_t t = t0; t < t1; ++t) {
    Piece<F32, VEC> hr, gr, sr;
    float h[VEC], g[VEC], s[VEC];
    hr.load(h_src, t * d + c, true);
    gr.load(dy, t * d + c, true);
    sr.load(dsum, t * d + c, dsum != nullptr);
    hr.get(h);
    gr.get(g);
    sr.get(s);
    const float rs = rs_in[t], k = k_in[t];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      dw[i] = fmaf(g[i], h[i] * rs, dw[i]);
      const float v = rs * fmaf(-h[i], k, g[i] * wf[i]);
      h[i] = dsum ? s[i] + v : v;
    }
    hr.set(h);
    hr.store(dx, t * d + c);
  }
  Piece<true, VEC> p;
  p.set(dw);
  p.store(part, (int64_t)blockIdx.y * d + c);
}

// dw[c] = the sum of n partial rows: 32 columns per workgroup, every 32nd row
// per thread, 16 of them on their way at once whatever their number (gradient of
// 800 x 1024, 200 rows here: 8.1 -> 7.3 us against a loop unrolled 8 times, the
// same at 512 rows), the 32 threads of a column added in order.
__global__ __launch_bounds__(1024) void rmsnorm_dw_kernel(const float* __restrict__ part, int n,
                                                          int d, float* __restrict__ dw) {
  __shared__ float lds[32][33];
  const int c = blockIdx.x * 32 + threadIdx.x % 32, g = threadIdx.x / 32;
  float s = 0.0f;
  if (c < d) {
    for (int r0 = g; r0 < n; r0 += 32 * 16) {
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = r0 + 32 * i;
        v[i] = r < n ? part[(int64_t)r * d + c] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) s += v[i];
    }
  }
  lds[g][threadIdx.x % 32] = s;
  __syncthreads();
  if (g == 0 && c < d) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += lds[i][threadIdx.x];
    dw[c] = s;
  }
}

unsigned norm_grid(int64_t rows, int per_wg, unsigned most) {
  const int64_t n = ceil_div(rows, per_wg);
  return (unsigned)(n < (int64_t)most ? n : (int64_t)most);
}

}  // namespace

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

hipError_t launch_rmsnorm(const void* x, const void* residual, const float* w, int64_t T, int d,
                          float eps, bool f32, void* sum, void* y, void* q, float* scales,
                          hipStream_t s) {
  uint8_t* q8 = static_cast<uint8_t*>(q);
#define MHL_NORM(F32, VEC, LANES, NV)                                                              \
  hipLaunchKernelGGL((rmsnorm_kernel<F32, VEC, LANES, NV>),                                        \
                     dim3(norm_grid(T, norm_threads(LANES) / LANES, kNormMaxGrid)),                \
                     dim3(norm_threads(LANES)), 0, s, x, residual, w, T, d, eps, sum, y, q8, scales)
#define MHL_NORM_WIDE(F32, VEC)                                                                   \
  hipLaunchKernelGGL((rmsnorm_wide_kernel<F32, VEC>), dim3(norm_grid(T, 1, kNormMaxGrid)),        \
                     dim3(kNormThreads), 0, s, x, residual, w, T, d, eps, sum, y, q8, scales)
#define MHL_NORM_TYPE(F32)                                       \
  switch (norm_form(d)) {                                        \
    MHL_NORM_FORMS(F32, MHL_NORM)                                \
    case NormForm::kLarge8: MHL_NORM(F32, 8, 512, 8); break;     \
    case NormForm::kWide8: MHL_NORM_WIDE(F32, 8); break;         \
    case NormForm::kWide1: MHL_NORM_WIDE(F32, 1); break;         \
  }
  if (f32)
    MHL_NORM_TYPE(true)
  else
    MHL_NORM_TYPE(false)
#undef MHL_NORM_TYPE
#undef MHL_NORM_WIDE
#undef MHL_NORM
  return hipGetLastError();
}

hipError_t launch_rmsnorm_bwd(const void* h, const float* w, const void* dy, const void* dsum,
                              int64_t T, int d, float eps, bool f32, void* dx, float* part,
                              float* rows, hipStream_t s) {
  const unsigned n = (unsigned)rmsnorm_bwd_parts(T, d);
#define MHL_NORM(F32, VEC, LANES, NV)                                                              \
  hipLaunchKernelGGL((rmsnorm_bwd_kernel<F32, VEC, LANES, NV>), dim3(n),                           \
                     dim3(norm_threads(LANES)), 0, s, h, w, dy, dsum, T, d, eps, dx, part)
#define MHL_NORM_WIDE(F32, VEC)                                                                    \
  do {                                                                                             \
    hipLaunchKernelGGL((rmsnorm_bwd_wide_kernel<F32, VEC>), dim3(norm_grid(T, 1, kNormMaxGrid)),   \
                       dim3(kNormThreads), 0, s, h, w, dy, T, d, eps, rows, rows + T);             \
    hipLaunchKernelGGL((rmsnorm_bwd_columns_kernel<F32, VEC>),                                     \
                       dim3((unsigned)ceil_div(d, kNormThreads * VEC), n), dim3(kNormThreads), 0,  \
                       s, h, w, dy, dsum, T, d, rows, rows + T, dx, part);                         \
  } while (0)
#define MHL_NORM_TYPE(F32)                                                                       \
  switch (norm_form(d)) {                                                                        \
    MHL_NORM_FORMS(F32, MHL_NORM)                                                                \
    case NormForm::kLarge8:                                                                      \
    case NormForm::kWide8: MHL_NORM_WIDE(F32, 8); break;                                         \
    case NormForm::kWide1: MHL_NORM_WIDE(F32, 1); break;                                         \
  }
  if (f32)
    MHL_NORM_TYPE(true)
  else
    MHL_NORM_TYPE(false)
#undef MHL_NORM_TYPE
#undef MHL_NORM_WIDE
#undef MHL_NORM
  return hipGetLastError();
}

hipError_t launch_rmsnorm_dw(const float* part, int64_t n, int d, float* dw, hipStream_t s) {
  hipLaunchKernelGGL(rmsnorm_dw_kernel, dim3((unsigned)ceil_div(d, 32)), dim3(1024), 0, s, part,
                     (int)n, d, dw);
  return hipGetLastError();
}

}  // namespace mhl
