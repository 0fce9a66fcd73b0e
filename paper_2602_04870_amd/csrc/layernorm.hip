// The residual sum and layer norm in front of the layer, and their gradient.
//
//   h = round(x + residual);  mu = mean_c h;  rs = 1 / sqrt(mean_c (h - mu)^2 + eps)
//   n = (h - mu) rs;  y = n w + b
//
// and, for a gradient dy of y and dsum of h (from h's other readers),
//
//   g = dy w;  dx = dsum + rs (g - mean_c g - n mean_c(g n));
//   dw = sum_t dy n;  db = sum_t dy.
//
// The norm is that of the stored (rounded) h, so the gradient, which has only h,
// differentiates what the forward computed.  Sums are in fp32.  The mean is taken
// first and the squares from it, so rows far from zero keep their variance; what
// the mean's own rounding leaves, r = mean (h - mu), is found in the same sums and
// taken off:  mean (h - mu)^2 - r^2  and  n = (h - mu - r) rs.
//
// HBM bounds both (16384 x 2048 in bf16 with a residual: 51 us, 5.3 TB/s; the gradient with
// dsum 52 us, 5.1 TB/s, and 5 us of layernorm_dw_kernel): every element is read once, rows in
// registers as in norm.hip (NormForm).  Widths that are no multiple of 8 take the form of the next one (ODD): their
// rows begin anywhere, so pieces are loaded and stored at any address, the last one by
// elements (column by column, as the RMS norm has them, 30000 x 100 in bf16 took 17 us
// and its gradient 26).  Rows too wide for registers are walked three times by a
// workgroup (the second and third time out of the caches).

#include "norm_rows.hpp"
#include "training_launch.hpp"

namespace mhl {
namespace {

// row_sum of N values at once.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* lds) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lane_sum<(LANES < kWave ? LANES : kWave)>(v[i]);
  if (LANES <= kWave) return;
  __syncthreads();  // the readers of the sums before
  if (lane_id() == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) lds[i * kNormWaves + (threadIdx.x >> 6)] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = lds[i * kNormWaves];
#pragma unroll
    for (int w = 1; w < LANES / kWave; ++w) v[i] += lds[i * kNormWaves + w];
  }
}

// Eight elements from column col on of a row of d (none of it past d), zeros behind.
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
template <bool F32, bool ODD>
__device__ __forceinline__ Raw8<F32> load_piece(const void* row, uint32_t col, int d) {
  if constexpr (!ODD) {
    return load8<F32>(row, col, col < (uint32_t)d);
  } else {
    Raw8<F32> r;
    const int n = d - (int)col;
    if (n >= 8) {
      const u32x4_any* p = static_cast<const u32x4_any*>(from<F32>(row, col));
#pragma unroll
      for (int i = 0; i < (F32 ? 2 : 1); ++i) r.v[i] = p[i];
    } else {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < n ? load1<F32>(row, col + i) : 0.0f;
      r = pack8<F32>(f);  // exactly: they are of the type
    }
    return r;
  }
}
template <bool F32, bool ODD>
__device__ __forceinline__ void store_piece(void* row, uint32_t col, int d, const Raw8<F32>& r) {
  if constexpr (!ODD) {
    if (col < (uint32_t)d) store8<F32>(row, col, r);
  } else {
    const int n = d - (int)col;
    if (n >= 8) {
      u32x4_any* p = static_cast<u32x4_any*>(from<F32>(row, col));
#pragma unroll
      for (int i = 0; i < (F32 ? 2 : 1); ++i) p[i] = r.v[i];
    } else {
      float f[8];
      unpack8<F32>(r, f);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) store1<F32>(row, col + i, f[i]);
    }
  }
}
template <bool ODD>
__device__ __forceinline__ void load_weights(const float* w, uint32_t col, int d, float (&f)[8]) {
  unpack8<true>(load_piece<true, ODD>(w, col, d), f);
}

// 1 / sqrt(variance + eps) from the sum of (h - mu)^2 (the difference's rounding
// must not take a constant row's variance below zero).
__device__ __forceinline__ float row_rs(float squares, float r, float inv_d, float eps) {
  return 1.0f / sqrtf(fmaxf(fmaf(-r, r, squares * inv_d), 0.0f) + eps);
}

// LANES lanes per row, each with NV pieces of 8 columns, at most LANES * NV * 8 of them
// (a multiple of 8 unless ODD).  residual == NULL: h is x, and sum is not written.
// b may be NULL.  sum may be x or residual, y may be x: a lane stores only what
// it has read.
template <bool F32, bool ODD, int LANES, int NV>
__global__ __launch_bounds__(norm_threads(LANES)) void layernorm_kernel(
    const void* x, const void* residual, const float* __restrict__ w, const float* __restrict__ b,
    int64_t T, int d, float eps, void* sum, void* y, uint8_t* q, float* scales) {
  __shared__ float lds[2 * kNormWaves];
  constexpr int kRows = norm_threads(LANES) / LANES;
  const int l = threadIdx.x % LANES;
  const float inv_d = 1.0f / (float)d;
  for (int64_t row = first_row<LANES>(); row < T; row += (int64_t)gridDim.x * kRows) {
    const void *x_row = from<F32>(x, row * d), *r_row = from<F32>(residual, row * d);
    void* const sum_row = from<F32>(sum, row * d);
    Raw8<F32> hr[NV], rr[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) hr[v] = load_piece<F32, ODD>(x_row, (v * LANES + l) * 8, d);
    if (residual) {
#pragma unroll
      for (int v = 0; v < NV; ++v) rr[v] = load_piece<F32, ODD>(r_row, (v * LANES + l) * 8, d);
    }
    float s0[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float h[8];
      unpack8<F32>(hr[v], h);
      if (residual) {
        float r[8];
        unpack8<F32>(rr[v], r);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += r[i];
        hr[v] = pack8<F32>(h);
        store_piece<F32, ODD>(sum_row, (v * LANES + l) * 8, d, hr[v]);
        unpack8<F32>(hr[v], h);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s0[0] += h[i];
    }
    row_sums<LANES>(s0, lds);
    const float mu = s0[0] * inv_d;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int n = d - (v * LANES + l) * 8;
      float h[8];
      unpack8<F32>(hr[v], h);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float c = (ODD ? i : 0) < n ? h[i] - mu : 0.0f;
        s[0] += c;
        s[1] = fmaf(c, c, s[1]);
      }
    }
    row_sums<LANES>(s, lds);
    const float r = s[0] * inv_d;
    const float rs = row_rs(s[1], r, inv_d, eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const uint32_t col = (v * LANES + l) * 8;
      float h[8], wf[8], bf[8] = {};
      unpack8<F32>(hr[v], h);
      load_weights<ODD>(w, col, d, wf);
      if (b) load_weights<ODD>(b, col, d, bf);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = fmaf((h[i] - mu - r) * rs, wf[i], bf[i]);
      if constexpr (ODD)
        store_piece<F32, true>(from<F32>(y, row * d), col, d, pack8<F32>(h));
      else
        write_y<F32, 8>(h, col < (uint32_t)d, row, col, d, y, q, scales);
    }
  }
}

// Any width, one workgroup per row, VEC columns at a time (VEC 8: d a multiple
// of 8; VEC 1 writes no 8 bits).
template <bool F32, int VEC>
__global__ __launch_bounds__(kNormThreads) void layernorm_wide_kernel(
    const void* x, const void* residual, const float* __restrict__ w, const float* __restrict__ b,
    int64_t T, int d, float eps, void* sum, void* y, uint8_t* q, float* scales) {
  __shared__ float lds[2 * kNormWaves];
  const float inv_d = 1.0f / (float)d;
  for (int64_t row = blockIdx.x; row < T; row += gridDim.x) {
    const void* h_src = residual ? sum : x;  // each thread reads back what it wrote itself
    float s0[1] = {0.0f};
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
      for (int i = 0; i < VEC; ++i) s0[0] += h[i];
    }
    row_sums<kNormThreads>(s0, lds);
    const float mu = s0[0] * inv_d;
    float s[2] = {0.0f, 0.0f};
    for (int c = threadIdx.x * VEC; c < d; c += kNormThreads * VEC) {
      Piece<F32, VEC> p;
      float h[VEC];
      p.load(h_src, row * d + c, true);
      p.get(h);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float v = h[i] - mu;
        s[0] += v;
        s[1] = fmaf(v, v, s[1]);
      }
    }
    row_sums<kNormThreads>(s, lds);
    const float r = s[0] * inv_d;
    const float rs = row_rs(s[1], r, inv_d, eps);
    // whole wavefronts to the end: the 8-bit output reduces over 16 lanes
    for (int c0 = 0; c0 < d; c0 += kNormThreads * VEC) {
      const int c = c0 + threadIdx.x * VEC;
      Piece<F32, VEC> p;
      float h[VEC], wf[VEC], bf[VEC];
      p.load(h_src, row * d + c, c < d);
      p.get(h);
      load_weight<VEC>(w, c, c < d, wf);
      load_weight<VEC>(b, c, b && c < d, bf);
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[i] = fmaf((h[i] - mu - r) * rs, wf[i], bf[i]);
      write_y<F32, VEC>(h, c < d, row, c, d, y, q, scales);
    }
  }
}

// What a row's gradient needs beside its elements: mu + r as mu and r apart
// (their sum would be rounded), rs, mean g and mean (g n).
struct RowGrad {
  float mu, r, rs, g, gn;
};
// From the sums of (h - mu), (h - mu)^2, g and g (h - mu).
__device__ __forceinline__ RowGrad row_grad(const float (&s)[4], float mu, float inv_d, float eps) {
  RowGrad o;
  o.mu = mu;
  o.r = s[0] * inv_d;
  o.rs = row_rs(s[1], o.r, inv_d, eps);
  o.g = s[2] * inv_d;
  o.gn = fmaf(-o.r, s[2], s[3]) * inv_d * o.rs;
  return o;
}

// The gradient, rows as above; a workgroup goes over rows blockIdx.x,
// blockIdx.x + gridDim.x, ... (of kRows rows each) with its columns' dw and db in
// registers and leaves their sums in part[blockIdx.x][2][d], its rows' lanes added
// in order.  dx may be dy or dsum.
template <bool F32, bool ODD, int LANES, int NV>
__global__ __launch_bounds__(norm_threads(LANES)) void layernorm_bwd_kernel(
    const void* h_src, const float* __restrict__ w, const void* dy, const void* dsum, int64_t T,
    int d, float eps, void* dx, float* __restrict__ part) {
  constexpr int kRows = norm_threads(LANES) / LANES;
  constexpr int kRound = 16;  // of a lane's sums through LDS at once
  __shared__ float lds[4 * kNormWaves];
  __shared__ float add[kRows > 1 ? kNormThreads * kRound : 1];
  const int l = threadIdx.x % LANES;
  const float inv_d = 1.0f / (float)d;
  float wf[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    load_weights<ODD>(w, (v * LANES + l) * 8, d, wf[v]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[v][i] = db[v][i] = 0.0f;
  }
  for (int64_t row = first_row<LANES>(); row < T; row += (int64_t)gridDim.x * kRows) {
    const void *h_row = from<F32>(h_src, row * d), *dy_row = from<F32>(dy, row * d);
    const void* const dsum_row = from<F32>(dsum, row * d);
    void* const dx_row = from<F32>(dx, row * d);
    Raw8<F32> hr[NV], gr[NV], sr[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      hr[v] = load_piece<F32, ODD>(h_row, (v * LANES + l) * 8, d);
      gr[v] = load_piece<F32, ODD>(dy_row, (v * LANES + l) * 8, d);
    }
    if (dsum) {
#pragma unroll
      for (int v = 0; v < NV; ++v) sr[v] = load_piece<F32, ODD>(dsum_row, (v * LANES + l) * 8, d);
    }
    float s0[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float h[8];
      unpack8<F32>(hr[v], h);
#pragma unroll
      for (int i = 0; i < 8; ++i) s0[0] += h[i];
    }
    row_sums<LANES>(s0, lds);
    const float mu = s0[0] * inv_d;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int n = d - (v * LANES + l) * 8;
      float h[8], g[8];
      unpack8<F32>(hr[v], h);
      unpack8<F32>(gr[v], g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float c = (ODD ? i : 0) < n ? h[i] - mu : 0.0f;
        const float gw = g[i] * wf[v][i];
        s[0] += c;
        s[1] = fmaf(c, c, s[1]);
        s[2] += gw;
        s[3] = fmaf(gw, c, s[3]);
      }
    }
    row_sums<LANES>(s, lds);
    const RowGrad o = row_grad(s, mu, inv_d, eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float h[8], g[8], e[8];
      unpack8<F32>(hr[v], h);
      unpack8<F32>(gr[v], g);
      if (dsum) unpack8<F32>(sr[v], e);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n = (h[i] - o.mu - o.r) * o.rs;
        dw[v][i] = fmaf(g[i], n, dw[v][i]);
        db[v][i] += g[i];
        const float t = o.rs * fmaf(-n, o.gn, g[i] * wf[v][i] - o.g);
        h[i] = dsum ? e[i] + t : t;
      }
      store_piece<F32, ODD>(dx_row, (v * LANES + l) * 8, d, pack8<F32>(h));
    }
  }
  float* const out = part + (int64_t)blockIdx.x * 2 * d;
  if constexpr (kRows == 1) {
#pragma unroll
    for (int v = 0; v < 2 * NV; ++v)
      store_piece<true, ODD>(out + (int64_t)(v / NV) * d, ((v % NV) * LANES + l) * 8, d,
                             pack8<true>(v < NV ? dw[v % NV] : db[v % NV]));
  } else {
    // the rows' lanes: kPer of the round's sums added by each of the kRows groups of lanes
    constexpr int kPer = kRound / kRows;
    const int group = threadIdx.x / LANES;
#pragma unroll
    for (int at = 0; at < 2 * NV * 8; at += kRound) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRound; ++i) {
        const int v = (at + i) / 8;
        add[i * kNormThreads + threadIdx.x] = v < NV ? dw[v % NV][i % 8] : db[v % NV][i % 8];
      }
      __syncthreads();
      const int first = at + group * kPer, v = first / 8;
      float sum[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float* p = add + (group * kPer + i) * kNormThreads + l;
        sum[i] = p[0];
#pragma unroll
        for (int r = 1; r < kRows; ++r) sum[i] += p[r * LANES];
      }
      const int col = ((v % NV) * LANES + l) * 8 + first % 8;
      float* const to = out + (int64_t)(v / NV) * d + col;
      if (kPer == 4 && col + 4 <= d) {
        *reinterpret_cast<u32x4_any*>(to) =
            u32x4{__float_as_uint(sum[0]), __float_as_uint(sum[kPer > 1 ? 1 : 0]),
                  __float_as_uint(sum[kPer > 2 ? 2 : 0]), __float_as_uint(sum[kPer > 3 ? 3 : 0])};
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (col + i < d) to[i] = sum[i];
      }
    }
  }
}

// Any width, VEC columns at a time (VEC 8: d a multiple of 8): RowGrad of every
// row ...
template <bool F32, int VEC>
__global__ __launch_bounds__(kNormThreads) void layernorm_bwd_wide_kernel(
    const void* h_src, const float* __restrict__ w, const void* dy, int64_t T, int d, float eps,
    RowGrad* __restrict__ rows) {
  __shared__ float lds[4 * kNormWaves];
  const float inv_d = 1.0f / (float)d;
  for (int64_t row = blockIdx.x; row < T; row += gridDim.x) {
    float s0[1] = {0.0f};
    for (int c = threadIdx.x * VEC; c < d; c += kNormThreads * VEC) {
      Piece<F32, VEC> hr;
      float h[VEC];
      hr.load(h_src, row * d + c, true);
      hr.get(h);
#pragma unroll
      for (int i = 0; i < VEC; ++i) s0[0] += h[i];
    }
    row_sums<kNormThreads>(s0, lds);
    const float mu = s0[0] * inv_d;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
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
        const float v = h[i] - mu, gw = g[i] * wf[i];
        s[0] += v;
        s[1] = fmaf(v, v, s[1]);
        s[2] += gw;
        s[3] = fmaf(gw, v, s[3]);
      }
    }
    row_sums<kNormThreads>(s, lds);
    if (threadIdx.x == 0) rows[row] = row_grad(s, mu, inv_d, eps);
  }
}

// ... and, grid (ceil(d / (256 VEC)), chunks of rows), dx and the chunks' dw and
// db: a thread goes down VEC columns.
template <bool F32, int VEC>
__global__ __launch_bounds__(kNormThreads) void layernorm_bwd_columns_kernel(
    const void* h_src, const float* __restrict__ w, const void* dy, const void* dsum, int64_t T,
    int d, const RowGrad* __restrict__ rows, void* dx, float* __restrict__ part) {
  const int c = (blockIdx.x * kNormThreads + threadIdx.x) * VEC;
  if (c >= d) return;
  const int64_t t0 = T * blockIdx.y / gridDim.y, t1 = T * (blockIdx.y + 1) / gridDim.y;
  float wf[VEC], dw[VEC], db[VEC];
  load_weight<VEC>(w, c, true, wf);
#pragma unroll
  for (int i = 0; i < VEC; ++i) dw[i] = db[i] = 0.0f;
#pragma unroll 4
  for (int64_t t = t0; t < t1; ++t) {
    Piece<F32, VEC> hr, gr, sr;
    float h[VEC], g[VEC], e[VEC];
    hr.load(h_src, t * d + c, true);
    gr.load(dy, t * d + c, true);
    sr.load(dsum, t * d + c, dsum != nullptr);
    hr.get(h);
    gr.get(g);
    sr.get(e);
    const RowGrad o = rows[t];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float n = (h[i] - o.mu - o.r) * o.rs;
      dw[i] = fmaf(g[i], n, dw[i]);
      db[i] += g[i];
      const float v = o.rs * fmaf(-n, o.gn, g[i] * wf[i] - o.g);
      h[i] = dsum ? e[i] + v : v;
    }
    hr.set(h);
    hr.store(dx, t * d + c);
  }
  Piece<true, VEC> p;
  p.set(dw);
  p.store(part, (int64_t)blockIdx.y * 2 * d + c);
  p.set(db);
  p.store(part, ((int64_t)blockIdx.y * 2 + 1) * d + c);
}

// dw[c], and db[c] (NULL: not wanted) as columns d to 2 d - 1, are the sums of n
// partial rows of 2 d: 32 columns per workgroup, every 32nd row per thread, 16 of
// them on their way at once, the 32 threads of a column added in order.
__global__ __launch_bounds__(1024) void layernorm_dw_kernel(const float* __restrict__ part, int n,
                                                            int d, float* __restrict__ dw,
                                                            float* __restrict__ db) {
  __shared__ float lds[32][33];
  const int width = db ? 2 * d : d;
  const int c = blockIdx.x * 32 + threadIdx.x % 32, g = threadIdx.x / 32;
  float s = 0.0f;
  if (c < width) {
    for (int r0 = g; r0 < n; r0 += 32 * 16) {
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = r0 + 32 * i;
        v[i] = r < n ? part[(int64_t)r * 2 * d + c] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) s += v[i];
    }
  }
  lds[g][threadIdx.x % 32] = s;
  __syncthreads();
  if (g == 0 && c < width) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += lds[i][threadIdx.x];
    if (c < d)
      dw[c] = s;
    else
      db[c - d] = s;
  }
}

}  // namespace

// call(LANES, NV) of the register form of a row, as compile-time constants.
template <class F>
static void for_form(NormForm form, F&& call) {
  auto with = [&](auto lanes, auto nv) { call(lanes, nv); };
  using std::integral_constant;
  switch (form) {
    case NormForm::kPart16: with(integral_constant<int, 16>{}, integral_constant<int, 1>{}); break;
    case NormForm::kPart32: with(integral_constant<int, 32>{}, integral_constant<int, 1>{}); break;
    case NormForm::kWave1: with(integral_constant<int, 64>{}, integral_constant<int, 1>{}); break;
    case NormForm::kWave2: with(integral_constant<int, 64>{}, integral_constant<int, 2>{}); break;
    case NormForm::kWave4: with(integral_constant<int, 64>{}, integral_constant<int, 4>{}); break;
    case NormForm::kGroup2: with(integral_constant<int, 256>{}, integral_constant<int, 2>{}); break;
    case NormForm::kGroup4: with(integral_constant<int, 256>{}, integral_constant<int, 4>{}); break;
    case NormForm::kLarge4: with(integral_constant<int, 512>{}, integral_constant<int, 4>{}); break;
    default: with(integral_constant<int, 512>{}, integral_constant<int, 8>{}); break;  // kLarge8
  }
}

// call(X in fp32, a width that is no multiple of 8)
template <class F>
static void for_rows(bool f32, int d, F&& call) {
  if (f32 && d % 8)
    call(std::true_type{}, std::true_type{});
  else if (f32)
    call(std::true_type{}, std::false_type{});
  else if (d % 8)
    call(std::false_type{}, std::true_type{});
  else
    call(std::false_type{}, std::false_type{});
}

hipError_t launch_layernorm(const void* x, const void* residual, const float* w, const float* b,
                            int64_t T, int d, float eps, bool f32, void* sum, void* y, void* q,
                            float* scales, hipStream_t s) {
  uint8_t* q8 = static_cast<uint8_t*>(q);
  const NormForm form = layernorm_form(d);
  for_rows(f32, d, [&](auto F32, auto ODD) {
    constexpr bool kF32 = decltype(F32)::value, kOdd = decltype(ODD)::value;
    if (form == NormForm::kWide8) {
      hipLaunchKernelGGL((layernorm_wide_kernel<kF32, kOdd ? 1 : 8>),
                         dim3(norm_grid(T, 1, kNormMaxGrid)), dim3(kNormThreads), 0, s, x, residual,
                         w, b, T, d, eps, sum, y, q8, scales);
      return;
    }
    for_form(form, [&](auto LANES, auto NV) {
      constexpr int kLanes = decltype(LANES)::value, kThreads = norm_threads(kLanes);
      hipLaunchKernelGGL((layernorm_kernel<kF32, kOdd, kLanes, decltype(NV)::value>),
                         dim3(norm_grid(T, kThreads / kLanes, kNormMaxGrid)), dim3(kThreads), 0, s,
                         x, residual, w, b, T, d, eps, sum, y, q8, scales);
    });
  });
  return hipGetLastError();
}

hipError_t launch_layernorm_bwd(const void* h, const float* w, const void* dy, const void* dsum,
                                int64_t T, int d, float eps, bool f32, void* dx, float* part,
                                float* rows, hipStream_t s) {
  const unsigned n = (unsigned)layernorm_bwd_parts(T, d);
  static_assert(sizeof(RowGrad) == sizeof(float) * kLayernormRowFloats, "workspace");
  RowGrad* rg = reinterpret_cast<RowGrad*>(rows);
  const NormForm form = layernorm_form(d);
  for_rows(f32, d, [&](auto F32, auto ODD) {
    constexpr bool kF32 = decltype(F32)::value, kOdd = decltype(ODD)::value;
    if (layernorm_bwd_wide(d)) {
      constexpr int VEC = kOdd ? 1 : 8;
      hipLaunchKernelGGL((layernorm_bwd_wide_kernel<kF32, VEC>), dim3(norm_grid(T, 1, kNormMaxGrid)),
                         dim3(kNormThreads), 0, s, h, w, dy, T, d, eps, rg);
      hipLaunchKernelGGL((layernorm_bwd_columns_kernel<kF32, VEC>),
                         dim3((unsigned)ceil_div(d, kNormThreads * VEC), n), dim3(kNormThreads), 0,
                         s, h, w, dy, dsum, T, d, rg, dx, part);
      return;
    }
    for_form(form, [&](auto LANES, auto NV) {
      constexpr int kLanes = decltype(LANES)::value, kNV = decltype(NV)::value;
      if constexpr (kNV <= 4)  // (kLarge8 is wide here)
        hipLaunchKernelGGL((layernorm_bwd_kernel<kF32, kOdd, kLanes, kNV>), dim3(n),
                           dim3(norm_threads(kLanes)), 0, s, h, w, dy, dsum, T, d, eps, dx, part);
    });
  });
  return hipGetLastError();
}

hipError_t launch_layernorm_dw(const float* part, int64_t n, int d, float* dw, float* db,
                               hipStream_t s) {
  hipLaunchKernelGGL(layernorm_dw_kernel, dim3((unsigned)ceil_div(db ? 2 * d : d, 32)), dim3(1024),
                     0, s, part, (int)n, d, dw, db);
  return hipGetLastError();
}

}  // namespace mhl
