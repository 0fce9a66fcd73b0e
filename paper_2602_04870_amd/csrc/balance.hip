// The loss that balances the experts by gradient, and the counts it goes by.  Per
// head, over the n tokens that count, with c_e the counts, p_t = softmax(W x_t):
//
//   f_e = c_e / sum c;  loss = E sum_e f_e mean_t p_t(e) = 1 + mean_t u_t,
//   u_t = sum_e p_t(e) f'_e,  f'_e = E f_e - 1
//
// (sum_e p_t(e) = 1).  Counts are no function of W; the gradient is
//
//   ds_t(e) = dloss / n p_t(e) (f'_e - u_t);  dX_t = sum_e ds_t(e) W_e;
//   dW_e = sum_t ds_t(e) x_t.
//
// The T x E scores stay on the chip: the loss takes one sweep over the experts with
// a running maximum, sum and weighted sum, and keeps log sum exp and u_t of every
// token; the gradient computes the scores again, once token by token for dX and
// once expert by expert for dW (a fixed order, no atomics).
//
// All products go to the bf16 matrix instructions at fp32 accuracy: an fp32 value
// is three bf16 ones, w = w0 + w1 + w2 exactly (each the nearest to what is left),
// and products of pieces w_i x_j with i + j <= 2 are kept: 3 with a bf16 x (exact),
// 6 with an fp32 x (2^-24 of the product left out); the fp32 matrix instructions
// take 2.7 times as long as the 6.

#include "device_common.hpp"
#include "training_launch.hpp"

namespace mhl {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxExperts = 1024;
constexpr int kTokenWaves = kBalanceTokens / 32;

// ---------------------------------------------------------------------------
// Counts
// ---------------------------------------------------------------------------
constexpr int kCountThreads = 256;

__global__ __launch_bounds__(kCountThreads) void counts_zero_kernel(int32_t* counts, int n) {
  const int i = blockIdx.x * kCountThreads + threadIdx.x;
  if (i < n) counts[i] = 0;
}

// Head blockIdx.y, tokens [blockIdx.x tokens, + tokens): a histogram in LDS, added
// to the counts (whole numbers, so in any order).
__global__ __launch_bounds__(kCountThreads) void expert_counts_kernel(
    const int32_t* __restrict__ idx, const uint8_t* __restrict__ mask, int64_t T, int Nh, int Ne,
    int k, DivMagic by_k, int tokens, int32_t* counts) {
  __shared__ int32_t hist[kMaxExperts];
  for (int e = threadIdx.x; e < Ne; e += kCountThreads) hist[e] = 0;
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int here = (int)(T - t0 < tokens ? T - t0 : tokens);
  for (int i = threadIdx.x; i < here * k; i += kCountThreads) {
    const int t = div_by_magic(i, by_k);
    if (mask && !mask[t0 + t]) continue;
    const int e = idx[((t0 + t) * Nh + blockIdx.y) * k + (i - t * k)];
    if ((unsigned)e < (unsigned)Ne) atomicAdd(&hist[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < Ne; e += kCountThreads)
    if (hist[e]) atomicAdd(&counts[(int64_t)blockIdx.y * Ne + e], hist[e]);
}

// ---------------------------------------------------------------------------
// Operands
// ---------------------------------------------------------------------------
// Eight values as N bf16 pieces, each the nearest to what the ones before left.
template <int N>
__device__ __forceinline__ void split8(const float (&f)[8], u32x4 (&out)[N]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int p = 0; p < N; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = pack_bf16x2(r[2 * i], r[2 * i + 1]);
      out[p][i] = w;
      r[2 * i] -= bf16_bits_to_f32(w & 0xFFFFu);
      r[2 * i + 1] -= __uint_as_float(w & 0xFFFF0000u);
    }
}

// Bytes of a block of 32 experts as operands: fragments of 64 lanes x 16 bytes.
//   scores: piece, k-step s: lane holds expert lane % 32, d = 16 s + 8 (lane / 32) + j
//   dX (transposed): piece, tile dt of 32 d, k-step s: lane holds d = 32 dt + lane % 32,
//       experts 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4, in the order in which a score
//       tile's rows lie in its registers
template <int DH>
constexpr int kScoreFrags = 3 * DH / 16;
template <int DH>
constexpr int kBackFrags = 3 * (DH / 32) * 2;

template <int DH, bool BWD>
__global__ __launch_bounds__(256) void balance_weights_kernel(const float* __restrict__ W, int Ne,
                                                              u32x4* __restrict__ out) {
  constexpr int kFrags = kScoreFrags<DH> + (BWD ? kBackFrags<DH> : 0);
  const int e0 = blockIdx.x * 32;
  const float* w = W + (int64_t)blockIdx.y * Ne * DH;
  u32x4* o = out + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kFrags * 64;
  for (int i = threadIdx.x; i < DH / 16 * 64; i += 256) {
    const int s = i >> 6, lane = i & 63, e = e0 + (lane & 31);
    float f[8];
    u32x4 p[3];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      f[j] = e < Ne ? w[(int64_t)e * DH + 16 * s + 8 * (lane >> 5) + j] : 0.0f;
    split8(f, p);
#pragma unroll
    for (int q = 0; q < 3; ++q) o[(q * (DH / 16) + s) * 64 + lane] = p[q];
  }
  if (!BWD) return;
  o += kScoreFrags<DH> * 64;
  for (int i = threadIdx.x; i < DH / 32 * 2 * 64; i += 256) {
    const int dt = i >> 7, s = (i >> 6) & 1, lane = i & 63;
    float f[8];
    u32x4 p[3];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = e0 + 16 * s + 8 * (j >> 2) + 4 * (lane >> 5) + (j & 3);
      f[j] = e < Ne ? w[(int64_t)e * DH + 32 * dt + (lane & 31)] : 0.0f;
    }
    split8(f, p);
#pragma unroll
    for (int q = 0; q < 3; ++q) o[(q * (DH / 32) * 2 + dt * 2 + s) * 64 + lane] = p[q];
  }
}

// f'_e of the head's experts (zeros up to the next multiple of 32) in LDS: exact
// whole numbers, one division.
template <int THREADS>
__device__ __forceinline__ void load_excess(const int32_t* __restrict__ counts, int Ne, float* f,
                                            long long* lds) {
  long long part = 0;
  for (int e = threadIdx.x; e < Ne; e += THREADS) part += counts[e];
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) part += __shfl_xor(part, d, kWave);
  if (lane_id() == 0) lds[threadIdx.x >> 6] = part;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) total += lds[w];
  const int padded = (Ne + 31) & ~31;
  for (int e = threadIdx.x; e < padded; e += THREADS)
    f[e] = e < Ne && total > 0
               ? (float)((double)((long long)counts[e] * Ne - total) / (double)total)
               : 0.0f;
  __syncthreads();
}

// One lane's operand of X: token row, d = 16 s + 8 g + j, as NX pieces.
template <int DH, bool F32>
struct XOperand {
  static constexpr int NX = F32 ? 3 : 1;
  u32x4 x[NX][DH / 16];
  __device__ __forceinline__ void load(const void* X, int64_t row, bool ok, int g) {
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) {
      const int64_t at = row * DH + 16 * s + 8 * g;
      if (F32) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(X) + at);
        const f32x4 a = ok ? p[0] : f32x4{0, 0, 0, 0}, b = ok ? p[1] : f32x4{0, 0, 0, 0};
        const float f[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        u32x4 o[NX];
        split8(f, o);
#pragma unroll
        for (int p2 = 0; p2 < NX; ++p2) x[p2][s] = o[p2];
      } else {
        x[0][s] = ok ? *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(X) + at)
                     : u32x4{0, 0, 0, 0};
      }
    }
  }
};

// Rows of a score tile past the last expert begin at -infinity: no weight.
__device__ __forceinline__ f32x16 score_start(int e0, int Ne, int g) {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v)
    z[v] = e0 + 8 * (v >> 2) + 4 * g + (v & 3) < Ne ? 0.0f : -INFINITY;
  return z;
}

// Scores of 32 experts (rows) x 32 tokens (lanes), small products first.
template <int DH, bool F32>
__device__ __forceinline__ f32x16 score_tile(const u32x4* w, const XOperand<DH, F32>& x,
                                             f32x16 z) {
  const int lane = lane_id();
#pragma unroll
  for (int q = 2; q >= 0; --q)
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) {
      const bf16x8 a = as_bf16x8(w[(q * (DH / 16) + s) * 64 + lane]);
#pragma unroll
      for (int p = XOperand<DH, F32>::NX - 1; p >= 0; --p)
        if (p + q <= 2) z = mfma32_bf16(a, as_bf16x8(x.x[p][s]), z);
    }
  return z;
}

template <int N>
__device__ __forceinline__ void copy_to_lds(const u32x4* __restrict__ src, u32x4* dst) {
#pragma unroll
  for (int i = 0; i < N; i += kTokenWaves * kWave)
    if (N % (kTokenWaves * kWave) == 0 || i + (int)threadIdx.x < N)
      dst[i + threadIdx.x] = src[i + threadIdx.x];
}

// ---------------------------------------------------------------------------
// The loss: 32 tokens of head blockIdx.y per wavefront, over all experts.
// ---------------------------------------------------------------------------
template <int DH, bool F32>
__global__ __launch_bounds__(kTokenWaves* kWave) void balance_loss_kernel(
    const void* __restrict__ X, const u32x4* __restrict__ weights,
    const int32_t* __restrict__ counts, const uint8_t* __restrict__ mask, int64_t T, int Nh, int Ne,
    float2* __restrict__ stats, double* __restrict__ part) {
  constexpr int kFrags = kScoreFrags<DH>;
  __shared__ u32x4 w[kFrags * 64];
  __shared__ __align__(16) float fex[kMaxExperts];
  __shared__ long long sums[kTokenWaves];
  __shared__ double loss[kTokenWaves];
  const int h = blockIdx.y, lane = lane_id(), g = lane >> 5, wave = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * kBalanceTokens + wave * 32 + (lane & 31);
  const bool ok = t < T && (!mask || mask[t < T ? t : 0]);
  load_excess<kTokenWaves * kWave>(counts + (int64_t)h * Ne, Ne, fex, sums);
  XOperand<DH, F32> x;
  x.load(X, t * Nh + h, ok, g);
  const int nb = (Ne + 31) / 32;
  const u32x4* src = weights + (int64_t)h * nb * kFrags * 64;
  float M = -INFINITY, l = 0.0f, u = 0.0f;  // maximum (times log2 e), sum, weighted sum
  for (int b = 0; b < nb; ++b) {
    __syncthreads();
    copy_to_lds<kFrags * 64>(src + (int64_t)b * kFrags * 64, w);
    __syncthreads();
    const f32x16 z = score_tile<DH, F32>(w, x, score_start(32 * b, Ne, g));
    float top = z[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) top = fmaxf(top, z[v]);
    const float Mn = fmaxf(M, top * kLog2e);
    const float ref = Mn == -INFINITY ? 0.0f : Mn;
    const float old = __builtin_amdgcn_exp2f(M - ref);
    l *= old;
    u *= old;
    M = Mn;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 f = *reinterpret_cast<const f32x4*>(&fex[32 * b + 8 * q + 4 * g]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(z[4 * q + i], kLog2e, -ref));
        l += p;
        u = fmaf(p, f[i], u);
      }
    }
  }
  // the two lanes of a token
  const float Mo = __shfl_xor(M, 32, kWave), lo = __shfl_xor(l, 32, kWave),
              uo = __shfl_xor(u, 32, kWave);
  const float Mt = fmaxf(M, Mo);
  const float a = __builtin_amdgcn_exp2f(M - Mt), c = __builtin_amdgcn_exp2f(Mo - Mt);
  l = l * a + lo * c;
  u = u * a + uo * c;
  const float lse = ok ? (Mt + __builtin_amdgcn_logf(l)) * kLn2 : 0.0f;
  const float share = ok ? u / l : 0.0f;
  if (g == 0 && t < T) stats[t * Nh + h] = float2{lse, share};
  double sum = g == 0 ? (double)share : 0.0;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor(sum, d, kWave);
  if (lane == 0) loss[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < kTokenWaves; ++i) sum += loss[i];
    part[(int64_t)h * gridDim.x + blockIdx.x] = sum;
  }
}

// The loss of head blockIdx.x from its token blocks' sums, and 1 / n behind the
// tokens' stats.
__global__ __launch_bounds__(256) void balance_loss_sum_kernel(
    const double* __restrict__ part, int64_t blocks, const int32_t* __restrict__ counts,
    const uint8_t* __restrict__ mask, int64_t T, int Nh, int Ne, float* __restrict__ loss,
    float2* __restrict__ stats) {
  __shared__ double sums[256];
  __shared__ long long tokens[256], slots[256];
  const int h = blockIdx.x;
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < blocks; i += 256) s += part[h * blocks + i];
  long long n = 0, c = 0;
  if (mask)
    for (int64_t t = threadIdx.x; t < T; t += 256) n += mask[t] != 0;
  for (int e = threadIdx.x; e < Ne; e += 256) c += counts[(int64_t)h * Ne + e];
  sums[threadIdx.x] = s;
  tokens[threadIdx.x] = n;
  slots[threadIdx.x] = c;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) {
      sums[threadIdx.x] += sums[threadIdx.x + w];
      tokens[threadIdx.x] += tokens[threadIdx.x + w];
      slots[threadIdx.x] += slots[threadIdx.x + w];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const long long all = mask ? tokens[0] : (long long)T;
    const double m = all > 0 ? (double)all : 1.0;
    loss[h] = slots[0] > 0 ? (float)(1.0 + sums[0] / m) : 0.0f;
    stats[T * Nh + h] = float2{(float)(1.0 / m), 0.0f};
  }
}

// ---------------------------------------------------------------------------
// dX: 32 tokens of head blockIdx.y per wavefront, over all experts.  Without the
// factor dloss / n, which comes at the end.
// ---------------------------------------------------------------------------
// ds of a score tile, whose 8 rows 8 s .. 8 s + 7 of a lane are the operand of
// k-step s: p (f' - u) in NP pieces.
template <int NP>
__device__ __forceinline__ void split_ds(const f32x16& ds, int s, u32x4 (&out)[NP]) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = ds[8 * s + j];
  split8(f, out);
}

template <int DH, bool F32>
__global__ __launch_bounds__(kTokenWaves* kWave) void balance_dx_kernel(
    const void* __restrict__ X, const u32x4* __restrict__ weights,
    const int32_t* __restrict__ counts, const float2* __restrict__ stats,
    const float* __restrict__ dloss, const uint8_t* __restrict__ mask, const void* dX_add,
    int64_t T, int Nh, int Ne, void* dX) {
  constexpr int kFrags = kScoreFrags<DH> + kBackFrags<DH>;
  constexpr int kLast = F32 ? 2 : 1;  // products of pieces i + j <= kLast
  __shared__ u32x4 w[kFrags * 64];
  __shared__ __align__(16) float fex[kMaxExperts];
  __shared__ long long sums[kTokenWaves];
  const int h = blockIdx.y, lane = lane_id(), g = lane >> 5, wave = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * kBalanceTokens + wave * 32 + (lane & 31);
  const int64_t row = t * Nh + h;
  const bool ok = t < T && (!mask || mask[t < T ? t : 0]);
  load_excess<kTokenWaves * kWave>(counts + (int64_t)h * Ne, Ne, fex, sums);
  XOperand<DH, F32> x;
  x.load(X, row, ok, g);
  // a token that does not count: p = exp2(-infinity) = 0
  const float2 st = ok ? stats[row] : float2{INFINITY, 0.0f};
  const float lse = st.x * kLog2e, u = st.y;
  const float c = dloss[h] * stats[T * Nh + h].x;
  const int nb = (Ne + 31) / 32;
  const u32x4* src = weights + (int64_t)h * nb * kFrags * 64;
  f32x16 dx[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) dx[i] = zero16();
  for (int b = 0; b < nb; ++b) {
    __syncthreads();
    copy_to_lds<kFrags * 64>(src + (int64_t)b * kFrags * 64, w);
    __syncthreads();
    f32x16 z = score_tile<DH, F32>(w, x, score_start(32 * b, Ne, g));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 f = *reinterpret_cast<const f32x4*>(&fex[32 * b + 8 * q + 4 * g]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        z[4 * q + i] = __builtin_amdgcn_exp2f(fmaf(z[4 * q + i], kLog2e, -lse)) * (f[i] - u);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 ds[kLast + 1];
      split_ds(z, s, ds);
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
        for (int q = kLast; q >= 0; --q) {
          const bf16x8 a = as_bf16x8(
              w[(kScoreFrags<DH> + q * (DH / 32) * 2 + dt * 2 + s) * 64 + lane]);
#pragma unroll
          for (int p = kLast - q; p >= 0; --p) dx[dt] = mfma32_bf16(a, as_bf16x8(ds[p]), dx[dt]);
        }
    }
  }
  if (t >= T) return;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t at = row * DH + 32 * dt + 8 * q + 4 * g;
      float f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = ok ? dx[dt][4 * q + i] * c : 0.0f;
      if (F32) {
        if (dX_add) {
          const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const float*>(dX_add) + at);
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] += a[i];
        }
        *reinterpret_cast<f32x4*>(static_cast<float*>(dX) + at) = f32x4{f[0], f[1], f[2], f[3]};
      } else {
        if (dX_add) {
          const u32x2 a = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(dX_add) + at);
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] += bf16_bits_to_f32((a[i >> 1] >> (16 * (i & 1))) & 0xFFFFu);
        }
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(dX) + at) =
            u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
      }
    }
}

// ---------------------------------------------------------------------------
// dW: a block of 32 experts per wavefront, whose weights stay in its registers,
// over a chunk of the tokens, 32 at a time through LDS.
// ---------------------------------------------------------------------------
template <int DH, bool F32>
__global__ __launch_bounds__(256) void balance_dw_kernel(
    const void* __restrict__ X, const u32x4* __restrict__ weights, int block_frags,
    const int32_t* __restrict__ counts, const float2* __restrict__ stats,
    const uint8_t* __restrict__ mask, int64_t T, int Nh, int Ne, int groups,
    float* __restrict__ part) {
  constexpr int NX = F32 ? 3 : 1;
  constexpr int kUnits = DH / 8;  // 16-byte units of a row
  __shared__ __align__(16) uint8_t xs[NX][32 * DH * 2];
  __shared__ __align__(16) float lse[32], us[32];
  __shared__ __align__(16) float fex[kMaxExperts];
  __shared__ long long sums[4];
  const int threads = blockDim.x;
  const int h = blockIdx.x / groups, lane = lane_id(), g = lane >> 5;
  const int nb = (Ne + 31) / 32;
  const int b = (blockIdx.x % groups) * (threads / kWave) + (int)(threadIdx.x >> 6);
  const bool live = b < nb;
  // f' of the lane's expert
  {
    long long s = 0;
    for (int e = threadIdx.x; e < Ne; e += threads) s += counts[(int64_t)h * Ne + e];
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d, kWave);
    if (lane == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
  }
  long long total = 0;
  for (int i = 0; i < threads / kWave; ++i) total += sums[i];
  const int e = 32 * b + (lane & 31);
  const float f = e < Ne && total > 0
                      ? (float)((double)((long long)counts[(int64_t)h * Ne + e] * Ne - total) /
                                (double)total)
                      : 0.0f;
  u32x4 w[3][DH / 16];
  const u32x4* src = weights + ((int64_t)h * nb + (live ? b : 0)) * block_frags * 64;
#pragma unroll
  for (int q = 0; q < 3; ++q)
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) w[q][s] = src[(q * (DH / 16) + s) * 64 + lane];
  f32x16 dw[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) dw[i] = zero16();
  const int64_t tiles = (T + 31) / 32;
  const int64_t begin = tiles * blockIdx.y / gridDim.y, end = tiles * (blockIdx.y + 1) / gridDim.y;
  auto addr = [](int row, int col) {
    return row * DH * 2 + swz_tr<kUnits>(col >> 3, row) * 16 + (col & 7) * 2;
  };
  for (int64_t tile = begin; tile < end; ++tile) {
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * kUnits; i += threads) {
      const int r = i / kUnits, j = i % kUnits;
      const int64_t t = tile * 32 + r;
      const bool ok = t < T && (!mask || mask[t]);
      const int64_t at = (t * Nh + h) * DH + 8 * j;
      u32x4 o[NX];
      if (F32) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(X) + at);
        const f32x4 a = ok ? p[0] : f32x4{0, 0, 0, 0}, c = ok ? p[1] : f32x4{0, 0, 0, 0};
        const float v[8] = {a[0], a[1], a[2], a[3], c[0], c[1], c[2], c[3]};
        split8(v, o);
      } else {
        o[0] = ok ? *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(X) + at)
                  : u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int p = 0; p < NX; ++p) *reinterpret_cast<u32x4*>(xs[p] + addr(r, 8 * j)) = o[p];
    }
    if (threadIdx.x < 32) {
      const int64_t t = tile * 32 + threadIdx.x;
      const bool ok = t < T && (!mask || mask[t]);
      const float2 st = ok ? stats[t * Nh + h] : float2{INFINITY, 0.0f};
      lse[threadIdx.x] = st.x * kLog2e;
      us[threadIdx.x] = st.y;
    }
    __syncthreads();
    // scores of 32 tokens (rows) x 32 experts (lanes)
    f32x16 z = zero16();
#pragma unroll
    for (int p = NX - 1; p >= 0; --p)
#pragma unroll
      for (int s = 0; s < DH / 16; ++s) {
        const bf16x8 a = as_bf16x8(
            *reinterpret_cast<const u32x4*>(xs[p] + addr(lane & 31, 16 * s + 8 * g)));
#pragma unroll
        for (int q = 2 - p; q >= 0; --q) z = mfma32_bf16(a, as_bf16x8(w[q][s]), z);
      }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 l4 = *reinterpret_cast<const f32x4*>(&lse[8 * q + 4 * g]);
      const f32x4 u4 = *reinterpret_cast<const f32x4*>(&us[8 * q + 4 * g]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        z[4 * q + i] = __builtin_amdgcn_exp2f(fmaf(z[4 * q + i], kLog2e, -l4[i])) * (f - u4[i]);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 ds[3];
      split_ds(z, s, ds);
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
        for (int p = NX - 1; p >= 0; --p) {
          const bf16x8 a = tr_fragment(xs[p], addr, 16 * s, 16 * s + 4, 16 * s + 8, 16 * s + 12,
                                       32 * dt);
#pragma unroll
          for (int q = 2 - p; q >= 0; --q) dw[dt] = mfma32_bf16(a, as_bf16x8(ds[q]), dw[dt]);
        }
    }
  }
  if (!live) return;
  float* o = part + (((int64_t)blockIdx.y * Nh + h) * nb * 32 + e) * DH;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4*>(o + 32 * dt + 8 * q + 4 * g) =
          f32x4{dw[dt][4 * q], dw[dt][4 * q + 1], dw[dt][4 * q + 2], dw[dt][4 * q + 3]};
}

// dW = dW_add + dloss / n times the sum of n partial results, in order.
__global__ __launch_bounds__(256) void balance_dw_sum_kernel(
    const f32x4* __restrict__ part, int64_t n, int64_t stride, const float2* __restrict__ inv_n,
    const float* __restrict__ dloss, const f32x4* dW_add, int Ne, int padded, int dh4, f32x4* dW) {
  const int h = blockIdx.y;
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= Ne * dh4) return;
  const f32x4* p = part + (int64_t)h * padded * dh4 + i;
  f32x4 s{0, 0, 0, 0};
  for (int64_t r = 0; r < n; ++r) s += p[r * stride];
  const float c = dloss[h] * inv_n[h].x;
  f32x4 o;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = s[k] * c;
  const int64_t at = (int64_t)h * Ne * dh4 + i;
  if (dW_add) o += dW_add[at];
  dW[at] = o;
}

}  // namespace

hipError_t launch_expert_counts(const int32_t* idx, const uint8_t* mask, int64_t T, int Nh, int Ne,
                                int k, int32_t* counts, hipStream_t s) {
  const int n = Nh * Ne;
  hipLaunchKernelGGL(counts_zero_kernel, dim3((unsigned)ceil_div(n, kCountThreads)),
                     dim3(kCountThreads), 0, s, counts, n);
  if (T == 0) return hipGetLastError();
  // about 1024 workgroups, of at least 128 tokens
  int64_t blocks = ceil_div(1024, Nh);
  if (blocks > ceil_div(T, 128)) blocks = ceil_div(T, 128);
  // (a workgroup's slots are counted in 31 bits: T k is)
  const int64_t tokens = ceil_div(T, blocks);
  hipLaunchKernelGGL(expert_counts_kernel, dim3((unsigned)ceil_div(T, tokens), (unsigned)Nh),
                     dim3(kCountThreads), 0, s, idx, mask, T, Nh, Ne, k, div_magic(k), (int)tokens,
                     counts);
  return hipGetLastError();
}

hipError_t launch_balance_weights(const float* W, int Nh, int dh, int Ne, bool backward, void* out,
                                  hipStream_t s) {
  const dim3 grid((unsigned)balance_blocks(Ne), (unsigned)Nh);
  u32x4* o = static_cast<u32x4*>(out);
#define MHL_WEIGHTS(DH, BWD) \
  hipLaunchKernelGGL((balance_weights_kernel<DH, BWD>), grid, dim3(256), 0, s, W, Ne, o)
  if (dh == 128) {
    if (backward)
      MHL_WEIGHTS(128, true);
    else
      MHL_WEIGHTS(128, false);
  } else {
    if (backward)
      MHL_WEIGHTS(64, true);
    else
      MHL_WEIGHTS(64, false);
  }
#undef MHL_WEIGHTS
  return hipGetLastError();
}

#define MHL_BALANCE_TYPES(CALL) \
  if (dh == 128) {              \
    if (f32)                    \
      CALL(128, true);          \
    else                        \
      CALL(128, false);         \
  } else {                      \
    if (f32)                    \
      CALL(64, true);           \
    else                        \
      CALL(64, false);          \
  }

hipError_t launch_balance_loss(const void* X, const void* weights, const int32_t* counts,
                               const uint8_t* mask, int64_t T, int Nh, int dh, int Ne, bool f32,
                               float* stats, double* part, hipStream_t s) {
  const dim3 grid((unsigned)balance_token_blocks(T), (unsigned)Nh);
#define MHL_LOSS(DH, F32)                                                                      \
  hipLaunchKernelGGL((balance_loss_kernel<DH, F32>), grid, dim3(kTokenWaves* kWave), 0, s, X,  \
                     static_cast<const u32x4*>(weights), counts, mask, T, Nh, Ne,              \
                     reinterpret_cast<float2*>(stats), part)
  MHL_BALANCE_TYPES(MHL_LOSS)
#undef MHL_LOSS
  return hipGetLastError();
}

hipError_t launch_balance_loss_sum(const double* part, const int32_t* counts, const uint8_t* mask,
                                   int64_t T, int Nh, int Ne, float* loss, float* stats,
                                   hipStream_t s) {
  hipLaunchKernelGGL(balance_loss_sum_kernel, dim3((unsigned)Nh), dim3(256), 0, s, part,
                     balance_token_blocks(T), counts, mask, T, Nh, Ne, loss,
                     reinterpret_cast<float2*>(stats));
  return hipGetLastError();
}

hipError_t launch_balance_dx(const void* X, const void* weights, const int32_t* counts,
                             const float* stats, const float* dloss, const uint8_t* mask,
                             const void* dX_add, int64_t T, int Nh, int dh, int Ne, bool f32,
                             void* dX, hipStream_t s) {
  const dim3 grid((unsigned)balance_token_blocks(T), (unsigned)Nh);
#define MHL_DX(DH, F32)                                                                       \
  hipLaunchKernelGGL((balance_dx_kernel<DH, F32>), grid, dim3(kTokenWaves* kWave), 0, s, X,   \
                     static_cast<const u32x4*>(weights), counts,                              \
                     reinterpret_cast<const float2*>(stats), dloss, mask, dX_add, T, Nh, Ne, dX)
  MHL_BALANCE_TYPES(MHL_DX)
#undef MHL_DX
  return hipGetLastError();
}

hipError_t launch_balance_dw(const void* X, const void* weights, const int32_t* counts,
                             const float* stats, const uint8_t* mask, int64_t T, int Nh, int dh,
                             int Ne, bool f32, float* part, hipStream_t s) {
  const int waves = balance_dw_waves(Ne), groups = (int)ceil_div(balance_blocks(Ne), waves);
  const dim3 grid((unsigned)(Nh * groups), (unsigned)balance_splits(T, Nh, Ne));
#define MHL_DW(DH, F32)                                                                          \
  hipLaunchKernelGGL((balance_dw_kernel<DH, F32>), grid, dim3((unsigned)(waves * kWave)), 0, s,  \
                     X, static_cast<const u32x4*>(weights), kScoreFrags<DH> + kBackFrags<DH>,    \
                     counts, reinterpret_cast<const float2*>(stats), mask, T, Nh, Ne, groups, part)
  MHL_BALANCE_TYPES(MHL_DW)
#undef MHL_DW
  return hipGetLastError();
}

hipError_t launch_balance_dw_sum(const float* part, const float* stats, const float* dloss,
                                 const float* dW_add, int64_t T, int Nh, int dh, int Ne, float* dW,
                                 hipStream_t s) {
  const int padded = 32 * balance_blocks(Ne), dh4 = dh / 4;
  const dim3 grid((unsigned)ceil_div(Ne * dh4, 256), (unsigned)Nh);
  hipLaunchKernelGGL(balance_dw_sum_kernel, grid, dim3(256), 0, s,
                     reinterpret_cast<const f32x4*>(part), balance_splits(T, Nh, Ne),
                     (int64_t)Nh * padded * dh4, reinterpret_cast<const float2*>(stats) + T * Nh,
                     dloss, reinterpret_cast<const f32x4*>(dW_add), Ne, padded, dh4,
                     reinterpret_cast<f32x4*>(dW));
  return hipGetLastError();
}

}  // namespace mhl
