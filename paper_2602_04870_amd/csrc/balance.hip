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
// All products go to the fp16 matrix instructions at fp32 accuracy.  A value scaled
// by a power of two is two fp16 ones, w = w0 + w1, each the nearest to what is left:
// off by 2^-23 of itself, or by 2^-39 of the largest of those that share the scale
// (a token's row of X; 32 experts' rows of W, for dW all of a workgroup's, up to 256; the
// head's ds for dX, an expert's ds so far, times 2^60 at most, for dW).  A bf16 x is one
// fp16 value, exactly (down to 2^-31 of its row's largest).  Products of pieces kept:
// w0 x, w1 x with a bf16 x; w0 x0, w0 x1, w1 x0 with an fp32 x (up to 2^-22 of the
// product left out).  So a score takes 2 or 3 passes; in three bf16 pieces each it took 3 or 6
// (gradient at 65536 tokens x 8 heads x 1024 experts: 1855 us so), and one pass of the
// fp32 matrix instructions lasts as long as 16.

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

// A head's slots of T tokens into a histogram in LDS, eight of a thread on their way at
// once.
template <int THREADS>
__device__ __forceinline__ void count_slots(const int32_t* __restrict__ idx,
                                            const uint8_t* __restrict__ mask, int T, int Nh, int Ne,
                                            int k, DivMagic by_k, int32_t* hist) {
  const int n = T * k;
  for (int i0 = threadIdx.x; i0 < n; i0 += 8 * THREADS) {
    int e[8];
    uint8_t counted[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = i0 < n - j * THREADS ? i0 + j * THREADS : i0;
      const int t = div_by_magic(i, by_k);
      e[j] = idx[(int64_t)t * Nh * k + (i - t * k)];
      counted[j] = mask ? mask[t] : 1;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i0 < n - j * THREADS && counted[j] && (unsigned)e[j] < (unsigned)Ne)
        atomicAdd(&hist[e[j]], 1);
  }
}

// All of head blockIdx.x's slots, where they are few: no launch in front to clear the
// counts.
constexpr int kCountAllThreads = 1024;
constexpr int64_t kCountAllSlots = 1 << 13;  // 32768 of them take 19 us, in two launches 8

__global__ __launch_bounds__(kCountAllThreads) void expert_counts_all_kernel(
    const int32_t* __restrict__ idx, const uint8_t* __restrict__ mask, int64_t T, int Nh, int Ne,
    int k, DivMagic by_k, int32_t* __restrict__ counts) {
  __shared__ int32_t hist[kMaxExperts];
  if ((int)threadIdx.x < Ne) hist[threadIdx.x] = 0;
  __syncthreads();
  count_slots<kCountAllThreads>(idx + blockIdx.x * k, mask, (int)T, Nh, Ne, k, by_k, hist);
  __syncthreads();
  if ((int)threadIdx.x < Ne) counts[(int64_t)blockIdx.x * Ne + threadIdx.x] = hist[threadIdx.x];
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
  count_slots<kCountThreads>(idx + (t0 * Nh + blockIdx.y) * k, mask ? mask + t0 : nullptr, here, Nh,
                             Ne, k, by_k, hist);
  __syncthreads();
  for (int e = threadIdx.x; e < Ne; e += kCountThreads)
    if (hist[e]) atomicAdd(&counts[(int64_t)blockIdx.y * Ne + e], hist[e]);
}

// ---------------------------------------------------------------------------
// Operands
// ---------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

__device__ __forceinline__ f32x16 mfma32_f16(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// v less one half of a register of two fp16 values, in one instruction.
template <int HALF>
__device__ __forceinline__ float minus_half(float v, uint32_t pair) {
  float r;
  if (HALF == 0)
    asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(pair), "v"(v));
  else
    asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(pair), "v"(v));
  return r;
}

// Eight values times a power of two as N fp16 pieces, each the nearest to what the ones
// before left.  The multiply comes with the conversion (v_fma_mix*_f16).
template <int N>
__device__ __forceinline__ void split8(const float (&f)[8], float up, u32x4 (&out)[N]) {
  static_assert(N <= 2, "pieces");
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w;
    asm("v_fma_mixlo_f16 %0, %1, %2, 0" : "=v"(w) : "v"(f[2 * i]), "v"(up));
    asm("v_fma_mixhi_f16 %0, %1, %2, 0" : "+v"(w) : "v"(f[2 * i + 1]), "v"(up));
    out[0][i] = w;
  }
  if constexpr (N == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[0,0,0] op_sel_hi:[0,0,1]"
          : "=v"(a) : "v"(f[2 * i]), "v"(up), "v"(out[0][i]));
      asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[0,0,1] op_sel_hi:[0,0,1]"
          : "=v"(b) : "v"(f[2 * i + 1]), "v"(up), "v"(out[0][i]));
      out[1][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
    }
  }
}

// Eight values as N fp16 pieces, each the nearest to what the ones before left.
template <int N>
__device__ __forceinline__ void split8(const float (&f)[8], u32x4 (&out)[N]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int p = 0; p < N; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f16x2 h = __builtin_convertvector((f32x2{r[2 * i], r[2 * i + 1]}), f16x2);
      out[p][i] = __builtin_bit_cast(uint32_t, h);
      if (p + 1 < N) {
        r[2 * i] = minus_half<0>(r[2 * i], out[p][i]);
        r[2 * i + 1] = minus_half<1>(r[2 * i + 1], out[p][i]);
      }
    }
}

// The power of two that takes values of magnitude up to `most` (its bits) below 2^15,
// and its inverse (a row below 2^-112 is not lifted further).
struct Pow2 {
  float up, down;
};
__device__ __forceinline__ Pow2 pow2_below_2_15(uint32_t most) {
  uint32_t e = most >> 23;
  e = e < 15u ? 15u : e > 254u ? 254u : e;
  return Pow2{__uint_as_float((268u - e) << 23), __uint_as_float((e - 14u) << 23)};
}
__device__ __forceinline__ float log2_of(float power) {  // exactly
  return (float)((int)(__float_as_uint(power) >> 23) - 127);
}
__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v)));
}
// What takes a block's scores (the products of x up and w up) to powers of two: log2 e
// over both powers.  At least 2^-126: an expert that is not there has the score -infinity,
// which times zero (a row of zeros, weights below 2^-9) would be NaN.  The scores are below
// 2^37 in the products' unit, so none moves by more than 2^-89.
__device__ __forceinline__ float score_scale(float x_down, float w_down) {
  return fmaxf(x_down * w_down * kLog2e, 0x1p-126f);
}
__device__ __forceinline__ uint32_t bits_abs(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Maximum over the LANES (8 or 16) lanes that share a row.
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  auto over = [&](auto ctrl) {
    v = umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF,
                                                      true));
  };
  over(std::integral_constant<int, 0xB1>{});   // quad_perm [1, 0, 3, 2]
  over(std::integral_constant<int, 0x4E>{});   // quad_perm [2, 3, 0, 1]
  over(std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (LANES == 16) over(std::integral_constant<int, 0x140>{});  // row_mirror
  return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = row_max<16>(v);
  v = umax(v, __shfl_xor(v, 16, kWave));
  return umax(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ long long wave_sum(long long v) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d, kWave);
  return v;
}

// f' = E c / total - 1 from exact whole numbers, with one division.
__device__ __forceinline__ float excess(int32_t c, int Ne, long long total) {
  return total > 0 ? (float)((double)((long long)c * Ne - total) / (double)total) : 0.0f;
}
// |f' - u| <= max f' - min f': the exponent F with |f' - u| 2^F < 2^14.
__device__ __forceinline__ float ds_exponent(uint32_t most, uint32_t least, int Ne,
                                             long long total) {
  const double R = total > 0 ? (double)((long long)(most - least) * Ne) / (double)total : 0.0;
  return R > 0.0 ? (float)(13 - ilogb(R)) : 0.0f;
}

// A matrix of rows of DH fp16 values in LDS, 16-byte units swizzled (swz_tr), and a lane's
// places in 32 of its rows as an operand: with the rows as the operand's rows (lane: row
// lane % 32, columns 16 s + 8 (lane / 32) + j), and transposed (lane: column 32 dt + lane
// % 32, rows 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4, the order in which the rows of a
// 32 x 32 product lie in a lane's registers).  The swizzle is linear and repeats after
// 16 rows, so everything but the lane's base is an exclusive or or an offset.
template <int DH>
struct Tile {
  static constexpr int kRow = DH * 2;
  static constexpr int kBytes = 32 * kRow;
  static __device__ __forceinline__ int unit(int row, int j) {
    return row * kRow + swz_tr<DH / 8>(j, row) * 16;
  }
  int rows, cols[2];
  __device__ __forceinline__ Tile() {
    const int lane = lane_id(), g = lane >> 5, c = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    rows = unit(lane & 31, g);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      cols[k] = unit(4 * g + 8 * k + ((lane & 15) >> 2), c >> 3) + (c & 7) * 2;
  }
  __device__ __forceinline__ u32x4 row_operand(const uint8_t* p, int s) const {
    return *reinterpret_cast<const u32x4*>(p + (rows ^ (s * 32)));
  }
  __device__ __forceinline__ u32x4 col_operand(const uint8_t* p, int dt, int s) const {
    const u32x2 lo = lds_read_tr16(p + 16 * s * kRow + (cols[0] ^ (dt * 64)));
    const u32x2 hi = lds_read_tr16(p + 16 * s * kRow + (cols[1] ^ (dt * 64)));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
};

// What lies behind the weights in the workspace, per head: f'_e of the experts (zeros up
// to the next multiple of 32), the blocks' powers of two (down) and F.
struct HeadInfo {
  float f[kMaxExperts];
  float down[kMaxExperts / 32];
  float F;
  float pad[31];
};
static_assert(sizeof(HeadInfo) == kBalanceHeadBytes, "workspace");

// The router's weights, grid (blocks of 32 experts, heads): two Tiles per block, the
// pieces of w up.
template <int DH>
__global__ __launch_bounds__(256) void balance_weights_kernel(const float* __restrict__ W,
                                                              const int32_t* __restrict__ counts,
                                                              int Ne, uint8_t* __restrict__ out,
                                                              HeadInfo* __restrict__ info) {
  constexpr int kUnits = DH / 8, kPer = 32 * kUnits / 256;
  __shared__ long long totals[4];
  __shared__ uint32_t tops[3][4];
  const int e0 = blockIdx.x * 32, h = blockIdx.y, lane = lane_id(), wave = threadIdx.x >> 6;
  const float* src = W + ((int64_t)h * Ne + e0) * DH;
  float v[kPer][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int unit = i * 256 + threadIdx.x;
    const bool ok = e0 + unit / kUnits < Ne;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const f32x4 x = ok ? *reinterpret_cast<const f32x4*>(src + unit * 8 + 4 * k) : f32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[i][4 * k + j] = x[j];
        top = umax(top, bits_abs(x[j]));
      }
    }
  }
  long long total = 0;
  uint32_t most = 0, least = 0xFFFFFFFFu;
  for (int e = threadIdx.x; e < Ne; e += 256) {
    const uint32_t c = (uint32_t)counts[(int64_t)h * Ne + e];
    total += (int32_t)c;
    most = umax(most, c);
    least = c < least ? c : least;
  }
  total = wave_sum(total);
  top = wave_max(top);
  most = wave_max(most);
  least = ~wave_max(~least);
  if (lane == 0) {
    totals[wave] = total;
    tops[0][wave] = top;
    tops[1][wave] = most;
    tops[2][wave] = ~least;
  }
  __syncthreads();
  total = totals[0] + totals[1] + totals[2] + totals[3];
  auto over_waves = [&](int k) {
    return umax(umax(tops[k][0], tops[k][1]), umax(tops[k][2], tops[k][3]));
  };
  const Pow2 scale = pow2_below_2_15(over_waves(0));
  if (threadIdx.x < 32) {
    const int e = e0 + threadIdx.x;
    info[h].f[e] = e < Ne ? excess(counts[(int64_t)h * Ne + e], Ne, total) : 0.0f;
    if (threadIdx.x == 0) {
      info[h].down[blockIdx.x] = scale.down;
      if (blockIdx.x == 0) info[h].F = ds_exponent(over_waves(1), ~over_waves(2), Ne, total);
    }
  }
  uint8_t* o = out + ((int64_t)h * gridDim.x + blockIdx.x) * 2 * Tile<DH>::kBytes;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int unit = i * 256 + threadIdx.x;
    u32x4 p[2];
    split8(v[i], scale.up, p);
#pragma unroll
    for (int q = 0; q < 2; ++q)
      *reinterpret_cast<u32x4*>(o + q * Tile<DH>::kBytes +
                                Tile<DH>::unit(unit / kUnits, unit % kUnits)) = p[q];
  }
}

// One lane's operand of X: token row, d = 16 s + 8 g + j, as NX pieces of x up, the
// row's power of two.
template <int DH, bool F32>
struct XOperand {
  static constexpr int NX = F32 ? 2 : 1;
  u32x4 x[NX][DH / 16];
  float down;
  u32x4 raw[DH / 16][F32 ? 2 : 1];
  // A readable row on its way; then as an operand, zeros unless ok (it counts).
  __device__ __forceinline__ void fetch(const void* X, int64_t row, int g) {
    const uint8_t* p = static_cast<const uint8_t*>(X) + (row * DH + 8 * g) * (F32 ? 4 : 2);
#pragma unroll
    for (int s = 0; s < DH / 16; ++s)
#pragma unroll
      for (int i = 0; i < (F32 ? 2 : 1); ++i)
        raw[s][i] = *reinterpret_cast<const u32x4*>(p + 16 * s * (F32 ? 4 : 2) + 16 * i);
  }
  __device__ __forceinline__ void convert(bool ok) {
    if (__any(!ok)) {
#pragma unroll
      for (int s = 0; s < DH / 16; ++s)
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i)
          if (!ok) raw[s][i] = u32x4{0, 0, 0, 0};
    }
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) top = top_of(raw[s], top);
    top = widen(top);
    top = umax(top, __shfl_xor(top, 32, kWave));
    const Pow2 scale = pow2_below_2_15(top);
    down = scale.down;
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) {
      float f[8];
      u32x4 o[NX];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = value(raw[s], i);
      split8(f, scale.up, o);
#pragma unroll
      for (int q = 0; q < NX; ++q) x[q][s] = o[q];
    }
  }
  __device__ __forceinline__ void load(const void* X, int64_t row, bool ok, int g) {
    fetch(X, row, g);
    convert(ok);
  }
  // The largest magnitude of eight and of top, for bf16 two at once, and its bits as fp32.
  template <int N>
  static __device__ __forceinline__ uint32_t top_of(const u32x4 (&raw)[N], uint32_t top) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
          top = umax(top, raw[n][i] & 0x7FFFFFFFu);
        } else {
          const uint32_t w = raw[n][i] & 0x7FFF7FFFu;
          top = __builtin_bit_cast(
              uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                  __builtin_bit_cast(u16x2, w)));
        }
      }
    return top;
  }
  static __device__ __forceinline__ uint32_t widen(uint32_t top) {
    return F32 ? top : umax(top << 16, top & 0xFFFF0000u);
  }
  // element i of eight as they lie in memory
  template <int N>
  static __device__ __forceinline__ float value(const u32x4 (&raw)[N], int i) {
    if constexpr (F32) return __uint_as_float(raw[i >> 2][i & 3]);
    const uint32_t w = raw[0][i >> 1];
    return __uint_as_float((i & 1) ? w & 0xFFFF0000u : w << 16);
  }
};

// One lane's operand of W, straight from memory: expert e, d = 16 s + 8 g + j, as two
// pieces of w up, the power of two of its wavefront's (or workgroup's) experts.
template <int DH>
struct WOperand {
  float v[DH / 16][8];
  u32x4 w[2][DH / 16];
  float down;
  // Head's weights Wh; zeros past the last expert.  Returns the lane's largest magnitude.
  __device__ __forceinline__ uint32_t load(const float* __restrict__ Wh, int e, int Ne, int g) {
    const float* src = Wh + (int64_t)(e < Ne ? e : Ne - 1) * DH + 8 * g;
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < DH / 16; ++s)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(src + 16 * s + 4 * k);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[s][4 * k + j] = e < Ne ? x[j] : 0.0f;
          top = umax(top, bits_abs(v[s][4 * k + j]));
        }
      }
    return top;
  }
  __device__ __forceinline__ void split(uint32_t top) {
    const Pow2 scale = pow2_below_2_15(top);
    down = scale.down;
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) {
      u32x4 o[2];
      split8(v[s], scale.up, o);
      w[0][s] = o[0];
      w[1][s] = o[1];
    }
  }
};

// What a head's counts give: their sum, and whether the head has any; all of a
// workgroup of THREADS.
struct HeadCounts {
  long long total;
  uint32_t most, least;
};
template <int THREADS>
__device__ __forceinline__ HeadCounts head_counts(const int32_t* __restrict__ counts, int Ne,
                                                  long long* totals, uint32_t (*tops)[2]) {
  const int wave = threadIdx.x >> 6;
  HeadCounts c{0, 0u, 0xFFFFFFFFu};
  for (int e = threadIdx.x; e < Ne; e += THREADS) {
    const uint32_t n = (uint32_t)counts[e];
    c.total += (int32_t)n;
    c.most = umax(c.most, n);
    c.least = n < c.least ? n : c.least;
  }
  c.total = wave_sum(c.total);
  c.most = wave_max(c.most);
  c.least = wave_max(~c.least);
  if (lane_id() == 0) {
    totals[wave] = c.total;
    tops[wave][0] = c.most;
    tops[wave][1] = c.least;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) {
    if (w != wave) c.total += totals[w];
    c.most = umax(c.most, tops[w][0]);
    c.least = umax(c.least, tops[w][1]);
  }
  c.least = ~c.least;
  return c;
}

// Scores of 32 experts (rows) x 32 tokens (lanes), times both powers of two, small
// products first.  e0: the block's first expert; rows past the last one have no weight.
template <int DH, bool F32>
__device__ __forceinline__ f32x16 score_tile(const uint8_t* w, const Tile<DH>& at,
                                             const XOperand<DH, F32>& x, int e0, int Ne) {
  f32x16 z = zero16();
#pragma unroll
  for (int q = 1; q >= 0; --q)
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) {
      const u32x4 a = at.row_operand(w + q * Tile<DH>::kBytes, s);
#pragma unroll
      for (int p = XOperand<DH, F32>::NX - 1; p >= 0; --p)
        if (p + q <= 1) z = mfma32_f16(a, x.x[p][s], z);
    }
  if (e0 + 32 > Ne) {
    asm volatile("");  // a branch, not 48 instructions for every block
#pragma unroll
    for (int v = 0; v < 16; ++v)
      z[v] = e0 + mfma32_row(v, lane_id()) < Ne ? z[v] : -INFINITY;
  }
  return z;
}

// The same with the weights in registers.
template <int DH, bool F32>
__device__ __forceinline__ f32x16 score_tile(const WOperand<DH>& w, const XOperand<DH, F32>& x,
                                             int e0, int Ne) {
  f32x16 z = zero16();
#pragma unroll
  for (int q = 1; q >= 0; --q)
#pragma unroll
    for (int s = 0; s < DH / 16; ++s)
#pragma unroll
      for (int p = XOperand<DH, F32>::NX - 1; p >= 0; --p)
        if (p + q <= 1) z = mfma32_f16(w.w[q][s], x.x[p][s], z);
  if (e0 + 32 > Ne) {
    asm volatile("");
#pragma unroll
    for (int v = 0; v < 16; ++v)
      z[v] = e0 + mfma32_row(v, lane_id()) < Ne ? z[v] : -INFINITY;
  }
  return z;
}

// The running maximum (times log2 e), sum and weighted sum of a token's softmax.
struct Running {
  float M = -INFINITY, l = 0.0f, u = 0.0f;
  // 32 experts' scores times m = log2 e over their power of two; f: their f'.
  __device__ __forceinline__ void add(const f32x16& z, float m, const float* f, int g) {
    float top = z[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) top = fmaxf(top, z[v]);
    const float Mn = fmaxf(M, top * m);
    const float ref = Mn == -INFINITY ? 0.0f : Mn;
    const float old = __builtin_amdgcn_exp2f(M - ref);
    l *= old;
    u *= old;
    M = Mn;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 f4 = *reinterpret_cast<const f32x4*>(f + 8 * q + 4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(z[4 * q + i], m, -ref));
        l += p;
        u = fmaf(p, f4[i], u);
      }
    }
  }
  // Together with another part of the token's experts, one of which has a weight.
  __device__ __forceinline__ void join(float Mo, float lo, float uo) {
    const float Mt = fmaxf(M, Mo);
    const float a = __builtin_amdgcn_exp2f(M - Mt), c = __builtin_amdgcn_exp2f(Mo - Mt);
    l = l * a + lo * c;
    u = u * a + uo * c;
    M = Mt;
  }
  __device__ __forceinline__ void join_halves() {
    join(__shfl_xor(M, 32, kWave), __shfl_xor(l, 32, kWave), __shfl_xor(u, 32, kWave));
  }
  __device__ __forceinline__ float2 stats(bool ok) const {
    return float2{ok ? (M + __builtin_amdgcn_logf(l)) * kLn2 : 0.0f, ok ? u / l : 0.0f};
  }
};

// A block's weights to LDS, a KB per wavefront in turn, by DMA that the compiler does not
// track: barrier_vm<0> before they are read.
template <int DH>
__device__ __forceinline__ void fetch_block(u32x4 rsrc, int b, uint8_t* lds) {
  constexpr uint32_t kBlock = 2 * Tile<DH>::kBytes;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const uint32_t voff = lane_id() * 16;
#pragma unroll
  for (uint32_t i = 0; i < kBlock; i += kTokenWaves * 1024u)
    dma_lds16(rsrc, lds + i + wave * 1024u, voff, (uint32_t)b * kBlock + i + wave * 1024u);
}

// ---------------------------------------------------------------------------
// The loss: 32 tokens of a head per wavefront, over all experts, whose operands go
// through LDS in two buffers.  A workgroup's head is blockIdx.x % Nh: workgroups go
// round the dies, so with 8 heads a die has one head's weights in its L2.
// ---------------------------------------------------------------------------
template <int DH, bool F32>
__global__ __launch_bounds__(kTokenWaves* kWave) void balance_loss_kernel(
    const void* __restrict__ X, const uint8_t* __restrict__ weights,
    const HeadInfo* __restrict__ info, const uint8_t* __restrict__ mask, int64_t T, int Nh, int Ne,
    float2* __restrict__ stats, double* __restrict__ part) {
  constexpr uint32_t kBlock = 2 * Tile<DH>::kBytes;
  __shared__ __align__(16) uint8_t w[2][kBlock];
  __shared__ __align__(16) float fex[kMaxExperts];
  __shared__ double loss[kTokenWaves];
  const int h = blockIdx.x % Nh, lane = lane_id(), g = lane >> 5, wave = threadIdx.x >> 6;
  const int64_t tb = blockIdx.x / Nh, t = tb * kBalanceTokens + wave * 32 + (lane & 31);
  const int64_t near = t < T ? t : T - 1;
  const int nb = (Ne + 31) / 32;
  const u32x4 rsrc = buffer_words(weights + (int64_t)h * nb * kBlock, (uint32_t)nb * kBlock);
  fetch_block<DH>(rsrc, 0, w[0]);
  const Tile<DH> at;
  // (workgroups that go on to further tokens, fetched ahead, gave nothing: 322.9 -> 330 us at
  // 65536 x 8 heads x 1024 experts, 43.1 -> 43 at 16384 x 16 x 128 with its counts)
  XOperand<DH, F32> x;
  x.fetch(X, near * Nh + h, g);
  const bool ok = (mask ? mask[near] != 0 : true) && t < T;
  for (int e = threadIdx.x; e < nb * 32; e += kTokenWaves * kWave) fex[e] = info[h].f[e];
  x.convert(ok);
  Running run;
  for (int b = 0; b < nb; ++b) {
    const float m = score_scale(x.down, info[h].down[b]);
    barrier_vm<0>();
    if (b + 1 < nb) fetch_block<DH>(rsrc, b + 1, w[(b + 1) & 1]);
    run.add(score_tile<DH, F32>(w[b & 1], at, x, 32 * b, Ne), m, fex + 32 * b, g);
  }
  run.join_halves();
  const float2 st = run.stats(ok);
  if (g == 0 && t < T) stats[t * Nh + h] = st;
  double sum = g == 0 ? (double)st.y : 0.0;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor(sum, d, kWave);
  if (lane == 0) loss[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < kTokenWaves; ++i) sum += loss[i];
    part[h * ceil_div(T, kBalanceTokens) + tb] = sum;
  }
}

// The loss where there are few tokens: eight wavefronts, EG of them for the blocks of
// experts in turn, the others for as many groups of 32 tokens; weights straight from
// memory, no launch in front.  A head's tokens in one workgroup: also its loss, with no
// launch behind.
constexpr int kFewThreads = kBalanceFewWaves * kWave;

template <int DH, bool F32, int EG>
__global__ __launch_bounds__(kFewThreads) void balance_loss_few_kernel(
    const void* __restrict__ X, const float* __restrict__ W, const int32_t* __restrict__ counts,
    const uint8_t* __restrict__ mask, int64_t T, int Nh, int Ne, float2* __restrict__ stats,
    double* __restrict__ part, float* __restrict__ loss) {
  constexpr int TG = kBalanceFewWaves / EG;
  __shared__ __align__(16) float fex[kMaxExperts];
  __shared__ long long totals[kBalanceFewWaves];
  __shared__ uint32_t tops[kBalanceFewWaves][2];
  __shared__ float runs[EG][3][TG * 32];
  __shared__ double sums[TG];
  __shared__ int tokens[TG];
  const int h = blockIdx.x % Nh, lane = lane_id(), g = lane >> 5, wave = threadIdx.x >> 6;
  const int eg = wave % EG, tg = wave / EG;
  const int64_t tb = blockIdx.x / Nh, t = tb * (TG * 32) + tg * 32 + (lane & 31);
  const int64_t near = t < T ? t : T - 1;
  const bool counted = mask ? mask[near] != 0 : true;
  const float* Wh = W + (int64_t)h * Ne * DH;
  WOperand<DH> w;
  uint32_t top = w.load(Wh, 32 * eg + (lane & 31), Ne, g);
  const HeadCounts c = head_counts<kFewThreads>(counts + (int64_t)h * Ne, Ne, totals, tops);
  for (int e = threadIdx.x; e < ((Ne + 31) & ~31); e += kFewThreads)
    fex[e] = e < Ne ? excess(counts[(int64_t)h * Ne + e], Ne, c.total) : 0.0f;
  const bool ok = t < T && counted;
  XOperand<DH, F32> x;
  x.load(X, near * Nh + h, ok, g);
  __syncthreads();
  Running run;
  for (int b = eg; b * 32 < Ne; b += EG) {
    w.split(wave_max(top));
    const float m = score_scale(x.down, w.down);
    const f32x16 z = score_tile<DH, F32>(w, x, 32 * b, Ne);
    if ((b + EG) * 32 < Ne) top = w.load(Wh, 32 * (b + EG) + (lane & 31), Ne, g);
    run.add(z, m, fex + 32 * b, g);
  }
  // (a wavefront without experts has M = -infinity, which join_halves would make NaN)
  if (eg * 32 < Ne) run.join_halves();
  if constexpr (EG > 1) {
    if (g == 0) {
      runs[eg][0][tg * 32 + lane] = run.M;
      runs[eg][1][tg * 32 + lane] = run.l;
      runs[eg][2][tg * 32 + lane] = run.u;
    }
    __syncthreads();
    if (eg == 0) {
      const int at = tg * 32 + (lane & 31);
#pragma unroll
      for (int i = 1; i < EG; ++i) run.join(runs[i][0][at], runs[i][1][at], runs[i][2][at]);
    }
  }
  if (eg == 0) {
    const float2 st = run.stats(ok);
    if (g == 0 && t < T) stats[t * Nh + h] = st;
    double sum = g == 0 ? (double)st.y : 0.0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor(sum, d, kWave);
    if (lane == 0) sums[tg] = sum;
    const int n = __popcll(__ballot(ok && g == 0));
    if (lane == 0) tokens[tg] = n;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double sum = sums[0];
    int n = tokens[0];
#pragma unroll
    for (int i = 1; i < TG; ++i) {
      sum += sums[i];
      n += tokens[i];
    }
    if (T > TG * 32) {
      part[h * ceil_div(T, TG * 32) + tb] = sum;
    } else {
      const double m = n > 0 ? (double)n : 1.0;
      loss[h] = c.total > 0 ? (float)(1.0 + sum / m) : 0.0f;
      stats[T * Nh + h] = float2{(float)(1.0 / m), 0.0f};
    }
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
  if (mask) {
    // 16 bytes at once: the number that is not zero, by folding each to its low bit
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < T / 16; i += 256) {
      const u32x4 m = reinterpret_cast<const u32x4*>(mask)[i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t v = m[k];
        v |= v >> 4;
        v |= v >> 2;
        v |= v >> 1;  // (bits from the next byte reach only the upper seven)
        n += __popc(v & 0x01010101u);
      }
    }
    for (int64_t t = T / 16 * 16 + threadIdx.x; t < T; t += 256) n += mask[t] != 0;
  }
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
// dX: 32 tokens of a head per wavefront, over all experts, as in the loss; ds and W as two
// fp16 values each, whatever X's type: dX is rounded once, when dX_add is added (one
// value each, 2^-10 off per term, took 415 us where two take 598: bf16, 65536 tokens x 8
// heads x 1024 experts).  ds comes out of the exponential as ds 2^(F + K - k_b), with the
// block's power k_b and the head's smallest K, so that all blocks' products add up alike;
// the rest of the factors come at the end.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void split_ds(const f32x16& ds, int s, u32x4 (&out)[2]) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = ds[8 * s + j];
  split8(f, out);
}

// dX^T += W^T ds of 32 experts x 32 tokens.
template <int DH>
__device__ __forceinline__ void add_dx(const f32x16& z, const uint8_t* w, const Tile<DH>& at,
                                       f32x16 (&dx)[DH / 32]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    u32x4 ds[2];
    split_ds(z, s, ds);
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
      for (int q = 1; q >= 0; --q) {
        const u32x4 a = at.col_operand(w + q * Tile<DH>::kBytes, dt, s);
#pragma unroll
        for (int p = 1 - q; p >= 0; --p) dx[dt] = mfma32_f16(a, ds[p], dx[dt]);
      }
  }
}

// A lane's part of its token's row of dX, times c, added to dX_add's.  c = 0 is for a
// token that does not count, whose sums are dropped.
template <int DH, bool F32>
__device__ __forceinline__ void store_dx(const f32x16 (&dx)[DH / 32], float c, int64_t row,
                                         const void* dX_add, void* dX) {
  const int g = lane_id() >> 5;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t to = row * DH + 32 * dt + 8 * q + 4 * g;
      float f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = c != 0.0f ? dx[dt][4 * q + i] * c : 0.0f;
      if (F32) {
        if (dX_add) {
          const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const float*>(dX_add) + to);
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] += a[i];
        }
        *reinterpret_cast<f32x4*>(static_cast<float*>(dX) + to) = f32x4{f[0], f[1], f[2], f[3]};
      } else {
        if (dX_add) {
          const u32x2 a = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(dX_add) + to);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            f[i] += bf16_bits_to_f32((a[i >> 1] >> (16 * (i & 1))) & 0xFFFFu);
        }
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(dX) + to) =
            u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
      }
    }
}

// The same for a wavefront's 32 tokens from t0 on, through a Tile of LDS, so that whole
// rows are read and written (by lanes' own pieces of 8 bytes the kernel took 80 us where
// it took 55 so, 48 now: 16384 x 16 heads x 16 experts).
template <int DH, bool F32>
__device__ __forceinline__ void store_dx_rows(const f32x16 (&dx)[DH / 32], bool ok, float c,
                                              int64_t t0, int64_t T, int Nh, int h, uint8_t* tile,
                                              const void* dX_add, void* dX) {
  constexpr int kUnits = DH / 8, kRows = kWave / kUnits;  // 16-byte units, rows per access
  constexpr int kPasses = F32 ? 2 : 1;                    // fp32: half a row at a time
  const int lane = lane_id(), g = lane >> 5, r0 = lane / kUnits, j = lane % kUnits;
#pragma unroll
  for (int pass = 0; pass < kPasses; ++pass) {
    auto row = [&](int i) { return t0 + r0 + kRows * i; };
    auto address = [&](int i) {
      return ((row(i) * Nh + h) * DH) * (F32 ? 4 : 2) + pass * DH * 2 + 16 * j;
    };
    auto place = [&](int i) {
      return reinterpret_cast<u32x4*>(tile + Tile<DH>::unit(r0 + kRows * i, j));
    };
    if (dX_add) {
      u32x4 add[32 / kRows];
#pragma unroll
      for (int i = 0; i < 32 / kRows; ++i)
        add[i] = row(i) < T ? *reinterpret_cast<const u32x4*>(
                                  static_cast<const uint8_t*>(dX_add) + address(i))
                            : u32x4{0, 0, 0, 0};
      wave_lds_order();  // the readers of what was there
#pragma unroll
      for (int i = 0; i < 32 / kRows; ++i) *place(i) = add[i];
    }
    wave_lds_order();
#pragma unroll
    for (int i = 0; i < DH / 8 / kPasses; ++i) {
      const int dt = i / 4 + pass * (DH / 32 / kPasses), q = i % 4;
      float f[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = ok ? dx[dt][4 * q + k] * c : 0.0f;
      if constexpr (F32) {
        f32x4* p = reinterpret_cast<f32x4*>(tile + Tile<DH>::unit(lane & 31, 2 * i + g));
        f32x4 v{f[0], f[1], f[2], f[3]};
        if (dX_add) v += *p;
        *p = v;
      } else {
        u32x2* p = reinterpret_cast<u32x2*>(tile + Tile<DH>::unit(lane & 31, i) + 8 * g);
        if (dX_add) {
          const u32x2 a = *p;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            f[k] += bf16_bits_to_f32((a[k >> 1] >> (16 * (k & 1))) & 0xFFFFu);
        }
        *p = u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
      }
    }
    wave_lds_order();
#pragma unroll
    for (int i = 0; i < 32 / kRows; ++i)
      if (row(i) < T)
        *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(dX) + address(i)) = *place(i);
  }
}

// The largest of the head's blocks' powers down (2^-K), in every lane.
__device__ __forceinline__ float head_down(const HeadInfo& info, int nb) {
  float d = lane_id() < nb ? info.down[lane_id()] : 0.0f;
#pragma unroll
  for (int i = 1; i < 32; i <<= 1) d = fmaxf(d, __shfl_xor(d, i, kWave));
  return uniform(d);
}

struct DxArgs {
  const void* X;
  const uint8_t* weights;
  const HeadInfo* info;
  const float2* stats;
  const float* dloss;
  const uint8_t* mask;
  const void* dX_add;
  int64_t T;
  int Nh, Ne;
  void* dX;
};
template <int DH>
struct DxShared {
  __align__(16) uint8_t w[2][2 * Tile<DH>::kBytes];
  __align__(16) float fex[kMaxExperts];
};

template <int DH, bool F32>
__device__ __forceinline__ void balance_dx(const DxArgs& a, unsigned block, DxShared<DH>& sm) {
  constexpr uint32_t kBlock = 2 * Tile<DH>::kBytes;
  const float2* __restrict__ stats = a.stats;
  const HeadInfo* __restrict__ info = a.info;
  const uint8_t* __restrict__ mask = a.mask;
  const int64_t T = a.T;
  const int Nh = a.Nh, Ne = a.Ne;
  auto& w = sm.w;
  auto& fex = sm.fex;
  const int h = block % Nh, lane = lane_id(), g = lane >> 5, wave = threadIdx.x >> 6;
  const int64_t t = (int64_t)(block / Nh) * kBalanceTokens + wave * 32 + (lane & 31);
  const int64_t row = t * Nh + h;
  const bool ok = t < T && (!mask || mask[t < T ? t : 0]);
  const int nb = (Ne + 31) / 32;
  const u32x4 rsrc = buffer_words(a.weights + (int64_t)h * nb * kBlock, (uint32_t)nb * kBlock);
  fetch_block<DH>(rsrc, 0, w[0]);
  const Tile<DH> at;
  for (int e = threadIdx.x; e < nb * 32; e += kTokenWaves * kWave) fex[e] = info[h].f[e];
  XOperand<DH, F32> x;
  x.load(a.X, (t < T ? t : T - 1) * Nh + h, ok, g);
  // a token that does not count: p = exp2(-infinity) = 0
  const float2 st = ok ? stats[row] : float2{INFINITY, 0.0f};
  const float down = head_down(info[h], nb), F = info[h].F;
  const float u = st.y, lse = st.x * kLog2e - F;
  const float c = a.dloss[h] * stats[T * Nh + h].x * __builtin_amdgcn_ldexpf(down, -(int)F);
  f32x16 dx[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) dx[i] = zero16();
  for (int b = 0; b < nb; ++b) {
    const float down_b = info[h].down[b];
    const float m = score_scale(x.down, down_b);
    const float ref = lse - (log2_of(down_b) - log2_of(down));
    barrier_vm<0>();
    if (b + 1 < nb) fetch_block<DH>(rsrc, b + 1, w[(b + 1) & 1]);
    const uint8_t* wb = w[b & 1];
    f32x16 z = score_tile<DH, F32>(wb, at, x, 32 * b, Ne);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 f = *reinterpret_cast<const f32x4*>(&fex[32 * b + 8 * q + 4 * g]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        z[4 * q + i] = __builtin_amdgcn_exp2f(fmaf(z[4 * q + i], m, -ref)) * (f[i] - u);
    }
    add_dx<DH>(z, wb, at, dx);
  }
  __syncthreads();  // the weights' LDS is the rows' now
  store_dx_rows<DH, F32>(dx, ok, c, t - (lane & 31), T, Nh, h, &w[0][0] + wave * Tile<DH>::kBytes,
                         a.dX_add, a.dX);
}

template <int DH, bool F32>
__global__ __launch_bounds__(kTokenWaves* kWave) void balance_dx_kernel(const DxArgs a) {
  __shared__ DxShared<DH> sm;
  balance_dx<DH, F32>(a, blockIdx.x, sm);
}

// ---------------------------------------------------------------------------
// dW: a block of 32 experts per wavefront, whose weights stay in its registers, over
// a chunk of the tokens, 32 SUB at a time through LDS in two buffers (EW blocks of
// experts in a workgroup; SUB = 4 / EW wavefronts share one where there are fewer than
// four, each with 32 tokens of its own).  X lies in LDS as pieces of x up (a token's power of
// two), read along d for the scores and transposed for dW; what up adds is taken off
// ds in its exponential.  ds is two fp16 values times S, a power of two that every
// expert (lane) has for itself: it is lowered, and the sums with it, when a ds does not
// fit any more, so an expert that gets little weight keeps its digits.
// ---------------------------------------------------------------------------
constexpr int kDwWaves = 4;
constexpr int dw_waves(int blocks) { return blocks > kDwWaves ? blocks : kDwWaves; }
constexpr float kDwFirst = 0x1p60f;  // S before the first ds: any above 2^-45 lowers it

template <int DH, bool F32, int EW>
struct DwShared {
  static constexpr int NX = F32 ? 2 : 1, SUB = dw_waves(EW) / EW;
  static constexpr int kTiles = 2 * NX * SUB * Tile<DH>::kBytes;
  static constexpr int kSums = (SUB - 1) * EW * 32 * DH * 4;  // of all but a block's first wavefront
  __align__(16) uint8_t xs[kTiles > kSums ? kTiles : kSums];
  __align__(16) float ms[2][32 * SUB], refs[2][32 * SUB], us[2][32 * SUB];
  long long totals[dw_waves(EW)];
  uint32_t tops[dw_waves(EW)][2];
};

struct DwArgs {
  const void* X;
  const float* W;
  const int32_t* counts;
  const float2* stats;
  const float* dloss;
  const uint8_t* mask;
  const float* dW_add;
  int64_t T;
  int Nh, Ne, groups, splits;
  float *dW, *part;
};

// Where a lane's largest ds (top, of its half of the rows) does not fit fp16 any more, S, ds
// and the sums down by a power of two that takes it to [2^10, 2^11).
template <int N>
__device__ __forceinline__ bool lower_to_fit(float top, f32x16& z, f32x16 (&dw)[N], float& S) {
  const u32x2 both = permlane32_swap(__float_as_uint(top), __float_as_uint(top));
  top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
  if (!__any(top >= 32768.0f)) return false;
  uint32_t ex = __float_as_uint(top) >> 23;
  ex = ex > 254u ? 254u : ex;
  const float k = top >= 32768.0f ? __uint_as_float((264u - ex) << 23) : 1.0f;
  S *= k;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] *= k;
#pragma unroll
  for (int dt = 0; dt < N; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) dw[dt][v] *= k;
  return true;
}

// A lane's expert's part of dW: c times it where there is one chunk, else a partial result.
template <int DH>
__device__ __forceinline__ void store_dw(const DwArgs& a, const f32x16 (&dw)[DH / 32], int h,
                                         int split, int nb, int e, float c) {
  if (e >= a.Ne) return;
  const int g = lane_id() >> 5;
  const bool whole = a.splits == 1;
  const int64_t row = ((int64_t)h * a.Ne + e) * DH;
  float* o = whole ? a.dW + row : a.part + (((int64_t)split * a.Nh + h) * nb * 32 + e) * DH;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int d = 32 * dt + 8 * q + 4 * g;
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = dw[dt][4 * q + i] * (whole ? c : 1.0f);
      if (whole && a.dW_add) v += *reinterpret_cast<const f32x4*>(a.dW_add + row + d);
      *reinterpret_cast<f32x4*>(o + d) = v;
    }
}

template <int DH, bool F32, int EW>
__device__ __forceinline__ void balance_dw(const DwArgs& a, unsigned block,
                                           DwShared<DH, F32, EW>& sm) {
  constexpr int NX = F32 ? 2 : 1, SUB = dw_waves(EW) / EW, kTokens = 32 * SUB;
  constexpr int kUnits = DH / 8;                               // 16-byte units of a row
  constexpr int kPer = kTokens * kUnits / (dw_waves(EW) * kWave);  // units per thread
  constexpr int kPiece = SUB * Tile<DH>::kBytes;
  const void* __restrict__ X = a.X;
  const float* __restrict__ W = a.W;
  const int32_t* __restrict__ counts = a.counts;
  const float2* __restrict__ stats = a.stats;
  const uint8_t* __restrict__ mask = a.mask;
  const int64_t T = a.T;
  const int Nh = a.Nh, Ne = a.Ne, groups = a.groups, splits = a.splits;
  uint8_t* const xs = sm.xs;
  auto& ms = sm.ms;
  auto& refs = sm.refs;
  auto& us = sm.us;
  const int lane = lane_id(), g = lane >> 5, wave = threadIdx.x >> 6;
  // all groups of a (head, chunk) on one die, which then reads its tokens once
  const int slot = block / kXcds, group = slot % groups;
  const int64_t pair = (int64_t)(slot / groups) * kXcds + block % kXcds;
  if (pair >= (int64_t)Nh * splits) return;
  const int h = (int)(pair % Nh), split = (int)(pair / Nh);
  const int nb = (Ne + 31) / 32, b = group * EW + wave % EW, sub = wave / EW;
  const int e = 32 * b + (lane & 31);
  const bool live = e < Ne;
  const int64_t tiles = (T + kTokens - 1) / kTokens;
  const int64_t begin = tiles * split / splits, end = tiles * (split + 1) / splits;
  // a tile's rows and their stats on their way (nothing waits for the mask: what a token
  // that does not count has is read and dropped), then in LDS
  u32x4 raw[kPer][F32 ? 2 : 1];
  float2 st[kPer];
  uint8_t counted[kPer];
  auto fetch = [&](int64_t tile) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int unit = i * dw_waves(EW) * kWave + threadIdx.x;
      int64_t t = tile * kTokens + unit / kUnits;
      t = t < T ? t : T - 1;
      const uint8_t* p = static_cast<const uint8_t*>(X) +
                         ((t * Nh + h) * DH + 8 * (unit % kUnits)) * (F32 ? 4 : 2);
#pragma unroll
      for (int k = 0; k < (F32 ? 2 : 1); ++k)
        raw[i][k] = *reinterpret_cast<const u32x4*>(p + 16 * k);
      st[i] = stats[t * Nh + h];
      counted[i] = mask ? mask[t] : 1;
    }
  };
  if (begin < end) fetch(begin);
  // the lane's expert: f' and, scaled alike for all of the workgroup's experts, its weights
  WOperand<DH> w;
  const uint32_t top = w.load(W + (int64_t)h * Ne * DH, e, Ne, g);
  const HeadCounts hc =
      head_counts<dw_waves(EW) * kWave>(counts + (int64_t)h * Ne, Ne, sm.totals, sm.tops);
  const float f = live ? excess(counts[(int64_t)h * Ne + e], Ne, hc.total) : 0.0f;
  {
    uint32_t most = wave_max(top);
    __syncthreads();  // the readers of tops
    if (lane == 0) sm.tops[wave][0] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < dw_waves(EW); ++i) most = umax(most, sm.tops[i][0]);
    w.split(most);
  }
  const float down = w.down;
  f32x16 dw[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) dw[i] = zero16();
  float S = kDwFirst, fS = f * kDwFirst;  // S and f' S
  auto store = [&](int64_t tile, int buf) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int unit = i * dw_waves(EW) * kWave + threadIdx.x, r = unit / kUnits;
      const bool ok = tile * kTokens + r < T && counted[i];
      if (__any(!ok)) {
#pragma unroll
        for (int k = 0; k < (F32 ? 2 : 1); ++k)
          if (!ok) raw[i][k] = u32x4{0, 0, 0, 0};
      }
      using Row = XOperand<DH, F32>;
      const Pow2 scale =
          pow2_below_2_15(row_max<kUnits>(Row::widen(Row::top_of(raw[i], 0u))));
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = Row::value(raw[i], k);
      u32x4 o[NX];
      split8(v, scale.up, o);
#pragma unroll
      for (int p = 0; p < NX; ++p)
        *reinterpret_cast<u32x4*>(xs + (buf * NX + p) * kPiece +
                                  Tile<DH>::unit(r, unit % kUnits)) = o[p];
      if (unit % kUnits == 0) {
        // a token that does not count: p = exp2(-infinity) = 0
        ms[buf][r] = scale.down * down * kLog2e;
        refs[buf][r] = ok ? fmaf(st[i].x, kLog2e, -log2_of(scale.down)) : INFINITY;
        us[buf][r] = ok ? st[i].y : 0.0f;
      }
    }
  };
  const Tile<DH> at;
  if (begin < end) store(begin, 0);
  for (int64_t tile = begin; tile < end; ++tile) {
    const int buf = (int)(tile - begin) & 1;
    __syncthreads();
    if (tile + 1 < end) fetch(tile + 1);
    const uint8_t* xb = xs + buf * NX * kPiece + sub * Tile<DH>::kBytes;
    // scores of 32 tokens (rows) x 32 experts (lanes)
    f32x16 z = zero16();
#pragma unroll
    for (int p = NX - 1; p >= 0; --p)
#pragma unroll
      for (int s = 0; s < DH / 16; ++s) {
        const u32x4 a = at.row_operand(xb + p * kPiece, s);
#pragma unroll
        for (int q = 1 - p; q >= 0; --q) z = mfma32_f16(a, w.w[q][s], z);
      }
    float top = 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = 32 * sub + 8 * q + 4 * g;
      const f32x4 m4 = *reinterpret_cast<const f32x4*>(&ms[buf][r]);
      const f32x4 r4 = *reinterpret_cast<const f32x4*>(&refs[buf][r]);
      const f32x4 u4 = *reinterpret_cast<const f32x4*>(&us[buf][r]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[4 * q + i] =
            __builtin_amdgcn_exp2f(fmaf(z[4 * q + i], m4[i], -r4[i])) * fmaf(-S, u4[i], fS);
        top = fmaxf(top, fabsf(z[4 * q + i]));
      }
    }
    if (lower_to_fit(top, z, dw, S)) fS = f * S;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 ds[2];
      split_ds(z, s, ds);
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
        for (int p = NX - 1; p >= 0; --p) {
          const u32x4 a = at.col_operand(xb + p * kPiece, dt, s);
#pragma unroll
          for (int q = 1 - p; q >= 0; --q) dw[dt] = mfma32_f16(a, ds[q], dw[dt]);
        }
    }
    if (tile + 1 < end) store(tile + 1, buf ^ 1);
  }
  const float k = 1.0f / S;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) dw[dt][v] *= k;
  // the wavefronts that share a block, in order
  if constexpr (SUB > 1) {
    f32x4* sums = reinterpret_cast<f32x4*>(xs);
    auto place = [&](int w, int i) { return ((w - EW) * (DH / 8) + i) * kWave + lane; };
    __syncthreads();
    if (sub > 0) {
#pragma unroll
      for (int i = 0; i < DH / 8; ++i)
        sums[place(wave, i)] = f32x4{dw[i / 4][4 * (i % 4)], dw[i / 4][4 * (i % 4) + 1],
                                     dw[i / 4][4 * (i % 4) + 2], dw[i / 4][4 * (i % 4) + 3]};
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int r = 1; r < SUB; ++r)
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) {
        const f32x4 v = sums[place(wave + r * EW, i)];
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i / 4][4 * (i % 4) + j] += v[j];
      }
  }
  store_dw<DH>(a, dw, h, split, nb, e, splits == 1 ? a.dloss[h] * stats[T * Nh + h].x : 1.0f);
}

template <int DH, bool F32, int EW>
__global__ __launch_bounds__(dw_waves(EW)* kWave) void balance_dw_kernel(const DwArgs a) {
  __shared__ DwShared<DH, F32, EW> sm;
  balance_dw<DH, F32, EW>(a, blockIdx.x, sm);
}

// dW (first, its workgroups take longest) and dX in one launch, where neither fills the
// card.
template <int DH, bool F32, int EW>
__global__ __launch_bounds__(kDwWaves* kWave) void balance_dw_dx_kernel(const DwArgs dw,
                                                                        const DxArgs dx,
                                                                        unsigned dw_blocks) {
  static_assert(kDwWaves == kTokenWaves, "one launch");
  __shared__ union Shared {
    DwShared<DH, F32, EW> dw;
    DxShared<DH> dx;
    __device__ Shared() {}
  } sm;
  if (blockIdx.x < dw_blocks)
    balance_dw<DH, F32, EW>(dw, blockIdx.x, sm.dw);
  else
    balance_dx<DH, F32>(dx, blockIdx.x - dw_blocks, sm.dx);
}

// ---------------------------------------------------------------------------
// The gradient where there are few tokens, in one launch: the first workgroups make dX,
// the others dW.  For dX EG wavefronts of a workgroup take the blocks of experts in turn,
// the others as many groups of 32 tokens; weights straight from memory, and through
// a Tile of the wavefront's own to be read transposed.  The products add up in the unit
// of the largest weights so far (down), to which both are lowered when larger ones come.
// ---------------------------------------------------------------------------
template <int DH, int EG>
struct DxFewShared {
  static constexpr int kTiles = kDwWaves * 2 * Tile<DH>::kBytes;
  static constexpr int kSums = (kDwWaves - kDwWaves / EG) * 32 * DH * 4;
  __align__(16) uint8_t ws[kTiles > kSums ? kTiles : kSums];
  __align__(16) float fex[kMaxExperts];
  long long totals[kDwWaves];
  uint32_t tops[kDwWaves][2];
};

template <int DH, bool F32, int EG>
__device__ __forceinline__ void balance_dx_few(const DwArgs& a, const void* dX_add, void* dX,
                                               unsigned block,
                                               DxFewShared<DH, EG>& sm) {
  constexpr int TG = kDwWaves / EG;
  const int64_t T = a.T;
  const int Nh = a.Nh, Ne = a.Ne;
  const int h = block % Nh, lane = lane_id(), g = lane >> 5, wave = threadIdx.x >> 6;
  const int eg = wave % EG, tg = wave / EG;
  const int64_t t = (int64_t)(block / Nh) * (TG * 32) + tg * 32 + (lane & 31);
  const int64_t near = t < T ? t : T - 1;
  const bool counted = a.mask ? a.mask[near] != 0 : true;
  const float* Wh = a.W + (int64_t)h * Ne * DH;
  const int32_t* counts = a.counts + (int64_t)h * Ne;
  WOperand<DH> w;
  uint32_t top = w.load(Wh, 32 * eg + (lane & 31), Ne, g);
  float2 st = a.stats[near * Nh + h];
  const HeadCounts hc = head_counts<kDwWaves * kWave>(counts, Ne, sm.totals, sm.tops);
  for (int e = threadIdx.x; e < ((Ne + 31) & ~31); e += kDwWaves * kWave)
    sm.fex[e] = e < Ne ? excess(counts[e], Ne, hc.total) : 0.0f;
  const float F = ds_exponent(hc.most, hc.least, Ne, hc.total);
  const bool ok = t < T && counted;
  if (!ok) st = float2{INFINITY, 0.0f};  // p = exp2(-infinity) = 0
  XOperand<DH, F32> x;
  x.load(a.X, near * Nh + h, ok, g);
  const float lse = st.x * kLog2e - F;
  f32x16 dx[DH / 32];
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) dx[i] = zero16();
  const Tile<DH> at;
  uint8_t* const ws = sm.ws + wave * 2 * Tile<DH>::kBytes;
  float down = 0x1p-126f;
  __syncthreads();
  for (int b = eg; b * 32 < Ne; b += EG) {
    w.split(wave_max(top));
    const float down_b = uniform(w.down);
    wave_lds_order();  // the readers of the block before
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int s = 0; s < DH / 16; ++s)
        *reinterpret_cast<u32x4*>(ws + q * Tile<DH>::kBytes + (at.rows ^ (s * 32))) = w.w[q][s];
    wave_lds_order();
    const float m = score_scale(x.down, down_b);
    f32x16 z = score_tile<DH, F32>(w, x, 32 * b, Ne);
    if ((b + EG) * 32 < Ne) top = w.load(Wh, 32 * (b + EG) + (lane & 31), Ne, g);
    if (down_b > down) {
      const float k = down / down_b;
      down = down_b;
#pragma unroll
      for (int i = 0; i < DH / 32; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) dx[i][v] *= k;
    }
    const float ref = lse - (log2_of(down_b) - log2_of(down));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 f = *reinterpret_cast<const f32x4*>(&sm.fex[32 * b + 8 * q + 4 * g]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        z[4 * q + i] = __builtin_amdgcn_exp2f(fmaf(z[4 * q + i], m, -ref)) * (f[i] - st.y);
    }
    add_dx<DH>(z, ws, at, dx);
  }
  const float c = a.dloss[h] * a.stats[T * Nh + h].x * __builtin_amdgcn_ldexpf(down, -(int)F);
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) dx[i][v] *= c;
  if constexpr (EG > 1) {
    // the wavefronts that share tokens, in order
    f32x4* sums = reinterpret_cast<f32x4*>(sm.ws);
    auto place = [&](int e, int i) { return (((e - 1) * TG + tg) * (DH / 8) + i) * kWave + lane; };
    __syncthreads();
    if (eg > 0) {
#pragma unroll
      for (int i = 0; i < DH / 8; ++i)
        sums[place(eg, i)] = f32x4{dx[i / 4][4 * (i % 4)], dx[i / 4][4 * (i % 4) + 1],
                                   dx[i / 4][4 * (i % 4) + 2], dx[i / 4][4 * (i % 4) + 3]};
    }
    __syncthreads();
    if (eg > 0) return;
#pragma unroll
    for (int r = 1; r < EG; ++r)
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) {
        const f32x4 v = sums[place(r, i)];
#pragma unroll
        for (int j = 0; j < 4; ++j) dx[i / 4][4 * (i % 4) + j] += v[j];
      }
  }
  if (t < T) store_dx<DH, F32>(dx, ok ? 1.0f : 0.0f, t * Nh + h, dX_add, dX);
}

// EG: also the blocks of experts per workgroup of dW.
template <int DH, bool F32, int EG>
__global__ __launch_bounds__(kDwWaves* kWave) void balance_bwd_few_kernel(
    const DwArgs a, const void* dX_add, void* dX, unsigned dx_blocks) {
  __shared__ union Shared {
    DxFewShared<DH, EG> dx;
    DwShared<DH, F32, EG> dw;
    __device__ Shared() {}
  } sm;
  if (blockIdx.x < dx_blocks)
    balance_dx_few<DH, F32, EG>(a, dX_add, dX, blockIdx.x, sm.dx);
  else
    balance_dw<DH, F32, EG>(a, blockIdx.x - dx_blocks, sm.dw);
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
#pragma unroll 8
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
  if (T * k <= kCountAllSlots) {
    hipLaunchKernelGGL(expert_counts_all_kernel, dim3((unsigned)Nh), dim3(kCountAllThreads), 0, s,
                       idx, mask, T, Nh, Ne, k, div_magic(k), counts);
    return hipGetLastError();
  }
  const int n = Nh * Ne;
  hipLaunchKernelGGL(counts_zero_kernel, dim3((unsigned)ceil_div(n, kCountThreads)),
                     dim3(kCountThreads), 0, s, counts, n);
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

// A head's part of the workspace behind the operands.
static HeadInfo* head_info(const void* weights, int Nh, int dh, int Ne) {
  return reinterpret_cast<HeadInfo*>(
      const_cast<uint8_t*>(static_cast<const uint8_t*>(weights)) +
      balance_operand_bytes(Nh, dh, Ne));
}

hipError_t launch_balance_weights(const float* W, const int32_t* counts, int Nh, int dh, int Ne,
                                  void* out, hipStream_t s) {
  const dim3 grid((unsigned)balance_blocks(Ne), (unsigned)Nh);
#define MHL_WEIGHTS(DH)                                                                  \
  hipLaunchKernelGGL((balance_weights_kernel<DH>), grid, dim3(256), 0, s, W, counts, Ne, \
                     static_cast<uint8_t*>(out), head_info(out, Nh, dh, Ne))
  if (dh == 128)
    MHL_WEIGHTS(128);
  else
    MHL_WEIGHTS(64);
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

hipError_t launch_balance_loss(const void* X, const float* W, const void* weights,
                               const int32_t* counts, const uint8_t* mask, int64_t T, int Nh,
                               int dh, int Ne, bool f32, float* stats, double* part, float* loss,
                               hipStream_t s) {
  const dim3 grid((unsigned)(Nh * balance_token_blocks(T, Nh, Ne)));
  float2* st = reinterpret_cast<float2*>(stats);
  if (balance_few(T, Nh, Ne)) {
    const int eg = balance_few_groups(Ne, kBalanceFewWaves);
#define MHL_LOSS_EG(DH, F32, EG)                                                                 \
  hipLaunchKernelGGL((balance_loss_few_kernel<DH, F32, EG>), grid, dim3(kFewThreads), 0, s, X,   \
                     W, counts, mask, T, Nh, Ne, st, part, loss)
#define MHL_LOSS(DH, F32)          \
  do {                             \
    if (eg == 1)                   \
      MHL_LOSS_EG(DH, F32, 1);     \
    else if (eg == 2)              \
      MHL_LOSS_EG(DH, F32, 2);     \
    else if (eg == 4)              \
      MHL_LOSS_EG(DH, F32, 4);     \
    else                           \
      MHL_LOSS_EG(DH, F32, 8);     \
  } while (0)
    MHL_BALANCE_TYPES(MHL_LOSS)
#undef MHL_LOSS
#undef MHL_LOSS_EG
    return hipGetLastError();
  }
#define MHL_LOSS(DH, F32)                                                                      \
  hipLaunchKernelGGL((balance_loss_kernel<DH, F32>), grid, dim3(kTokenWaves* kWave), 0, s, X,  \
                     static_cast<const uint8_t*>(weights), head_info(weights, Nh, dh, Ne), mask, \
                     T, Nh, Ne, st, part)
  MHL_BALANCE_TYPES(MHL_LOSS)
#undef MHL_LOSS
  return hipGetLastError();
}

hipError_t launch_balance_loss_sum(const double* part, const int32_t* counts, const uint8_t* mask,
                                   int64_t T, int Nh, int Ne, float* loss, float* stats,
                                   hipStream_t s) {
  hipLaunchKernelGGL(balance_loss_sum_kernel, dim3((unsigned)Nh), dim3(256), 0, s, part,
                     balance_token_blocks(T, Nh, Ne), counts, mask, T, Nh, Ne, loss,
                     reinterpret_cast<float2*>(stats));
  return hipGetLastError();
}

static DwArgs dw_args(const void* X, const float* W, const int32_t* counts, const float* stats,
                      const float* dloss, const uint8_t* mask, const float* dW_add, int64_t T,
                      int Nh, int dh, int Ne, float* dW, float* part) {
  return DwArgs{X, W, counts, reinterpret_cast<const float2*>(stats), dloss, mask, dW_add, T, Nh,
                Ne, (int)ceil_div(balance_blocks(Ne), balance_dw_blocks(T, Nh, dh, Ne)),
                (int)balance_splits(T, Nh, dh, Ne), dW, part};
}
static unsigned dw_workgroups(const DwArgs& a) {
  return (unsigned)(ceil_div((int64_t)a.Nh * a.splits, kXcds) * kXcds * a.groups);
}

template <int V>
using Int = std::integral_constant<int, V>;

// call(d_h, X in fp32, blocks of experts per workgroup of dW) as compile-time constants.
template <class F>
static void for_dw(int dh, bool f32, int ew, F&& call) {
  auto blocks = [&](auto DH, auto F32) {
    if (ew == 1)
      call(DH, F32, Int<1>{});
    else if (ew == 2)
      call(DH, F32, Int<2>{});
    else if (ew == 4)
      call(DH, F32, Int<4>{});
    else if constexpr (decltype(DH)::value == 128)
      call(DH, F32, Int<8>{});
  };
  if (dh == 128 && f32)
    blocks(Int<128>{}, std::true_type{});
  else if (dh == 128)
    blocks(Int<128>{}, std::false_type{});
  else if (f32)
    blocks(Int<64>{}, std::true_type{});
  else
    blocks(Int<64>{}, std::false_type{});
}

hipError_t launch_balance_dx(const void* X, const void* weights, const float* stats,
                             const float* dloss, const uint8_t* mask, const void* dX_add, int64_t T,
                             int Nh, int dh, int Ne, bool f32, void* dX, hipStream_t s) {
  const DxArgs a{X, static_cast<const uint8_t*>(weights), head_info(weights, Nh, dh, Ne),
                 reinterpret_cast<const float2*>(stats), dloss, mask, dX_add, T, Nh, Ne, dX};
  const dim3 grid((unsigned)(Nh * ceil_div(T, kBalanceTokens)));
#define MHL_DX(DH, F32) \
  hipLaunchKernelGGL((balance_dx_kernel<DH, F32>), grid, dim3(kTokenWaves* kWave), 0, s, a)
  MHL_BALANCE_TYPES(MHL_DX)
#undef MHL_DX
  return hipGetLastError();
}

hipError_t launch_balance_dw(const void* X, const float* W, const int32_t* counts,
                             const float* stats, const float* dloss, const uint8_t* mask,
                             const float* dW_add, int64_t T, int Nh, int dh, int Ne, bool f32,
                             float* dW, float* part, hipStream_t s) {
  const DwArgs a = dw_args(X, W, counts, stats, dloss, mask, dW_add, T, Nh, dh, Ne, dW, part);
  for_dw(dh, f32, balance_dw_blocks(T, Nh, dh, Ne), [&](auto DH, auto F32, auto EW) {
    hipLaunchKernelGGL((balance_dw_kernel<decltype(DH)::value, decltype(F32)::value,
                                          decltype(EW)::value>),
                       dim3(dw_workgroups(a)), dim3(dw_waves(decltype(EW)::value) * kWave), 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_balance_dw_dx(const void* X, const float* W, const void* weights,
                                const int32_t* counts, const float* stats, const float* dloss,
                                const uint8_t* mask, const void* dX_add, const float* dW_add,
                                int64_t T, int Nh, int dh, int Ne, bool f32, void* dX, float* dW,
                                float* part, hipStream_t s) {
  const DwArgs dw = dw_args(X, W, counts, stats, dloss, mask, dW_add, T, Nh, dh, Ne, dW, part);
  const DxArgs dx{X, static_cast<const uint8_t*>(weights), head_info(weights, Nh, dh, Ne),
                  reinterpret_cast<const float2*>(stats), dloss, mask, dX_add, T, Nh, Ne, dX};
  const unsigned dw_blocks = dw_workgroups(dw);
  const dim3 grid(dw_blocks + (unsigned)(Nh * ceil_div(T, kBalanceTokens)));
  for_dw(dh, f32, balance_dw_blocks(T, Nh, dh, Ne), [&](auto DH, auto F32, auto EW) {
    if constexpr (decltype(EW)::value <= kDwWaves)
      hipLaunchKernelGGL((balance_dw_dx_kernel<decltype(DH)::value, decltype(F32)::value,
                                               decltype(EW)::value>),
                         grid, dim3(kDwWaves * kWave), 0, s, dw, dx, dw_blocks);
  });
  return hipGetLastError();
}

hipError_t launch_balance_bwd_few(const void* X, const float* W, const int32_t* counts,
                                  const float* stats, const float* dloss, const uint8_t* mask,
                                  const void* dX_add, const float* dW_add, int64_t T, int Nh,
                                  int dh, int Ne, bool f32, void* dX, float* dW, float* part,
                                  hipStream_t s) {
  const DwArgs a = dw_args(X, W, counts, stats, dloss, mask, dW_add, T, Nh, dh, Ne, dW, part);
  for_dw(dh, f32, balance_dw_blocks(T, Nh, dh, Ne), [&](auto DH, auto F32, auto EW) {
    constexpr int EG = decltype(EW)::value;
    if constexpr (EG <= kDwWaves) {
      const unsigned dx_blocks = (unsigned)(Nh * ceil_div(T, 32 * (kDwWaves / EG)));
      hipLaunchKernelGGL((balance_bwd_few_kernel<decltype(DH)::value, decltype(F32)::value, EG>),
                         dim3(dx_blocks + dw_workgroups(a)), dim3(kDwWaves * kWave), 0, s, a,
                         dX_add, dX, dx_blocks);
    }
  });
  return hipGetLastError();
}

hipError_t launch_balance_dw_sum(const float* part, const float* stats, const float* dloss,
                                 const float* dW_add, int64_t T, int Nh, int dh, int Ne, float* dW,
                                 hipStream_t s) {
  const int padded = 32 * balance_blocks(Ne), dh4 = dh / 4;
  const dim3 grid((unsigned)ceil_div(Ne * dh4, 256), (unsigned)Nh);
  hipLaunchKernelGGL(balance_dw_sum_kernel, grid, dim3(256), 0, s,
                     reinterpret_cast<const f32x4*>(part), balance_splits(T, Nh, dh, Ne),
                     (int64_t)Nh * padded * dh4, reinterpret_cast<const float2*>(stats) + T * Nh,
                     dloss, reinterpret_cast<const f32x4*>(dW_add), Ne, padded, dh4,
                     reinterpret_cast<f32x4*>(dW));
  return hipGetLastError();
}

}  // namespace mhl
