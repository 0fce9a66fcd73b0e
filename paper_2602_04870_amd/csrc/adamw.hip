// AdamW over many tensors at once.  Per element, with g = grad_scale * grad,
//
//   m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps) - lr wd p
//
// in fp32.  HBM bounds it (6.3 GB of bf16 weights, fp32 masters, gradients and states: 1139
// us, 5.5 TB/s; 0.95 GB with 8-bit states 197 us, 4.8 TB/s): every tensor's elements are
// read once and written once by the workgroup that has them, the tensors' addresses being
// kernel arguments (one launch for kAdamTensors tensors, nothing to upload).
//
// States in 8 bits are m and sqrt(v), e4m3 with a scale per 128 elements (16 lanes
// of 8 elements).  m changes by (1 - b1) (g - m), v by (1 - b2) (g^2 - v): where the betas
// are near 1, or g near m, often less than half a step of e4m3 (2^-4), and rounding to
// the nearest would leave the state where it is.  Each is rounded up with the probability
// of the part below the step instead, so that it moves by the update on average.  The
// random numbers are a hash of the key and the element's place, nothing is kept.  sqrt(v)
// is held rather than v: it has half the exponents, and what is not zero is not rounded
// to zero, which would make a step as large as m / eps.
//
// The states' arithmetic is one rounding per operation, with no fused multiply-add:
// an 8-bit value that falls on the other side of its random border is a whole step
// off, so states of 8 bits are the same wherever the same operations are made.

#include "scaled_common.hpp"
#include "training_launch.hpp"

namespace mhl {
namespace {

constexpr int kAdamThreads = 256;
static_assert(kAdamThreads * 8 == kAdamChunk, "8 elements per thread");

__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}
// 32 random bits of element i.
__device__ __forceinline__ uint32_t random_bits(uint32_t key, int64_t i) {
  return mix((uint32_t)i * 0x9E3779B9u + (uint32_t)(i >> 32) * 0x3C6EF373u + key);
}

// Eight elements of a float or bf16 tensor (uniform kind), n <= 8 of them there.
__device__ __forceinline__ void load_any(const void* p, bool bf16, int64_t at, int n,
                                         float (&f)[8]) {
  if (n == 8) {
    if (bf16)
      unpack8<false>(load8<false>(p, at, true), f);
    else
      unpack8<true>(load8<true>(p, at, true), f);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    f[i] = i < n ? (bf16 ? load1<false>(p, at + i) : load1<true>(p, at + i)) : 0.0f;
}
__device__ __forceinline__ void store_any(void* p, bool bf16, int64_t at, int n,
                                          const float (&f)[8]) {
  if (n == 8) {
    if (bf16)
      store8<false>(p, at, pack8<false>(f));
    else
      store8<true>(p, at, pack8<true>(f));
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) {
      if (bf16)
        store1<false>(p, at + i, f[i]);
      else
        store1<true>(p, at + i, f[i]);
    }
}

// Eight e4m3 values times their block's scale.
__device__ __forceinline__ void load_q8(const void* p, const float* scales, int64_t at, int n,
                                        float (&f)[8]) {
  const uint8_t* s = static_cast<const uint8_t*>(p) + at;
  u32x2 w{0u, 0u};
  if (n == 8) {
    w = *reinterpret_cast<const u32x2*>(s);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) w[i >> 2] |= (uint32_t)s[i] << (8 * (i & 3));
  }
  const float scale = n > 0 ? scales[at / kScaleBlock] : 0.0f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
    f[4 * j] = lo[0] * scale;
    f[4 * j + 1] = lo[1] * scale;
    f[4 * j + 2] = hi[0] * scale;
    f[4 * j + 3] = hi[1] * scale;
  }
}

// |y| (at most 448 (1 + 2^-22), or NaN) to e4m3, up where the part below a step
// is over 1 - u / 2^16.  Above 2^-6 a step is 2^20 in fp32's bits, so u is added
// there and the bits below cut off; under it the values are whole numbers of 2^-9.
__device__ __forceinline__ uint32_t e4m3_random(float y, uint32_t u, bool keep) {
  const uint32_t a = magnitude(y);
  uint32_t q;
  if (a >= 0x3C800000u)
    q = ((a + (u << 4)) >> 20) - (120u << 3);
  else
    q = (uint32_t)fmaf(__uint_as_float(a), 512.0f, (float)u * 0x1p-16f);
  if (keep && a != 0u && q == 0u) q = 1u;
  q = a > 0x7F800000u ? 0x7Fu : q;
  return q | ((__float_as_uint(y) >> 24) & 0x80u);
}

// b1 m + (1 - b1) g, each operation rounded.
__device__ __forceinline__ float blend(float state, float beta, float g, float rest) {
#pragma clang fp contract(off)
  const float a = state * beta, b = g * rest;
  return a + b;
}

// The block's scale (largest magnitude times 1 / 448, so at most an ulp from the
// quotient) and its values in 8 bits (16 lanes, all of a wavefront active).  SHIFT: the
// random numbers' half of u.
template <int SHIFT, bool KEEP>
__device__ __forceinline__ void store_q8(void* p, float* scales, int64_t at, int n,
                                         const float (&f)[8], const uint32_t (&u)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = i < n ? magnitude(f[i]) : 0u;
    top = b > top ? b : top;
  }
  const float most = __uint_as_float(max16(top)) * (1.0f / kE4m3Max);
  const float s = most < kScaleMin ? kScaleMin : most;
  const float inv = __builtin_amdgcn_rcpf(s);
  u32x2 w{0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    w[i >> 2] |= e4m3_random(over_scale(f[i], s, inv), (u[i] >> SHIFT) & 0xFFFFu, KEEP)
                 << (8 * (i & 3));
  uint8_t* d = static_cast<uint8_t*>(p) + at;
  if (n == 8) {
    *reinterpret_cast<u32x2*>(d) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) d[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
  if (n > 0 && (threadIdx.x & 15) == 0) scales[at / kScaleBlock] = s;
}

__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamLaunch a) {
  int i = 0;  // the last tensor that begins at or before this workgroup
#pragma unroll
  for (int j = 1; j < kAdamTensors; ++j) i += blockIdx.x >= a.first[j] ? 1 : 0;
  const AdamTensor& t = a.t[i];
  const AdamStep& c = a.step;
  const float scale = c.grad_scale ? *c.grad_scale : 1.0f;
  const int64_t begin = (int64_t)(blockIdx.x - a.first[i]) * a.chunk;
  for (int64_t at0 = begin; at0 < begin + a.chunk && at0 < t.n; at0 += kAdamChunk) {
    const int64_t at = at0 + threadIdx.x * 8;
    const int64_t left = t.n - at;
    const int n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
    float g[8], p[8], m[8], v[8], root[8];
    load_any(t.grad, t.grad_bf16, at, n, g);
    if (t.master)
      load_any(t.master, false, at, n, p);
    else
      load_any(t.param, t.param_bf16, at, n, p);
    if (t.m_scale) {
      load_q8(t.m, t.m_scale, at, n, m);
      load_q8(t.v, t.v_scale, at, n, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = v[k] * v[k];
    } else {
      load_any(t.m, false, at, n, m);
      load_any(t.v, false, at, n, v);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float s = g[k] * scale;
      m[k] = blend(m[k], c.beta1, s, c.rest1);
      v[k] = blend(v[k], c.beta2, s * s, c.rest2);
      root[k] = sqrtf(v[k]);
      p[k] = p[k] - fmaf(c.rate, m[k] / fmaf(root[k], c.root, c.eps), t.decay * p[k]);
    }
    store_any(t.param, t.param_bf16, at, n, p);
    if (t.master) store_any(t.master, false, at, n, p);
    if (t.m_scale) {
      uint32_t u[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] = random_bits(t.key, at + k);
      store_q8<0, false>(t.m, t.m_scale, at, n, m, u);
      store_q8<16, true>(t.v, t.v_scale, at, n, root, u);
    } else {
      store_any(t.m, false, at, n, m);
      store_any(t.v, false, at, n, v);
    }
  }
}

}  // namespace

hipError_t launch_adamw(const AdamLaunch& a, unsigned workgroups, hipStream_t s) {
  hipLaunchKernelGGL(adamw_kernel, dim3(workgroups), dim3(kAdamThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace mhl
