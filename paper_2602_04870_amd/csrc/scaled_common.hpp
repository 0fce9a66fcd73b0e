// Rows of bf16 or fp32 in and out of registers, and blocks of 128 values held
// in 8 bits (e4m3: largest value 448) with one fp32 scale.  Shared by the norm
// and quantisation kernels.
#pragma once

#include "device_common.hpp"

namespace mhl {

constexpr int kScaleBlock = 128;       // values along the contraction per scale
constexpr float kE4m3Max = 448.0f;
constexpr float kScaleMin = 0x1p-126f;  // keeps 1 / scale finite: a block below 448 * 2^-126 loses its last bits

// Eight consecutive elements as they lie in memory.
template <bool F32>
struct Raw8 {
  u32x4 v[F32 ? 2 : 1];
};

// Element at of p.
template <bool F32>
__device__ __forceinline__ const void* from(const void* p, int64_t at) {
  return static_cast<const uint8_t*>(p) + at * (F32 ? 4 : 2);
}
template <bool F32>
__device__ __forceinline__ void* from(void* p, int64_t at) {
  return static_cast<uint8_t*>(p) + at * (F32 ? 4 : 2);
}

template <bool F32>
__device__ __forceinline__ const u32x4* row_ptr(const void* p, int64_t at) {
  return reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(p) + at * (F32 ? 4 : 2));
}
template <bool F32>
__device__ __forceinline__ u32x4* row_ptr(void* p, int64_t at) {
  return reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(p) + at * (F32 ? 4 : 2));
}

// Elements at .. at + 7 (16-byte aligned), zeros unless ok.
template <bool F32>
__device__ __forceinline__ Raw8<F32> load8(const void* p, int64_t at, bool ok) {
  Raw8<F32> r;
  const u32x4* s = row_ptr<F32>(p, at);
#pragma unroll
  for (int i = 0; i < (F32 ? 2 : 1); ++i) r.v[i] = ok ? s[i] : u32x4{0u, 0u, 0u, 0u};
  return r;
}

template <bool F32>
__device__ __forceinline__ void unpack8(const Raw8<F32>& r, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (F32)
      f[i] = __uint_as_float(r.v[i >> 2][i & 3]);
    else
      f[i] = (i & 1) ? __uint_as_float(r.v[0][i >> 1] & 0xFFFF0000u) : bf16_bits_to_f32(r.v[0][i >> 1]);
  }
}

// Rounded to the type (bf16: nearest even).
template <bool F32>
__device__ __forceinline__ Raw8<F32> pack8(const float (&f)[8]) {
  Raw8<F32> r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F32) {
      r.v[0][i] = __float_as_uint(f[i]);
      r.v[F32 ? 1 : 0][i] = __float_as_uint(f[4 + i]);
    } else {
      r.v[0][i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    }
  }
  return r;
}

template <bool F32>
__device__ __forceinline__ void store8(void* p, int64_t at, const Raw8<F32>& r) {
  u32x4* d = row_ptr<F32>(p, at);
#pragma unroll
  for (int i = 0; i < (F32 ? 2 : 1); ++i) d[i] = r.v[i];
}

// One element (rows whose width is no multiple of 8).
template <bool F32>
__device__ __forceinline__ float load1(const void* p, int64_t at) {
  if (F32) return reinterpret_cast<const float*>(p)[at];
  return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[at]);
}
template <bool F32>
__device__ __forceinline__ float round1(float v) {
  return F32 ? v : bf16_bits_to_f32(pack_bf16x2(v, v) & 0xFFFFu);
}
template <bool F32>
__device__ __forceinline__ void store1(void* p, int64_t at, float v) {
  if (F32)
    reinterpret_cast<float*>(p)[at] = v;
  else
    reinterpret_cast<uint16_t*>(p)[at] = (uint16_t)pack_bf16x2(v, v);
}

// VEC (8 or 1) consecutive elements.
template <bool F32, int VEC>
struct Piece {
  Raw8<F32> r;
  __device__ __forceinline__ void load(const void* p, int64_t at, bool ok) { r = load8<F32>(p, at, ok); }
  __device__ __forceinline__ void get(float (&f)[8]) const { unpack8<F32>(r, f); }
  __device__ __forceinline__ void set(const float (&f)[8]) { r = pack8<F32>(f); }  // rounds
  __device__ __forceinline__ void store(void* p, int64_t at) const { store8<F32>(p, at, r); }
};
template <bool F32>
struct Piece<F32, 1> {
  float v;
  __device__ __forceinline__ void load(const void* p, int64_t at, bool ok) {
    v = 0.0f;
    if (ok) v = load1<F32>(p, at);
  }
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = v; }
  __device__ __forceinline__ void set(const float (&f)[1]) { v = round1<F32>(f[0]); }
  __device__ __forceinline__ void store(void* p, int64_t at) const { store1<F32>(p, at, v); }
};

// The bits of |v|: ordered as integers they order magnitudes, with infinity
// above every finite value and NaN above infinity, so one integer maximum
// finds a block's largest magnitude and lets no NaN pass unseen.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
  return v > o ? v : o;
}
// Maximum over aligned groups of 16 lanes, in every lane of the group (all 64
// lanes active): pairs, quads, halves of 8, the two halves.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = dpp_max<0xB1>(v);   // quad_perm [1, 0, 3, 2]
  v = dpp_max<0x4E>(v);   // quad_perm [2, 3, 0, 1]
  v = dpp_max<0x141>(v);  // row_half_mirror
  return dpp_max<0x140>(v);  // row_mirror
}

// Sum over aligned groups of LANES lanes, the same in each of them (each step
// adds a pair's two values, whose sum does not depend on their order).
template <int LANES>
__device__ __forceinline__ float lane_sum(float v) {
#pragma unroll
  for (int d = 1; d < LANES; d <<= 1) v += __shfl_xor(v, d, kWave);
  return v;
}

// a / b by one multiply with (about) 1 / b and a correction: r + (a - r b) / b.
__device__ __forceinline__ float quotient(float a, float b, float inv) {
  const float r = a * inv;
  return fmaf(fmaf(-r, b, a), inv, r);
}

// A block's scale from its largest magnitude (NaN from an infinity or a NaN),
// and the scale's reciprocal to an ulp.
__device__ __forceinline__ float block_scale(uint32_t amax, float& inv) {
  const float q = quotient(__uint_as_float(amax), kE4m3Max, 1.0f / kE4m3Max);
  const float s = q < kScaleMin ? kScaleMin : q;
  inv = __builtin_amdgcn_rcpf(s);
  return s;
}

// v over its block's scale s, less than 2^-44 of itself off before its rounding to
// fp32 (an ulp for v below 2^-106, whose remainder is a denormal number; the bare
// multiply, 2^-22 off, moved values that lie on a border between two of e4m3's, as
// bf16 inputs often do).  At most 448 (1 + 2^-22), which e4m3 rounds to
// 448, so nothing has to be clamped.  A block whose scale is not finite becomes NaN
// as a whole.
__device__ __forceinline__ float over_scale(float v, float s, float inv) {
  return quotient(v, s, inv);
}

// Four values to e4m3 (nearest even), in one word.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

}  // namespace mhl
