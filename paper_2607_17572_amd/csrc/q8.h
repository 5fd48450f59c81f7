// Device helpers of the 8-bit formats (OCP E4M3 and E5M2, E8M0 exponents).
#pragma once
#include "ops8.h"

namespace jg {

// 16 bytes at any alignment of the element (global accesses need none on gfx950)
typedef unsigned int u32x4a __attribute__((ext_vector_type(4), aligned(2)));

// eight consecutive elements as fp32
__device__ __forceinline__ void load8(const uint16_t* p, float* v) {
  const u32x4a u = *(const u32x4a*)p;
#pragma unroll
  for (int w = 0; w < 4; ++w) { v[2 * w] = bf2f(u[w] & 0xffffu); v[2 * w + 1] = bf2f(u[w] >> 16); }
}
__device__ __forceinline__ void load8(const float* p, float* v) {
  const u32x4a a = *(const u32x4a*)p, b = *(const u32x4a*)(p + 4);
#pragma unroll
  for (int w = 0; w < 4; ++w) { v[w] = __uint_as_float(a[w]); v[4 + w] = __uint_as_float(b[w]); }
}
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
  u32x4a u;
#pragma unroll
  for (int w = 0; w < 4; ++w) u[w] = (uint32_t)f2bf(v[2 * w]) | ((uint32_t)f2bf(v[2 * w + 1]) << 16);
  *(u32x4a*)p = u;
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  u32x4a a, b;
#pragma unroll
  for (int w = 0; w < 4; ++w) { a[w] = __float_as_uint(v[w]); b[w] = __float_as_uint(v[4 + w]); }
  *(u32x4a*)p = a;
  *(u32x4a*)(p + 4) = b;
}
// columns c .. c+7 of a row of `cols` elements; zeros past its end
template <typename T>
__device__ __forceinline__ void load8(const T* row, int c, int cols, float* v) {
  if (c + 8 <= cols) { load8(row + c, v); return; }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? ldf(row, c + e) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store8(T* row, int c, int cols, const float* v) {
  if (c + 8 <= cols) { store8(row + c, v); return; }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < cols) stf(row, c + e, v[e]);
}

// |v| as an ordered whole number: NaN above infinity above every finite value
__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Exponent byte of a block whose largest magnitude has the bits m: the least s with
// |largest| <= MAX 2^(s - 127), MAX = 1.75 2^8 (E4M3) or 1.75 2^15 (E5M2), at least 0;
// 255 (NaN) if the block holds an infinity or a NaN.
template <int F>
__device__ __forceinline__ uint32_t exp_byte(uint32_t m) {
  const int e = (int)(m >> 23);
  const int s = e - (F == E5M2 ? 15 : 8) + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e == 255 ? 255u : (uint32_t)(s > 0 ? s : 0);
}
// 2^(127 - s), exact; NaN for s = 255 (so that every value of the block becomes NaN)
__device__ __forceinline__ float inv_scale(uint32_t s) {
  return __uint_as_float(s == 255u ? 0x7fc00000u : (254u - s) << 23);
}
// four values as bytes, rounded to nearest even (none exceeds the format: inv_scale sees to it)
template <int F>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int r = 0;
  if (F == E5M2) {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  }
  return (uint32_t)r;
}

// the first n of eight bytes, zeros for the rest: padding is zero bytes, whatever the
// factors and the scale (0 times a negative factor is -0, 0 times NaN NaN)
__device__ __forceinline__ uint2 first_bytes(uint2 w, int n) {
  if (n >= 8) return w;
  const uint64_t m = n > 0 ? ~0ull >> (64 - 8 * n) : 0;
  return make_uint2(w.x & (uint32_t)m, w.y & (uint32_t)(m >> 32));
}

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
// largest over the 16 lanes of a row of 16
__device__ __forceinline__ uint32_t max16(uint32_t v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = umax(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

}  // namespace jg
