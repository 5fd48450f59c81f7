// Product of two 8-bit matrices with a power-of-two scale per block of 128.
//
//   C[m][n] = beta C + sum_k A(m, k) B(n, k) + bias[n]
//
// Two ways through the matrix cores:
//
// bf16 results: v_mfma_scale_f32_32x32x64_f8f6f4, 64 of k an instruction; its scale
// operands take the block exponents as they are stored, so the product needs no
// arithmetic beside the matrix instructions.  The instruction adds its products in
// groups of 8 neighbours of k, aligned to the largest of the group: a product loses
// what lies 13 bits below that one; between the groups the sums are fp32 (found with
// operands of one large and one small product).  On normally distributed data with
// spread scales the sums are 1e-5 to 3e-5 off (relative, 2-norm, whatever k is), a
// fiftieth of the rounding to bf16 that follows.
//
// fp32 results: the values as bf16 (every 8-bit value with its scale is one:
// v_cvt_scalef32_pk_bf16_fp8) through v_mfma_f32_32x32x16_bf16, whose sums are fp32,
// at half the rate.
#include "q8.h"

namespace jg {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// scale byte as the factor it stands for (as the conversion takes it)
__device__ __forceinline__ float scale_of(int s) { return __uint_as_float(s == 255 ? 0x7fc00000u : (uint32_t)s << 23); }

// eight 8-bit values (two words) times a scale, as bf16
template <int F>
__device__ __forceinline__ bf16x8 widen8(int w0, int w1, float s) {
  bf16x2 a, b, c, d;
  if constexpr (F == E5M2) {
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w0, s, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w0, s, true);
    c = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w1, s, false);
    d = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w1, s, true);
  } else {
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, true);
    c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, false);
    d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, true);
  }
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One wave per 32 x 32 tile of C, operands straight from memory.
template <int FA, typename T>
__global__ __launch_bounds__(256) void matmul8_k(Matmul8Args g) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tiles_n = (g.b.rows + 63) / 64;
  const int m0 = (int)(blockIdx.x / tiles_n) * 64 + (wave >> 1) * 32, n0 = (int)(blockIdx.x % tiles_n) * 64 + (wave & 1) * 32;
  const int l = lane & 31, h = lane >> 5;
  const int ra = min(m0 + l, g.a.rows - 1), rb = min(n0 + l, g.b.rows - 1);
  const uint8_t* pa = g.a.q + (size_t)ra * g.a.ld + 32 * h;
  const uint8_t* pb = g.b.q + (size_t)rb * g.b.ld + 32 * h;
  f32x16 acc;
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  const int nk = (g.a.k + 127) / 128;
  for (int b = 0; b < nk; ++b) {
    const int sa = (int)((g.a.sc[(size_t)(b >> 2) * g.a.rows + ra] >> (8 * (b & 3))) & 255u);
    const int sb = (int)((g.b.sc[(size_t)(b >> 2) * g.b.rows + rb] >> (8 * (b & 3))) & 255u);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const i32x4 a0 = *(const i32x4*)(pa + b * 128 + t * 64), a1 = *(const i32x4*)(pa + b * 128 + t * 64 + 16);
      const i32x4 b0 = *(const i32x4*)(pb + b * 128 + t * 64), b1 = *(const i32x4*)(pb + b * 128 + t * 64 + 16);
      const i32x8 va = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
      const i32x8 vb = __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7);
      if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, acc, FA, 0, 0, sa, 0, sb);
      } else {
        // k in any order, the same on both sides
#pragma unroll
        for (int w = 0; w < 8; w += 2)
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FA>(va[w], va[w + 1], scale_of(sa)),
                                                        widen8<E4M3>(vb[w], vb[w + 1], scale_of(sb)), acc, 0, 0, 0);
      }
    }
  }
  const int n = n0 + l;
  if (n >= g.b.rows) return;
  const float bias = g.bias ? ldf((const T*)g.bias, n) : 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int m = m0 + 8 * (e / 4) + 4 * h + e % 4;
    if (m >= g.a.rows) continue;
    float v = acc[e] + bias;
    T* c = (T*)g.out + (size_t)m * g.ldo;
    if (g.beta != 0.f) v += ldf(c, n);
    stf(c, n, v);
  }
}

template <int FA>
static void launch_matmul8(const Matmul8Args& g, hipStream_t s) {
  const dim3 grid((unsigned)((g.a.rows + 63) / 64) * (unsigned)((g.b.rows + 63) / 64));
  if (g.out_dt == BF16) hipLaunchKernelGGL((matmul8_k<FA, uint16_t>), grid, dim3(256), 0, s, g);
  else hipLaunchKernelGGL((matmul8_k<FA, float>), grid, dim3(256), 0, s, g);
}

int matmul8(const Matmul8Args& g, hipStream_t s) {
  if (g.a.fmt == E5M2) launch_matmul8<1>(g, s);
  else launch_matmul8<0>(g, s);
  JG_CHECK_LAUNCH("matmul8");
  return 0;
}

}  // namespace jg
