// Matrices in 8 bits with one power-of-two scale per block of 128.
//
// For a block with largest magnitude a: 2^e with the least e such that a <= MAX 2^e
// (MAX: 448 for E4M3, 57344 for E5M2), q = round(y 2^-e) to nearest even.  Powers of
// two cost no precision (both formats are floating point: only values 2^-15 (E4M3)
// below the block's largest lose bits), are exact to apply, and are what the
// matrix cores' scale operand takes.
//
// One workgroup per 128 x 128 tile: a thread holds 8 rows x 8 columns in registers, so
// the row blocks (16 lanes), the column blocks (16 thread rows) and the transposed
// bytes all come from one read of x.  The transposed bytes go through LDS so that
// every store is a whole 128-byte line.  Bound by memory: 2 or 4 bytes read and 1 or 2
// written per element.
#include "q8.h"

namespace jg {

template <typename T, int F, bool TILE>
__global__ __launch_bounds__(256) void quant8_k(Quant8Args a) {
  constexpr int TS = 144;  // bytes per transposed line in LDS
  __shared__ __attribute__((aligned(16))) uint8_t tr[128 * TS];
  __shared__ uint32_t cmax[4][128];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int cg = t & 15, rg = t >> 4;  // columns 8 cg .. +7, rows 8 rg .. +7 of the tile
  const int tiles_c = (a.cols + 127) / 128;
  const int tr_i = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  const int r0 = tr_i * 128 + rg * 8, c0 = tc * 128 + cg * 8;
  float v[8][8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    if (r0 + p < a.rows) load8((const T*)a.x + (size_t)(r0 + p) * a.ldx, c0, a.cols, v[p]);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) v[p][e] = 0.f;
  }
  if (a.row_mul) {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const float m = r0 + p < a.rows ? a.row_mul[r0 + p] : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[p][e] *= m;
    }
  }
  if (a.col_mul) {
    float m[8];
    load8((const T*)a.col_mul, c0, a.cols, m);
#pragma unroll
    for (int p = 0; p < 8; ++p)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[p][e] *= m[e];
  }

  const int blocks_r = (a.rows + 127) / 128;
  uint32_t tile_s = 0;
  if (TILE) {
    uint32_t m = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = umax(m, mag(v[p][e]));
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = umax(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if (lane == 0) cmax[wave][0] = m;
    __syncthreads();
    m = umax(umax(cmax[0][0], cmax[1][0]), umax(cmax[2][0], cmax[3][0]));
    tile_s = exp_byte<F>(m);
  }

  if (a.out.q) {
    uint8_t* sc = (uint8_t*)a.out.sc;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      uint32_t s = tile_s;
      if (!TILE) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = umax(m, mag(v[p][e]));
        s = exp_byte<F>(max16(m));
      }
      const float k = inv_scale(s);
      const uint2 w = make_uint2(pack4<F>(v[p][0] * k, v[p][1] * k, v[p][2] * k, v[p][3] * k),
                                 pack4<F>(v[p][4] * k, v[p][5] * k, v[p][6] * k, v[p][7] * k));
      if (r0 + p < a.rows) {
        *(uint2*)(a.out.q + (size_t)(r0 + p) * a.out.ld + c0) = first_bytes(w, a.cols - c0);
        if (cg == 0) {
          uint8_t* b = sc + ((size_t)(tc >> 2) * a.rows + r0 + p) * 4 + (tc & 3);
          *b = (uint8_t)s;
          if (tc == tiles_c - 1)  // blocks past the last one
            for (int j = (tc & 3) + 1; j < 4; ++j) *++b = 0;
        }
      }
    }
  }

  if (a.out_t.q) {
    uint32_t s[8];
    if (TILE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = tile_s;
    } else {
      // column c0 + e: over this thread's rows, the wave's four thread rows, the four waves
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t m = 0;
#pragma unroll
        for (int p = 0; p < 8; ++p) m = umax(m, mag(v[p][e]));
        m = umax(m, (uint32_t)__shfl_xor((int)m, 16, 64));
        m = umax(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        if (lane < 16) cmax[wave][cg * 8 + e] = m;
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = cg * 8 + e;
        s[e] = exp_byte<F>(umax(umax(cmax[0][c], cmax[1][c]), umax(cmax[2][c], cmax[3][c])));
      }
    }
    uint8_t* sc = (uint8_t*)a.out_t.sc;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float k = inv_scale(s[e]);
      const uint2 w = make_uint2(pack4<F>(v[0][e] * k, v[1][e] * k, v[2][e] * k, v[3][e] * k),
                                 pack4<F>(v[4][e] * k, v[5][e] * k, v[6][e] * k, v[7][e] * k));
      *(uint2*)(tr + (cg * 8 + e) * TS + rg * 8) = first_bytes(w, a.rows - r0);
      if (rg == 0 && c0 + e < a.cols) {
        uint8_t* b = sc + ((size_t)(tr_i >> 2) * a.cols + c0 + e) * 4 + (tr_i & 3);
        *b = (uint8_t)s[e];
        if (tr_i == blocks_r - 1)
          for (int j = (tr_i & 3) + 1; j < 4; ++j) *++b = 0;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // 8 lanes per line of 128 bytes
      const int c = i * 32 + (t >> 3), g = tc * 128 + c;
      if (g < a.cols)
        *(uint4*)(a.out_t.q + (size_t)g * a.out_t.ld + (size_t)tr_i * 128 + (t & 7) * 16) =
            *(const uint4*)(tr + c * TS + (t & 7) * 16);
    }
  }
}

template <typename T, int F>
static void launch_quant8(const Quant8Args& a, hipStream_t s) {
  const unsigned grid = (unsigned)((a.rows + 127) / 128) * (unsigned)((a.cols + 127) / 128);
  if (a.tile) hipLaunchKernelGGL((quant8_k<T, F, true>), dim3(grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((quant8_k<T, F, false>), dim3(grid), dim3(256), 0, s, a);
}

int quant8(const Quant8Args& a, hipStream_t s) {
  const size_t tiles = (((size_t)a.rows + 127) / 128) * (((size_t)a.cols + 127) / 128);
  if (int rc = too_many(tiles, 256, "quantize8: too many 128 x 128 tiles")) return rc;
  if (a.dt == BF16) {
    if (a.fmt == E5M2) launch_quant8<uint16_t, E5M2>(a, s);
    else launch_quant8<uint16_t, E4M3>(a, s);
  } else {
    if (a.fmt == E5M2) launch_quant8<float, E5M2>(a, s);
    else launch_quant8<float, E4M3>(a, s);
  }
  JG_CHECK_LAUNCH("quant8");
  return 0;
}

}  // namespace jg
