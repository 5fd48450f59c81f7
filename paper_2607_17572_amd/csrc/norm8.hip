// Residual addition + RMS norm with the normalised rows in 8 bits, and its backward.
//
//   h = round(x + r),  rstd = 1 / sqrt(mean(h^2) + eps),  y = (h rstd) gain -> 8 bits
//   dx = dh + rstd (a - h rstd^2 mean(a h)),  a = dy gain      (dx: gradient of x and of r)
//   dgain = beta dgain + sum over rows of dy h rstd
// The 8-bit rounding is passed straight through.  Sums are fp64 forward, fp32 backward.
//
// A row stays in registers between its two uses: NT threads (a wave, 256 or 1024 threads)
// hold NV vectors of 8 columns each, vector i of thread t at column 8 (i NT + t); 16
// neighbouring lanes then hold one block of 128 columns and a wave one exponent
// word.  Both are bound by memory: every tensor is read or written once (9216 x 4096 in
// bf16 with the residual: 51 us, 5.2 TB/s).
#include <algorithm>

#include "q8.h"
#include "tile.h"

namespace jg {

// Sum over the NT threads of a row (in every thread); `sh`: 16 floats per row.
template <int NT>
__device__ __forceinline__ float row_sum(float v, float* sh) {
  if constexpr (NT == 64) return wave_sum(v);
  else return block_sum(v, sh);
}

// The same in fp64.
template <int NT>
__device__ __forceinline__ double row_sum64(double v, double* sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) v += sh[i];
  }
  return v;
}

// The sum of squares is fp64 (the kernel waits for memory all the same), so that rstd is
// off by its own rounding alone: an 8-bit value next to a border of its rounding then
// falls to the exact side wherever fp32 factors can tell; and squares do not overflow.
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void rmsnorm8_k(Norm8Args a) {
  constexpr int RPB = NT < 256 ? 256 / NT : 1;  // rows per workgroup
  __shared__ double sh[16];
  const int t = threadIdx.x % NT, row = blockIdx.x * RPB + threadIdx.x / NT;
  if (row >= a.rows) return;  // whole waves: RPB > 1 only with NT = 64, which has no barrier
  const T* x = (const T*)a.x + (size_t)row * a.ldx;
  float v[NV][8];
  double ss = 0.0;
#pragma unroll
  for (int i = 0; i < NV; ++i) load8(x, 8 * (i * NT + t), a.cols, v[i]);
  if (a.r) {
    const T* r = (const T*)a.r + (size_t)row * a.ldr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float w[8];
      load8(r, 8 * (i * NT + t), a.cols, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[i][e] += w[e];
        // h as it is stored: the backward reads it
        if constexpr (sizeof(T) == 2) v[i][e] = bf2f(f2bf(v[i][e]));
      }
    }
  }
  if (a.h) {
    T* h = (T*)a.h + (size_t)row * a.ldh;
#pragma unroll
    for (int i = 0; i < NV; ++i) store8(h, 8 * (i * NT + t), a.cols, v[i]);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma((double)v[i][e], (double)v[i][e], ss);
  ss = row_sum64<NT>(ss, sh);
  const float rstd = (float)(1.0 / sqrt(ss / a.cols + a.eps));
  if (a.rstd && t == 0) a.rstd[row] = rstd;
  uint8_t* q = a.y.q + (size_t)row * a.y.ld;
  const int kp = (a.cols + 127) / 128 * 128;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = 8 * (i * NT + t);
    float g[8];
    load8((const T*)a.gain, c, a.cols, g);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      g[e] *= v[i][e] * rstd;
      // columns past the end hold zeros, but zero times an infinite rstd is NaN
      if (c + 8 > a.cols && c + e >= a.cols) g[e] = 0.f;
      m = umax(m, mag(g[e]));
    }
    const uint32_t s = exp_byte<E4M3>(max16(m));
    const float k = inv_scale(s);
    if (c < kp) {
      *(uint2*)(q + c) = first_bytes(make_uint2(pack4<E4M3>(g[0] * k, g[1] * k, g[2] * k, g[3] * k),
                                                pack4<E4M3>(g[4] * k, g[5] * k, g[6] * k, g[7] * k)),
                                     a.cols - c);
    }
    // the wave's four blocks, one word (blocks past the end hold zeros: byte 0)
    const uint32_t w = (uint32_t)__shfl((int)s, 0, 64) | (uint32_t)__shfl((int)s, 16, 64) << 8 |
                       (uint32_t)__shfl((int)s, 32, 64) << 16 | (uint32_t)__shfl((int)s, 48, 64) << 24;
    if ((t & 63) == 0 && c < a.cols) a.y.sc[(size_t)(c / 512) * a.rows + row] = w;
  }
}

template <typename T, int NT, int NV>
static void launch_norm8(const Norm8Args& a, hipStream_t s) {
  constexpr int RPB = NT < 256 ? 256 / NT : 1;
  hipLaunchKernelGGL((rmsnorm8_k<T, NT, NV>), dim3((a.rows + RPB - 1) / RPB), dim3(NT < 256 ? 256 : NT), 0, s, a);
}

// The threads of a row: enough that each holds at most 4 vectors.
template <template <typename, int, int> class L, typename T, typename A>
static void by_width(const A& a, hipStream_t s) {
  const int c = a.cols;
  if (c <= 512) L<T, 64, 1>::go(a, s);
  else if (c <= 1024) L<T, 64, 2>::go(a, s);
  else if (c <= 2048) L<T, 64, 4>::go(a, s);
  else if (c <= 4096) L<T, 256, 2>::go(a, s);
  else if (c <= 8192) L<T, 256, 4>::go(a, s);
  else if (c <= 16384) L<T, 1024, 2>::go(a, s);
  else L<T, 1024, 4>::go(a, s);
}
template <typename T, int NT, int NV>
struct Norm8 {
  static void go(const Norm8Args& a, hipStream_t s) { launch_norm8<T, NT, NV>(a, s); }
};

int rmsnorm8(const Norm8Args& a, hipStream_t s) {
  const unsigned nt = a.cols <= 2048 ? 64 : a.cols <= 8192 ? 256 : 1024;  // a row's threads (by_width)
  if (int rc = too_many((size_t)a.rows + 3, nt, "rmsnorm8: too many rows")) return rc;
  if (a.dt == BF16) by_width<Norm8, uint16_t>(a, s);
  else by_width<Norm8, float>(a, s);
  JG_CHECK_LAUNCH("rmsnorm8");
  return 0;
}

// ------------------------------------------------------------------ backward
// A workgroup takes rows w, w + workgroups, ... (with NT = 64 each of its four waves does) and
// keeps its sums of dgain in registers; they go to part[workgroup][cols] and are
// added in that order.  A row's loads are issued together and stay in their storage type
// until they are used.  9216 x 4096 in bf16: 61 us, 4.9 TB/s (the copy of a large buffer: 5.2)
// with 512 workgroups; 73 with 256, 65 with 768, and 75 with a wave per row there.
static int norm8_workgroups(int rows, int cols) {
  const int per = cols <= 2048 ? 4 : 1;  // rows at a time (by_width)
  return (int)std::min(((long)rows + per - 1) / per, 512l);
}
size_t rmsnorm8_grad_bytes(int rows, int cols) {
  return (size_t)norm8_workgroups(rows, cols) * cols * sizeof(float);
}

// 16 bytes of a buffer; none (zeros) past its end
__device__ __forceinline__ u32x4a buf_load16(__amdgpu_buffer_rsrc_t r, int off) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}
__device__ __forceinline__ void buf_store16(u32x4a v, __amdgpu_buffer_rsrc_t r, int off) {
  __builtin_amdgcn_raw_buffer_store_b128(v, r, off, 0, 0);
}

// A row of a matrix (p == nullptr: zeros).  V8: its elements are a multiple of eight at a
// multiple of 16 bytes; vectors then are whole or past the end, where a buffer's
// range check gives zeros and stores nothing, without a branch.
template <typename T, bool V8>
struct Row8 {
  T* p;
  int cols;
  __device__ __forceinline__ Row8(const void* m, size_t ld, unsigned row, int n) {
    p = m ? (T*)m + row * ld : nullptr;
    cols = m ? n : 0;
  }
};

// eight elements of a row as stored
template <typename T, bool V8>
struct Raw8 {
  u32x4a r[sizeof(T) / 2];
  __device__ __forceinline__ void load(const Row8<T, V8>& row, int c) {
    if constexpr (V8) {
      const __amdgpu_buffer_rsrc_t b = make_rsrc(row.p, (long)row.cols * sizeof(T));
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = buf_load16(b, c * (int)sizeof(T) + 16 * i);
    } else {
      float v[8];
      load8(row.p, c, row.cols, v);
      set(v);
    }
  }
  __device__ __forceinline__ void store(const Row8<T, V8>& row, int c) const {
    if constexpr (V8) {
      const __amdgpu_buffer_rsrc_t b = make_rsrc(row.p, (long)row.cols * sizeof(T));
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) buf_store16(r[i], b, c * (int)sizeof(T) + 16 * i);
    } else {
      float v[8];
      get(v);
      store8(row.p, c, row.cols, v);
    }
  }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (sizeof(T) == 2) {
        r[0][w] = (uint32_t)f2bf(v[2 * w]) | (uint32_t)f2bf(v[2 * w + 1]) << 16;
      } else {
        r[0][w] = __float_as_uint(v[w]);
        r[1][w] = __float_as_uint(v[4 + w]);
      }
    }
  }
  // forgets what is known of the values: a later get() unpacks again, and the fp32
  // values need not be kept
  __device__ __forceinline__ void renew() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) asm("" : "+v"(r[i]));
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (sizeof(T) == 2) {
        v[2 * w] = bf2f(r[0][w] & 0xffffu);
        v[2 * w + 1] = bf2f(r[0][w] >> 16);
      } else {
        v[w] = __uint_as_float(r[0][w]);
        v[4 + w] = __uint_as_float(r[1][w]);
      }
    }
  }
};

template <typename T, int NT, int NV, bool V8>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void rmsnorm8_grad_k(Norm8Grad a) {
  constexpr int RPB = NT < 256 ? 256 / NT : 1;
  constexpr bool WAVE = NT == 64;
  __shared__ float sh[16];
  __shared__ __attribute__((aligned(16))) float sum[WAVE ? 512 * NV : 1];
  __shared__ __attribute__((aligned(16))) T gain[WAVE ? 512 * NV : 1];  // as the lanes hold it
  const int t = threadIdx.x % NT, sub = WAVE ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
  const unsigned workers = gridDim.x * RPB;
  Raw8<T, V8> g[WAVE ? 1 : NV];
  float dg[NV][8];
  if constexpr (WAVE) {
    for (int i = threadIdx.x; i < 512 * NV; i += 256) gain[i] = i < a.cols ? ((const T*)a.gain)[i] : (T)0;
    __syncthreads();
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) g[i].load(Row8<T, V8>(a.gain, 0, 0, a.cols), 8 * (i * NT + t));
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[i][e] = 0.f;
  const float inv_c = 1.f / (float)a.cols;
  for (unsigned row = blockIdx.x * RPB + sub; row < (unsigned)a.rows; row += workers) {
    Raw8<T, V8> dy[NV], h[NV], dh[NV];
    const Row8<T, V8> rdy(a.dy, a.lddy, row, a.cols), rh(a.h, a.ldh, row, a.cols), rdh(a.dh, a.lddh, row, a.cols),
        rdx(a.dx, a.lddx, row, a.cols);
#pragma unroll
    for (int i = 0; i < NV; ++i) dy[i].load(rdy, 8 * (i * NT + t));
#pragma unroll
    for (int i = 0; i < NV; ++i) h[i].load(rh, 8 * (i * NT + t));
#pragma unroll
    for (int i = 0; i < NV; ++i) dh[i].load(rdh, 8 * (i * NT + t));
    const float rs = a.rstd[row];
    auto up_of = [&](int i, float* up, float* n, float* d) {  // a = dy gain, n = h rstd, dy
      float gv[8];
      if constexpr (WAVE) load8(gain + 8 * (i * 64 + t), gv);
      else g[i].get(gv);
      dy[i].get(d);
      h[i].get(n);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[e] *= rs;
        up[e] = d[e] * gv[e];
      }
    };
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float up[8], n[8], d[8];
      up_of(i, up, n, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dg[i][e] = fmaf(d[e], n[e], dg[i][e]);
        dot = fmaf(up[e], n[e], dot);
      }
    }
    dot = row_sum<NT>(dot, sh) * inv_c;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      dy[i].renew();
      h[i].renew();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float up[8], n[8], d[8], o[8];
      up_of(i, up, n, d);
      dh[i].get(o);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += rs * (up[e] - n[e] * dot);
      dh[i].set(o);
      dh[i].store(rdx, 8 * (i * NT + t));
    }
  }
  float* p = a.part + (size_t)blockIdx.x * a.cols;
  if constexpr (WAVE) {  // the waves' sums, in wave order
    for (int w = 0; w < RPB; ++w) {
      __syncthreads();
      if (sub != w) continue;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float* const q = sum + 8 * (i * 64 + t);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = w ? q[e] + dg[i][e] : dg[i][e];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.cols; i += 256) p[i] = sum[i];
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) store8(p, 8 * (i * NT + t), a.cols, dg[i]);
  }
}

// dgain = beta dgain + sum of part over the workgroups: 64 columns per workgroup, its 16
// waves take every 16th row of part.
template <typename T>
__global__ __launch_bounds__(1024) void norm8_dgain_k(const float* part, int workers, int cols, T* dgain, float beta) {
  __shared__ float sh[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < cols)
#pragma unroll 8
    for (int w = wave; w < workers; w += 16) s += part[(size_t)w * cols + c];
  sh[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) {
    for (int i = 1; i < 16; ++i) s += sh[i][lane];
    if (beta != 0.f) s += ldf(dgain, c);
    stf(dgain, c, s);
  }
}

template <typename T, int NT, int NV>
struct Norm8G {
  static void go(const Norm8Grad& a, hipStream_t s) {
    const dim3 grid(norm8_workgroups(a.rows, a.cols)), block(NT < 256 ? 256 : NT);
    const size_t es = dsize(a.dt);
    const bool v8 = a.cols % 8 == 0 && (a.lddy * es | a.ldh * es | a.lddh * es | a.lddx * es) % 16 == 0 &&
                    ((uintptr_t)a.dy | (uintptr_t)a.h | (uintptr_t)a.dh | (uintptr_t)a.dx | (uintptr_t)a.gain) % 16 == 0;
    if (v8) hipLaunchKernelGGL((rmsnorm8_grad_k<T, NT, NV, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rmsnorm8_grad_k<T, NT, NV, false>), grid, block, 0, s, a);
  }
};

int rmsnorm8_grad(const Norm8Grad& a, hipStream_t s) {
  if (a.dt == BF16) by_width<Norm8G, uint16_t>(a, s);
  else by_width<Norm8G, float>(a, s);
  JG_CHECK_LAUNCH("rmsnorm8_grad");
  const int workers = norm8_workgroups(a.rows, a.cols);
  const dim3 grid((a.cols + 63) / 64);
  if (a.dgain_dt == BF16)
    hipLaunchKernelGGL(norm8_dgain_k<uint16_t>, grid, dim3(1024), 0, s, a.part, workers, a.cols, (uint16_t*)a.dgain, a.beta);
  else
    hipLaunchKernelGGL(norm8_dgain_k<float>, grid, dim3(1024), 0, s, a.part, workers, a.cols, (float*)a.dgain, a.beta);
  JG_CHECK_LAUNCH("rmsnorm8_grad dgain");
  return 0;
}

}  // namespace jg
