// Residual addition + RMS norm with the normalised rows in 8 bits, and its backward.
//
//   h = round(x + r),  rstd = 1 / sqrt(mean(h^2) + eps),  y = (h rstd) gain -> 8 bits
//   dx = dh + rstd (a - h rstd^2 mean(a h)),  a = dy gain      (dx: gradient of x and of r)
//   dgain = beta dgain + sum over rows of dy h rstd
// The 8-bit rounding is passed straight through.  Sums are fp32.
//
// A row stays in registers between its two uses: NT threads (a wave, 256 or 1024 threads)
// hold NV vectors of 8 columns each, vector i of thread t at column 8 (i NT + t); 16
// neighbouring lanes then hold one block of 128 columns and a wave one exponent
// word.  Both are bound by memory: every tensor is read or written once.
#include "q8.h"

namespace jg {

// Sum over the NT threads of a row (in every thread); `sh`: 16 floats per row.
template <int NT>
__device__ __forceinline__ float row_sum(float v, float* sh) {
  if constexpr (NT == 64) return wave_sum(v);
  else return block_sum(v, sh);
}

template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void rmsnorm8_k(Norm8Args a) {
  constexpr int RPB = NT < 256 ? 256 / NT : 1;  // rows per workgroup
  __shared__ float sh[16];
  const int t = threadIdx.x % NT, row = blockIdx.x * RPB + threadIdx.x / NT;
  if (row >= a.rows) return;  // whole waves: RPB > 1 only with NT = 64, which has no barrier
  const T* x = (const T*)a.x + (size_t)row * a.ldx;
  float v[NV][8], ss = 0.f;
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
    for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss);
  ss = row_sum<NT>(ss, sh);
  const float rstd = 1.f / sqrtf(ss / (float)a.cols + a.eps);
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
      *(uint2*)(q + c) = make_uint2(pack4<E4M3>(g[0] * k, g[1] * k, g[2] * k, g[3] * k),
                                    pack4<E4M3>(g[4] * k, g[5] * k, g[6] * k, g[7] * k));
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
  if (a.dt == BF16) by_width<Norm8, uint16_t>(a, s);
  else by_width<Norm8, float>(a, s);
  JG_CHECK_LAUNCH("rmsnorm8");
  return 0;
}

// ------------------------------------------------------------------ backward
// Each of `workers` thread rows takes rows w, w + workers, ... and keeps its sums of
// dgain in registers; they go to part[worker][cols] and are added in that order.
static int norm8_threads(int cols) { return cols <= 2048 ? 64 : cols <= 8192 ? 256 : 1024; }
static int norm8_workers(int rows, int cols) {
  const int per = norm8_threads(cols) == 64 ? 4 : 1;
  const int blocks = 512, want = (rows + per - 1) / per;
  return (want < blocks ? want : blocks) * per;
}
size_t rmsnorm8_grad_bytes(int rows, int cols) { return (size_t)norm8_workers(rows, cols) * cols * sizeof(float); }

template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void rmsnorm8_grad_k(Norm8Grad a) {
  constexpr int RPB = NT < 256 ? 256 / NT : 1;
  __shared__ float sh[16];
  const int t = threadIdx.x % NT, worker = blockIdx.x * RPB + threadIdx.x / NT, workers = gridDim.x * RPB;
  float g[NV][8], dg[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    load8((const T*)a.gain, 8 * (i * NT + t), a.cols, g[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[i][e] = 0.f;
  }
  const float inv_c = 1.f / (float)a.cols;
  for (int row = worker; row < a.rows; row += workers) {
    const T* dyp = (const T*)a.dy + (size_t)row * a.lddy;
    const T* hp = (const T*)a.h + (size_t)row * a.ldh;
    const float rs = a.rstd[row];
    float dy[NV][8], h[NV][8], dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      load8(dyp, 8 * (i * NT + t), a.cols, dy[i]);
      load8(hp, 8 * (i * NT + t), a.cols, h[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n = h[i][e] * rs, up = dy[i][e] * g[i][e];
        dg[i][e] = fmaf(dy[i][e], n, dg[i][e]);
        h[i][e] = n;
        dy[i][e] = up;
        dot = fmaf(up, n, dot);
      }
    dot = row_sum<NT>(dot, sh) * inv_c;
    T* dxp = (T*)a.dx + (size_t)row * a.lddx;
    const T* dhp = (const T*)a.dh + (size_t)row * a.lddh;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float o[8];
      if (a.dh) load8(dhp, 8 * (i * NT + t), a.cols, o);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = rs * (dy[i][e] - h[i][e] * dot);
        o[e] = a.dh ? o[e] + d : d;
      }
      store8(dxp, 8 * (i * NT + t), a.cols, o);
    }
  }
  float* p = a.part + (size_t)worker * a.cols;
#pragma unroll
  for (int i = 0; i < NV; ++i) store8(p, 8 * (i * NT + t), a.cols, dg[i]);
}

// dgain = beta dgain + sum of part over the workers: 64 columns per workgroup, its 16
// waves take every 16th worker.
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
    constexpr int RPB = NT < 256 ? 256 / NT : 1;
    const int workers = norm8_workers(a.rows, a.cols);
    hipLaunchKernelGGL((rmsnorm8_grad_k<T, NT, NV>), dim3(workers / RPB), dim3(NT < 256 ? 256 : NT), 0, s, a);
  }
};

int rmsnorm8_grad(const Norm8Grad& a, hipStream_t s) {
  if (a.dt == BF16) by_width<Norm8G, uint16_t>(a, s);
  else by_width<Norm8G, float>(a, s);
  JG_CHECK_LAUNCH("rmsnorm8_grad");
  const int workers = norm8_workers(a.rows, a.cols);
  const dim3 grid((a.cols + 63) / 64);
  if (a.dgain_dt == BF16)
    hipLaunchKernelGGL(norm8_dgain_k<uint16_t>, grid, dim3(1024), 0, s, a.part, workers, a.cols, (uint16_t*)a.dgain, a.beta);
  else
    hipLaunchKernelGGL(norm8_dgain_k<float>, grid, dim3(1024), 0, s, a.part, workers, a.cols, (float*)a.dgain, a.beta);
  JG_CHECK_LAUNCH("rmsnorm8_grad dgain");
  return 0;
}

}  // namespace jg
