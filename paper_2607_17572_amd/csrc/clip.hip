// Global norm of a list of gradient tensors, and the scaled copy that respects it.
//
//   norm = sqrt(sum of g^2) or max |g| over all elements of all tensors (fp64),
//   c = max_norm / norm if max_norm < norm < infinity, else 1;  dst = src c.
//
// Tensors travel as kernel arguments, up to GS a launch (neighbours in memory are one
// piece: the tensors of a flat gradient without padding between them need one launch
// however many they are).  Pieces are cut into chunks of CH elements, dealt to the
// workgroups in turn.  Each workgroup keeps one partial result, carried over the
// launches of a long list; the scaling pass adds the partials itself (2048 of them at
// most, in one order in every workgroup) instead of waiting for a launch that does.
// Bound by memory: every element is read twice and written once.
#include <algorithm>
#include <cmath>

#include "q8.h"

namespace jg {

// Elements of a chunk: 64 a thread, or 8 where the list then still has no more chunks
// than the card's CUs take at once (a small gradient: 0.3 million elements, 48 tensors).
constexpr int GS = 112, CH = 16384, CH_SMALL = 2048;
constexpr size_t SMALL = 1u << 21;

struct GradSegs {
  const void* src[GS];
  void* dst[GS];
  size_t n[GS];
  unsigned first[GS];  // chunk at which a piece begins
  unsigned char dt[GS];  // src type | dst type << 1
  int count;
  unsigned chunks, ch;
};
static_assert(sizeof(GradSegs) <= 3400, "kernel arguments");

// The piece of a chunk: the pieces' first chunks lie in the lanes, two each, so that
// finding one reads no memory.
static_assert(GS <= 128, "two pieces per lane");
struct Pieces {
  unsigned f0, f1;
  __device__ __forceinline__ explicit Pieces(const GradSegs& g) {
    const int lane = threadIdx.x & 63;
    f0 = lane < g.count ? g.first[lane] : ~0u;
    f1 = lane + 64 < g.count ? g.first[lane + 64] : ~0u;
  }
  __device__ __forceinline__ int of(unsigned c) const {
    return __popcll(__ballot(f0 <= c)) + __popcll(__ballot(f1 <= c)) - 1;
  }
};

template <bool MAX>
__device__ __forceinline__ void take(double& acc, uint32_t& top, const float* v) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (MAX) top = umax(top, mag(v[e]));
    else acc = fma((double)v[e], (double)v[e], acc);
  }
}
// The largest magnitude's bits as the value they stand for, exactly, so that partials
// of either kind are doubles.
__device__ __forceinline__ double merge(bool max, double a, double b) {
  if (!max) return a + b;
  return a != a || b != b ? a + b : a > b ? a : b;
}

template <typename T, bool MAX>
__device__ __forceinline__ void norm_chunk(const T* p, unsigned n, double& acc, uint32_t& top) {
  unsigned i = threadIdx.x * 8;
  if (n == CH) {  // eight vectors in flight
    float v[8][8];
#pragma unroll
    for (int u = 0; u < 8; ++u) load8(p + i + u * 2048, v[u]);
#pragma unroll
    for (int u = 0; u < 8; ++u) take<MAX>(acc, top, v[u]);
    return;
  }
  for (; i < n; i += 2048) {
    float v[8];
    load8(p, (int)i, (int)n, v);
    take<MAX>(acc, top, v);
  }
}

template <bool MAX>
__global__ __launch_bounds__(256) void grad_norm_k(GradSegs g, double* part, int carry) {
  __shared__ double sh[4];
  double acc = 0.0;
  uint32_t top = 0;
  const Pieces pieces(g);
  for (unsigned c = blockIdx.x; c < g.chunks; c += gridDim.x) {
    const int s = pieces.of(c);
    const size_t at = (size_t)(c - g.first[s]) * g.ch, left = g.n[s] - at;
    const unsigned n = left < g.ch ? (unsigned)left : g.ch;
    if (g.dt[s] & 1) norm_chunk<uint16_t, MAX>((const uint16_t*)g.src[s] + at, n, acc, top);
    else norm_chunk<float, MAX>((const float*)g.src[s] + at, n, acc, top);
  }
  if (MAX) acc = (double)__uint_as_float(top);
  for (int o = 32; o > 0; o >>= 1) acc = merge(MAX, acc, __shfl_xor(acc, o, 64));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    acc = merge(MAX, merge(MAX, sh[0], sh[1]), merge(MAX, sh[2], sh[3]));
    part[blockIdx.x] = carry ? merge(MAX, part[blockIdx.x], acc) : acc;
  }
}

// The norm from the partials, in every thread of the workgroup.
template <bool MAX>
__device__ __forceinline__ double whole_norm(const double* part, int nparts, double* sh) {
  double a = 0.0;
  for (int i = threadIdx.x; i < nparts; i += 256) a = merge(MAX, a, part[i]);
  for (int o = 32; o > 0; o >>= 1) a = merge(MAX, a, __shfl_xor(a, o, 64));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = a;
  __syncthreads();
  a = merge(MAX, merge(MAX, sh[0], sh[1]), merge(MAX, sh[2], sh[3]));
  return MAX ? a : sqrt(a);
}

template <bool MAX>
__global__ __launch_bounds__(256) void grad_norm_out_k(const double* part, int nparts, double* out) {
  __shared__ double sh[4];
  const double norm = whole_norm<MAX>(part, nparts, sh);
  if (threadIdx.x == 0) out[0] = norm;
}

template <typename T, typename D>
__device__ __forceinline__ void scale_chunk(const T* p, D* d, unsigned n, float c) {
  unsigned i = threadIdx.x * 8;
  if (n == CH) {
    float v[8][8];
#pragma unroll
    for (int u = 0; u < 8; ++u) load8(p + i + u * 2048, v[u]);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] *= c;
      store8(d + i + u * 2048, v[u]);
    }
    return;
  }
  for (; i < n; i += 2048) {
    float v[8];
    load8(p, (int)i, (int)n, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= c;
    store8(d, (int)i, (int)n, v);
  }
}

// a value that all lanes share, in scalar registers
__device__ __forceinline__ double scalar(double v) {
  return __hiloint2double(__builtin_amdgcn_readfirstlane(__double2hiint(v)), __builtin_amdgcn_readfirstlane(__double2loint(v)));
}

// With a factor below fp32's normal range, where fp32 would lose its digits or make it 0.
__device__ __noinline__ void scale_in_fp64(const void* src, void* dst, size_t at, unsigned n, int t, double c) {
  for (size_t i = at + threadIdx.x; i < at + n; i += 256) {
    const float v = (float)((double)(t & 1 ? ldf((const uint16_t*)src, i) : ldf((const float*)src, i)) * c);
    if (t & 2) stf((uint16_t*)dst, i, v);
    else stf((float*)dst, i, v);
  }
}

template <bool MAX>
__global__ __launch_bounds__(256) void grad_scale_k(GradSegs g, const double* part, int nparts, double max_norm,
                                                    double* out) {
  __shared__ double sh[4];
  const double norm = whole_norm<MAX>(part, nparts, sh);
  // false for NaN; an infinite norm keeps the gradients too
  const bool clip = norm > max_norm && norm <= 1.7976931348623157e308;
  const double c = scalar(clip ? max_norm / norm : 1.0);
  if (out && blockIdx.x == 0 && threadIdx.x == 0) { out[0] = norm; out[1] = c; }
  const float cf = (float)c;
  const Pieces pieces(g);
  for (unsigned k = blockIdx.x; k < g.chunks; k += gridDim.x) {
    const int s = pieces.of(k);
    if (!clip && g.src[s] == g.dst[s]) continue;
    const size_t at = (size_t)(k - g.first[s]) * g.ch, left = g.n[s] - at;
    const unsigned n = left < g.ch ? (unsigned)left : g.ch;
    const int t = g.dt[s];
    if (c < 0x1p-126) scale_in_fp64(g.src[s], g.dst[s], at, n, t, c);
    else if (t == 3) scale_chunk((const uint16_t*)g.src[s] + at, (uint16_t*)g.dst[s] + at, n, cf);
    else if (t == 1) scale_chunk((const uint16_t*)g.src[s] + at, (float*)g.dst[s] + at, n, cf);
    else if (t == 2) scale_chunk((const float*)g.src[s] + at, (uint16_t*)g.dst[s] + at, n, cf);
    else scale_chunk((const float*)g.src[s] + at, (float*)g.dst[s] + at, n, cf);
  }
}

// Calls f(pieces) for each launch's worth of the list, empty tensors left out.
template <class F>
static int for_pieces(GradAt at, const void* list, int count, int ch, F f) {
  GradSegs g;
  g.ch = ch;
  g.count = 0;
  g.chunks = 0;
  GradSeg cur{};
  bool have = false;
  auto flush = [&]() -> int {
    const int rc = g.count ? f(g) : 0;
    g.count = 0;
    g.chunks = 0;
    return rc;
  };
  auto put = [&](const GradSeg& s) -> int {
    // a launch's chunk numbers fit 31 bits: a longer piece is cut
    const size_t most = (size_t)ch << 28;
    for (size_t done = 0; done < s.n;) {
      const size_t n = std::min(s.n - done, most);
      const unsigned chunks = (unsigned)((n + ch - 1) / ch);
      if (g.count == GS || g.chunks > (1u << 28))
        if (int rc = flush()) return rc;
      const int i = g.count++;
      g.src[i] = (const char*)s.src + done * dsize(s.src_dt);
      g.dst[i] = s.dst ? (char*)s.dst + done * dsize(s.dst_dt) : nullptr;
      g.n[i] = n;
      g.first[i] = g.chunks;
      g.dt[i] = (unsigned char)(s.src_dt | s.dst_dt << 1);
      g.chunks += chunks;
      done += n;
    }
    return 0;
  };
  for (int i = 0; i < count; ++i) {
    const GradSeg s = at(list, i);
    if (s.n == 0) continue;
    if (have && s.src_dt == cur.src_dt && s.dst_dt == cur.dst_dt &&
        (const char*)cur.src + cur.n * dsize(cur.src_dt) == (const char*)s.src &&
        (cur.dst ? (char*)cur.dst + cur.n * dsize(cur.dst_dt) == (char*)s.dst : !s.dst)) {
      cur.n += s.n;
      continue;
    }
    if (have)
      if (int rc = put(cur)) return rc;
    cur = s;
    have = true;
  }
  if (have)
    if (int rc = put(cur)) return rc;
  return flush();
}

static int chunk_of(GradAt at, const void* list, int count) {
  size_t n = 0;
  for (int i = 0; i < count; ++i) n += at(list, i).n;
  return n <= SMALL ? CH_SMALL : CH;
}

// Partials of the norm of the whole list; returns their number (0: no elements), -1 on an error.
static int norm_pass(GradAt at, const void* list, int count, int ch, bool largest, double* part, hipStream_t s) {
  size_t chunks = 0;  // of the whole list: every launch has workgroups for the longest
  for (int i = 0; i < count; ++i) chunks += (at(list, i).n + ch - 1) / ch;
  const int nparts = (int)std::min<size_t>(chunks, GRAD_PART);
  bool carry = false;
  const int rc = for_pieces(at, list, count, ch, [&](const GradSegs& g) -> int {
    if (largest) hipLaunchKernelGGL(grad_norm_k<true>, dim3(nparts), dim3(256), 0, s, g, part, carry ? 1 : 0);
    else hipLaunchKernelGGL(grad_norm_k<false>, dim3(nparts), dim3(256), 0, s, g, part, carry ? 1 : 0);
    JG_CHECK_LAUNCH("grad_norm");
    carry = true;
    return 0;
  });
  return rc ? -1 : nparts;
}

int grad_norm(GradAt at, const void* list, int count, bool largest, double* part, double* out, hipStream_t s) {
  const int ch = chunk_of(at, list, count), nparts = norm_pass(at, list, count, ch, largest, part, s);
  if (nparts < 0) return 3;
  if (largest) hipLaunchKernelGGL(grad_norm_out_k<true>, dim3(1), dim3(256), 0, s, part, nparts, out);
  else hipLaunchKernelGGL(grad_norm_out_k<false>, dim3(1), dim3(256), 0, s, part, nparts, out);
  JG_CHECK_LAUNCH("grad_norm_out");
  return 0;
}

int grad_clip(GradAt at, const void* list, int count, bool largest, double max_norm, double* part, double* out,
              hipStream_t s) {
  const int ch = chunk_of(at, list, count), nparts = norm_pass(at, list, count, ch, largest, part, s);
  if (nparts < 0) return 3;
  auto scale = [&](const GradSegs& g) -> int {
    const unsigned grid = std::max(1u, std::min<unsigned>(g.chunks, 2048));
    if (largest) hipLaunchKernelGGL(grad_scale_k<true>, dim3(grid), dim3(256), 0, s, g, part, nparts, max_norm, out);
    else hipLaunchKernelGGL(grad_scale_k<false>, dim3(grid), dim3(256), 0, s, g, part, nparts, max_norm, out);
    JG_CHECK_LAUNCH("grad_scale");
    return 0;
  };
  if (nparts == 0) {  // no elements: norm 0, factor 1
    GradSegs none;
    none.count = 0;
    none.chunks = 0;
    none.ch = ch;
    return scale(none);
  }
  return for_pieces(at, list, count, ch, scale);
}

}  // namespace jg
