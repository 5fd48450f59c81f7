// Operators of an 8-bit linear layer and the clip of the gradient behind it:
// quantiser, residual + RMS norm with 8-bit rows and its backward, the 8-bit
// product, the global gradient norm.
#pragma once
#include "common.h"

namespace jg {

// A launch has fewer than 2^32 threads along x.  Returns 4 (unsupported) for more.
inline int too_many(size_t workgroups, unsigned threads, const char* what) {
  if (workgroups * threads < (1ull << 32)) return 0;
  set_error(std::string(what) + " for one launch (2^32 threads)");
  return 4;
}

enum Fmt8 { E4M3 = 0, E5M2 = 1 };

// 8-bit matrix of `rows` rows and k columns: bytes q[row * ld + col], zero from k to the
// next multiple of 128, and the exponents of its 128-column blocks, packed four
// to a word: byte j of sc[w * rows + row] belongs to columns 128 (4w + j) .. + 127
// and stands for 2^(byte - 127) (255: NaN; blocks past k: 0).  The packing lets 32
// lanes fetch the exponents of 32 rows and 512 columns as one 128-byte line.
struct Mat8 {
  uint8_t* q = nullptr;
  uint32_t* sc = nullptr;
  size_t ld = 0;
  int rows = 0, k = 0, fmt = E4M3;
};

struct Quant8Args {
  const void* x;
  size_t ldx;
  int rows, cols, dt;
  const float* row_mul;  // or nullptr
  const void* col_mul;   // or nullptr; dt
  int tile;              // one exponent per 128 x 128 instead of per 128 elements of a line
  Mat8 out, out_t;       // q == nullptr: not wanted
  int fmt;
};
int quant8(const Quant8Args& a, hipStream_t s);

constexpr int NORM8_MAX_COLS = 32768;

struct Norm8Args {
  const void* x; size_t ldx;
  const void* r; size_t ldr;  // residual or nullptr
  const void* gain;
  int rows, cols, dt;
  float eps;
  void* h; size_t ldh;        // or nullptr
  Mat8 y;
  float* rstd;                // or nullptr
};
int rmsnorm8(const Norm8Args& a, hipStream_t s);

struct Norm8Grad {
  const void* dy; size_t lddy;
  const void* h; size_t ldh;
  const float* rstd;
  const void* gain;
  const void* dh; size_t lddh;  // or nullptr
  int rows, cols, dt;
  void* dx; size_t lddx;
  void* dgain; int dgain_dt;
  float beta;
  float* part;                  // rmsnorm8_grad_bytes(rows, cols)
};
size_t rmsnorm8_grad_bytes(int rows, int cols);
int rmsnorm8_grad(const Norm8Grad& a, hipStream_t s);

struct Matmul8Args {
  Mat8 a, b;
  const void* bias;  // out_dt, or nullptr
  void* out; size_t ldo; int out_dt;
  float beta;        // 0 or 1
  // a long k over few tiles is split: sums of each split, added by a second launch
  float* part;
  int kind, splits, per_split;  // set by matmul8_plan
};
// Chooses the tiles and splits (from the sizes and out_dt); returns the bytes of `part`.
size_t matmul8_plan(Matmul8Args& a);
int matmul8(const Matmul8Args& a, hipStream_t s);

struct GradSeg {
  const void* src;
  void* dst;
  size_t n;
  int src_dt, dst_dt;
};
// Yields the i-th of `count` tensors of a list.
typedef GradSeg (*GradAt)(const void* list, int i);
// part: GRAD_PART doubles of workspace.  out[0] = norm; with dst also out[1] = the factor.
constexpr int GRAD_PART = 2048;
int grad_norm(GradAt at, const void* list, int count, bool largest, double* part, double* out, hipStream_t s);
int grad_clip(GradAt at, const void* list, int count, bool largest, double max_norm, double* part, double* out,
              hipStream_t s);

}  // namespace jg
