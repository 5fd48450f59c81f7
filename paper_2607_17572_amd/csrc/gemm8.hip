// Product of two 8-bit matrices with a power-of-two scale per block of 128.
//
//   C[m][n] = beta C + sum_k A(m, k) B(n, k) + bias[n]
//
// Two ways through the matrix cores:
//
// bf16 results of 128 x 128 and 256 x 256 tiles: v_mfma_scale_f32_32x32x64_f8f6f4, 64 of k
// an instruction; its scale operands take the block exponents as they are stored, so
// the product needs no arithmetic beside the matrix instructions.  The instruction adds
// its products in groups of 8 neighbours of k, aligned to the largest exponent of the
// group: a product loses what lies 13 bits below that one; between the groups the sums
// are fp32 (found with operands of one large and one small product).  So a sum is off by
// less than 2^-10 (7 2^-13) of the largest |product| of each group, added over the groups.
// On normally distributed data with spread scales that is 1e-5 to 3e-5 (relative, 2-norm,
// whatever k is), a fiftieth of the rounding to bf16 that follows; the fp32 sums below
// would take twice the time there (9216 x 16384, k 4096: 465 us).
//
// Everything else: the values as bf16 (v_cvt_scalef32_pk_bf16_fp8) through
// v_mfma_f32_32x32x16_bf16, whose sums are fp32, at half the rate.  With up to 16 rows and
// on 64 x 32 and 64 x 64 tiles the matrix instructions take a small part of the time, so
// bf16 results have these sums as well (us, against the 8-bit instruction's: one row,
// 16384 x 4096 14.9, 14.5; 37 x 4096, k 12288 20.3, 19.8; 33 x 1024, k 4096 8.9, 8.3; 512 x 1024,
// k 1024 6.3, 5.7; 1024 x 1024, k 8192 23.8, 20.8).  bf16 holds every value
// of a block whose scale is below 2^113 (E4M3: 2^120), down to multiples of 2^-133.  A
// wave that met a scale of 2^17 or more drops its sums and starts again with the 8-bit
// instruction, whose scales have no such limit, eight times for each 64 of k and each time
// with one of the 8 neighbours only (large_scales, one_of_8): fp32 sums again, and what
// bf16 rounds off of values below 2^-126 has met no factor of 2^32 or more.  4096 x 4096,
// k 9216 with large scales everywhere: 976 us instead of 223, of which looking for them
// takes 2.
#include <type_traits>

#include "q8.h"
#include "tile.h"

namespace jg {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// scale byte as the factor it stands for (as the conversion takes it)
__device__ __forceinline__ float scale_of(int s) { return __uint_as_float(s == 255 ? 0x7fc00000u : (uint32_t)s << 23); }

// Nonzero if one of a word's exponent bytes is 144 .. 254 (a scale of 2^17 or more).
__device__ __forceinline__ uint32_t large_scales(uint32_t w) {
  return ((w & 0x70707070u) + 0x70707070u) & ~((w & 0x7f7f7f7fu) + 0x01010101u) & w & 0x80808080u;
}
// The p-th of every eight bytes (two words), zeros for the rest.
__device__ __forceinline__ i32x8 one_of_8(i32x8 v, int p) {
  const int even = p < 4 ? (int)(0xffu << (8 * p)) : 0, odd = p < 4 ? 0 : (int)(0xffu << (8 * (p - 4)));
#pragma unroll
  for (int w = 0; w < 8; ++w) v[w] &= w & 1 ? odd : even;
  return v;
}

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

// --------------------------------------------------------------- tiled kernel
// BM x BN tiles, KG groups of WM x WN waves that split the k tiles and add their sums
// through LDS.  k tiles of 64 bytes pass through four LDS stages, loaded three ahead
// straight from memory (the layout, swizzle and barriers of the bf16 direct-to-LDS
// kernel: 64 bytes are 32 of its k and 64 here, so that loads and LDS reads have twice
// its matrix instructions to hide behind).  A fragment is 32 rows x 64 bytes: a lane takes chunks
// h and h + 2 of its row (h = lane / 32), the same on both sides, so the order of k
// inside the instruction differs from memory's and the sum does not.
//
// The instruction's left operand is B, so that a lane holds neighbouring columns of
// one row of C.  A's fragments are read half a tile ahead: step 0 multiplies the
// first half of A's fragments while the second half is read, step 1 the second half
// while the next tile's B and first half are read.
template <int ROWS, int NW, int WR>
struct Op8 {
  static constexpr int NL = ROWS / 16 / NW;  // direct loads of 1 KB per wave and k tile
  static_assert(NL * 16 * NW == ROWS, "every wave loads the same");
  int voff[NL];
  int fo;  // chunk h of this lane's row of fragment 0; chunk h + 2 lies at fo ^ 32
  __device__ inline void init(int ld, int wrow0) {
    const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % NW;
#pragma unroll
    for (int t = 0; t < NL; ++t) {
      const int row = 16 * (wave * NL + t) + lane / 4;
      voff[t] = row * ld + 16 * ((lane % 4) ^ swz_n(row));
    }
    const int r = lane & 31;
    fo = (wrow0 + r) * 64 + ((lane >> 5) ^ swz_n(r)) * 16;
  }
  __device__ inline void load(__amdgpu_buffer_rsrc_t R, char* S, int k0) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % NW;
#pragma unroll
    for (int t = 0; t < NL; ++t)
      load_lds16(R, S + (wave * NL + t) * 1024, voff[t] + k0);
  }
  __device__ inline i32x8 frag(const char* S, int i) const {
    const i32x4 a = *(const i32x4*)(S + fo + i * 2048), b = *(const i32x4*)(S + (fo ^ 32) + i * 2048);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// The part of k that this workgroup multiplies: split blockIdx.y of g.splits.
__device__ __forceinline__ void take_split(Matmul8Args& g) {
  if (g.splits == 1) return;
  const int b0 = (int)blockIdx.y * g.per_split;  // blocks of 128, whole exponent words
  g.a.q += (size_t)b0 * 128;
  g.b.q += (size_t)b0 * 128;
  g.a.sc += (size_t)(b0 / 4) * g.a.rows;
  g.b.sc += (size_t)(b0 / 4) * g.b.rows;
  g.a.k = min(g.a.k - b0 * 128, g.per_split * 128);
  g.part += (size_t)blockIdx.y * g.a.rows * g.b.rows;
}

// bias, old C and the store of eight (bf16) or four (fp32) columns of a row; a split
// stores its sums
template <typename T, int NC>
__device__ __forceinline__ void store_c(const Matmul8Args& g, int row, int col, float* v) {
  if (g.splits > 1) {
    float* p = g.part + (size_t)row * g.b.rows;
#pragma unroll
    for (int e = 0; e < NC; e += 4) {
      if (col + e + 4 <= g.b.rows) {
        *(u32x4a*)(p + col + e) = u32x4a{__float_as_uint(v[e]), __float_as_uint(v[e + 1]), __float_as_uint(v[e + 2]),
                                         __float_as_uint(v[e + 3])};
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (col + e + x < g.b.rows) p[col + e + x] = v[e + x];
      }
    }
    return;
  }
  T* c = (T*)g.out + (size_t)row * g.ldo + col;
  const T* b = (const T*)g.bias + col;
  if (col + NC <= g.b.rows) {
    if constexpr (NC == 8) {
      float o[8];
      if (g.bias) {
        load8(b, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += o[e];
      }
      if (g.beta != 0.f) {
        load8(c, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += o[e];
      }
      store8(c, v);
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < NC; ++e) {
        float x = v[e];
        if (g.bias) x += ldf(b, e);
        if (g.beta != 0.f) x += ldf(c, e);
        stf(c, e, x);
      }
    } else {
      u32x4a o;
      if (g.bias) {
        o = *(const u32x4a*)b;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += __uint_as_float(o[e]);
      }
      if (g.beta != 0.f) {
        o = *(const u32x4a*)c;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += __uint_as_float(o[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(v[e]);
      *(u32x4a*)c = o;
    }
  } else {
#pragma unroll
    for (int e = 0; e < NC; ++e)
      if (col + e < g.b.rows) {
        float x = v[e];
        if (g.bias) x += ldf(b, e);
        if (g.beta != 0.f) x += ldf(c, e);
        stf(c, e, x);
      }
  }
}

// Epilogue of a wave's FM x FN fragments of 32 x 32 (rows from row0, columns from col0): 32
// rows at a time through its own LDS at Ts (it reads back only what it wrote, in issue
// order), so that stores are whole lines.  A lane's columns are the same in every row:
// their bias is loaded once; old values of C are loaded a fragment row at a time,
// all in flight before the first use.
template <int FN>
constexpr int epi_floats() { return 32 * (32 * FN + 4); }

template <typename T, int FM, int FN>
__device__ __forceinline__ void epilogue8(const Matmul8Args& g, const f32x16 (&acc)[FM][FN], int row0, int col0, float* Ts) {
  constexpr int CS = 32 * FN + 4, NC = sizeof(T) == 2 ? 8 : 4;  // floats per staged row; columns per lane and store
  constexpr int LPR = 32 * FN / NC, RPP = 64 / LPR, P = 32 / RPP;  // lanes per row, rows per store, stores
  const int lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
  const int r_in = lane / LPR, c_in = lane % LPR * NC, col = col0 + c_in;
  const int M = g.a.rows, N = g.b.rows;
  const bool split = g.splits > 1, inner = row0 + 32 * FM <= M && col0 + 32 * FN <= N;
  float bias[NC];
#pragma unroll
  for (int e = 0; e < NC; ++e) bias[e] = 0.f;
  if (g.bias && !split && inner) {
#pragma unroll
    for (int e = 0; e < NC; ++e) bias[e] = ldf((const T*)g.bias, col + e);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(f32x4*)(Ts + l * CS + 32 * j + 8 * q + 4 * h) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    asm volatile("" ::: "memory");
    const int row = row0 + 32 * i + r_in;
    auto staged = [&](int p, float* v) {
#pragma unroll
      for (int q = 0; q < NC / 4; ++q) {
        const f32x4 x = *(const f32x4*)(Ts + (p * RPP + r_in) * CS + c_in + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] = x[e];
      }
    };
    if (!inner || split) {
#pragma unroll 1
      for (int p = 0; p < P; ++p) {
        float v[NC];
        staged(p, v);
        if (row + p * RPP < M) store_c<T, NC>(g, row + p * RPP, col, v);
      }
    } else {
      T* const c = (T*)g.out + (size_t)row * g.ldo + col;
      u32x4a old[P];
      if (g.beta != 0.f) {
#pragma unroll
        for (int p = 0; p < P; ++p) old[p] = *(const u32x4a*)(c + (size_t)(p * RPP) * g.ldo);
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p) old[p] = u32x4a{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float v[NC];
        staged(p, v);
#pragma unroll
        for (int e = 0; e < NC; ++e) {
          const uint32_t u = old[p][sizeof(T) == 2 ? e / 2 : e];
          v[e] += bias[e] + (sizeof(T) == 2 ? bf2f(e & 1 ? u >> 16 : u & 0xffffu) : __uint_as_float(u));
        }
        u32x4a o;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if constexpr (sizeof(T) == 2) o[w] = (uint32_t)f2bf(v[2 * w]) | (uint32_t)f2bf(v[2 * w + 1]) << 16;
          else o[w] = __float_as_uint(v[w]);
        }
        *(u32x4a*)(c + (size_t)(p * RPP) * g.ldo) = o;
      }
    }
    asm volatile("" ::: "memory");
  }
}

template <int FA, typename T, int BM, int BN, int WM, int WN, int KG>
__global__ __launch_bounds__(64 * WM * WN * KG) void matmul8_tile_k(Matmul8Args g) {
  take_split(g);
  constexpr int BK = 64, NW = WM * WN, FM = BM / (32 * WM), FN = BN / (32 * WN), HM = FM / 2;
  static_assert(FM % 2 == 0, "A's fragments go in two halves");
  constexpr int STG = (BM + BN) * BK, SB = BM * BK;
  // one variable per stage: accesses name their stage statically (see wait_vm_lds)
  __shared__ __attribute__((aligned(1024))) char st0[KG * STG];
  __shared__ __attribute__((aligned(1024))) char st1[KG * STG];
  __shared__ __attribute__((aligned(1024))) char st2[KG * STG];
  __shared__ __attribute__((aligned(1024))) char st3[KG * STG];

  const int M = g.a.rows, N = g.b.rows;
  const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + BN - 1) / BN;
  int tm, tn;
  tile_coords(xcd_remap(blockIdx.x, tiles_m * tiles_n), tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int grp = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW;
  const int lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
  const int wave = (threadIdx.x >> 6) % NW, wm = wave / WN, wn = wave % WN;

  typedef Op8<BM, NW, BM / WM> OpA;
  typedef Op8<BN, NW, BN / WN> OpB;
  OpA oa;
  OpB ob;
  oa.init((int)g.a.ld, wm * (BM / WM));
  ob.init((int)g.b.ld, wn * (BN / WN));
  // the tile's rows: offsets stay below 2^31 (ld <= 2^22), rows past the end and the
  // prefetch behind the last row read zeros
  const int kp = (g.a.k + 127) / 128 * 128;
  const __amdgpu_buffer_rsrc_t RA = make_rsrc(g.a.q + (size_t)m0 * g.a.ld, (min(BM, M - m0) - 1) * (long)g.a.ld + kp);
  const __amdgpu_buffer_rsrc_t RB = make_rsrc(g.b.q + (size_t)n0 * g.b.ld, (min(BN, N - n0) - 1) * (long)g.b.ld + kp);

  // exponent words of this lane's row of each fragment (four blocks = eight k tiles)
  uint32_t pa[FM], pb[FN];
#pragma unroll
  for (int i = 0; i < FM; ++i) pa[i] = min(m0 + wm * (BM / WM) + 32 * i + l, M - 1);
#pragma unroll
  for (int j = 0; j < FN; ++j) pb[j] = min(n0 + wn * (BN / WN) + 32 * j + l, N - 1);

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  auto stage = [&](auto ic) -> char* {
    constexpr int c = decltype(ic)::value & 3;
    if constexpr (c == 0) return st0 + grp * STG;
    else if constexpr (c == 1) return st1 + grp * STG;
    else if constexpr (c == 2) return st2 + grp * STG;
    else return st3 + grp * STG;
  };
  // the group's k tiles: kt0 .. kt0 + nk - 1, kt0 a multiple of 8 (whole exponent words)
  const int nkt = kp / BK, nkg = KG == 1 ? nkt : ((nkt + KG - 1) / KG + 7) / 8 * 8;
  const int kt0 = grp * nkg, nk = KG == 1 ? nkt : max(0, min(nkg, nkt - kt0));
  uint32_t wa[FM], wb[FN], na[FM], nb[FN];
  auto words = [&](int t) {  // of k tile t (a multiple of 8); the last ones again behind the end
    const size_t w = min(t, nkt - 1) / 8;
    const uint32_t *sa = g.a.sc + w * M, *sb = g.b.sc + w * N;
#pragma unroll
    for (int i = 0; i < FM; ++i) na[i] = sa[pa[i]];
#pragma unroll
    for (int j = 0; j < FN; ++j) nb[j] = sb[pb[j]];
  };

  uint64_t large = 0;  // lanes that met a scale beyond what bf16 is used for
  i32x8 fa[FM], fb[2][FN];
  bf16x8 xb[FN][4];
  auto mfma_half = [&](int half, int buf) {
    if (half == 0) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int w = 0; w < 4; ++w)
          xb[j][w] = widen8<E4M3>(fb[buf][j][2 * w], fb[buf][j][2 * w + 1], scale_of(wb[j] & 255u));
    }
#pragma unroll
    for (int i = half * HM; i < (half + 1) * HM; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const bf16x8 xa = widen8<FA>(fa[i][2 * w], fa[i][2 * w + 1], scale_of(wa[i] & 255u));
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[j][w], xa, acc[i][j], 0, 0, 0);
      }
  };

  constexpr int NL = OpA::NL + OpB::NL;
  words(kt0);
  auto load_tile = [&](char* S, int t) {
    oa.load(RA, S, (kt0 + t) * BK);
    ob.load(RB, S + SB, (kt0 + t) * BK);
  };
  load_tile(st0 + grp * STG, 0);
  load_tile(st1 + grp * STG, 1);
  load_tile(st2 + grp * STG, 2);
  wait_vm_lds<2 * NL>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < HM; ++i) fa[i] = oa.frag(st0 + grp * STG, i);
#pragma unroll
  for (int j = 0; j < FN; ++j) fb[0][j] = ob.frag(st0 + grp * STG + SB, j);

  // k tile kt is read from stage kt % 4, tile kt + 3 loads into the stage of tile kt - 1
  auto iter = [&](auto ic, int kt) {
    constexpr int c = decltype(ic)::value, buf = c & 1;
    const char* S = stage(std::integral_constant<int, c>());
    const char* Sn = stage(std::integral_constant<int, c + 1>());
    char* Sx = stage(std::integral_constant<int, c + 3>());
    if constexpr (c == 0) {
#pragma unroll
      for (int i = 0; i < FM; ++i) wa[i] = na[i];
#pragma unroll
      for (int j = 0; j < FN; ++j) wb[j] = nb[j];
      words(kt0 + kt + 8);
      uint32_t w = 0;
#pragma unroll
      for (int i = 0; i < FM; ++i) w |= large_scales(wa[i]);
#pragma unroll
      for (int j = 0; j < FN; ++j) w |= large_scales(wb[j]);
      large |= __ballot(w != 0);
    } else if constexpr (c % 2 == 0) {  // the next block of 128
#pragma unroll
      for (int i = 0; i < FM; ++i) wa[i] >>= 8;
#pragma unroll
      for (int j = 0; j < FN; ++j) wb[j] >>= 8;
    }
#pragma unroll
    for (int i = HM; i < FM; ++i) fa[i] = oa.frag(S, i);
    oa.load(RA, Sx, (kt0 + kt + 3) * BK);
    mfma_half(0, buf);
    __builtin_amdgcn_sched_barrier(0);
    // tile kt + 1 has landed once only the loads of tile kt + 2 and A's of kt + 3 fly
    wait_vm_lds<NL + OpA::NL>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < HM; ++i) fa[i] = oa.frag(Sn, i);
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[buf ^ 1][j] = ob.frag(Sn + SB, j);
    ob.load(RB, Sx + SB, (kt0 + kt + 3) * BK);
    mfma_half(1, buf);
    __builtin_amdgcn_sched_barrier(0);
  };
  int kt = 0;
  for (; kt + 7 < nk; kt += 8) {
    iter(std::integral_constant<int, 0>(), kt);
    iter(std::integral_constant<int, 1>(), kt + 1);
    iter(std::integral_constant<int, 2>(), kt + 2);
    iter(std::integral_constant<int, 3>(), kt + 3);
    iter(std::integral_constant<int, 4>(), kt + 4);
    iter(std::integral_constant<int, 5>(), kt + 5);
    iter(std::integral_constant<int, 6>(), kt + 6);
    iter(std::integral_constant<int, 7>(), kt + 7);
  }
  // the rest: k tiles come in pairs
  if (kt < nk) {
    iter(std::integral_constant<int, 0>(), kt);
    iter(std::integral_constant<int, 1>(), kt + 1);
  }
  if (kt + 2 < nk) {
    iter(std::integral_constant<int, 2>(), kt + 2);
    iter(std::integral_constant<int, 3>(), kt + 3);
  }
  if (kt + 4 < nk) {
    iter(std::integral_constant<int, 4>(), kt + 4);
    iter(std::integral_constant<int, 5>(), kt + 5);
  }
  // one barrier per k tile: a group with fewer joins the others' rest
  if constexpr (KG > 1)
    for (int i = nk; i < nkg; ++i) __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();

  if (large) {  // the wave's products once more, from memory
    auto chunks = [](const uint8_t* p) {
      return __builtin_shufflevector(*(const i32x4*)p, *(const i32x4*)(p + 32), 0, 1, 2, 3, 4, 5, 6, 7);
    };
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
#pragma unroll 1
    for (int t = kt0; t < kt0 + nk; ++t) {
      const int at = t * BK + 16 * h, sh = 8 * (t / 2 & 3);
      const uint32_t *sa = g.a.sc + (size_t)(t / 8) * M, *sb = g.b.sc + (size_t)(t / 8) * N;
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        fb[0][j] = chunks(g.b.q + pb[j] * g.b.ld + at);
        wb[j] = sb[pb[j]] >> sh;
      }
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const i32x8 a = chunks(g.a.q + pa[i] * g.a.ld + at);
        wa[i] = sa[pa[i]] >> sh;
#pragma unroll 1
        for (int p = 0; p < 8; ++p) {
          const i32x8 x = one_of_8(a, p);
#pragma unroll
          for (int j = 0; j < FN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[0][j], x, acc[i][j], 0, FA, 0, (int)wb[j], 0,
                                                                        (int)wa[i]);
        }
      }
    }
  }

  auto stn = [&](int i) { return i == 0 ? st0 : i == 1 ? st1 : i == 2 ? st2 : st3; };
  if constexpr (KG > 1) {
    // the other groups hand theirs to the first, added in group order
    constexpr int PW = FM * FN * 4096, PER = KG * STG / PW;  // bytes of a wave's sums; waves per stage
    static_assert(PER >= 1 && NW * (KG - 1) <= 4 * PER, "the sums must fit the stages");
    if (grp > 0) {
      const int slot = (grp - 1) * NW + wave;
      f32x4* const out = (f32x4*)(stn(slot / PER) + slot % PER * PW);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            out[((i * FN + j) * 4 + q) * 64 + lane] =
                f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    }
    __syncthreads();
    if (grp == 0) {
      for (int o = 0; o < KG - 1; ++o) {
        const int slot = o * NW + wave;
        const f32x4* const in = (const f32x4*)(stn(slot / PER) + slot % PER * PW);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4 x = in[((i * FN + j) * 4 + q) * 64 + lane];
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += x[e];
            }
      }
    }
    __syncthreads();  // the sums are read: their place is free
    if (grp > 0) return;
  }

  constexpr int TB = 4 * epi_floats<FN>(), EPS = KG * STG / TB;  // waves per stage
  static_assert(EPS >= 1 && NW <= 4 * EPS, "epilogue staging");
  epilogue8<T, FM, FN>(g, acc, m0 + wm * (BM / WM), n0 + wn * (BN / WN), (float*)(stn(wave / EPS) + wave % EPS * TB));
}

// ------------------------------------------------------- tiled kernel, 128 deep
// BM x BN tiles for bf16 results, four waves of (BM / 2) x (BN / 2) made of 32 x 32
// fragments, k tiles of 128 bytes (one block) through two LDS stages.  One wave per
// SIMD holds its part of C in 256 accumulator registers and reads (128 + 128) x 128
// bytes for 64 instructions, two thirds of what eight waves of 128 x 64 read: the card
// runs at its power limit here, and what LDS reads do not take, the clock gets.
//
// With one wave per SIMD nothing hides a wait, so every LDS read and direct load is
// issued a quarter of a k tile or more before its use.  A k tile is four quarters,
// (half of A) x (half of B); halves of A and B are named 0 and 1, and Bp is B's half p,
// p = the k tile's parity:
//   quarter 0: A0 Bp       while B(1-p) and A1 are read; barrier: the stage is read by all
//   quarter 1: A0 B(1-p)   while the first loads of k tile + 2 go into that stage
//   quarter 2: A1 B(1-p)   while more do; barrier: the next k tile has landed
//   quarter 3: A1 Bp       while the rest do and the next k tile's A0 and B(1-p) are read,
//                          its first quarter's operands
// Measured at 8192^3: all loads in quarters 2 and 3 401 us, spread over quarters 2, 3 and
// the next 0 398, reads early in their quarter 390, as above 385; one barrier per k tile
// with the loads in quarters 3 and 0 408.
// LDS rows are 128 bytes; chunk c (16 bytes) of row r lies at c ^ ((r >> 1) & 7): a
// read's 16 neighbouring lanes (16 rows, one chunk), and groups such as {0-3, 32-35},
// then cover the 64 banks once (with c ^ (r & 7) the counters showed 4 conflict cycles
// a read).
template <int ROWS, int WR>
struct Op8q {
  static constexpr int NL = ROWS / 32;  // direct loads of 1 KB (8 rows) per wave and k tile
  static_assert(NL % 2 == 0, "a load's parity is its rows' bit 3");
  int voff, step;                       // offset of the first; bytes from one to the next
  int fo;                               // chunk 4 h of this lane's row of fragment 0; chunk 4 h + x lies at fo ^ 16 x
  __device__ inline void init(int ld, int wrow0) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    voff = (8 * wave * NL + lane / 8) * ld + 16 * ((lane & 7) ^ (lane >> 4));
    step = 8 * ld;
    const int r = lane & 31;
    fo = (wrow0 + r) * 128 + ((4 * (lane >> 5)) ^ ((r >> 1) & 7)) * 16;
  }
  // loads t0 .. t0 + n - 1 of the k tile at k0 into the stage at S
  template <int T0, int N>
  __device__ inline void load(__amdgpu_buffer_rsrc_t R, char* S, int k0) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int t = T0; t < T0 + N; ++t) load_lds16(R, S + (wave * NL + t) * 1024, (t & 1 ? voff ^ 64 : voff) + (t * step + k0));
  }
  __device__ inline i32x8 frag(const char* S, int i, int kk) const {
    const i32x4 a = *(const i32x4*)(S + (fo ^ (32 * kk)) + i * 4096), b = *(const i32x4*)(S + (fo ^ (32 * kk + 16)) + i * 4096);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// Instruction interleave of a quarter: up to RP LDS reads behind each matrix instruction
// until all R are issued, the L direct loads evenly.
template <int MF, int R, int L, int RP, int I = 0>
__device__ __forceinline__ void quarter_sched() {
  if constexpr (I < MF) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    constexpr int r = I == MF - 1 ? R : (R < RP ? R : RP), l = L * (I + 1) / MF - L * I / MF;
    if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
    if constexpr (l > 0) __builtin_amdgcn_sched_group_barrier(0x020, l, 0);
    quarter_sched<MF, R - r, L, RP, I + 1>();
  }
}

// Epilogue of the streaming form: a wave's fragments by 32 rows x 64 columns through 4.5 KB
// of LDS of its own, already rounded (the bias is added in the accumulators' layout: a
// lane holds four neighbouring columns of a row).  Bs: the bias from col0 on, in LDS.
// N % 8 == 0, beta 0.
template <int SM, int SN>
__device__ __forceinline__ void store_stream(const Matmul8Args& g, f32x16 (&acc)[SM][SN], int row0, int col0, const uint16_t* Bs,
                                             uint16_t* Ts) {
  constexpr int CS = 72;  // bf16 per staged row
  int lane = threadIdx.x & 63;
  long ldo = g.ldo;
  asm volatile("" : "+v"(lane), "+s"(ldo));  // nothing of the epilogue is kept in registers over the products
  const int l = lane & 31, h = lane >> 5, r8 = lane >> 3, c8 = (lane & 7) * 8, M = g.a.rows, N = g.b.rows;
  uint16_t* const out = (uint16_t*)g.out + (size_t)(row0 + r8) * ldo + col0 + c8;
#pragma unroll
  for (int jj = 0; jj < SN; jj += 2) {
    __builtin_amdgcn_sched_barrier(0);
    float b[2][16];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint2 w = *(const uint2*)(Bs + 32 * (jj + j) + 8 * q + 4 * h);
        b[j][4 * q] = __uint_as_float(w.x << 16);
        b[j][4 * q + 1] = __uint_as_float(w.x & 0xffff0000u);
        b[j][4 * q + 2] = __uint_as_float(w.y << 16);
        b[j][4 * q + 3] = __uint_as_float(w.y & 0xffff0000u);
      }
#pragma unroll
    for (int i = 0; i < SM; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t o[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int n = 4 * q + 2 * e;
            o[e] = (uint32_t)f2bf(acc[i][jj + j][n] + b[j][n]) | (uint32_t)f2bf(acc[i][jj + j][n + 1] + b[j][n + 1]) << 16;
          }
          *(uint2*)(Ts + l * CS + 32 * j + 8 * q + 4 * h) = make_uint2(o[0], o[1]);
        }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const u32x4a o = *(const u32x4a*)(Ts + (8 * p + r8) * CS + c8);
        if (row0 + 32 * i + 8 * p + r8 < M && col0 + 32 * jj + c8 < N)
          *(u32x4a*)(out + (size_t)(32 * i + 8 * p) * ldo + 32 * jj) = o;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// STREAM: at most one workgroup per CU goes through the tiles id, id + grid, ...; the last
// two k tiles of one load the first two of the next, so that its first operands are in
// registers before the epilogue, which has its own LDS, and its loads fly meanwhile.
// Without it a workgroup waits 2 us for its first tile and 3 for its last stores.
// 9216 x 12288, k 512: 113 -> 95 us; 9216 x 16384, k 4096 with bias 474 -> 465 (loading the
// bias from memory in the epilogue 472: a wait for it is one for the loads before it).
template <int FA, int BM, int BN, int L2, int L3, bool STREAM>
__global__ __launch_bounds__(256) void matmul8_quad_k(Matmul8Args g) {
  take_split(g);
  constexpr int BK = 128, SM = BM / 64, SN = BN / 64, HM = SM / 2, HN = SN / 2;  // 32 x 32 fragments of a wave
  constexpr int SB = BM * BK;
  __shared__ __attribute__((aligned(1024))) char st0[(BM + BN) * BK];
  __shared__ __attribute__((aligned(1024))) char st1[(BM + BN) * BK];

  const int M = g.a.rows, N = g.b.rows;
  const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + BN - 1) / BN;
  const int tiles = tiles_m * tiles_n;
  auto place = [&](int id, int& m, int& n) {
    int tm, tn;
    tile_coords(xcd_remap(id, tiles), tiles_m, tiles_n, tm, tn);
    m = tm * BM;
    n = tn * BN;
  };
  int id = blockIdx.x, m0, n0, m1 = 0, n1 = 0;  // this tile and (STREAM) the next one
  place(id, m0, n0);
  const int lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;

  typedef Op8q<BM, BM / 2> OpA;
  typedef Op8q<BN, BN / 2> OpB;
  OpA oa;
  OpB ob;
  oa.init((int)g.a.ld, wm * (BM / 2));
  ob.init((int)g.b.ld, wn * (BN / 2));
  // the tile's rows: offsets stay below 2^31 (ld <= 2^22), rows past the end and the
  // prefetch behind the last row read zeros
  const int nk = (g.a.k + BK - 1) / BK;
  bool more = false;  // there is a next tile: otherwise its loads bring nothing
#define JG_ROWS8(x, r0, cnt, on) \
  make_rsrc(x.q + (size_t)(r0) * x.ld, (on) ? (min(cnt, x.rows - (r0)) - 1) * (long)x.ld + nk * BK : 0)
  __amdgpu_buffer_rsrc_t RA = JG_ROWS8(g.a, m0, BM, true), RB = JG_ROWS8(g.b, n0, BN, true);

  // exponent words of the tile's rows, four k tiles each: through LDS as well
  __shared__ __attribute__((aligned(256))) uint32_t stw[BM + BN];
  constexpr int NWL = (BM + BN) / 256;  // direct loads of 64 words per wave
  constexpr int NW = NWL + STREAM;      // and one of the bias
  __shared__ __attribute__((aligned(256))) uint32_t stb[STREAM ? 256 : 1];
  static_assert(BN <= 512, "a wave's 64 words of two columns");
  uint32_t wa[SM], wb[SN];
  // of k tile t (a multiple of 4) of the tile at m, n; the last ones again behind the end
  auto load_words = [&](int t, int m, int n, bool on) {
    const size_t w = min(t, nk - 1) / 4;
#pragma unroll
    for (int i = 0; i < NWL; ++i) {
      const int row = 64 * (4 * i + wave);  // of A's rows, then B's
      const bool a = BM >= 256 ? i < BM / 256 : wave < BM / 64;
      const int rows = a ? M : N, r0 = a ? m : n;
      const __amdgpu_buffer_rsrc_t W =
          make_rsrc((a ? g.a.sc : g.b.sc) + w * rows + r0, on ? min(a ? BM : BN, rows - r0) * 4 : 0);
      load_lds4(W, (char*)(stw + row), ((a ? row : row - BM) + lane) * 4);
    }
  };

  f32x16 acc[SM][SN];
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < SM; ++i)
#pragma unroll
      for (int j = 0; j < SN; ++j) {
        float z = 0.f;
        if constexpr (STREAM) asm volatile("" : "+v"(z));  // or one fragment of zeros is kept and copied
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = z;
      }
  };
  clear();

  i32x8 fa[SM][2], fb[SN][2];
  auto read_a = [&](const char* S, int half, bool w) {  // w: the exponent words too
#pragma unroll
    for (int i = half * HM; i < (half + 1) * HM; ++i) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) fa[i][kk] = oa.frag(S, i, kk);
      if (w) wa[i] = stw[wm * (BM / 2) + 32 * i + l];
    }
  };
  auto read_b = [&](const char* S, int half, bool w) {
#pragma unroll
    for (int j = half * HN; j < (half + 1) * HN; ++j) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) fb[j][kk] = ob.frag(S + SB, j, kk);
      if (w) wb[j] = stw[BM + wn * (BN / 2) + 32 * j + l];
    }
  };
  auto quarter = [&](auto cc, int ah, int bh) {  // cc: byte of the exponent words
    constexpr int c = decltype(cc)::value;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = ah * HM; i < (ah + 1) * HM; ++i)
#pragma unroll
        for (int j = bh * HN; j < (bh + 1) * HN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j][kk], fa[i][kk], acc[i][j], 0, FA, c, (int)wb[j], c,
                                                                      (int)wa[i]);
  };

  // direct loads LO .. HI - 1 (A's, then B's) of k tile t
  auto load = [&](auto lo, auto hi, const __amdgpu_buffer_rsrc_t& A, const __amdgpu_buffer_rsrc_t& B, char* S, int t) {
    constexpr int LO = decltype(lo)::value, HI = decltype(hi)::value, NA = OpA::NL;
    if constexpr (LO < NA) oa.template load<LO, (HI < NA ? HI : NA) - LO>(A, S, t * BK);
    if constexpr (HI > NA) ob.template load<(LO > NA ? LO - NA : 0), HI - (LO > NA ? LO : NA)>(B, S + SB, t * BK);
  };
  constexpr int NL = OpA::NL + OpB::NL;
  typedef std::integral_constant<int, 0> C0;
  typedef std::integral_constant<int, NL * L2 / 16> C1;
  typedef std::integral_constant<int, NL * (L2 + L3) / 16> C2;
  typedef std::integral_constant<int, NL> C3;
  load_words(0, m0, n0, true);
  load(C0(), C3(), RA, RB, st0, 0);
  load(C0(), C3(), RA, RB, st1, 1);
  wait_vm_lds<NL>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read_a(st0, 0, true);
  read_b(st0, 0, true);

  constexpr int MF = 2 * HM * HN;
  // one k tile; loads the k tile t2 of A, B into its place and, in the second of four, the
  // words of k tile tw of the tile at mw, nw
  auto iter = [&](auto cc, const __amdgpu_buffer_rsrc_t& A, const __amdgpu_buffer_rsrc_t& B, int t2, int tw = 0, int mw = 0,
                  int nw = 0, bool on = true) __attribute__((always_inline)) {
    constexpr int c = decltype(cc)::value, p = c & 1;
    char* S = p ? st1 : st0;
    const char* Sn = p ? st0 : st1;
    // keeps the fragments' addresses (too far apart for one base) from being held in
    // registers over the loop: an addition each instead
    asm("" : "+v"(oa.fo), "+v"(ob.fo));
    if constexpr (STREAM) asm("" : "+v"(oa.voff), "+v"(ob.voff), "+s"(oa.step), "+s"(ob.step));
    read_b(S, 1 - p, c == 0);
    read_a(S, 1, c == 0);
    quarter(cc, 0, p);
    quarter_sched<MF, (c == 0 ? 5 : 4) * (HN + HM), 0, 2>();
    __builtin_amdgcn_sched_barrier(0);
    // every wave's reads of this stage are done
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    load(C0(), C1(), A, B, S, t2);
    quarter(cc, 0, 1 - p);
    quarter_sched<MF, 0, C1::value, 1>();
    __builtin_amdgcn_sched_barrier(0);
    // (the words of the four k tiles under way are in registers since the first of them)
    if constexpr (c == 1) load_words(tw, mw, nw, on);
    if constexpr (c == 1 && STREAM)  // this tile's bias, zeros if there is none
      load_lds4(make_rsrc((const uint16_t*)g.bias + n0, g.bias ? min(BN, N - n0) * 2 : 0), (char*)(stb + 64 * wave), threadIdx.x * 4);
    load(C1(), C2(), A, B, S, t2);
    quarter(cc, 1, 1 - p);
    quarter_sched<MF, 0, C2::value - C1::value + (c == 1 ? NW : 0), 1>();
    __builtin_amdgcn_sched_barrier(0);
    // the next k tile has landed once only the loads of the one after it (and the words) fly
    wait_vm_lds<C2::value + (c == 1 ? NW : 0)>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    load(C2(), C3(), A, B, S, t2);
    read_a(Sn, 0, c == 3);
    read_b(Sn, 1 - p, c == 3);
    quarter(cc, 1, p);
    quarter_sched<MF, (c == 3 ? 5 : 4) * (HM + HN), NL - C2::value, 3>();
    __builtin_amdgcn_sched_barrier(0);
  };
  typedef std::integral_constant<int, 0> I0;
  typedef std::integral_constant<int, 1> I1;
  typedef std::integral_constant<int, 2> I2;
  typedef std::integral_constant<int, 3> I3;
  const int row_in = wm * (BM / 2), col_in = wn * (BN / 2);
  if constexpr (STREAM) {
    __shared__ __attribute__((aligned(16))) uint16_t ste[4][32 * 72];
    for (;;) {
      more = id + (int)gridDim.x < tiles;
      if (more) {
        id += gridDim.x;
        place(id, m1, n1);
      }
      const __amdgpu_buffer_rsrc_t RA1 = JG_ROWS8(g.a, m1, BM, more), RB1 = JG_ROWS8(g.b, n1, BN, more);
      int kt = 0;
      do {
        const bool end = kt + 4 >= nk;
        const __amdgpu_buffer_rsrc_t A = end ? RA1 : RA, B = end ? RB1 : RB;
        const int t = end ? 0 : kt + 4;
        iter(I0(), RA, RB, kt + 2);
        iter(I1(), RA, RB, kt + 3, t, end ? m1 : m0, end ? n1 : n0, !end || more);
        iter(I2(), A, B, t);
        iter(I3(), A, B, t + 1);
        kt += 4;
      } while (kt < nk);
      store_stream<SM, SN>(g, acc, m0 + row_in, n0 + col_in, (const uint16_t*)stb + col_in, ste[wave]);
      if (!more) break;
      clear();
      m0 = m1;
      n0 = n1;
      RA = RA1;
      RB = RB1;
    }
    __builtin_amdgcn_s_waitcnt(0);  // no load into LDS outlives the workgroup
  } else {
    int kt = 0;
    for (; kt + 3 < nk; kt += 4) {
      iter(I0(), RA, RB, kt + 2);
      iter(I1(), RA, RB, kt + 3, kt + 4, m0, n0);
      iter(I2(), RA, RB, kt + 4);
      iter(I3(), RA, RB, kt + 5);
    }
    if (kt < nk) iter(I0(), RA, RB, kt + 2);
    if (kt + 1 < nk) iter(I1(), RA, RB, kt + 3, kt + 4, m0, n0);
    if (kt + 2 < nk) iter(I2(), RA, RB, kt + 4);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    constexpr int TB = 4 * epi_floats<SN>();
    static_assert(2 * TB <= (BM + BN) * BK, "epilogue staging");
    epilogue8<uint16_t, SM, SN>(g, acc, m0 + row_in, n0 + col_in, (float*)((wave & 2 ? st1 : st0) + (wave & 1) * TB));
  }
#undef JG_ROWS8
}

// ------------------------------------------------------------------- few rows
// Up to 16 rows of A: bound by reading B once.  A workgroup takes 16 rows of B, its eight
// waves every eighth block of 128 (neighbouring blocks of a row are read together),
// operands straight to registers with four blocks in flight a wave.  The waves' sums
// are added through LDS in wave order.  A lane takes chunks q and q + 4 of a row's block
// (q = lane / 16), the same on both sides.  One row, 16384 x 4096 (68 MB from memory): 15.8
// us, 4.3 TB/s; 4096 x 12288 (50 MB): 13.2.  With four weights in turn, which the 256 MB
// cache holds in part: 13.5 and 10.9, where 32 rows of B a workgroup took 14.5 and 15.5, two
// blocks in flight 16.3 and 10.0 (these six with the 8-bit instruction).
template <int FA, typename T>
__global__ __launch_bounds__(512) void matmul8_few_k(Matmul8Args g) {
  constexpr int KW = 8, U = 4;
  __shared__ f32x4 red[KW][64];
  const int lane = threadIdx.x & 63, l = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int M = g.a.rows, N = g.b.rows, n0 = blockIdx.x * 16, nk = (g.a.k + 127) / 128;
  const uint32_t ra = min(l, M - 1), rb = min(n0 + l, N - 1);
  const uint8_t* const pa = g.a.q + ra * g.a.ld + 16 * q;
  const uint8_t* const pb = g.b.q + rb * g.b.ld + 16 * q;
  const int sh = 8 * (wave & 3);  // the blocks of a wave have one place in their exponent words
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  uint32_t large = 0;

  // blocks b0, b0 + KW, ... (UU of them): all loads, then all products
  auto blocks = [&](auto uu, int b0) {
    constexpr int UU = decltype(uu)::value;
    i32x8 fa[UU], fb[UU];
    uint32_t wa[UU], wb[UU];
#pragma unroll
    for (int u = 0; u < UU; ++u) {
      const size_t b = b0 + KW * u;
      fb[u] = __builtin_shufflevector(*(const i32x4*)(pb + b * 128), *(const i32x4*)(pb + b * 128 + 64), 0, 1, 2, 3, 4, 5, 6, 7);
      wb[u] = (g.b.sc + b / 4 * N)[rb];
      fa[u] = __builtin_shufflevector(*(const i32x4*)(pa + b * 128), *(const i32x4*)(pa + b * 128 + 64), 0, 1, 2, 3, 4, 5, 6, 7);
      wa[u] = (g.a.sc + b / 4 * M)[ra];
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < UU; ++u) {
      large |= large_scales(wa[u]) | large_scales(wb[u]);
#pragma unroll
      for (int w = 0; w < 8; w += 2)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<E4M3>(fb[u][w], fb[u][w + 1], scale_of((wb[u] >> sh) & 255u)),
                                                      widen8<FA>(fa[u][w], fa[u][w + 1], scale_of((wa[u] >> sh) & 255u)), acc, 0,
                                                      0, 0);
    }
  };
  int b0 = wave;
  for (; b0 + KW * (U - 1) < nk; b0 += KW * U) blocks(std::integral_constant<int, U>(), b0);
  for (; b0 < nk; b0 += KW) blocks(std::integral_constant<int, 1>(), b0);
  if (__ballot(large != 0)) {  // the wave's products once more
    auto chunks = [](const uint8_t* p) {
      return __builtin_shufflevector(*(const i32x4*)p, *(const i32x4*)(p + 64), 0, 1, 2, 3, 4, 5, 6, 7);
    };
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
    for (size_t b = wave; b < (size_t)nk; b += KW) {
      const i32x8 fa = chunks(pa + b * 128), fb = chunks(pb + b * 128);
      const uint32_t wa = (g.a.sc + b / 4 * M)[ra] >> sh, wb = (g.b.sc + b / 4 * N)[rb] >> sh;
#pragma unroll 1
      for (int p = 0; p < 8; ++p)
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, one_of_8(fa, p), acc, 0, FA, 0, (int)wb, 0, (int)wa);
    }
  }
  red[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && l < M) {
#pragma unroll
    for (int w = 1; w < KW; ++w) acc += red[w][lane];
    float y[4] = {acc[0], acc[1], acc[2], acc[3]};
    store_c<T, 4>(g, l, n0 + 4 * q, y);
  }
}

// The splits' sums in their order, bias and old C.
template <typename T>
__global__ __launch_bounds__(256) void matmul8_join_k(Matmul8Args g) {
  const size_t N = g.b.rows, n4 = (N + 3) / 4, all = (size_t)g.a.rows * N;
  const size_t x = (size_t)blockIdx.x * 256 + threadIdx.x, row = x / n4;
  const int col = (int)(x % n4) * 4;
  if (row >= (size_t)g.a.rows) return;
  const float* p = g.part + row * N + col;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (col + 4 <= (int)N) {
    for (int i = 0; i < g.splits; ++i, p += all) {
      const u32x4a u = *(const u32x4a*)p;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += __uint_as_float(u[e]);
    }
  } else {
    for (int i = 0; i < g.splits; ++i, p += all)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < (int)N) v[e] += p[e];
  }
  g.splits = 1;
  store_c<T, 4>(g, (int)row, col, v);
}

// The streaming form of 256 x 256 tiles: whole groups of four k tiles, 16-byte stores
static bool streams(const Matmul8Args& g) { return ((long)g.a.k + 127) / 128 % 4 == 0 && g.b.rows % 8 == 0; }

template <int FA, int BM, int BN>
static void launch_quad(const Matmul8Args& g, hipStream_t s) {
  const dim3 grid((unsigned)((g.a.rows + BM - 1) / BM) * (unsigned)((g.b.rows + BN - 1) / BN), g.splits);
  if constexpr (BM == 256) {
    if (g.splits == 1 && streams(g) && (uintptr_t)g.bias % 4 == 0 && g.beta == 0.f) {
      hipLaunchKernelGGL((matmul8_quad_k<FA, BM, BN, 6, 5, true>), dim3(grid.x < 256 ? grid.x : 256), dim3(256), 0, s, g);
      return;
    }
  }
  hipLaunchKernelGGL((matmul8_quad_k<FA, BM, BN, 6, 5, false>), grid, dim3(256), 0, s, g);
}

template <int FA, typename T, int BM, int BN, int WM, int WN, int KG>
static void launch_tile(const Matmul8Args& g, hipStream_t s) {
  const dim3 grid((unsigned)((g.a.rows + BM - 1) / BM) * (unsigned)((g.b.rows + BN - 1) / BN), g.splits);
  hipLaunchKernelGGL((matmul8_tile_k<FA, T, BM, BN, WM, WN, KG>), grid, dim3(64 * WM * WN * KG), 0, s, g);
}

// ---------------------------------------------------------------------- launch
enum Kind8 { K8_FEW, K8_32, K8_64, K8_128, K8_256 };

// Tiles and splits of k: the least estimated time (us) = rounds of the 256 CUs x (blocks
// of 128 of a split x time per block + prologue and epilogue), and for a split the
// second launch and the sums' way through memory.  The times per block are those
// measured with every CU busy: 0.29 (64 x 64); bf16 0.58 (128 x 128; 1.0 for two on a CU), 1.4
// (256 x 256); fp32 0.78 (1.65), 3.2.  64 x 32 tiles, each of four groups of waves with a
// quarter of k, need no second launch but read the left operand twice as often: 0.53 per
// block of a group on up to 32 CUs, 0.63 (17 rows) to 0.98 (64) above, 1.25 in more than one
// round.  Over 110 sizes drawn from 17 .. 9000 rows, 64 .. 16384 columns and k the choice takes
// 0.99 times the best of four tiles x eight splits in the mean and 1.19 times at most.
// Examples (us, bf16; 64 x 32, 64 x 64 in one and four splits, 128 x 128): 37 x 4096, k 12288:
// 21.5, 28.5, 16.6, 42.7; 18 x 7040, k 4864: 11.1, 14.1, 16.2, 19.5; 31 x 326, k 5248: 10.4, 15.8,
// 12.1, 16.6; 1024 x 4096, k 4096: 78, 47, 73, 21; 8192 x 8192, k 512: 128 x 128 80, 256 x 256 64;
// 6144 x 6144, k 1024: 51.8, 54.2.  The single-token kernel up to 16 rows: 14.3 at 16 x 4096,
// k 12288 (64 x 64 tiles in four splits with 17 rows: 15.7).

size_t matmul8_plan(Matmul8Args& g) {
  const int M = g.a.rows, N = g.b.rows, nb = (int)(((long)g.a.k + 127) / 128);
  g.kind = K8_FEW;
  g.splits = 1;
  g.per_split = nb;
  if (M <= 16) return 0;
  const bool f32 = g.out_dt == F32;
  double bt = 1e300;
  for (int kind = K8_32; kind <= K8_256; ++kind) {
    const int b = kind <= K8_64 ? 64 : kind == K8_128 ? 128 : 256, bn = kind == K8_32 ? 32 : b;
    const long tiles = ((long)M + b - 1) / b * (((long)N + bn - 1) / bn);
    for (int s = 1; s <= 16; ++s) {
      const int ps = s == 1 ? nb : ((nb + s - 1) / s + 3) / 4 * 4;
      const long wgs = tiles * s;
      if (s > 1 && (ps < 8 || wgs > 1024)) break;  // more only costs more
      if ((nb + ps - 1) / ps != s) continue;
      double t;
      if (kind == K8_32) {
        if (s > 1) break;  // its four groups of k are the split
        const double one = wgs > 256 ? 1.25 : wgs > 32 ? 0.625 + 0.0075 * ((M < 64 ? M : 64) - 17) : 0.525;
        t = 2.8 + (wgs + 255) / 256 * ((nb + 15) / 16 * 4 * one);
      } else if (kind == K8_64) {
        t = 2.0 + (wgs + 255) / 256 * (ps * 0.29 + 1.5);
      } else if (kind == K8_128) {  // two workgroups per CU
        const double one = ps * (f32 ? 0.78 : 0.58) + 2.5, two = ps * (f32 ? 1.65 : 1.0) + 3.5;
        const long rest = wgs % 512;
        t = 2.0 + wgs / 512 * two + (rest == 0 ? 0.0 : rest <= 256 ? one : two);
      } else {
        t = 4.0 + (wgs + 255) / 256 * (ps * (f32 ? 3.2 : 1.4) + (s == 1 && streams(g) ? 6.5 : 8.5));
      }
      if (s > 1) t += 4.0 + (double)M * N * s * 8 / 4.5e6;
      if (t < bt) {
        bt = t;
        g.kind = kind;
        g.splits = s;
        g.per_split = ps;
      }
    }
  }
  return g.splits > 1 ? (size_t)g.splits * M * N * sizeof(float) : 0;
}

template <int FA, typename T>
static void launch_matmul8(const Matmul8Args& g, hipStream_t s) {
  if (g.kind == K8_FEW) {
    hipLaunchKernelGGL((matmul8_few_k<FA, T>), dim3((g.b.rows + 15) / 16), dim3(512), 0, s, g);
    return;
  }
  if (g.kind == K8_32) return launch_tile<FA, T, 64, 32, 1, 1, 4>(g, s);
  if (g.kind == K8_64) return launch_tile<FA, T, 64, 64, 1, 2, 2>(g, s);
  if constexpr (sizeof(T) == 2) {
    if (g.kind == K8_128) launch_quad<FA, 128, 128>(g, s);
    else launch_quad<FA, 256, 256>(g, s);
  } else {
    if (g.kind == K8_128) launch_tile<FA, T, 128, 128, 2, 2, 1>(g, s);
    else launch_tile<FA, T, 256, 256, 2, 4, 1>(g, s);
  }
}

int matmul8(const Matmul8Args& g, hipStream_t s) {
  const size_t M = g.a.rows, N = g.b.rows;
  const size_t bm = g.kind == K8_128 ? 128 : g.kind == K8_256 ? 256 : 64, bn = g.kind == K8_32 ? 32 : bm;
  const size_t wgs = g.kind == K8_FEW ? (N + 15) / 16 : (M + bm - 1) / bm * ((N + bn - 1) / bn);
  const char* const many = "matmul8: too many rows";
  if (int rc = too_many(wgs, g.kind == K8_FEW || (g.kind == K8_256 && g.out_dt == F32) ? 512 : 256, many)) return rc;
  if (int rc = too_many(M > N ? M + 256 : N + 256, 2, many)) return rc;  // (row numbers of the last tile are ints)
  if (g.out_dt == BF16) {
    if (g.a.fmt == E5M2) launch_matmul8<E5M2, uint16_t>(g, s);
    else launch_matmul8<E4M3, uint16_t>(g, s);
  } else {
    if (g.a.fmt == E5M2) launch_matmul8<E5M2, float>(g, s);
    else launch_matmul8<E4M3, float>(g, s);
  }
  JG_CHECK_LAUNCH("matmul8");
  if (g.splits > 1) {
    const size_t n = M * ((N + 3) / 4);
    const dim3 grid((unsigned)((n + 255) / 256));
    if (g.out_dt == BF16) hipLaunchKernelGGL(matmul8_join_k<uint16_t>, grid, dim3(256), 0, s, g);
    else hipLaunchKernelGGL(matmul8_join_k<float>, grid, dim3(256), 0, s, g);
    JG_CHECK_LAUNCH("matmul8_join");
  }
  return 0;
}

}  // namespace jg
