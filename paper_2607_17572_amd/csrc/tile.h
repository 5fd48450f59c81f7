// Device helpers of the LDS-tiled matrix-core kernels: tile order, buffer resources,
// direct-to-LDS loads, instruction interleave.
#pragma once
#include "common.h"

namespace jg {

// Workgroups are dealt to the 8 XCDs round-robin: consecutive tiles of one XCD.
__device__ inline int xcd_remap(int b, int total) {
  const int per = total / 8, rem = total % 8;
  const int xcd = b % 8, local = b / 8;
  return xcd < rem ? xcd * (per + 1) + local : rem * (per + 1) + (xcd - rem) * per + local;
}

__device__ inline void tile_coords(int id, int tiles_m, int tiles_n, int& tm, int& tn) {
  constexpr int GROUP_M = 8;
  const int in_group = GROUP_M * tiles_n;
  const int gid = id / in_group;
  const int first = gid * GROUP_M;
  const int gsz = min(tiles_m - first, GROUP_M);
  const int r = id % in_group;
  tm = first + r % gsz;
  tn = r / gsz;
}

__device__ inline __amdgpu_buffer_rsrc_t make_rsrc(const void* p, long bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, (short)0, (int)bytes, 0x00020000);
}

#define JG_LDS(p) ((__attribute__((address_space(3))) void*)(p))
// 16 bytes per lane from a buffer straight into 1 KB of LDS at S (wave-uniform)
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t R, char* S, int off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(R, JG_LDS(S), 16, off, 0, 0, 0);
}
// 4 bytes per lane into 256 bytes
__device__ __forceinline__ void load_lds4(__amdgpu_buffer_rsrc_t R, char* S, int off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(R, JG_LDS(S), 4, off, 0, 0, 0);
}

// First half of the workgroup barrier for the direct-loaded stages: this
// wave's LDS reads done (lgkmcnt 0) and at most NV of its direct loads still
// in flight (the loads of the two newest k tiles); s_barrier follows.  Unlike
// __syncthreads there is no release fence, which would wait for every direct
// load (they are LDS writes) and drain the prefetch; the empty asm statements
// keep the compiler from moving memory accesses across it.
template <int NV>
__device__ __forceinline__ void wait_vm_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((NV & 15) | ((NV >> 4) << 14) | 0x70);  // vmcnt(NV) expcnt(7) lgkmcnt(0)
}

__device__ __forceinline__ int swz_n(int row) { return (((row >> 1) & 1) * 2) ^ (((row >> 2) & 1) * 3) ^ ((row >> 3) & 1); }

// Instruction interleave of one MFMA step: MF MFMAs, with R LDS reads, W LDS
// writes and L global loads dealt out between them (reads and writes
// alternating, then loads), in that order.
template <int O, int HI, int R, int W>
__device__ __forceinline__ void sched_ops() {
  if constexpr (O < HI) {
    constexpr int RW = 2 * (R < W ? R : W);
    constexpr int kind = O < RW ? O % 2 : (O < R + W ? (R > W ? 0 : 1) : 2);
    __builtin_amdgcn_sched_group_barrier(kind == 0 ? 0x100 : (kind == 1 ? 0x200 : 0x020), 1, 0);
    sched_ops<O + 1, HI, R, W>();
  }
}
template <int MF, int R, int W, int L, int I = 0>
__device__ __forceinline__ void pipe_sched() {
  if constexpr (I < MF) {
    constexpr int T = R + W + L;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    sched_ops<I * T / MF, (I + 1) * T / MF, R, W>();
    pipe_sched<MF, R, W, L, I + 1>();
  }
}

}  // namespace jg
