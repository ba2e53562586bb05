// Tiles of K and V in LDS: copies that do not pass through registers, swizzles, waits and the cross-lane steps of a row that
// two lanes share (gfx950).
#pragma once

#include "prism_common.h"

namespace prism {

// Asynchronous global -> LDS tile copies (buffer_load_dwordx4 ... lds: every lane fetches 16
// bytes at rsrc.base + voffset + soffset and the wave's 64 pieces land contiguously in LDS
// at M0-base + 16*lane).  LDS slot p (16-byte units) of a tile belongs to (row, c') with c'
// the swizzled chunk position; the lane that fills it reads global chunk
// c = c' ^ swizzle(row), i.e. the swizzle is applied on the global side.
// Buffer (not flat/global) addressing is used on purpose: LDS reads issued while such
// copies are in flight then keep exact lgkmcnt tracking in the compiler.
typedef __attribute__((address_space(3))) void* lptr_t;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
  // raw buffer, 32-bit data format, no swizzle, no TID addition
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}

// XOR applied to the chunk index of K-tile row `row` so that 16 consecutive rows put the same
// chunk on 16 different LDS bank groups: rows of 128 bytes (d = 64) come two to a 256-byte line,
// rows of 512 bytes (d = 256) wrap the banks twice.
template <int D>
__device__ __forceinline__ int k_row_swizzle(int row) {
  return D == 64 ? ((row >> 1) & 7) : (row & 15);
}

// XOR applied to the 64-byte groups of V-tile row `row`, so that the four keys of a transposing read lie in four bank groups: rows
// of 128 bytes (d = 64) come two to a 256-byte line.
template <int D>
__device__ __forceinline__ int v_row_swizzle(int row) {
  return D == 64 ? ((row >> 1) & 1) : (row & 3);
}
// this wave's first LDS slot of a tile's piece 0, wave-uniform and re-materialised per step so that the per-piece M0
// values are formed with scalar adds instead of being kept live (and spilled) across the whole loop
__device__ __forceinline__ int first_slot(int t) {
  int wave_base = __builtin_amdgcn_readfirstlane(t & ~63);
  asm volatile("" : "+s"(wave_base));
  return wave_base;
}

// One piece of such a copy, written as asm: the compiler, seeing the builtin, would wait for a copy into one of two buffers before
// it reads the other.  Waited for with wait_async_loads.
struct TileRsrc {
  u32x4 w;
};
__device__ __forceinline__ TileRsrc make_tile_rsrc(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  TileRsrc r;
  r.w[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)b);
  r.w[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(b >> 32) & 0xffffu));
  r.w[2] = __builtin_amdgcn_readfirstlane((int)bytes);
  r.w[3] = 0x00020000u;
  return r;
}
__device__ __forceinline__ void async_piece(const TileRsrc& rs, int lane_off, int tile_off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(lane_off), "s"(rs.w),
               "s"(tile_off)
               : "m0", "memory");
}

// Waits on the vector-memory counter, written with the builtin (immediate: vmcnt in bits 3:0,
// expcnt = 7 and lgkmcnt = 15 meaning "no wait") rather than inline asm, so that the compiler's
// own wait-count bookkeeping sees them: it then knows which tile copies have landed and adds no
// conservative vmcnt(0) of its own in front of the LDS reads of a finished tile.
__device__ __forceinline__ void wait_async_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0)
  asm volatile("" ::: "memory");
}
// max / sum of a value with the lane 32 away (the two lanes that share a query), on the
// v_permlane32_swap cross-lane path: an LDS shuffle here would queue behind the tile traffic
// on the critical path of every step.
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float other_half_max(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Workgroup barrier of the tile loop: this wave's LDS accesses are complete, then s_barrier.
// Unlike __syncthreads() it carries no memory fence, so the compiler adds no wait for the global
// loads, stores and atomics in flight (the next tile copies, the previous row's output, the
// queue pull); the tile copies are waited for explicitly with vmcnt where their data is needed.
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace prism
