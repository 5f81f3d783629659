// What the bf16 matrix-core attentions have in common: tiles of 64 keys in LDS, their loads,
// layout and barriers.
#pragma once

#include "common.h"

namespace infllm {
namespace {

constexpr int KB = 64;      // keys per tile

typedef short i16x4 __attribute__((ext_vector_type(4)));
#define INFLLM_LDS __attribute__((address_space(3)))

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Direct global->LDS loads (16 bytes per lane; lane i lands at LDS byte
// lds + 16*i, lds taken from M0).  Written as inline assembly so that the
// compiler does not guard every later LDS read with a wait for these loads: the
// kernel waits for them itself (s_waitcnt before the barrier that publishes a
// tile).  No compiler-generated code in these kernels uses M0.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// Wave-uniform base address plus a per-lane 32-bit byte offset.
__device__ __forceinline__ void lds_load(uint32_t lds, const void* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "m0");
}
// A full per-lane address.
__device__ __forceinline__ void lds_load_lane(uint32_t lds, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(p) : "m0");
}
#pragma clang diagnostic pop

// Values the compiler must treat as produced here (keeps derived addresses from
// being hoisted out of the tile loop into long-lived registers).
__device__ __forceinline__ uint32_t opaque_v(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ uint32_t opaque_s(uint32_t x) {
  asm volatile("" : "+s"(x));
  return x;
}

// Both LDS tiles are key-major [64 keys][D], unpadded, with the 16-byte granules
// of row r XOR-swizzled (granule g stored at g ^ swz(r)), and a 1 KB direct-load
// instruction still writes one contiguous LDS range.  gfx950 LDS serves 256
// bytes per clock (64 banks); for D = 128 (256-byte rows) the 4-bit swizzle
// below makes both fragment reads conflict-free: the K reads (16 consecutive
// rows, one granule each, per clock) and the transposed V reads (per 32 lanes:
// 4 consecutive rows x 64 bytes).  For D = 64 the 3-bit swizzle r & 7.
template <int D>
__device__ __forceinline__ int swz(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return r & 7;
}
template <int D>
__device__ __forceinline__ int tile_off(int r, int g) { return r * D + 8 * (g ^ swz<D>(r)); }

constexpr uint32_t kNoRow = 0xFFFFFFFFu;  // in a table of positions: an entry to skip

// Publish LDS tiles to the workgroup: wait until at most N of this wave's
// direct loads are still in flight (older loads -- the tiles about to be read
// -- have landed in LDS) and its own LDS traffic is done, then barrier.  Written
// out so that no wait for the younger loads is implied.
template <int N>
__device__ __forceinline__ void publish_barrier() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N));
  lds_barrier();
}

}  // namespace
}  // namespace infllm
