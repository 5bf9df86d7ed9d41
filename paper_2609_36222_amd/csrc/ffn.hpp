// Building blocks of the expert FFN kernels (16-bit and 4-bit weights): the
// matrix instruction, buffer loads to registers and to LDS, waits.
#pragma once

#include <type_traits>

#include "common.hpp"

namespace basek {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Buffer loads: a wave-uniform resource (base, size) in scalar registers,
// a 32-bit per-lane offset and a uniform scalar offset.  Reads past the
// resource's size return zero without touching memory.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
typedef __attribute__((address_space(3))) void *lds_ptr_t;
constexpr int RSRC_CFG = 0x00020000;
constexpr uint32_t OOB = 0x40000000u;   // a scalar offset past every resource used here

__device__ __forceinline__ rsrc_t make_rsrc(const void *base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, RSRC_CFG);
}

__device__ __forceinline__ bf16x8 bload(rsrc_t r, uint32_t voff, uint32_t soff) {
  return __builtin_bit_cast(bf16x8,
                            __builtin_amdgcn_raw_buffer_load_b128(r, (int)voff, (int)soff, 0));
}

// 16 bytes per lane from a buffer straight into LDS: lane l's bytes land at
// lds + 16 l (lds: uniform over the wavefront).  Counted by vmcnt like any
// buffer load; the compiler does not track these writes, so every reader
// waits for them explicitly (wait_vm, then a barrier).
__device__ __forceinline__ void load_lds(rsrc_t r, void *lds, uint32_t voff, uint32_t soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)lds, 16, voff, soff, 0, 0);
}

// Wait until at most N vector-memory operations of this wavefront are in
// flight (they complete in issue order).
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt field");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ void wg_barrier() { asm volatile("s_barrier" ::: "memory"); }

// f with the tile count nt (1 .. NT) as a compile-time value
template <int NT, typename Fn>
__device__ __forceinline__ void sp_tiles(int nt, Fn f) {
  if constexpr (NT > 1) {
    if (nt < NT) return sp_tiles<NT - 1>(nt, f);
  }
  f(std::integral_constant<int, NT>{});
}

}  // namespace basek
