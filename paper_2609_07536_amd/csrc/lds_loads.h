// Buffer loads into LDS and the waits for them (gfx950).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// One 16-byte-per-lane buffer -> LDS load: lane L's 16 bytes, at byte
// offset voff of the buffer rsrc describes, land at lds_base + 16 L; an
// offset at or past the buffer's extent reads zeros.  Issued as asm so the
// compiler does not serialise later LDS reads behind it; completion is
// tracked with explicit vmcnt waits.  (Buffer addressing, a 32-bit offset
// per lane against a base in scalar registers, keeps the texture
// addresser's work per load lower than 64-bit global addresses: measured,
// the same ring with global_load_lds_dwordx4 spends up to a third more
// time per stage.)
typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void dma16(i32x4 rsrc, uint32_t voff, uint32_t lds_base) {
  // (the resource is wave-uniform; readfirstlane keeps it in scalar
  // registers also where the compiler cannot prove that)
  i32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(rsrc[i]);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(voff), "s"(r)
               : "memory", "m0");
}

// The same with a further offset that the lanes share, less than the buffer's extent
// (what the range check does with a larger one is not relied on).  Not one function with
// an offset of zero: that took a scalar register and a move in every ring of the bf16
// kernels (up-projection of 16384 tokens, 32 experts of 2048 x 704, top 6: 513 us, and 517).
__device__ __forceinline__ void dma16(i32x4 rsrc, uint32_t voff, uint32_t lds_base, uint32_t soff) {
  i32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(rsrc[i]);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(voff), "s"(r),
                 "s"(__builtin_amdgcn_readfirstlane(soff))
               : "memory", "m0");
}

// ... and to lds_base + kLdsOffset, for unrolled loops: the sum goes straight to
// m0 (as C++ it is hoisted out of the loop, and there are more such sums than
// scalar registers).
template <int kLdsOffset>
__device__ __forceinline__ void dma16_at(i32x4 rsrc, uint32_t voff, uint32_t lds_base, uint32_t soff) {
  i32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(rsrc[i]);
  asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(voff), "s"(r),
                 "s"(__builtin_amdgcn_readfirstlane(soff)), "i"(kLdsOffset)
               : "memory", "m0", "scc");
}

// A raw buffer resource: base address, no stride, `bytes` readable (at most
// 2^31 - 1, so that kOutOfRange is always past it), wave-uniform.
constexpr uint32_t kOutOfRange = 0x80000000u;
__device__ __forceinline__ i32x4 buffer_rsrc(const void* base, long long bytes) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  const long long n = bytes < 0 ? 0 : (bytes > 0x7fffffffLL ? 0x7fffffffLL : bytes);
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)b);
  r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)((b >> 32) & 0xffffu));
  r[2] = __builtin_amdgcn_readfirstlane((int)n);
  r[3] = 0x00020000;   // raw 32-bit data format (gfx9 family)
  return r;
}

template <int N>
__device__ __forceinline__ void waitcnt_vm() {
  // s_waitcnt encoding: vmcnt[3:0] | expcnt[6:4] | lgkmcnt[11:8] | vmcnt_hi[15:14]
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (0 << 8) | ((N >> 4) << 14));
}

__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace
