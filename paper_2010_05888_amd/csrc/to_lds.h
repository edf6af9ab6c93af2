// Loads from memory straight to LDS, waited for by count. The compiler's own
// loads of this kind make it wait for all of them before any read of LDS that it
// cannot tell apart from them; these it does not know, so a kernel says itself
// what it waits for: wait_for(n) ends when at most the wave's n latest loads are
// outstanding (loads end in order).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "block8.h"

namespace garfield {

// The compiler does not look into them either for what must lie between two
// instructions: a scalar register that a vector instruction has written (a buffer's,
// say) may be read by a load five wait states later at the earliest, and m0 one after
// it is set. s_mov and s_nop 3 before every load are five.

typedef __attribute__((address_space(3))) void* LocalPtr;

__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((LocalPtr)(p)));
}

// `bytes` bytes from p on; reads beyond them give 0.
__device__ __forceinline__ u4 buffer_of(const void* p, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  u4 r;
  r.x = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a));
  r.y = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32) & 0xffffu);
  r.z = __builtin_amdgcn_readfirstlane(bytes);
  r.w = 0x00020000u;
  return r;
}

// 16 bytes a lane, from the lane's offset in the buffer to LDS at to + 16 * lane.
// `to` is the wave's.
__device__ __forceinline__ void load_to_lds16(u4 buffer, uint32_t from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from), "s"(buffer)
               : "memory");
}

// 16 and 4 bytes a lane from the lane's address.
__device__ __forceinline__ void load_to_lds16(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
               : "memory");
}

__device__ __forceinline__ void load_to_lds4(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
               : "memory");
}

// One byte a lane, to the low byte of a word of LDS at to + 4 * lane (the others 0).
__device__ __forceinline__ void load_to_lds1(u4 buffer, uint32_t from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_ubyte %1, %2, 0 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from), "s"(buffer)
               : "memory");
}

template <int N>
__device__ __forceinline__ void wait_for() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

__device__ __forceinline__ void wait_for_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
}

// A barrier that waits for none of the wave's accesses.
__device__ __forceinline__ void barrier_alone() { asm volatile("s_barrier" : : : "memory"); }

// A barrier that waits for the wave's LDS accesses and for none of its loads.
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

// Between accesses to LDS by which the lanes of one wave give each other values: what any of them
// did before is done for all of them after. The hardware keeps a wave's accesses in order, so
// this is no instruction; it keeps the compiler from putting them in another order.
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

}  // namespace garfield
