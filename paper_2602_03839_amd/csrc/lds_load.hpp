// lds_load.hpp -- loads from global memory straight into LDS, as instructions of
// their own: the compiler would make every later transposing LDS read wait for a
// load that it knows of.  They write no register and leave m0 as it was; whoever
// issues them waits for them (s_waitcnt vmcnt) before the LDS is read, and has
// the LDS reads of what lay there done before.
#pragma once

#include "device_common.hpp"

namespace pulse {

// Memory from p on as a buffer: no stride and no bound, since every offset used
// is in the tensor by construction.
__device__ __forceinline__ u32x4_t buffer_at(const void* p) {
  const uint64_t base = (uint64_t)p;
  return u32x4_t{(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, 0xFFFFFFFFu, 0x00027000u};
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}

// 16 bytes a lane, from byte offset `off` of the buffer into 1,024 adjacent bytes.
// STREAM: read once, so not kept in the caches.
template <bool STREAM>
__device__ __forceinline__ void load_to_lds(char* lds, uint32_t off, u32x4_t buffer) {
  uint32_t m0;
  if constexpr (STREAM)
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
        "buffer_load_dwordx4 %2, %3, 0 offen nt lds\n\ts_mov_b32 m0, %0"
        : "=&s"(m0)
        : "s"(lds_address(lds)), "v"(off), "s"(buffer));
  else
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
        "buffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
        : "=&s"(m0)
        : "s"(lds_address(lds)), "v"(off), "s"(buffer));
}

// 4 bytes a lane into 256 adjacent bytes.
__device__ __forceinline__ void load4_to_lds(char* lds, uint32_t off, u32x4_t buffer) {
  uint32_t m0;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
      "buffer_load_dword %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
      : "=&s"(m0)
      : "s"(lds_address(lds)), "v"(off), "s"(buffer));
}

}  // namespace pulse
