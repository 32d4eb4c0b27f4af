// Loads from memory straight into LDS (gfx950).
#pragma once
#include "rl_common.h"

// Buffer descriptor of `bytes` bytes at p in scalar registers (p and bytes are the same in every lane).
__device__ __forceinline__ u32x4 buffer_rsrc(const void* p, unsigned bytes) {
  const uint64_t a = (uint64_t)p;
  u32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((unsigned)a);
  r[1] = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32) & 0xffffu);
  r[2] = __builtin_amdgcn_readfirstlane(bytes);
  r[3] = 0x00027000u;
  return r;
}
// One load of 16 bytes per lane straight into LDS (lane l's piece at lds + 16 l).  Inline assembly: after
// the builtin the compiler waits for all such loads before any LDS read.  Whoever uses it waits with an
// explicit vmcnt (the loads return in order), puts a barrier before other waves read, and drains all of
// them before the workgroup ends.  Pieces whose offset lies behind the buffer's end arrive as zeros.
// The compiler counts no wait states for the instructions in here: the scalar operands come from scalar
// arithmetic (one that a vector instruction wrote would have to be five wait states old).
template <bool NT = false>     // past the caches
__device__ __forceinline__ void load_to_lds(unsigned lds, int voff, u32x4 rsrc, unsigned soff) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds" ::"s"(lds), "v"(voff), "s"(rsrc),
               "s"(soff)
               : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc),
               "s"(soff)
               : "memory", "m0");
}
// Scalars that vector instructions wrote have to be five wait states old when the loads above read them.  The wait takes them as its operand:
// one that only stood between them in the source could be moved ahead of them.
__device__ __forceinline__ void settle(u32x4& rsrc) { asm volatile("s_nop 4" : "+s"(rsrc)); }
// The same with 4 bytes per lane (lane l's at lds + 4 l), whatever wrote the scalars: few of them, so each waits by itself.
__device__ __forceinline__ void load_dword_to_lds(unsigned lds, int voff, u32x4 rsrc, unsigned soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc),
               "s"(soff)
               : "memory", "m0");
}
