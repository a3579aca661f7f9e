// Device helpers of the differential-attention kernels, which copy tiles into LDS and feed them to the matrix cores. attn_fwd.hip
// holds the same helpers: its counter profiles are keyed to the source of that one file.
#pragma once

#include "common.h"

// s_waitcnt with only the vector-memory counter constrained (gfx9 encoding)
#define WA_WAIT_VM(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (7 << 4) | (15 << 8) | (((n) >> 4) << 14))
// workgroup barrier after this wavefront's LDS reads have completed; the compiler may not move
// memory accesses across it
#define WA_BARRIER() asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory")

// Scheduling fence: no instruction moves across it. Placed between the operand reads of k-step s+1
// and the MFMAs of k-step s, it keeps those reads in flight while the MFMAs run (left alone, the
// scheduler sinks every read to just before its MFMA, and each MFMA then waits out an LDS latency).
#define WA_SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)

namespace wa {

typedef __attribute__((address_space(3))) void lds_void_t;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// two floats -> two bf16 (round to nearest even; one v_cvt_pk_bf16_f32 on gfx950)
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

// One 16-byte-per-lane copy from global memory (uniform base + per-lane byte offset) into LDS at the
// uniform address lds (lane i writes lds + 16 i). Written as inline assembly so that only the
// explicit vmcnt waits of the pipeline order it against LDS reads of the other tile; M0 (the LDS
// base of the copy), which a copy may read one wait state after it is written, is restored afterwards.
__device__ __forceinline__ void dma16(const void* gbase, uint32_t voff, const unsigned char* lds) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)lds);
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %3\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(m0), "v"(voff), "s"(gbase)
      : "memory");
}

}  // namespace wa
