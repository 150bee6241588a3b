// Pieces shared by the attention kernels that read tiles by key rows: copies to LDS that the
// compiler does not see, transposed fragments of them, a three-way maximum.
#pragma once

#include "common.h"

namespace dit {
namespace {

// 16 bytes per lane from base + off (valid up to `bytes`; zeros past it) to LDS at
// dst + 16 lane, as an instruction that the compiler does not see through: it
// would have every transposing read of LDS wait for all copies in flight.  The
// kernel's own waits and barriers order them.  (No registers come back; the
// address escapes, so that the barriers' memory clobbers cover what is written.  m0 is
// a reserved register, set before each use: clang warns against it among the clobbers.)
__device__ __forceinline__ void copy16_unseen(const void* base, uint32_t bytes, const void* dst, uint32_t off) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const uint64_t b = (uint64_t)base;  // (wave-uniform, also where the compiler holds it in vector registers)
  const u32x4 r = {(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b),
                   (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) & 0xffffu,
                   (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
  const uint32_t l = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)dst;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(l), "v"(off), "s"(r));
#endif
}

// Largest of three in one instruction (a NaN gives way to a number, as with fmaxf,
// which the compiler makes of several to quiet signalling NaNs first).
__device__ __forceinline__ float max3(float a, float b, float c) {
#if defined(__HIP_DEVICE_COMPILE__)
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
#else
  return fmaxf(fmaxf(a, b), c);
#endif
}

// Transposed V fragment from LDS: four keys from p and four from 16 rows further down.
__device__ __forceinline__ bf16x8_t vt_frag(const char* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
  const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p));
  const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 16 * 256)));
  return __builtin_bit_cast(bf16x8_t, make_uint4(lo.x, lo.y, hi.x, hi.y));
#else
  return bf16x8_t{};
#endif
}

}  // namespace
}  // namespace dit
