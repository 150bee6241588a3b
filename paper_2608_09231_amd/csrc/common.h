// Shared device helpers of the gfx950 kernels: bf16 bit handling, vector
// types for the MFMA builtins, wave reductions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

typedef uint16_t bf16_t;  // raw bfloat16 bit pattern in memory

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_to_f32(bf16_t b) {
  return __uint_as_float(((uint32_t)b) << 16);
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// Round to nearest, ties to even (hardware v_cvt_pk_bf16_f32).
__device__ __forceinline__ bf16_t f32_to_bf16(float f) {
  return __builtin_bit_cast(bf16_t, (__bf16)f);
}

// Two floats -> packed bf16 pair (lo in bits 0..15), one conversion instruction.
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  bf16x2_t v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

// Storage-type traits: load to f32 / round-and-store from f32.
template <typename T> struct St;
template <> struct St<float> {
  static __device__ __forceinline__ float ld(const float* p) { return *p; }
  static __device__ __forceinline__ float rd(float v) { return v; }
  static __device__ __forceinline__ void st(float* p, float v) { *p = v; }
};
template <> struct St<bf16_t> {
  static __device__ __forceinline__ float ld(const bf16_t* p) { return bf16_to_f32(*p); }
  static __device__ __forceinline__ float rd(float v) { return bf16_to_f32(f32_to_bf16(v)); }
  static __device__ __forceinline__ void st(bf16_t* p, float v) { *p = f32_to_bf16(v); }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

__device__ __forceinline__ double warp_sum_d(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Block-wide sum for blockDim.x = 64 * nwaves; `red` holds >= nwaves floats.
template <int NW>
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = warp_sum(v);
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  __syncthreads();
  if (l == 0) red[w] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) s += red[i];
  return s;
}

// GELU, tanh form: 0.5 x (1 + tanh(u)) = x * sigmoid(2u), u = sqrt(2/pi)(x + 0.044715 x^3).
// The sigmoid form has no cancellation for large negative x.  exp via the
// hardware base-2 exponential and a hardware reciprocal (about 1 ulp each,
// far below the bf16 rounding of the stored result).
__device__ __forceinline__ float gelu_tanh_f(float x) {
  const float k0 = 0.7978845608028654f * -2.f * 1.4426950408889634f;  // -2 sqrt(2/pi) log2(e)
  const float e = __builtin_amdgcn_exp2f(k0 * (x + 0.044715f * x * x * x));
  return x * __builtin_amdgcn_rcpf(1.f + e);
}

__device__ __forceinline__ float silu_f(float x) {
  return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x));
}

// ---- row-streaming helpers shared by the fused streaming kernels ----

__device__ __forceinline__ void unpack8(const uint4& u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                    pack_bf16x2(v[6], v[7]));
}

// Streamed tensors (read or written once per step) bypass L2 retention so the
// embedding and projection weights, re-read by every workgroup, stay cached.
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 ld_stream(const bf16_t* p) {
  const u32x4_t v = __builtin_nontemporal_load((const u32x4_t*)p);
  return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void st_stream(bf16_t* p, uint4 v) {
  const u32x4_t w = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(w, (u32x4_t*)p);
}

__device__ __forceinline__ void load_f8(const float* p, float (&m)[8]) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  m[0] = a.x; m[1] = a.y; m[2] = a.z; m[3] = a.w; m[4] = b.x; m[5] = b.y; m[6] = b.z; m[7] = b.w;
}

// Workgroup barrier after this wave's LDS operations have completed, without
// the workgroup-scope fence of __syncthreads (which would also wait for every
// outstanding global load of the wave).  The memory clobber keeps the
// compiler from moving memory operations across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  asm volatile("s_barrier" ::: "memory");
}

// Largest of v over the 8 or 16 neighbouring lanes of a lane, on the VALU (data
// parallel primitives: pairs, quads, halves of 8, 16).
template <int LANES>
__device__ __forceinline__ uint32_t max_over(uint32_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  static_assert(LANES == 8 || LANES == 16, "lanes");
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));   // lane ^ 1
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));   // lane ^ 2
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));  // 7 - lane, of 8
  if (LANES == 16) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));  // 15 - lane
#endif
  return v;
}

// ---- 8-bit floating point (e4m3) with power-of-two scales (E8M0 bytes) ----

// Scale byte of values whose largest magnitude has the bits `top` (compared as
// integers, so that a NaN stays the largest): the least e >= -127 with
// top <= 448 * 2^e, plus 127; 255 where the largest is not finite.  448 =
// 1.75 * 2^8: adding 0x1fffff to the bits carries into the exponent exactly
// for mantissas above 1.75.
__device__ __forceinline__ uint32_t e8m0_of(uint32_t top) {
  const int e = (int)((top + 0x1fffffu) >> 23) - 8;
  return top >= 0x7f800000u ? 255u : (uint32_t)(e < 0 ? 0 : e);
}
// 1 / 2^(byte - 127), exact; NaN for 255, which turns the whole block into NaNs.
__device__ __forceinline__ float e8m0_inverse(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float((254u - byte) << 23);
}
// Four floats of magnitude <= 448 (or NaN) to e4m3, round to nearest even.
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
#else
  return 0;
#endif
}

#define DIT_LN_EPS 1e-6f
#define DIT_RMS_EPS 1e-6f
