// Pieces shared by the tiled GEMMs: the order of tiles over the XCDs, copies to
// LDS and the waits for them, and the LDS-staged epilogue.
#pragma once

#include "common.h"
#include "kernels.h"

namespace dit {
namespace {

__device__ __forceinline__ int xcd_remap(int bid, int n) {
  const int x = bid & 7, idx = bid >> 3;
  const int q = n >> 3, r = n & 7;
  return x * q + (x < r ? x : r) + idx;
}

typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(1))) void glb_void_t;

// s_waitcnt with only the vector-memory counter constrained (gfx9 encoding:
// vmcnt[3:0] | expcnt[6:4] = 7 | lgkmcnt[11:8] = 15 | vmcnt[5:4] at [15:14]).
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// vmcnt(N) and lgkmcnt(0) in one wait (same encoding as wait_vmcnt).
template <int N>
__device__ __forceinline__ void wait_vmcnt_lgkm0() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | ((N >> 4) << 14));
}

// Workgroup barrier without the workgroup-scope fence of __syncthreads: that
// fence waits for every outstanding global load of the wave, copies to LDS
// included, which would drain the copies a deeper pipeline keeps in flight.
// The memory clobber keeps the compiler from moving memory operations across
// it; callers wait for their own LDS reads and copies first.
__device__ __forceinline__ void barrier_no_fence() { asm volatile("s_barrier" ::: "memory"); }

// 16 bytes per lane from base + voff + soff (bytes, 32-bit offsets) into LDS
// at dst + 16 lane: a raw buffer load with an LDS destination.  Offsets past
// 4 GiB - 1 read zeros; the host admits this path only when every row of
// the operand lies below that bound.
__device__ __forceinline__ void buf_lds16(const void* base, lds_void_t* dst, uint32_t voff, uint32_t soff) {
#if defined(__HIP_DEVICE_COMPILE__)
  const __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, (int)0xffffffffu, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, voff, soff, 0, 0);
#endif
}

// LDS-staged epilogue for waves that own 128 output columns (WN == 128).
// Per 32-row slab: the raw f32 accumulators go to this wave's 16 KB of LDS
// (columns XOR 32 on rows with bit 2 set, so the two lane halves of a write
// hit different banks); then lane l handles rows l/16 + 4p (p = 0..7) and
// columns 4(l%16) + [0,4) and 64 + 4(l%16) + [0,4): bias, per-head RMS (a
// head is the 16 lanes of one row: 4 shuffles), GELU / SiLU, gated
// residual, and 8-byte stores that coalesce to 128 bytes per row.
// Requires N % 8 == 0, gelu_from and gap_at multiples of 4.
// KIND selects a specialised body: EPI_K_STORE (bf16 store; the per-head RMS
// norm, GELU and column gap each apply to whole 128-column groups, so they
// are wave-uniform), EPI_K_GATED (gated residual only), EPI_K_ANY (every
// flag, per column).
// EPI_K_FP8 (each lane row's 128 columns quantised to e4m3 with their own
// power-of-two scale; norm and GELU as in EPI_K_STORE).  ROWS: rows of a slab.
enum { EPI_K_STORE = 0, EPI_K_GATED = 1, EPI_K_ANY = 2, EPI_K_FP8 = 3 };
template <int KIND, typename Prob>
struct EpiLdsT {
  const Prob& P;
  int m_base, ncol0, cq, rq, lrow, lhalf;
  bool f32out, gated, silu, rms, gelu_u;
  float bv[2][4], gv[2][4];
  int col[2];
  bool ok[2], gl[2];
  float* slab;

  __device__ __forceinline__ EpiLdsT(const Prob& P_, int m_base_, int ncol0_, int lrow_, int lhalf_, float* slab_)
      : P(P_), m_base(m_base_), ncol0(ncol0_), lrow(lrow_), lhalf(lhalf_), slab(slab_) {}

  // Flags, column map, bias and gate values of this lane's 8 columns.
  __device__ __forceinline__ void prep() {
    const int lane = lhalf * 32 + lrow;
    cq = lane & 15;
    rq = lane >> 4;
    f32out = KIND == EPI_K_ANY && (P.flags & DIT_EPI_F32);
    gated = KIND == EPI_K_GATED || (KIND == EPI_K_ANY && (P.flags & DIT_EPI_GATED_RES));
    silu = (KIND == EPI_K_ANY || KIND == EPI_K_FP8) && (P.flags & DIT_EPI_SILU);
    rms = KIND != EPI_K_GATED && ncol0 < P.rms_cols;
    gelu_u = (KIND == EPI_K_STORE || KIND == EPI_K_FP8) && ncol0 >= P.gelu_from;
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int n = ncol0 + 64 * hh + 4 * cq;
      ok[hh] = n < P.N;
      gl[hh] = n >= P.gelu_from;
      col[hh] = n + (n >= P.gap_at ? P.gap : 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bv[hh][e] = (P.bias && ok[hh]) ? bf16_to_f32(P.bias[n + e]) : 0.f;
        gv[hh][e] = (gated && ok[hh]) ? P.gate[n + e] : 0.f;
      }
    }
  }

  // Residual values C[m][col .. col+3] of slab i (gated epilogue), loaded
  // before any slab is staged so their latency overlaps the staging.
  __device__ __forceinline__ void load_old(int i, uint2 (&old)[8][2]) const {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int m = min(m_base + i * 32 + rq + 4 * p, P.M - 1);
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
        old[p][hh] = ok[hh] ? *(const uint2*)((const bf16_t*)P.C + (int64_t)m * P.ldc + col[hh]) : make_uint2(0, 0);
    }
  }

  // One 32-row slab: accumulators -> LDS -> 8-column row segments -> global.
  // Nothing waits on global memory here: a wave's LDS operations complete in
  // order, so neither the read-back nor the next slab's writes need more
  // than the wait for this wave's own slab writes.
  __device__ __forceinline__ void slab_pass(const f32x16_t (&a)[4], int i, const uint2 (&old)[8][2]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = 8 * (r >> 2) + 4 * lhalf + (r & 3);
        const int c = (j * 32 + lrow) ^ (((row >> 2) & 1) << 5);
        slab[row * 128 + c] = a[j][r];
      }
    slab_rows<1, 5>(i, old);
  }

  // The same for 16 x 16 blocks (a: rows 0..15, b: rows 16..31): lane (lr, lq)
  // holds column lr and rows 4 lq .. 4 lq + 3 of each; columns XOR 16 ((row >> 2) & 3)
  // send the four lane quarters of a write to different banks.
  __device__ __forceinline__ void slab_pass16(const f32x4_t (&a)[8], const f32x4_t (&b)[8], int i,
                                              const uint2 (&old)[8][2], int lr, int lq) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int c = (16 * j + lr) ^ (lq << 4);
        slab[(4 * lq + r) * 128 + c] = a[j][r];
        slab[(16 + 4 * lq + r) * 128 + c] = b[j][r];
      }
    slab_rows<3, 4>(i, old);
  }

  // Reads the staged slab back as 8-column row segments (columns XOR
  // ((row >> 2) & MASK) << SH), applies the epilogue and stores.
  template <int MASK, int SH, int ROWS = 32>
  __device__ __forceinline__ void slab_rows(int i, const uint2 (&old)[8][2]) {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0) only
#pragma unroll
    for (int p = 0; p < ROWS / 4; ++p) {
      const int row = rq + 4 * p;
      const int sw = ((row >> 2) & MASK) << SH;
      float v[2][4];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const float4 t = *(const float4*)(slab + row * 128 + ((64 * hh + 4 * cq) ^ sw));
        v[hh][0] = t.x + bv[hh][0]; v[hh][1] = t.y + bv[hh][1];
        v[hh][2] = t.z + bv[hh][2]; v[hh][3] = t.w + bv[hh][3];
      }
      if (KIND != EPI_K_GATED && rms) {
        float ss = 0.f;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int e = 0; e < 4; ++e) ss += v[hh][e] * v[hh][e];
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) ss += __shfl_xor(ss, o, 64);
        const float sc = rsqrtf(ss * (1.f / 128.f) + DIT_RMS_EPS);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[hh][e] *= sc;
      }
      const int m = m_base + i * 32 + row;
      if constexpr (KIND == EPI_K_STORE) {
        if (gelu_u)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[hh][e] = gelu_tanh_f(v[hh][e]);
        if (m < P.M)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
            if (ok[hh])
              *(uint2*)((bf16_t*)P.C + (int64_t)m * P.ldc + col[hh]) =
                  make_uint2(pack_bf16x2(v[hh][0], v[hh][1]), pack_bf16x2(v[hh][2], v[hh][3]));
        continue;
      } else if constexpr (KIND == EPI_K_GATED) {
        if (m < P.M)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
            if (ok[hh]) {
              const uint2 o = old[p][hh];
              const float y0 = __uint_as_float(o.x << 16) + gv[hh][0] * v[hh][0];
              const float y1 = __uint_as_float(o.x & 0xffff0000u) + gv[hh][1] * v[hh][1];
              const float y2 = __uint_as_float(o.y << 16) + gv[hh][2] * v[hh][2];
              const float y3 = __uint_as_float(o.y & 0xffff0000u) + gv[hh][3] * v[hh][3];
              *(uint2*)((bf16_t*)P.C + (int64_t)m * P.ldc + col[hh]) =
                  make_uint2(pack_bf16x2(y0, y1), pack_bf16x2(y2, y3));
            }
        continue;
      } else if constexpr (KIND == EPI_K_FP8) {
        // (the flags are wave-uniform: one branch each, not one per value)
        if (gelu_u) {
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[hh][e] = gelu_tanh_f(v[hh][e]);
        }
        if (silu) {
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[hh][e] = silu_f(v[hh][e]);
        }
        uint32_t top = 0;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(v[hh][e]) & 0x7fffffffu);
        top = max_over<16>(top);
        const uint32_t byte = e8m0_of(top);
        const float inv = e8m0_inverse(byte);
        if (m < P.M && ncol0 < P.N) {
          uint8_t* c = (uint8_t*)P.C + (int64_t)m * P.ldc + ncol0 + 4 * cq;
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
            *(uint32_t*)(c + 64 * hh) = pack_fp8x4(v[hh][0] * inv, v[hh][1] * inv, v[hh][2] * inv, v[hh][3] * inv);
          if (cq == 0) P.Cs[(int64_t)m * P.ldcs + (ncol0 >> 7)] = (uint8_t)byte;
        }
        continue;
      }
      if (m < P.M) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          if (!ok[hh]) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (gl[hh]) v[hh][e] = gelu_tanh_f(v[hh][e]);
            if (silu) v[hh][e] = silu_f(v[hh][e]);
          }
          if (f32out) {
            *(float4*)((float*)P.C + (int64_t)m * P.ldc + col[hh]) =
                make_float4(v[hh][0], v[hh][1], v[hh][2], v[hh][3]);
          } else {
            bf16_t* c = (bf16_t*)P.C + (int64_t)m * P.ldc + col[hh];
            if (gated) {
              const uint2 o = old[p][hh];
              v[hh][0] = __uint_as_float(o.x << 16) + gv[hh][0] * v[hh][0];
              v[hh][1] = __uint_as_float(o.x & 0xffff0000u) + gv[hh][1] * v[hh][1];
              v[hh][2] = __uint_as_float(o.y << 16) + gv[hh][2] * v[hh][2];
              v[hh][3] = __uint_as_float(o.y & 0xffff0000u) + gv[hh][3] * v[hh][3];
            }
            *(uint2*)c = make_uint2(pack_bf16x2(v[hh][0], v[hh][1]), pack_bf16x2(v[hh][2], v[hh][3]));
          }
        }
      }
    }
  }
};

}  // namespace
}  // namespace dit
