// 4-bit floating point: rows quantised to e2m1 with one power-of-two scale (an
// E8M0 byte) per 32 values, back from them, and the product of two such matrices,
//   C = epi(sum over blocks b of K: 2^(sa[m,b] + sw[n,b] - 254) sum over k in b: a[m,k] w[n,k], + bias).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes four blocks of 32 per instruction, each
// lane the 32 values of one row's block with a scale byte of its own.  Products of two e2m1 values are
// multiples of 1/4 up to 36: 32 of them add up exactly, and blocks enter the f32 sum
// without loss where their scales lie within 2^8 of each other (measured: no bit off; 1e-7
// in the 2-norm for scales spread over 2^30).  So bf16, f32 and 4-bit outputs all come from it.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "gemm_tile.h"
#include "kernels.h"

namespace dit {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

struct Fp4Prob {
  const uint8_t* A; int64_t lda;
  const uint8_t* W; int64_t ldw;
  const uint8_t* As; int64_t ldas;
  const uint8_t* Ws; int64_t ldws;
  const bf16_t* bias;
  void* C; int64_t ldc;
  uint8_t* Cs; int64_t ldcs;
  const float* gate;
  int M, N, K;
  int flags, rms_cols, gelu_from, gap_at, gap;
  int tiles_m, tiles_n;
};

// ---------------------------------------------------------------- 4-bit rows

// Scale byte of values whose largest magnitude has the bits `top` (compared as
// integers, so that a NaN stays the largest): the least e >= -127 with top <= 6 *
// 2^e, plus 127; 255 where the largest is not finite.  6 = 1.5 * 2^2: adding
// 0x3fffff to the bits carries into the exponent exactly for mantissas above 1.5.
__device__ __forceinline__ uint32_t scale4_of(uint32_t top) {
  const int e = (int)((top + 0x3fffffu) >> 23) - 2;
  return top >= 0x7f800000u ? 255u : (uint32_t)(e < 0 ? 0 : e);
}

// Eight floats of magnitude <= 6 to e2m1, round to nearest even, the first lowest.
__device__ __forceinline__ uint32_t pack_fp4x8(const float (&v)[8]) {
#if defined(__HIP_DEVICE_COMPILE__)
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], 1.f, 3);
#else
  return 0;
#endif
}

// Largest of v over a lane and its neighbours of 2 or 4.
template <int LANES>
__device__ __forceinline__ uint32_t max_near(uint32_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  static_assert(LANES == 2 || LANES == 4, "lanes");
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));              // lane ^ 1
  if (LANES == 4) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));  // lane ^ 2
#endif
  return v;
}

// Two lanes per block of 32, 16 values each; a wave takes 1024 values of a row.
// One pass, bound by memory: 32760 x 5120 bf16 (424 MB) 73 us, 5.8 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void quant_fp4_kernel(const T* __restrict__ x, int64_t ldx, uint8_t* __restrict__ q,
                                                        int64_t ldq, uint8_t* __restrict__ scale, int64_t lds, int M,
                                                        int K, int per_row) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t m = unit / per_row;
  if (m >= M) return;
  const int k = (int)(unit - m * per_row) * 1024 + 16 * lane;
  if (k >= K) return;  // K % 32 == 0: both lanes of a block are inside or not
  float v[16];
  const T* p = x + m * ldx + k;
  if constexpr (sizeof(T) == 2) {
    float a[8], b[8];
    unpack8(*(const uint4*)p, a);
    unpack8(*(const uint4*)(p + 8), b);
#pragma unroll
    for (int i = 0; i < 8; ++i) { v[i] = a[i]; v[8 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 t = *(const float4*)(p + 4 * i);
      v[4 * i] = t.x; v[4 * i + 1] = t.y; v[4 * i + 2] = t.z; v[4 * i + 3] = t.w;
    }
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max_near<2>(top);
  const uint32_t byte = scale4_of(top);
  const float inv = e8m0_inverse(byte);
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo[i] = v[i] * inv; hi[i] = v[8 + i] * inv; }
  *(uint2*)(q + m * ldq + (k >> 1)) = make_uint2(pack_fp4x8(lo), pack_fp4x8(hi));
  if ((lane & 1) == 0) scale[m * lds + (k >> 5)] = (uint8_t)byte;
}

// 16 bytes of values a lane and store, 2048 values of a row a wave with all loads in
// flight.  e2m1 as an f32 number times the scale, both exact.  Bound by memory: 32760 x 5120 to bf16 (424 MB) 72 us,
// 5.9 TB/s (with one load at a time 110).
template <typename T>
__global__ __launch_bounds__(256) void dequant_fp4_kernel(const uint8_t* __restrict__ q, int64_t ldq,
                                                          const uint8_t* __restrict__ scale, int64_t lds,
                                                          T* __restrict__ y, int64_t ldy, int M, int K, int per_row) {
  constexpr int V = 16 / sizeof(T), U = 32 / V;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t m = unit / per_row;
  if (m >= M) return;
  const int k0 = (int)(unit - m * per_row) * 2048 + V * lane;
  uint32_t w[U], byte[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int k = min(k0 + 64 * V * u, K - V);
    const uint8_t* p = q + m * ldq + (k >> 1);
    w[u] = V == 8 ? *(const uint32_t*)p : *(const uint16_t*)p;
    byte[u] = scale[m * lds + (k >> 5)];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int k = k0 + 64 * V * u;
    if (k >= K) return;
    // 2^(byte - 127): subnormal for 0, NaN for 255
    const float s = __uint_as_float(byte[u] == 0 ? 0x00400000u : byte[u] == 255 ? 0x7fc00000u : byte[u] << 23);
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t c = w[u] >> (4 * i);
      // 0, 1/2, then 1.m * 2^(e - 1)
      const uint32_t mag = (c & 7) < 2 ? (c & 1) * 0x3f000000u : 0x3f800000u + (((c & 7) - 2) << 22);
      v[i] = __uint_as_float(mag | (c & 8) << 28) * s;
    }
    uint4 out;
    if constexpr (V == 8) out = pack8(v);
    else out = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    st_stream((bf16_t*)(y + m * ldy + k), out);  // (16 bytes)
  }
}

// ---------------------------------------------------------------- products

// The 128-deep step of one 16 x 16 block: lane (lr, lq) holds row lr's values 32 lq .. + 31
// and, in byte B of sa or sw, their scale.
template <int B = 0>
__device__ __forceinline__ f32x4_t mfma_fp4(const i32x4_t& a, const i32x4_t& w, const f32x4_t& c, int sa, int sw) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i32x8_t x = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  const i32x8_t y = __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, B, sa, B, sw);
#else
  return c;
#endif
}

// The same of a 32 x 32 block and 64 of K: lane (lr, lh) holds row lr's values 32 lh .. + 31.
template <int B>
__device__ __forceinline__ f32x16_t mfma_fp4_32(const i32x4_t& a, const i32x4_t& w, const f32x16_t& c, int sa, int sw) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i32x8_t x = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  const i32x8_t y = __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, B, sa, B, sw);
#else
  return c;
#endif
}

// 16 bytes per lane from base + voff + soff to LDS at dst + 16 lane; lanes with voff
// >= OOB write zeros.  Offsets in bounds lie below OOB: the bases are those of a
// tile's first row, and the host bounds 256 rows of an operand.  An instruction that the compiler does
// not see through: it would have reads of LDS wait for all copies in flight.  The kernels' own waits
// and barriers order them, and scheduling fences keep their place.
constexpr uint32_t OOB = 0x80000000u;
__device__ __forceinline__ void copy16_unseen(const void* base, const void* dst, uint32_t voff, uint32_t soff) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const uint64_t b = (uint64_t)base;
  const u32x4 r = {(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, OOB, 0x00020000u};
  const uint32_t l = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)dst;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(l), "v"(voff), "s"(r),
               "s"(__builtin_amdgcn_readfirstlane(soff)));
#endif
}
// 4 bytes per lane the same way.
__device__ __forceinline__ void copy4_unseen(const void* base, const void* dst, uint32_t voff, uint32_t soff) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const uint64_t b = (uint64_t)base;
  const u32x4 r = {(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, OOB, 0x00020000u};
  const uint32_t l = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)dst;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(l), "v"(voff), "s"(r),
               "s"(__builtin_amdgcn_readfirstlane(soff)));
#endif
}

__device__ __forceinline__ i32x4_t lds_chunk(const char* p) { return *(const i32x4_t*)p; }

// Scale bytes in LDS.  A row has nd dwords of them, one per 128 of K; a group is DW of
// them (DW / 2 slices), 4 DW bytes a row, and the last group begins early enough to lie in
// the row: dword d is at d - start(group).  DW = 8: the halves of a row's 32 bytes change
// places on rows with bit 3 set, so that 16 rows' dwords lie in different banks.
//
// A row's bytes are far from the next row's, so that a request to L2 serves one row: with groups of 16
// bytes they were a third of the kernel's requests.
template <int DW>
struct Scales {
  int nd, blocks;  // dwords of a row, blocks of 32
  __device__ __forceinline__ explicit Scales(int K) : nd((K + 127) >> 7), blocks(K >> 5) {}
  __device__ __forceinline__ int start(int g) const { return g == 0 ? 0 : min(DW * g, nd - DW); }
  // place of dword d of group g
  __device__ __forceinline__ int place(int g, int d) const { return min(d - start(g), DW - 1); }
  // bytes of dword d that belong to blocks, the rest zeros (a NaN there would spoil sums of zeros)
  __device__ __forceinline__ uint32_t valid(int d) const {
    const int n = blocks - 4 * d;
    return n >= 4 ? ~0u : (1u << (8 * max(n, 0))) - 1u;
  }
  static __device__ __forceinline__ int swap(int row) { return DW == 8 ? (row >> 3) & 1 : 0; }
  // group 0 of a row, through registers: its dwords that exist
  __device__ __forceinline__ void first(const uint8_t* p, char* rows, int row) const {
#pragma unroll
    for (int h = 0; h < DW / 4; ++h) {
      i32x4_t x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *(const int*)(p + 4 * min(4 * h + i, nd - 1));
      *(i32x4_t*)(rows + 4 * DW * row + 16 * (h ^ swap(row))) = x;
    }
  }
};

// Origin of tile lt: M-grouped order, eight tile rows per group.
__device__ __forceinline__ void tile_at(const Fp4Prob& P, int lt, int& tm, int& tn) {
  constexpr int GROUP = 8;
  const int in_group = GROUP * P.tiles_n;
  const int gid = lt / in_group;
  const int first_m = gid * GROUP;
  const int gsz = min(P.tiles_m - first_m, GROUP);
  tm = first_m + (lt % in_group) % gsz;
  tn = (lt % in_group) / gsz;
}

// The LDS-staged epilogue for waves that own 128 output columns, and its variant
// that writes 4-bit rows: 8 lanes hold a block's 32 columns, 4 each.
enum { EPI_K_FP4 = 4 };
template <int KIND>
struct Epi : EpiLdsT<KIND == EPI_K_FP4 ? EPI_K_ANY : KIND, Fp4Prob> {
  using Base = EpiLdsT<KIND == EPI_K_FP4 ? EPI_K_ANY : KIND, Fp4Prob>;
  using Base::Base;
  using Base::P;

  template <int MASK, int SH, int ROWS>
  __device__ __forceinline__ void rows(int i, const uint2 (&old)[8][2]) {
    if constexpr (KIND != EPI_K_FP4) {
      Base::template slab_rows<MASK, SH, ROWS>(i, old);
    } else {
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0) only
#pragma unroll
      for (int p = 0; p < ROWS / 4; ++p) {
        const int row = this->rq + 4 * p, cq = this->cq;
        const int sw = ((row >> 2) & MASK) << SH;
        float v[2][4];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const float4 t = *(const float4*)(this->slab + row * 128 + ((64 * hh + 4 * cq) ^ sw));
          v[hh][0] = t.x + this->bv[hh][0]; v[hh][1] = t.y + this->bv[hh][1];
          v[hh][2] = t.z + this->bv[hh][2]; v[hh][3] = t.w + this->bv[hh][3];
        }
        if (this->rms) {
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
        if (this->ncol0 >= P.gelu_from) {  // (a multiple of 128: wave-uniform)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[hh][e] = gelu_tanh_f(v[hh][e]);
        }
        if (this->silu) {
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[hh][e] = silu_f(v[hh][e]);
        }
        const int m = this->m_base + i * 32 + row;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          uint32_t top = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(v[hh][e]) & 0x7fffffffu);
          const uint32_t byte = scale4_of(max_over<8>(top));
          [[maybe_unused]] const float inv = e8m0_inverse(byte);
          const int n = this->ncol0 + 64 * hh + 4 * cq;
          if (m < P.M && n < P.N) {
            uint32_t w = 0;
#if defined(__HIP_DEVICE_COMPILE__)
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[hh][0] * inv, v[hh][1] * inv, 1.f, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[hh][2] * inv, v[hh][3] * inv, 1.f, 1);
#endif
            *(uint16_t*)((uint8_t*)P.C + (int64_t)m * P.ldc + (n >> 1)) = (uint16_t)w;
            if ((cq & 7) == 0) P.Cs[(int64_t)m * P.ldcs + (n >> 5)] = (uint8_t)byte;
          }
        }
      }
    }
  }
};

// 4-bit rows straight from the accumulators of 32 x 32 blocks whose operands changed places:
// lane (lr, lh) holds row 32 i + lr's columns 8 q + 4 lh .. + 3 of block j, so that a
// lane and its other half hold a row's 32 TN columns.  (bf16 rows so stored, 32 bytes at a time, take
// 1 us a tile more than whole lines by way of LDS.)
template <int TM, int TN>
__device__ __forceinline__ void store_fp4(const Fp4Prob& P, f32x16_t (&acc)[TM][TN], int m0, int n0, int lr, int lh) {
#if defined(__HIP_DEVICE_COMPILE__)
  static_assert(TN == 4, "a head's 128 columns, a dword of scales");
  typedef uint32_t half_run __attribute__((ext_vector_type(2), aligned(2)));
  auto other_half = [](uint32_t v) {
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & 32) ? s[0] : s[1];
  };
  if (P.bias) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + 32 * j + 8 * q + 4 * lh;  // (N % 32 == 0)
        const half_run b = *(const half_run*)(P.bias + min(n, P.N - 4));
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < TM; ++i) acc[i][j][4 * q + e] += __uint_as_float(e & 1 ? b[e >> 1] & 0xffff0000u : b[e >> 1] << 16);
      }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = m0 + 32 * i + lr;
    if (n0 < P.rms_cols) {
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) ss += acc[i][j][r] * acc[i][j][r];
      ss += __uint_as_float(other_half(__float_as_uint(ss)));
      const float f = rsqrtf(ss * (1.f / 128.f) + DIT_RMS_EPS);
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] *= f;
    }
    if (n0 >= P.gelu_from) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = gelu_tanh_f(acc[i][j][r]);
    }
    if (P.flags & DIT_EPI_SILU) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = silu_f(acc[i][j][r]);
    }
    uint32_t scales = 0;
    uint8_t* c = (uint8_t*)P.C + (int64_t)m * P.ldc + (n0 >> 1) + 8 * lh;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      uint32_t top = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) top = max(top, __float_as_uint(acc[i][j][r]) & 0x7fffffffu);
      const uint32_t byte = scale4_of(max(top, other_half(top)));
      const float inv = e8m0_inverse(byte);
      scales |= byte << (8 * j);
      uint32_t w[2];  // 16 bits for q = 0, 1 and for 2, 3
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = acc[i][j][8 * h + e] * inv;
        w[h] = pack_fp4x8(v);
      }
      // the lower half takes both halves' first two, the upper one the last two
      const auto s = __builtin_amdgcn_permlane32_swap(w[0], w[1], false, false);
      if (m < P.M && n0 + 32 * j < P.N)
        *(uint2*)(c + 16 * j) = make_uint2((s[0] & 0xffffu) | s[1] << 16, s[0] >> 16 | (s[1] & 0xffff0000u));
    }
    if (m < P.M && lh == 0) {
      uint8_t* cs = P.Cs + (int64_t)m * P.ldcs + (n0 >> 5);
      if (n0 + 128 <= P.N) {
        *(uint32_t*)cs = scales;
      } else {
#pragma unroll
        for (int j = 0; j < TN; ++j)
          if (n0 + 32 * j < P.N) cs[j] = (uint8_t)(scales >> (8 * j));
      }
    }
  }
#endif
}

// 256 x 256 tiles, 8 waves of 64 x 128.  LDS: two slices of 256 of K each of W and A
// (32 KB, 16-byte chunks of a 128-byte row XOR-swizzled by ((row >> 1) & 7)) and two groups of
// both's scales.  32x32x64 MFMAs: a slice is four substeps of eight, and a
// substep's six fragments are read under the MFMAs of the one before it.
//
// The waves meet after substep 2, whose reads were the last of their slice: slice kt +
// 1 has landed, and slice kt's places take slice kt + 2 during substep 3.  Slices past the
// last one are copied as zeros (no memory traffic), which keeps every iteration alike.
//
// 32760 x 5120 x 13824 1.04 ms, 4.4 PFLOP/s; 32760 x 13824 x 5120 1.25 ms, with 4-bit rows out 1.05, with GELU, too, 1.16.
// What bounds it is power (the clock falls to 1.85 - 1.94 GHz, MFMAs busy 0.53 - 0.57 there) and the way through LDS (0.42, and 0.15
// in conflicts of the scale reads, 2.5 % of the time): of 1.08 ms the loop takes 0.93 without copies, 1.1 without
// fragment reads, 0.87 without both.  A tile's beginning and end take 5 us, 10 with bf16 rows out
// (3 more where the first products waited for both slices and the scales came by way of registers),
// which only another work-group on the CU could hide, and LDS has no room for it.
template <int KIND>
__global__ __launch_bounds__(512) void gemm_fp4_ring_kernel(Fp4Prob P) {
  constexpr int UNIT = 256 * 128, INS = 4, TM = 2, TN = 4, SC = 4 * UNIT, GROUP = 512 * 32;
  __shared__ __attribute__((aligned(1024))) char smem[SC + 2 * GROUP];
  int tm, tn;
  tile_at(P, xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n), tm, tn);
  const int m0 = tm * 256, n0 = tn * 256;
  const int nk = (P.K + 255) >> 8;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int lr = lane & 31, lh = lane >> 5;

  // copy j of this wave moves rows 8 (4 wave + j) .. + 7 of an operand's slice
  const uint8_t* Ab = P.A + (int64_t)m0 * P.lda;
  const uint8_t* Wb = P.W + (int64_t)n0 * P.ldw;
  const int c0 = (lane & 7) ^ (lane >> 4);  // chunk of even copies; odd ones: c0 ^ 4
  uint32_t aoff[INS], woff[INS];
#pragma unroll
  for (int j = 0; j < INS; ++j) {
    const int row = 8 * (wave * INS + j) + (lane >> 3);
    aoff[j] = (uint32_t)min(row, P.M - 1 - m0) * (uint32_t)P.lda + 16 * (c0 ^ (4 * (j & 1)));
    woff[j] = (uint32_t)min(row, P.N - 1 - n0) * (uint32_t)P.ldw + 16 * (c0 ^ (4 * (j & 1)));
  }
  auto issue1 = [&](const uint8_t* base, const uint32_t (&off)[INS], int u, int s, int j) {
    copy16_unseen(base, smem + u + (wave * INS + j) * 1024,
                  16 * (c0 ^ (4 * (j & 1))) < (P.K >> 1) - 128 * s ? off[j] : OOB, (uint32_t)s * 128);
  };
  // scales: waves 0 .. 3 rows of A, 4 .. 7 rows of W, 64 each, two lanes a row
  const Scales<8> sc(P.K);
  const uint8_t* sbase = wave < 4 ? P.As + (int64_t)m0 * P.ldas : P.Ws + (int64_t)n0 * P.ldws;
  auto scale_row = [&](int row) {  // of the work-group's 512
    return wave < 4 ? (uint32_t)min(row, P.M - 1 - m0) * (uint32_t)P.ldas
                    : (uint32_t)min(row - 256, P.N - 1 - n0) * (uint32_t)P.ldws;
  };
  uint32_t soff[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = 64 * wave + 32 * j + (lane >> 1);
    soff[j] = scale_row(row) + 16 * ((lane & 1) ^ sc.swap(row));
  }
  // (no branches between MFMAs: the compiler would sink products behind them, past the
  // barriers; a group past the last one is zeros)
  auto issue_scales = [&](int g) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      copy16_unseen(sbase, smem + SC + (g & 1) * GROUP + wave * 2048 + j * 1024, 8 * g < sc.nd ? soff[j] : OOB,
                    4 * max(sc.start(g), 0));
  };
  const int srow = SC + 32 * (64 * wm + lr), wrow = SC + 32 * (256 + 128 * wn + lr), sswap = 16 * sc.swap(lr);
  // scales of a half slice: of the substeps 0 and 1, and of 2 and 3
  struct Half { uint32_t a[TM], w[TN]; };
  auto read_scales = [&](Half& x, int d) {  // dword d of K (past the last one: any)
    const int g = d >> 3, at = ((g & 1) * GROUP + 4 * sc.place(g, d)) ^ sswap;
#pragma unroll
    for (int i = 0; i < TM; ++i) x.a[i] = *(const uint32_t*)(smem + srow + at + 1024 * i);
#pragma unroll
    for (int j = 0; j < TN; ++j) x.w[j] = *(const uint32_t*)(smem + wrow + at + 1024 * j);
  };
  auto place_scales = [&](Half& x, int d) {  // this lane's block of each substep into bytes 0 and 2
    const uint32_t v = sc.valid(d);
#pragma unroll
    for (int i = 0; i < TM; ++i) x.a[i] = (x.a[i] & v) >> (8 * lh);
#pragma unroll
    for (int j = 0; j < TN; ++j) x.w[j] = (x.w[j] & v) >> (8 * lh);
  };

  // this lane's chunk inside 32 rows of a unit: half lh of substep s
  int loff[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) loff[s] = lr * 128 + (((2 * s + lh) ^ ((lr >> 1) & 7)) << 4);
  const int wa = wm * 64 * 128, ww = wn * 128 * 128;
  f32x16_t acc[TM][TN] = {};
  // A substep's MFMAs, and between them one by one the fragment reads of the next
  // substep (s of the slice in units uw, ua) in the order of their use and a copy.
  // The fences keep that order.
  auto substep = [&](const i32x4_t(&a)[TM], const i32x4_t(&w)[TN], i32x4_t(&an)[TM], i32x4_t(&wn2)[TN], int uw, int ua,
                     int s, const Half& x, auto b_, auto copy) {
    constexpr int B = decltype(b_)::value;
#pragma unroll
    for (int q = 0; q < TM * TN; ++q) {
      const int i = q & 1, j = q >> 1;
      if constexpr (KIND == EPI_K_FP4) acc[i][j] = mfma_fp4_32<B>(w[j], a[i], acc[i][j], x.w[j], x.a[i]);
      else acc[i][j] = mfma_fp4_32<B>(a[i], w[j], acc[i][j], x.a[i], x.w[j]);
      __builtin_amdgcn_sched_barrier(0);
      if (q == 0 || q == 2) an[q >> 1] = lds_chunk(smem + ua + wa + (q >> 1) * 4096 + loff[s]);
      else if (q < 6) wn2[q == 1 ? 0 : q - 2] = lds_chunk(smem + uw + ww + (q == 1 ? 0 : q - 2) * 4096 + loff[s]);
      copy(q);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto none = [](int) {};
  using std::integral_constant;
  const integral_constant<int, 0> b0{};
  const integral_constant<int, 2> b2{};

  // W slice kt in unit kt % 2, A slice kt in unit 2 + kt % 2; a row that fills no group: by way of registers
  if (sc.nd >= 8) issue_scales(0);
  else sc.first(sbase + scale_row(tid), smem + SC, tid);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
#pragma unroll
    for (int j = 0; j < INS; ++j) {
      issue1(Wb, woff, s * UNIT, s, j);
      issue1(Ab, aoff, (2 + s) * UNIT, s, j);
    }
  }
  issue_scales(1);
  wait_vmcnt_lgkm0<2 * INS + 2>();  // slice 1 and group 1 may be on their way
  barrier_no_fence();
  i32x4_t a0[TM], w0[TN], a1[TM], w1[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) a0[i] = lds_chunk(smem + 2 * UNIT + wa + i * 4096 + loff[0]);
#pragma unroll
  for (int j = 0; j < TN; ++j) w0[j] = lds_chunk(smem + ww + j * 4096 + loff[0]);
  Half x0, x1;
  read_scales(x0, 0);
  place_scales(x0, 0);
  // slice kt, slice F = kt % 4 of a group of scales
  auto slice = [&](int kt, auto f_) {
    constexpr int F = decltype(f_)::value;
    constexpr int wu = (F & 1) * UNIT, au = wu + 2 * UNIT;
    __builtin_amdgcn_sched_barrier(0);
    substep(a0, w0, a1, w1, wu, au, 1, x0, b0, none);
    read_scales(x1, 2 * kt + 1);
    __builtin_amdgcn_sched_barrier(0);
    substep(a1, w1, a0, w0, wu, au, 2, x0, b2, none);
    place_scales(x1, 2 * kt + 1);
    __builtin_amdgcn_sched_barrier(0);
    substep(a0, w0, a1, w1, wu, au, 3, x1, b0, none);
    // this wave's reads of slice kt and its copies of slice kt + 1 are done; then everyone's are
    wait_vmcnt_lgkm0<0>();
    barrier_no_fence();
    // (slice kt's group of scales is read, too: the next but one takes its place)
    if constexpr (F == 3) issue_scales((kt >> 2) + 2);
    read_scales(x0, 2 * kt + 2);
    __builtin_amdgcn_sched_barrier(0);
    substep(a1, w1, a0, w0, wu ^ UNIT, au ^ UNIT, 0, x1, b2, [&](int q) {
      if (q & 1) issue1(Ab, aoff, au, kt + 2, q >> 1);
      else issue1(Wb, woff, wu, kt + 2, q >> 1);
    });
    place_scales(x0, 2 * kt + 2);
  };
  int kt = 0;
#pragma unroll 1
  for (; kt + 4 <= nk; kt += 4) {
    slice(kt, integral_constant<int, 0>{});
    slice(kt + 1, integral_constant<int, 1>{});
    slice(kt + 2, integral_constant<int, 2>{});
    slice(kt + 3, integral_constant<int, 3>{});
  }
  if (kt < nk) slice(kt, integral_constant<int, 0>{});
  if (kt + 1 < nk) slice(kt + 1, integral_constant<int, 1>{});
  if (kt + 2 < nk) slice(kt + 2, integral_constant<int, 2>{});
  __builtin_amdgcn_s_waitcnt(0);  // the copies past the end have landed
  __syncthreads();
  if constexpr (KIND == EPI_K_FP4) {
    store_fp4<TM, TN>(P, acc, m0 + 64 * wm, n0 + 128 * wn, lr, lh);
    return;
  }
  float* slab = (float*)smem + wave * (32 * 128);
  Epi<KIND> epi(P, m0 + 64 * wm, n0 + 128 * wn, lr, lh, slab);
  epi.prep();
  uint2 old[2][8][2];
  if (epi.gated) { epi.load_old(0, old[0]); epi.load_old(1, old[1]); }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = 8 * (r >> 2) + 4 * lh + (r & 3);
        slab[row * 128 + ((j * 32 + lr) ^ (((row >> 2) & 1) << 5))] = acc[i][j][r];
      }
    epi.template rows<1, 5, 32>(i, old[i]);
  }
}

// BM x 128 tiles, waves of 64 x 64 (BM = 64: 32 x 64, 192: 48 x 64), a ring of slices of 256 of K
// in LDS: two work-groups of 64 x 128 (three slices) or 128 x 128 (two) per CU, or
// one of 192 x 128 (three).  For launches that 256 x 256 tiles would not fill.  The waves
// meet before every step kt; slice kt + 1 has landed, and slice kt, whose fragments are all in
// registers, gives its place to slice kt + ST at once (late in the step: 20 K slices of 192 and 128 x 128
// tiles 29 and 30 us for 27 and 29).  The fragments of kt + 1 are read under the MFMAs of kt.
//
// 512 x 10240 x 5120 (192 x 128 tiles): 27 us, 2.0 PFLOP/s, and 0.86 us for each further 256 of K: without the
// copies 0.58, without the reads of fragments 0.86, MFMAs alone 0.47.  What bounds it is the way
// from L2: 40 KB a slice and CU, 11 TB/s over the chip.
template <int BM, int KIND>
__global__ __launch_bounds__(BM == 192 ? 512 : 256, 2) void gemm_fp4_tile_kernel(Fp4Prob P) {
  constexpr int ST = BM == 128 ? 2 : 3;
  constexpr int NW = BM == 192 ? 8 : 4, WM = BM / (NW / 2);  // waves, rows of a wave
  constexpr int TM = WM / 16, TN = 4, NF = TM + TN;
  constexpr int SLICE = (BM + 128) * 128, RING = ST * SLICE, GROUP = (BM + 128) * 16;
  constexpr int A_INS = BM / 8 / NW, W_INS = 128 / 8 / NW, INS = A_INS + W_INS;
  constexpr int TILE = BM * 128 * 4;
  constexpr int LDS = RING + 2 * GROUP + 16;  // (16: behind the last row's scales, see read_scales)
  __shared__ __attribute__((aligned(1024))) char smem[LDS > TILE ? LDS : TILE];
  int tm, tn;
  tile_at(P, xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n), tm, tn);
  const int m0 = tm * BM, n0 = tn * 128;
  const int nk = (P.K + 255) >> 8;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int lr = lane & 15, lq = lane >> 4;

  const uint8_t* Ab = P.A + (int64_t)m0 * P.lda;
  const uint8_t* Wb = P.W + (int64_t)n0 * P.ldw;
  // copy j of this wave: rows 8 (A_INS wave + j) .. + 7 of A, then the like of W
  uint32_t off[INS];
  int ch[INS];
#pragma unroll
  for (int j = 0; j < INS; ++j) {
    const int row = 8 * (j < A_INS ? wave * A_INS + j : wave * W_INS + j - A_INS) + (lane >> 3);
    ch[j] = 16 * ((lane & 7) ^ ((row >> 1) & 7));
    off[j] = (uint32_t)min(row, (j < A_INS ? P.M - 1 - m0 : P.N - 1 - n0)) * (uint32_t)(j < A_INS ? P.lda : P.ldw) + ch[j];
  }
  auto issue1 = [&](int u, int s, int j) {
    const int at = j < A_INS ? (wave * A_INS + j) * 1024 : BM * 128 + (wave * W_INS + j - A_INS) * 1024;
    copy16_unseen(j < A_INS ? Ab : Wb, smem + u + at, ch[j] < (P.K >> 1) - 128 * s ? off[j] : OOB, (uint32_t)s * 128);
  };
  // scales: 64 rows a wave, of A, then of W
  const Scales<4> sc(P.K);
  const int swave = wave % ((BM + 128) / 64), srow = 64 * swave + lane;
  const bool of_a = 64 * swave < BM;
  const uint8_t* sbase = of_a ? P.As + (int64_t)m0 * P.ldas : P.Ws + (int64_t)n0 * P.ldws;
  const uint32_t soff = of_a ? (uint32_t)min(srow, P.M - 1 - m0) * (uint32_t)P.ldas
                             : (uint32_t)min(srow - BM, P.N - 1 - n0) * (uint32_t)P.ldws;
  // (no branches between MFMAs: the compiler would sink products behind them, past the barriers; a
  // group past the last one is zeros, and a wave without rows repeats another's)
  auto issue_scales = [&](int g) {
    copy16_unseen(sbase, smem + RING + (g & 1) * GROUP + swave * 1024, 4 * g < sc.nd ? soff : OOB, 4 * max(sc.start(g), 0));
  };
  // (two dwords in one read; a second one past the row's last is another row's, and valid() clears it)
  auto read_scales = [&](int kt, uint32_t(&x)[NF][2], int f) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int g = kt >> 1, at = RING + (g & 1) * GROUP + 4 * sc.place(g, 2 * kt) + 4 * h;
      x[f][h] = *(const uint32_t*)(smem + at + 16 * ((f < TM ? WM * wm + 16 * f : BM + 64 * wn + 16 * (f - TM)) + lr));
    }
  };
  auto place_scales = [&](int kt, uint32_t(&x)[NF][2]) {  // this lane's block into byte 0
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t v = sc.valid(2 * kt + h);
#pragma unroll
      for (int f = 0; f < NF; ++f) x[f][h] = (x[f][h] & v) >> (8 * lq);
    }
  };
  int loff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) loff[h] = lr * 128 + (((4 * h + lq) ^ ((lr >> 1) & 7)) << 4);
  auto rd = [&](int u, int f, int h) {  // fragment f: A, then W
    const int at = u + (f < TM ? wm * WM * 128 + f * 2048 : BM * 128 + wn * 64 * 128 + (f - TM) * 2048);
    return lds_chunk(smem + at + loff[h]);
  };
  f32x4_t acc[TM][TN] = {};

#pragma unroll
  for (int s = 0; s < ST; ++s) {
#pragma unroll
    for (int j = 0; j < INS; ++j) issue1(s * SLICE, s, j);
    if (s == 0) {
      issue_scales(1);
      if (sc.nd >= 4) issue_scales(0);
      else if (tid < BM + 128) sc.first(sbase + soff, smem + RING, tid);  // (waits for slice 0, too)
    }
  }
  wait_vmcnt_lgkm0<(ST - 1) * INS>();
  barrier_no_fence();
  i32x4_t f0[NF][2], f1[NF][2];
  uint32_t s0[NF][2], s1[NF][2];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    f0[f][0] = rd(0, f, 0);
    f0[f][1] = rd(0, f, 1);
    read_scales(0, s0, f);
  }
  place_scales(0, s0);
  int u = 0;  // place of slice kt
  auto step = [&](int kt, i32x4_t(&f)[NF][2], i32x4_t(&fn)[NF][2], uint32_t(&x)[NF][2], uint32_t(&xn)[NF][2],
                  auto odd) {
    const int un = u == (ST - 1) * SLICE ? 0 : u + SLICE;
    // this wave's reads of slice kt and its copies of slice kt + 1 are done (those
    // of the next ST - 2 may stay in flight); then everyone's are
    wait_vmcnt_lgkm0<(ST - 2) * INS>();
    barrier_no_fence();
    if constexpr (decltype(odd)::value) issue_scales((kt >> 1) + 2);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 2 * TM * TN; ++q) {
      const int h = q / (TM * TN), i = q % TM, j = q % (TM * TN) / TM;
      acc[i][j] = mfma_fp4(f[i][h], f[TM + j][h], acc[i][j], x[i][h], x[TM + j][h]);
      __builtin_amdgcn_sched_barrier(0);
      // in the order of their use: A 0, W 0, the other A, the other W
      if (q < 2 * NF) {
        const int hq = q / NF, e = q % NF, r = e == 0 ? 0 : e == 1 ? TM : e <= TM ? e - 1 : e;
        fn[r][hq] = rd(un, r, hq);
        if (hq == 0) read_scales(kt + 1, xn, r);
      }
      if (q < INS) issue1(u, kt + ST, q);
      __builtin_amdgcn_sched_barrier(0);
    }
    place_scales(kt + 1, xn);
    u = un;
  };
  int kt = 0;
#pragma unroll 1
  for (; kt + 2 <= nk; kt += 2) {
    step(kt, f0, f1, s0, s1, std::false_type{});
    step(kt + 1, f1, f0, s1, s0, std::true_type{});
  }
  if (kt < nk) step(kt, f0, f1, s0, s1, std::false_type{});
  __builtin_amdgcn_s_waitcnt(0);  // the copies past the end have landed
  __syncthreads();
  // The tile in LDS as slabs of ROWS rows x 128, one per wave, columns XOR 16
  // ((row >> 2) & 3): then each wave has whole 128-column rows.
  constexpr int ROWS = BM == 192 ? 16 : BM / NW;
  float* tile = (float*)smem;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        tile[(wm * WM + 16 * i + 4 * lq + r) * 128 + ((64 * wn + 16 * j + lr) ^ (lq << 4))] = acc[i][j][r];
  __syncthreads();
#pragma unroll 1
  for (int slab = wave; slab < BM / ROWS; slab += NW) {
    Epi<KIND> epi(P, m0 + ROWS * slab, n0, lane & 31, lane >> 5, tile + ROWS * slab * 128);
    epi.prep();
    uint2 old[8][2];
    if (epi.gated) epi.load_old(0, old);
    epi.template rows<3, 4, ROWS>(0, old);
  }
}

// Few rows or few tiles: 16 RB x NT outputs per work-group, eight waves of 16 RB x 32
// that share K (NT = 32: eight ways, 64: four, 128, of 16 rows alone: two).  Each wave copies its own
// rows' slices and their scales to a ring of its own in LDS, so that no wave waits for another until
// their sums meet at the end; the copies read whole 128-byte lines, eight lanes
// each.  Bound by the way of W from memory: 1 x 13824 x 5120 9.6 us, 3.9 TB/s.
template <int NT, int RB, int KIND>
__global__ __launch_bounds__(512) void gemm_fp4_small_kernel(Fp4Prob P) {
  constexpr int NH = NT / 32, KS = 8 / NH, NF = 2 + RB, ST = RB == 1 ? 3 : 2;
  constexpr int INS = 2 * NF, SLICE = INS * 1024 + 512, LD = 36;  // W's two fragments, A's, scales
  constexpr int RING = 8 * ST * SLICE, PART = 8 * 16 * RB * LD * 4;
  static_assert(PART <= RING, "the waves' sums take the rings' place");
  __shared__ __attribute__((aligned(1024))) char smem[RING];
  const int lt = xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n);
  const int m0 = lt % P.tiles_m * (16 * RB), n0 = lt / P.tiles_m * NT;  // neighbours share the weights
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int ks = wave % KS, nh = wave / KS;
  const int nw = min(n0 + 32 * nh, P.N - 1);  // (a wave past the last column repeats it)
  const uint8_t* Wb = P.W + (int64_t)nw * P.ldw;
  const uint8_t* Ab = P.A + (int64_t)m0 * P.lda;
  // copy j: rows 8 j .. + 7 of W, then of A
  uint32_t off[INS];
  int ch[INS];
#pragma unroll
  for (int j = 0; j < INS; ++j) {
    const int row = 8 * (j < 4 ? j : j - 4) + (lane >> 3);
    ch[j] = 16 * ((lane & 7) ^ ((row >> 1) & 7));
    off[j] = (uint32_t)min(row, (j < 4 ? P.N - 1 - nw : P.M - 1 - m0)) * (uint32_t)(j < 4 ? P.ldw : P.lda) + ch[j];
  }
  // scales of row lane: 32 of W, 16 RB of A, each from its own operand
  const Scales<4> sc(P.K);
  const uint8_t* Wsb = P.Ws + (int64_t)nw * P.ldws;
  const uint8_t* Asb = P.As + (int64_t)m0 * P.ldas;
  const uint32_t soff = lane < 32 ? (uint32_t)min(lane, P.N - 1 - nw) * (uint32_t)P.ldws
                                  : (uint32_t)min((lane - 32) % (16 * RB), P.M - 1 - m0) * (uint32_t)P.ldas;
  const int steps = (P.K + 255) >> 8, per = (steps + KS - 1) / KS;
  const int s0 = ks * per, s1 = min(steps, s0 + per);
  char* ring = smem + wave * (ST * SLICE);
  // slice s of K (past the wave's last one: zeros) and its scales
  auto issue = [&](int s, int u) {
    const int left = s < s1 ? (P.K >> 1) - 128 * s : 0;
    char* d = ring + u * SLICE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t at = 4 * min(2 * s + h, sc.nd - 1);
      if (lane < 32) copy4_unseen(Wsb, d + INS * 1024 + 256 * h, soff, at);
      else copy4_unseen(Asb, d + INS * 1024 + 256 * h, soff, at);
    }
#pragma unroll
    for (int j = 0; j < INS; ++j)
      copy16_unseen(j < 4 ? Wb : Ab, d + j * 1024, ch[j] < left ? off[j] : OOB, (uint32_t)s * 128);
  };
  int loff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) loff[h] = lr * 128 + (((4 * h + lq) ^ ((lr >> 1) & 7)) << 4);
  f32x4_t acc[RB][2] = {};
#pragma unroll
  for (int u = 0; u < ST; ++u) issue(s0 + u, u);
  for (int s = s0; s < s1; s += ST) {
#pragma unroll
    for (int u = 0; u < ST; ++u) {  // (a slice past s1 adds zeros)
      wait_vmcnt<(ST - 1) * (INS + 4)>();  // this slice and its scales have landed
      asm volatile("" ::: "memory");
      i32x4_t f[NF][2];
      uint32_t b[NF][2];
#pragma unroll
      for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f[i][h] = lds_chunk(ring + u * SLICE + i * 2048 + loff[h]);
          const uint32_t x = *(const uint32_t*)(ring + u * SLICE + INS * 1024 + 256 * h + 4 * (16 * i + lr));
          b[i][h] = (x & (s + u < s1 ? sc.valid(2 * (s + u) + h) : 0u)) >> (8 * lq);
        }
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): read, its place is free
      asm volatile("" ::: "memory");
      issue(s + u + ST, u);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = mfma_fp4(f[2 + i][h], f[j][h], acc[i][j], b[2 + i][h], b[j][h]);
    }
  }
  __builtin_amdgcn_s_waitcnt(0);  // the copies past the end have landed
  __syncthreads();
  float(*part)[16 * RB][LD] = (float(*)[16 * RB][LD])smem;
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[wave][16 * i + 4 * lq + r][16 * j + lr] = acc[i][j][r];
  __syncthreads();

  // NT / 4 threads per row, 4 columns each, the waves' sums added in their order
  constexpr int TPR = NT / 4, PASS = 512 / TPR;
  const int c = tid % TPR, n = n0 + 4 * c;
#pragma unroll
  for (int r0 = 0; r0 < 16 * RB; r0 += PASS) {
    const int row = r0 + tid / TPR, m = m0 + row;
    if (row >= 16 * RB) return;  // whole waves
    f32x4_t t = {};
#pragma unroll
    for (int w = 0; w < KS; ++w) t += *(const f32x4_t*)&part[KS * (c / 8) + w][row][4 * (c % 8)];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = t[e] + (P.bias && n < P.N ? bf16_to_f32(P.bias[n + e]) : 0.f);
    if constexpr (NT == 128) {
      if (n0 < P.rms_cols) {  // one 128-wide head per tile
        float ss = v[0] * v[0] + v[1] * v[1] + v[2] * v[2] + v[3] * v[3];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) ss += __shfl_xor(ss, o, 64);
        const float f = rsqrtf(ss * (1.f / 128.f) + DIT_RMS_EPS);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= f;
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (n >= P.gelu_from) v[e] = gelu_tanh_f(v[e]);
      if (P.flags & DIT_EPI_SILU) v[e] = silu_f(v[e]);
      top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    }
    if constexpr (KIND == EPI_K_FP4) {
      // (eight threads hold a block; those past the last column are whole blocks)
      const uint32_t byte = scale4_of(max_over<8>(top));
      [[maybe_unused]] const float inv = e8m0_inverse(byte);
      if (m >= P.M || n >= P.N) continue;
      uint32_t w = 0;
#if defined(__HIP_DEVICE_COMPILE__)
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0] * inv, v[1] * inv, 1.f, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * inv, v[3] * inv, 1.f, 1);
#endif
      *(uint16_t*)((uint8_t*)P.C + (int64_t)m * P.ldc + (n >> 1)) = (uint16_t)w;
      if ((c & 7) == 0) P.Cs[(int64_t)m * P.ldcs + (n >> 5)] = (uint8_t)byte;
      continue;
    }
    if (m >= P.M || n >= P.N) continue;
    const int64_t at = (int64_t)m * P.ldc + n + (n >= P.gap_at ? P.gap : 0);
    if (P.flags & DIT_EPI_F32) {
      *(float4*)((float*)P.C + at) = make_float4(v[0], v[1], v[2], v[3]);
      continue;
    }
    uint2* o = (uint2*)((bf16_t*)P.C + at);
    if (P.flags & DIT_EPI_GATED_RES) {
      const uint2 x = *o;
      const float4 g = *(const float4*)(P.gate + n);
      v[0] = __uint_as_float(x.x << 16) + g.x * v[0];
      v[1] = __uint_as_float(x.x & 0xffff0000u) + g.y * v[1];
      v[2] = __uint_as_float(x.y << 16) + g.z * v[2];
      v[3] = __uint_as_float(x.y & 0xffff0000u) + g.w * v[3];
    }
    *o = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

}  // namespace

hipError_t launch_quant_fp4(const void* x, bool bf16, int64_t ldx, void* q, int64_t ldq, void* scale, int64_t lds, int M,
                            int K, hipStream_t s) {
  if (M == 0 || K == 0) return hipSuccess;
  const int per_row = (K + 1023) / 1024;
  const int64_t groups = ((int64_t)M * per_row + 3) / 4;
  if (bf16)
    hipLaunchKernelGGL(quant_fp4_kernel<bf16_t>, dim3((uint32_t)groups), dim3(256), 0, s, (const bf16_t*)x, ldx,
                       (uint8_t*)q, ldq, (uint8_t*)scale, lds, M, K, per_row);
  else
    hipLaunchKernelGGL(quant_fp4_kernel<float>, dim3((uint32_t)groups), dim3(256), 0, s, (const float*)x, ldx,
                       (uint8_t*)q, ldq, (uint8_t*)scale, lds, M, K, per_row);
  return hipGetLastError();
}

hipError_t launch_dequant_fp4(const void* q, int64_t ldq, const void* scale, int64_t lds, void* y, bool bf16, int64_t ldy,
                              int M, int K, hipStream_t s) {
  if (M == 0 || K == 0) return hipSuccess;
  const int per_row = (K + 2047) / 2048;
  const int64_t groups = ((int64_t)M * per_row + 3) / 4;
  if (bf16)
    hipLaunchKernelGGL(dequant_fp4_kernel<bf16_t>, dim3((uint32_t)groups), dim3(256), 0, s, (const uint8_t*)q, ldq,
                       (const uint8_t*)scale, lds, (bf16_t*)y, ldy, M, K, per_row);
  else
    hipLaunchKernelGGL(dequant_fp4_kernel<float>, dim3((uint32_t)groups), dim3(256), 0, s, (const uint8_t*)q, ldq,
                       (const uint8_t*)scale, lds, (float*)y, ldy, M, K, per_row);
  return hipGetLastError();
}

hipError_t launch_gemm_fp4(const GemmFp4Args& g, hipStream_t s, int n_cu) {
  if (g.M == 0 || g.N == 0) return hipSuccess;
  Fp4Prob p{};
  p.A = (const uint8_t*)g.A; p.lda = g.lda;
  p.W = (const uint8_t*)g.W; p.ldw = g.ldw;
  p.As = (const uint8_t*)g.As; p.ldas = g.ldas;
  p.Ws = (const uint8_t*)g.Ws; p.ldws = g.ldws;
  p.bias = (const bf16_t*)g.bias;
  p.C = g.C; p.ldc = g.ldc;
  p.Cs = (uint8_t*)g.Cs; p.ldcs = g.ldcs;
  p.gate = g.gate;
  p.M = g.M; p.N = g.N; p.K = g.K;
  p.flags = g.flags; p.rms_cols = g.rms_cols; p.gelu_from = g.gelu_from; p.gap_at = g.gap_at; p.gap = g.gap;
  auto go = [&](void (*fn)(Fp4Prob), int bm, int bn, int threads) {
    p.tiles_m = (g.M + bm - 1) / bm;
    p.tiles_n = (g.N + bn - 1) / bn;
    hipLaunchKernelGGL(fn, dim3((uint32_t)p.tiles_m * p.tiles_n), dim3(threads), 0, s, p);
    return hipGetLastError();
  };
  const bool f32 = g.flags & DIT_EPI_F32, fp4 = g.flags & DIT_EPI_FP4, gated = g.flags & DIT_EPI_GATED_RES;
  const bool plain = !(g.flags & DIT_EPI_SILU);
  const bool store = plain && !gated && !fp4 && !f32 && (g.gelu_from >= g.N || g.gelu_from % 128 == 0) &&
                     (g.gap == 0 || g.gap_at % 128 == 0);
  const bool only_gate = plain && gated && g.rms_cols == 0 && g.gelu_from >= g.N && g.gap == 0;
  auto tiles = [&](int bm, int bn) { return (int64_t)((g.M + bm - 1) / bm) * ((g.N + bn - 1) / bn); };
  // Few rows or few tiles: the narrowest tiles that fit the CUs once, to spread the way of W over them.  In us,
  // against 64 x 128 tiles: 1 x 13824 x 5120 10.4 14.8, 16 x 5120 x 13824 13.4 30.3, 32 x 5120 x 5120 9.0 14.7,
  // 64 x 5120 x 5120 11.8 14.7, 128 x 1024 x 1024 9.2 9.4, 256 x 512 x 4096 8.8 12.0, 128 x 128 x 8192 9.2 19.3.
  const bool one = g.M <= 16;
  const int rows = one ? 16 : 32, widest = one ? 128 : 64;
  int nt = g.rms_cols > 0 ? 128 : 32;
  while (nt < widest && tiles(rows, nt) > n_cu) nt *= 2;
  if (nt <= widest && tiles(rows, nt) <= n_cu) {
#define DIT_SMALL(K)                                                                                         \
  go(!one ? (nt == 64 ? gemm_fp4_small_kernel<64, 2, K> : gemm_fp4_small_kernel<32, 2, K>)                   \
          : nt == 128 ? gemm_fp4_small_kernel<128, 1, K>                                                     \
                      : nt == 64 ? gemm_fp4_small_kernel<64, 1, K> : gemm_fp4_small_kernel<32, 1, K>, rows, nt, 512)
    return fp4 ? DIT_SMALL(EPI_K_FP4) : DIT_SMALL(EPI_K_ANY);
#undef DIT_SMALL
  }
  // Rounds of the chip times a tile's time, which is some us and some per slice of 256 of K, fewer in a round
  // that fills at most half of the chip (fitted to each kernel over the sizes below).  In us, 64 x 128, 128 x 128,
  // 192 x 128 and 256 x 256 tiles (256 x 128 ones were nowhere the fastest):
  //   512 x 10240 x 5120  34 29 27 39    1024 x 10240 x 5120 53 48 48 42    512 x 5120 x 5120  21 20 23 36
  //   2048 x 4096 x 4096  35 28 38 34    4096 x 4096 x 1024  29 22 27 21    1333 x 1000 x 2336 10 12 14 21
  struct Tile { int bm, bn, per_cu; double half_us, slice_us, us; };
  auto cost = [&](const Tile& c) {
    const int64_t slots = (int64_t)n_cu * c.per_cu, n = tiles(c.bm, c.bn), full = (n - 1) / slots, slices = (g.K + 255) / 256;
    return full * (slices * c.slice_us + c.us) + slices * (2 * (n - full * slots) <= slots ? c.half_us : c.slice_us) + c.us;
  };
  const Tile cfg[] = {{64, 128, 2, 0.55, 0.8, 4}, {128, 128, 2, 0.69, 1.25, 6}, {192, 128, 1, 0.75, 1.0, 6},
                      {256, 256, 1, 1.35, 1.75, 12}};
  int best = 0;
  for (int c = 1; c < 4; ++c)
    if (cost(cfg[c]) < cost(cfg[best])) best = c;
  if (best == 3)
    return go(fp4 ? gemm_fp4_ring_kernel<EPI_K_FP4> : store ? gemm_fp4_ring_kernel<EPI_K_STORE>
              : only_gate ? gemm_fp4_ring_kernel<EPI_K_GATED> : gemm_fp4_ring_kernel<EPI_K_ANY>, 256, 256, 512);
#define DIT_TILE(BM, THREADS)                                                                                  \
  go(fp4 ? gemm_fp4_tile_kernel<BM, EPI_K_FP4> : store ? gemm_fp4_tile_kernel<BM, EPI_K_STORE>                  \
                                                       : gemm_fp4_tile_kernel<BM, EPI_K_ANY>, BM, 128, THREADS)
  if (best == 2) return DIT_TILE(192, 512);
  if (best == 1) return DIT_TILE(128, 256);
  return DIT_TILE(64, 256);
#undef DIT_TILE
}

}  // namespace dit
