// 8-bit floating point: rows quantised to e4m3 with one power-of-two scale (an
// E8M0 byte) per 128 values, and the product of two such matrices,
//   C = epi(sum over blocks b of K: 2^(sa[m,b] + sw[n,b] - 254) sum over k in b: a[m,k] w[n,k], + bias).
//
// The scales are powers of two because the matrix cores take them as they are:
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies one block of 128 of K per
// instruction and applies both operands' scale bytes for nothing, so the
// accumulators run through all of K without a VALU instruction between.  x / 2^e
// is exact, too: the one rounding of a value is the one to e4m3.
//
// That instruction adds the products of a few neighbouring k in about 14 bits
// below the largest of them (measured: 2^-14 of it is lost between neighbours
// and kept between far k; normal data come out 1.8e-5 off in the 2-norm, at
// any K).  A bf16 or e4m3 output rounds by 2^-9 or 2^-4, a hundred times that.
// An f32 output would carry it, so for those the operands are widened to bf16
// with their scale in registers and multiplied by bf16 MFMAs (WIDE).  That is exact
// for scale bytes up to 236; a wave that meets a larger one, or whose sums overflow,
// forms them anew (wide_sums).
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "gemm_tile.h"
#include "kernels.h"

namespace dit {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

struct Fp8Prob {
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

template <int KIND = EPI_K_ANY>
using EpiLds = EpiLdsT<KIND, Fp8Prob>;

// ---------------------------------------------------------------- quantise

// Eight lanes per block of 128, 16 values each; a wave takes eight blocks of a
// row.  One pass, bound by memory: 32760 x 5120 bf16 (504 MB) 86 us, 5.9 TB/s (a
// copy of 1 GiB: 5.2).
template <typename T>
__global__ __launch_bounds__(256) void quant_fp8_kernel(const T* __restrict__ x, int64_t ldx, uint8_t* __restrict__ q,
                                                        int64_t ldq, uint8_t* __restrict__ scale, int64_t lds, int M,
                                                        int K, int per_row) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t m = unit / per_row;
  if (m >= M) return;
  const int k = (int)(unit - m * per_row) * 1024 + 16 * lane;
  const bool in = k < K;  // K % 16 == 0: a lane's 16 values are inside or not
  float v[16];
  if (in) {
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
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.f;
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max_over<8>(top);
  const uint32_t byte = e8m0_of(top);
  const float inv = e8m0_inverse(byte);
  if (!in) return;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_fp8x4(v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv, v[4 * i + 3] * inv);
  *(uint4*)(q + m * ldq + k) = make_uint4(w[0], w[1], w[2], w[3]);
  if ((lane & 7) == 0) scale[m * lds + (k >> 7)] = (uint8_t)byte;
}

// ---------------------------------------------------------------- products

// 16 bytes per lane from base + voff + soff into LDS at dst + 16 lane; lanes
// with voff >= OOB write zeros.  Offsets in bounds lie below OOB: the bases are
// those of a tile's first row, and the host bounds 256 rows of an operand.
constexpr uint32_t OOB = 0x80000000u;
__device__ __forceinline__ void copy16_oob(const void* base, lds_void_t* dst, uint32_t voff, uint32_t soff) {
#if defined(__HIP_DEVICE_COMPILE__)
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, (int)OOB, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, voff, soff, 0, 0);
#endif
}

// 4 bytes from each lane's p to LDS at dst + 4 lane.
__device__ __forceinline__ void copy4(const uint8_t* p, lds_void_t* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p, dst, 4, 0, 0);
#endif
}

// The 128 x 128-deep step of one 16 x 16 block.  A lane holds row lr's 16-byte
// chunks lq and lq + 4 of the block of 128 (the sum over k does not mind their
// order, and these are the chunks that a swizzled LDS row serves without bank
// conflicts).  sa and sw: scale bytes of the lane's rows for four blocks of K; B: which.
template <int B = 0>
__device__ __forceinline__ f32x4_t mfma_scaled(const i32x8_t& a, const i32x8_t& w, const f32x4_t& c, int sa, int sw) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, w, c, 0, 0, B, sa, B, sw);
#else
  return c;
#endif
}

// The same of a 32 x 32 block and 64 of K: lane (lr, lh) holds 32 of row lr.
template <int B>
__device__ __forceinline__ f32x16_t mfma_scaled32(const i32x8_t& a, const i32x8_t& w, const f32x16_t& c, int sa,
                                                  int sw) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, w, c, 0, 0, B, sa, B, sw);
#else
  return c;
#endif
}

typedef int i32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x8_t frag8(i32x4_t lo, i32x4_t hi) {
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Both chunks of a fragment from LDS.  (Loads of a vector type keep their type
// information; without it the compiler has every one of them wait for all copies
// to LDS in flight.)
__device__ __forceinline__ i32x8_t lds_frag(const char* lo, const char* hi) {
  return frag8(*(const i32x4_t*)lo, *(const i32x4_t*)hi);
}

// The fragment widened to bf16, times 2^(byte - 127): four 32-deep operands.
__device__ __forceinline__ void widen(const i32x8_t& f, int byte, bf16x8_t (&w)[4]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const float s = __uint_as_float((uint32_t)(byte & 255) << 23);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    uint32_t u[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * t + h], s, false));
      u[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * t + h], s, true));
    }
    w[t] = __builtin_bit_cast(bf16x8_t, make_uint4(u[0], u[1], u[2], u[3]));
  }
#endif
}

// Other than zero, e4m3 values are 2^-9 .. 448, and bf16 numbers are normal from 2^-126
// to below 2^128.  Widened with a scale 2^UP times their own, values of bytes 0 .. 236 are
// normal bf16 numbers, the 2^-126 that a block of zeros has included; the sums then
// are 2^(2 UP) times too large.  (Without UP the least values of bytes below 3 lose bits.)
constexpr int UP = 10, LAST_BYTE = 236;
// Whether one of the lowest `valid` bytes lies above LAST_BYTE.  (A byte of ~x that is less
// than n borrows into its top bit, which is clear; one of x that is not leaves it.)
__device__ __forceinline__ uint32_t any_too_large(uint32_t x, int valid) {
  const uint32_t last = valid >= 4 ? ~0u : (1u << (8 * max(valid, 0))) - 1u;
  return (~x - 0x01010101u * (255 - LAST_BYTE)) & x & 0x80808080u & last;
}

// Sums over slices k0 .. k1 - 1 of 16 TM x 16 TN outputs from row m0 and column n0 on, for
// any scale bytes: each block of K is summed without its scales (e4m3 is exact in bf16),
// and the sum takes both at once.  Straight from memory, for waves that need it: 4096^3
// takes 1.26 ms where all do, and 0.12 where none does.
template <int TM, int TN>
__device__ __forceinline__ void wide_sums(const Fp8Prob& P, int m0, int n0, int k0, int k1, f32x4_t (&acc)[TM][TN]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
  auto frag = [&](const uint8_t* row, int k) {  // the lane's chunks of the block from k on
    const i32x4_t none = {0, 0, 0, 0};
    const int a = k + 16 * lq, b = a + 64;
    return frag8(a < P.K ? *(const i32x4_t*)(row + a) : none, b < P.K ? *(const i32x4_t*)(row + b) : none);
  };
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int m = min(m0 + 16 * i + lr, P.M - 1), n = min(n0 + 16 * j + lr, P.N - 1);
      f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int k = k0; k < k1; ++k) {
        bf16x8_t a[4], w[4];
        widen(frag(P.A + m * P.lda, 128 * k), 127, a);
        widen(frag(P.W + n * P.ldw, 128 * k), 127, w);
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 4; ++t) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], w[t], x, 0, 0, 0);
        const int sw = P.Ws[n * P.ldws + k];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int sa = P.As[min(m0 + 16 * i + 4 * lq + r, P.M - 1) * P.ldas + k];
          sum[r] += sa == 255 || sw == 255 ? __uint_as_float(0x7fc00000u) : ldexpf(x[r], sa + sw - 254);
        }
      }
      acc[i][j] = sum;
    }
#endif
}

// The end of a wave's sums of operands widened with 2^UP.  too_large: a lane met a byte above LAST_BYTE.
template <int TM, int TN>
__device__ __forceinline__ void finish_wide(const Fp8Prob& P, int m0, int n0, int k0, int k1, bool too_large,
                                            f32x4_t (&acc)[TM][TN]) {
#if defined(__HIP_DEVICE_COMPILE__)
  f32x4_t zero = {};  // NaN where a sum is not finite, which the true one may still be
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        acc[i][j][r] *= 1.f / (1 << 2 * UP);
        zero[r] = __builtin_fmaf(acc[i][j][r], 0.f, zero[r]);
      }
  const bool overflow = (zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.f;
  if (__builtin_amdgcn_ballot_w64(too_large || overflow)) wide_sums<TM, TN>(P, m0, n0, k0, k1, acc);
#endif
}

// Origin of tile lt: M-grouped order, eight tile rows per group.
__device__ __forceinline__ void tile_at(const Fp8Prob& P, int lt, int& tm, int& tn) {
  constexpr int GROUP = 8;
  const int in_group = GROUP * P.tiles_n;
  const int gid = lt / in_group;
  const int first_m = gid * GROUP;
  const int gsz = min(P.tiles_m - first_m, GROUP);
  tm = first_m + (lt % in_group) % gsz;
  tn = (lt % in_group) / gsz;
}

// 256 x 256 tiles, 8 waves of 64 x 128, the whole 160 KB of LDS as three W and
// two A slices of 128 of K (32 KB each, 16-byte chunks of a 128-byte row
// XOR-swizzled by ((row >> 1) & 7)).  32x32x64 MFMAs: a slice is two substeps of
// eight, and a substep's six fragments are read under the MFMAs of the one
// before it, evenly.
//
// The waves meet after substep 0, whose reads were the last of their slice: its
// units take A slice kt + 2 (in substep 1) and W slice kt + 3 (in the next
// substep 0).  Slices past the last one are copied as zeros (no memory
// traffic), which keeps every iteration and wait alike.
//
// 32760 x 13824 x 5120: bf16 out 1.87 ms (2.48 PFLOP/s), GELU and 8-bit rows out
// 2.02 ms (2.30).  Power bounds it: the same launch on operands of zeros runs at
// 3.65 PFLOP/s; on normal data the clock falls to 1.9 - 2.15 GHz.  Slices of 64
// and 128 x 128 tiles of four waves were slower.
template <int KIND>
__global__ __launch_bounds__(512) void gemm_fp8_ring_kernel(Fp8Prob P) {
  constexpr int UNIT = 256 * 128, INS = 4, TM = 2, TN = 4;
  __shared__ __attribute__((aligned(1024))) char smem[5 * UNIT];
  int tm, tn;
  tile_at(P, xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n), tm, tn);
  const int m0 = tm * 256, n0 = tn * 256;
  const int nk = (P.K + 127) >> 7;

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
    copy16_oob(base, (lds_void_t*)(smem + u + (wave * INS + j) * 1024),
               16 * (c0 ^ (4 * (j & 1))) < P.K - 128 * s ? off[j] : OOB, (uint32_t)s * 128);
  };
  auto issue = [&](const uint8_t* base, const uint32_t (&off)[INS], int u, int s) {
#pragma unroll
    for (int j = 0; j < INS; ++j) issue1(base, off, u, s, j);
  };
  // scales of this wave's rows, four slices to a dword: lane l loads rows l (and
  // 64 + l of W), a lane permutation hands them to the lanes that multiply
  const uint8_t* sap = P.As + (int64_t)min(m0 + 64 * wm + lane, P.M - 1) * P.ldas;
  const uint8_t* swp0 = P.Ws + (int64_t)min(n0 + 128 * wn + lane, P.N - 1) * P.ldws;
  const uint8_t* swp1 = P.Ws + (int64_t)min(n0 + 128 * wn + 64 + lane, P.N - 1) * P.ldws;
  int sna, snw0, snw1;
  auto load_scales = [&](int g) {
    const int at = 4 * min(g, (nk - 1) >> 2);
    sna = *(const int*)(sap + at);
    snw0 = *(const int*)(swp0 + at);
    snw1 = *(const int*)(swp1 + at);
  };
  int sa[TM], sw[TN];
  auto spread_scales = [&]() {
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = __builtin_amdgcn_ds_bpermute(4 * lr + 128 * i, sna);
#pragma unroll
    for (int j = 0; j < TN; ++j) sw[j] = __builtin_amdgcn_ds_bpermute(4 * lr + 128 * (j & 1), j < 2 ? snw0 : snw1);
  };

  // this lane's chunks inside 32 rows of a unit: half lh of substep s, 32 of its 64 k
  int loff[2][2];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int h = 0; h < 2; ++h) loff[s][h] = lr * 128 + (((4 * s + 2 * h + lh) ^ ((lr >> 1) & 7)) << 4);
  const int wa = wm * 64 * 128, ww = wn * 128 * 128;
  auto rd = [&](int at, int s) { return lds_frag(smem + at + loff[s][0], smem + at + loff[s][1]); };
  f32x16_t acc[TM][TN] = {};
  // A substep's MFMAs, and between them one by one the fragment reads of the next
  // substep (s of the slice in units uw, ua) in the order of their use and four
  // copies.  The fences keep that order.
  auto substep = [&](const i32x8_t(&a)[TM], const i32x8_t(&w)[TN], i32x8_t(&an)[TM], i32x8_t(&wn2)[TN], int uw, int ua,
                     int s, auto b_, auto copy) {
    constexpr int B = decltype(b_)::value;
#pragma unroll
    for (int q = 0; q < TM * TN; ++q) {
      const int i = q & 1, j = q >> 1;
      acc[i][j] = mfma_scaled32<B>(a[i], w[j], acc[i][j], sa[i], sw[j]);
      __builtin_amdgcn_sched_barrier(0);
      if (q == 0 || q == 2) an[q >> 1] = rd(ua + wa + (q >> 1) * 4096, s);
      else if (q < 6) wn2[q == 1 ? 0 : q - 2] = rd(uw + ww + (q == 1 ? 0 : q - 2) * 4096, s);
      if (q & 1) copy(q >> 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // W slice kt in unit kt % 3, A slice kt in unit 3 + kt % 2
  int wu = 0, au = 3 * UNIT;
  auto next_w = [](int u) { return u == 2 * UNIT ? 0 : u + UNIT; };
  load_scales(0);
  issue(Wb, woff, 0, 0);
  issue(Ab, aoff, 3 * UNIT, 0);
  issue(Wb, woff, UNIT, 1);
  issue(Ab, aoff, 4 * UNIT, 1);
  wait_vmcnt<2 * INS>();  // scales and slice 0 have landed
  barrier_no_fence();
  i32x8_t a0[TM], w0[TN], a1[TM], w1[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) a0[i] = rd(au + wa + i * 4096, 0);
#pragma unroll
  for (int j = 0; j < TN; ++j) w0[j] = rd(wu + ww + j * 4096, 0);
  spread_scales();
  // Slice kt, block B = kt % 4 of a dword of scales.
  auto slice = [&](int kt, auto b_) {
    constexpr int B = decltype(b_)::value;
    const int wn_ = next_w(wu), an_ = 7 * UNIT - au;
    if constexpr (B == 0) load_scales((kt >> 2) + 1);
    __builtin_amdgcn_sched_barrier(0);
    substep(a0, w0, a1, w1, wu, au, 1, b_, [&](int j) { issue1(Wb, woff, next_w(wn_), kt + 2, j); });
    // this wave's reads of slice kt and its copies of slice kt + 1 are done (W
    // slice kt + 2 may stay in flight); then everyone's are
    wait_vmcnt_lgkm0<INS>();
    barrier_no_fence();
    substep(a1, w1, a0, w0, wn_, an_, 0, b_, [&](int j) { issue1(Ab, aoff, au, kt + 2, j); });
    if constexpr (B == 3) spread_scales();
    wu = wn_;
    au = an_;
  };
  using std::integral_constant;
  int kt = 0;
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
  EpiLds<KIND> epi(P, m0 + 64 * wm, n0 + 128 * wn, lr, lh, (float*)smem + wave * (32 * 128));
  epi.prep();
  uint2 old[2][8][2];
  if (epi.gated) { epi.load_old(0, old[0]); epi.load_old(1, old[1]); }
  epi.slab_pass(acc[0], 0, old[0]);
  epi.slab_pass(acc[1], 1, old[1]);
}

// BM x 128 tiles, waves of 64 x 64 (BM = 64: 32 x 64), a ring of slices of 128 of K
// in LDS: two work-groups of 64 x 128 (three slices) or 128 x 128 (two) per CU, or
// one of 256 x 128 (three).  For launches that 256 x 256 tiles would not fill, and
// (WIDE) f32 outputs.  What bounds it is the way of a slice from L2 to LDS, so
// slices in flight count: the waves meet before every step kt; slice kt + 1 has
// landed, and slice kt, whose fragments are all in registers, gives its place to
// slice kt + ST.  The fragments of kt + 1 are read under the MFMAs of kt.
// 512 x 10240 x 5120 with the norm: 37 us (1.45 PFLOP/s) on 160 tiles of 256 x 128,
// which leave a third of the CUs without one.  Three work-groups of 64 x 128 per CU
// with two slices each lose: 1333 x 1000 x 2320 13 -> 17 us.
//
// KG = 2: two groups of four waves with rings of their own take the halves of K;
// their sums meet in LDS.  1333 x 1000 x 2320, f32: 17 us (0.37 PFLOP/s), a chain of
// ten slices on 168 CUs.
template <int BM, int KIND, bool WIDE, int KG = 1>
__global__ __launch_bounds__(BM == 256 ? 512 : 256 * KG, 2) void gemm_fp8_tile_kernel(Fp8Prob P) {
  constexpr int ST = BM == 128 ? 2 : 3;
  constexpr int NW = BM == 256 ? 8 : 4, WM = BM / (NW / 2);  // waves (of a group), rows of a wave
  constexpr int TM = WM / 16, TN = 4, NF = TM + TN;
  constexpr int SLICE = (BM + 128) * 128;
  constexpr int A_INS = BM / 8 / NW, W_INS = 128 / 8 / NW, INS = A_INS + W_INS;
  constexpr int TILE = BM * 128 * 4, RING = ST * SLICE;
  __shared__ __attribute__((aligned(1024))) char lds[KG * (RING > TILE ? RING : TILE)];
  int tm, tn;
  tile_at(P, xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n), tm, tn);
  const int m0 = tm * BM, n0 = tn * 128;
  const int nk = (P.K + 127) >> 7;

  const int tid = threadIdx.x, lane = tid & 63;
  const int grp = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 8);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) % NW;
  char* smem = lds + grp * RING;
  // slices k0 .. k1 - 1 are the group's
  const int half = (nk + 1) >> 1;
  const int k0 = KG == 1 || grp == 0 ? 0 : half, k1 = KG == 1 || grp ? nk : half;
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
    copy16_oob(j < A_INS ? Ab : Wb, (lds_void_t*)(smem + u + at), ch[j] < P.K - 128 * s ? off[j] : OOB, (uint32_t)s * 128);
  };
  // scales of this wave's rows, four slices to a dword: lane l loads rows l, a lane
  // permutation hands them to the lanes that multiply (A's fragments, then W's)
  const uint8_t* sap = P.As + (int64_t)min(m0 + WM * wm + (lane & (WM - 1)), P.M - 1) * P.ldas;
  const uint8_t* swp = P.Ws + (int64_t)min(n0 + 64 * wn + lane, P.N - 1) * P.ldws;
  int sna, snw, sna1 = 0, snw1 = 0, sc[NF];
  auto load_scales = [&](int g) {  // of slices k0 + 4 g .. + 3; KG = 2: from two dwords
    const int at = 4 * min((k0 >> 2) + g, (nk - 1) >> 2);
    sna = *(const int*)(sap + at);
    snw = *(const int*)(swp + at);
    if constexpr (KG == 2) {
      const int next = 4 * min((k0 >> 2) + g + 1, (nk - 1) >> 2);
      sna1 = *(const int*)(sap + next);
      snw1 = *(const int*)(swp + next);
    }
  };
  uint32_t too_large = 0;
  auto spread_scales = [&](int slices) {  // that are left
    if constexpr (KG == 2) {
      sna = __builtin_amdgcn_alignbyte(sna1, sna, k0 & 3);
      snw = __builtin_amdgcn_alignbyte(snw1, snw, k0 & 3);
    }
    if constexpr (WIDE) {  // (a byte past 255 carries into the next slice's, but is too large)
      too_large |= any_too_large(sna, slices) | any_too_large(snw, slices);
      sna += 0x01010101 * UP;
      snw += 0x01010101 * UP;
    }
#pragma unroll
    for (int f = 0; f < NF; ++f)
      sc[f] = __builtin_amdgcn_ds_bpermute(4 * lr + 64 * (f < TM ? f : f - TM), f < TM ? sna : snw);
  };
  int loff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) loff[h] = lr * 128 + (((4 * h + lq) ^ ((lr >> 1) & 7)) << 4);
  auto rd = [&](int u, int f) {  // fragment f: A, then W
    const int at = u + (f < TM ? wm * WM * 128 + f * 2048 : BM * 128 + wn * 64 * 128 + (f - TM) * 2048);
    return lds_frag(smem + at + loff[0], smem + at + loff[1]);
  };
  f32x4_t acc[TM][TN] = {};

  load_scales(0);
#pragma unroll
  for (int s = 0; s < ST; ++s)
#pragma unroll
    for (int j = 0; j < INS; ++j) issue1(s * SLICE, k0 + s, j);
  wait_vmcnt<(ST - 1) * INS>();  // scales and slice 0 have landed
  barrier_no_fence();
  i32x8_t f0[NF], other[WIDE ? 1 : NF];
  auto& f1 = [&]() -> auto& {
    if constexpr (WIDE) return f0;
    else return other;
  }();
#pragma unroll
  for (int f = 0; f < NF; ++f) f0[f] = rd(0, f);
  spread_scales(k1 - k0);
  int u = 0;  // place of slice kt
  auto step = [&](int kt, i32x8_t(&f)[NF], i32x8_t(&fn)[NF], auto b_) {
    constexpr int B = decltype(b_)::value;
    const int un = u == (ST - 1) * SLICE ? 0 : u + SLICE;
    // this wave's reads of slice kt and its copies of slice kt + 1 are done (those
    // of the next ST - 2 may stay in flight); then everyone's are
    wait_vmcnt_lgkm0<(ST - 2) * INS>();
    barrier_no_fence();
    if constexpr (B == 0) load_scales(((kt - k0) >> 2) + 1);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (WIDE) {
      // A widened, then W's fragments one ahead of their MFMAs; a fragment's registers take
      // that of the next slice as soon as it is widened (f and fn are the same)
      bf16x8_t aw[TM][4], wv[2][4];
#pragma unroll
      for (int i = 0; i < TM; ++i) widen(f[i], sc[i] >> (8 * B), aw[i]);
      widen(f[TM], sc[TM] >> (8 * B), wv[0]);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        fn[TM + j] = rd(un, TM + j);
#pragma unroll
        for (int i = 0; i < TM; ++i)
          if (j == TN - 2) fn[i] = rd(un, i);
#pragma unroll
        for (int c = j * INS / TN; c < (j + 1) * INS / TN; ++c) issue1(u, kt + ST, c);
        if (j + 1 < TN) widen(f[TM + j + 1], sc[TM + j + 1] >> (8 * B), wv[(j + 1) & 1]);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < TM; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aw[i][t], wv[j & 1][t], acc[i][j], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    } else {
#pragma unroll
      for (int q = 0; q < TM * TN; ++q) {
        const int i = q % TM, j = q / TM;
        acc[i][j] = mfma_scaled<B>(f[i], f[TM + j], acc[i][j], sc[i], sc[TM + j]);
        __builtin_amdgcn_sched_barrier(0);
        // in the order of their use: A 0, W 0, the other A, the other W
        if (q < NF) {
          const int x = q == 0 ? 0 : q == 1 ? TM : q <= TM ? q - 1 : q;
          fn[x] = rd(un, x);
        }
        if (q >= TM * TN - INS) issue1(u, kt + ST, q - (TM * TN - INS));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (B == 3) spread_scales(k1 - kt - 1);
    u = un;
  };
  using std::integral_constant;
  int kt = k0;
  for (; kt + 4 <= k1; kt += 4) {
    step(kt, f0, f1, integral_constant<int, 0>{});
    step(kt + 1, f1, f0, integral_constant<int, 1>{});
    step(kt + 2, f0, f1, integral_constant<int, 2>{});
    step(kt + 3, f1, f0, integral_constant<int, 3>{});
  }
  if (kt < k1) step(kt, f0, f1, integral_constant<int, 0>{});
  if (kt + 1 < k1) step(kt + 1, f1, f0, integral_constant<int, 1>{});
  if (kt + 2 < k1) step(kt + 2, f0, f1, integral_constant<int, 2>{});
  if constexpr (KG == 2)
    for (int i = k1 - k0; i < half; ++i) barrier_no_fence();  // the first group may have one more step
  if constexpr (WIDE) finish_wide<TM, TN>(P, m0 + wm * WM, n0 + 64 * wn, k0, k1, too_large != 0, acc);
  __builtin_amdgcn_s_waitcnt(0);  // the copies past the end have landed
  __syncthreads();
  // The tile in LDS as slabs of ROWS rows x 128, one per wave, columns XOR 16
  // ((row >> 2) & MASK): then each wave has whole 128-column rows.
  constexpr int ROWS = BM / (NW * KG), MASK = ROWS == 8 ? 1 : 3;
  float* tile = (float*)lds + grp * (BM * 128);
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        tile[(wm * WM + 16 * i + 4 * lq + r) * 128 + ((64 * wn + 16 * j + lr) ^ ((lq & MASK) << 4))] = acc[i][j][r];
  __syncthreads();
  const int slab = grp * NW + wave;
  float* mine = (float*)lds + ROWS * slab * 128;
  if constexpr (KG == 2) {
#pragma unroll
    for (int i = 0; i < ROWS / 2; ++i) {
      f32x4_t* x = (f32x4_t*)mine + 64 * i + lane;
      *x += x[BM * 32];
    }
  }
  EpiLds<KIND> epi(P, m0 + ROWS * slab, n0, lane & 31, lane >> 5, mine);
  epi.prep();
  uint2 old[8][2];
  if (epi.gated) epi.load_old(0, old);
  epi.template slab_rows<MASK, 4, ROWS>(0, old);
}

// Few rows or few tiles: 16 RB x NT outputs per work-group, eight waves of 16 RB x 32
// that share K (NT = 32: eight ways, 64: four, 128: two).  Each wave copies its own
// rows' slices to a ring of its own in LDS, so that no wave waits for another until
// their sums meet at the end; the copies read whole 128-byte lines, eight lanes
// each (fragments loaded to registers, 16 rows an instruction, take a CU longer
// than the memory does: 8 x 5120 x 13824 20.7 us).  Bound by the way of W from
// memory: 8 x 5120 x 13824 13.8 us, 5.1 TB/s; 1 x 13824 x 5120 13.6 us, 5.2 TB/s.
template <int NT, int RB, int KIND, bool WIDE>
__global__ __launch_bounds__(512) void gemm_fp8_small_kernel(Fp8Prob P) {
  constexpr int NH = NT / 32, KS = 8 / NH, NF = 2 + RB, ST = RB == 1 ? 3 : 2;
  constexpr int INS = 2 * NF, SLICE = INS * 1024 + 256, LD = 36;  // W's two fragments, A's, scales
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
  // scales of four slices of row lane: 32 of W, 16 RB of A
  const uint8_t* sp = lane < 32 ? P.Ws + (int64_t)min(nw + lane, P.N - 1) * P.ldws
                                : P.As + (int64_t)min(m0 + (lane - 32) % (16 * RB), P.M - 1) * P.ldas;
  const int steps = (P.K + 127) >> 7, per = (steps + KS - 1) / KS;
  const int s0 = ks * per, s1 = min(steps, s0 + per);
  char* ring = smem + wave * (ST * SLICE);
  // slice s of K (past the wave's last one: zeros) and its scales
  auto issue = [&](int s, int u) {
    const int left = s < s1 ? P.K - 128 * s : 0;
    copy4(sp + 4 * (min(s, steps - 1) >> 2), (lds_void_t*)(ring + u * SLICE + INS * 1024));
#pragma unroll
    for (int j = 0; j < INS; ++j)
      copy16_oob(j < 4 ? Wb : Ab, (lds_void_t*)(ring + u * SLICE + j * 1024), ch[j] < left ? off[j] : OOB, (uint32_t)s * 128);
  };
  int loff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) loff[h] = lr * 128 + (((4 * h + lq) ^ ((lr >> 1) & 7)) << 4);
  f32x4_t acc[RB][2] = {};
  int largest = 0;
#pragma unroll
  for (int u = 0; u < ST; ++u) issue(s0 + u, u);
  for (int s = s0; s < s1; s += ST) {
#pragma unroll
    for (int u = 0; u < ST; ++u) {  // (a slice past s1 adds zeros)
      wait_vmcnt<(ST - 1) * (INS + 1)>();  // this slice and its scales have landed
      asm volatile("" ::: "memory");
      i32x8_t f[NF];
      int b[NF];
#pragma unroll
      for (int i = 0; i < NF; ++i) {
        f[i] = lds_frag(ring + u * SLICE + i * 2048 + loff[0], ring + u * SLICE + i * 2048 + loff[1]);
        const int x = *(const int*)(ring + u * SLICE + INS * 1024 + 4 * (16 * i + lr));
        b[i] = (x >> (8 * ((s + u) & 3))) & (s + u < s1 ? 255 : 0);
      }
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): read, its place is free
      asm volatile("" ::: "memory");
      issue(s + u + ST, u);
      if constexpr (WIDE) {
        bf16x8_t w[2][4];
#pragma unroll
        for (int i = 0; i < NF; ++i) largest = max(largest, b[i]);
        widen(f[0], b[0] + UP, w[0]);
        widen(f[1], b[1] + UP, w[1]);
#pragma unroll
        for (int i = 0; i < RB; ++i) {
          bf16x8_t a[4];
          widen(f[2 + i], b[2 + i] + UP, a);
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], w[j][t], acc[i][j], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = mfma_scaled(f[2 + i], f[j], acc[i][j], b[2 + i], b[j]);
      }
    }
  }
  if constexpr (WIDE) finish_wide<RB, 2>(P, m0, nw, s0, s1, largest > LAST_BYTE, acc);
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
    uint32_t byte = 127;
    float inv = 1.f;
    if constexpr (KIND == EPI_K_FP8) {
      top = max_over<16>(top);
      top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
      byte = e8m0_of(top);
      inv = e8m0_inverse(byte);
    }
    if (m >= P.M || n >= P.N) continue;
    if constexpr (KIND == EPI_K_FP8) {
      *(uint32_t*)((uint8_t*)P.C + (int64_t)m * P.ldc + n) = pack_fp8x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
      if (c == 0) P.Cs[(int64_t)m * P.ldcs + (n >> 7)] = (uint8_t)byte;
      continue;
    }
    const int64_t at = (int64_t)m * P.ldc + n + (n >= P.gap_at ? P.gap : 0);
    if constexpr (WIDE) {
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

hipError_t launch_quant_fp8(const void* x, bool bf16, int64_t ldx, void* q, int64_t ldq, void* scale, int64_t lds, int M,
                            int K, hipStream_t s) {
  if (M == 0 || K == 0) return hipSuccess;
  const int per_row = (K + 1023) / 1024;
  const int64_t groups = ((int64_t)M * per_row + 3) / 4;
  if (bf16)
    hipLaunchKernelGGL(quant_fp8_kernel<bf16_t>, dim3((uint32_t)groups), dim3(256), 0, s, (const bf16_t*)x, ldx,
                       (uint8_t*)q, ldq, (uint8_t*)scale, lds, M, K, per_row);
  else
    hipLaunchKernelGGL(quant_fp8_kernel<float>, dim3((uint32_t)groups), dim3(256), 0, s, (const float*)x, ldx,
                       (uint8_t*)q, ldq, (uint8_t*)scale, lds, M, K, per_row);
  return hipGetLastError();
}

hipError_t launch_gemm_fp8(const GemmFp8Args& g, hipStream_t s, int n_cu) {
  if (g.M == 0 || g.N == 0) return hipSuccess;
  const bool f32 = g.flags & DIT_EPI_F32, fp8 = g.flags & DIT_EPI_FP8, gated = g.flags & DIT_EPI_GATED_RES;
  const bool groups = g.rms_cols > 0 || fp8;  // need a 128-column group in one place
  Fp8Prob p{};
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
  auto tiles = [&](int bm, int bn) { return (int64_t)((g.M + bm - 1) / bm) * ((g.N + bn - 1) / bn); };
  auto go = [&](void (*fn)(Fp8Prob), int bm, int bn, int threads) {
    p.tiles_m = (g.M + bm - 1) / bm;
    p.tiles_n = (g.N + bn - 1) / bn;
    hipLaunchKernelGGL(fn, dim3((uint32_t)p.tiles_m * p.tiles_n), dim3(threads), 0, s, p);
    return hipGetLastError();
  };
  const bool plain = !(g.flags & DIT_EPI_SILU);
  const bool store = plain && !gated && !fp8 && (g.gelu_from >= g.N || g.gelu_from % 128 == 0) &&
                     (g.gap == 0 || g.gap_at % 128 == 0);
  const bool only_gate = plain && gated && g.rms_cols == 0 && g.gelu_from >= g.N && g.gap == 0;
  // Few rows or few tiles: the narrowest tiles that fit the CUs once, to spread the
  // way of W over them.  In us, these tiles (their width) and 64 x 128 ones: 1 x 5120 x 5120 9 (32) and 17, 8 x
  // 5120 x 13824 13.8 (32) and 37, 64 x 5120 x 5120 12 (64) and 18, 32 x 16384 x 5120 16 (64) and 19, 1 x 28672 x
  // 5120 29 (128) and 30.  128 columns of 32 rows only for f32, 128 x 8192 x 5120 21 and 26; bf16
  // 19.5 and 18.6, 32 x 28672 x 5120 39 and 33.  Two rounds of them lose: 512 x 2560 x 5120 35 and 19.
  const bool one = g.M <= 16;
  const int rows = one ? 16 : 32, widest = one || f32 ? 128 : 64;
  int nt = groups ? 128 : 32;
  while (nt < widest && tiles(rows, nt) > n_cu) nt *= 2;
  if (nt <= widest && tiles(rows, nt) <= n_cu) {
    if (fp8) return go(gemm_fp8_small_kernel<128, 1, EPI_K_FP8, false>, rows, 128, 512);
    if (f32 && one)
      return go(nt == 128  ? gemm_fp8_small_kernel<128, 1, EPI_K_ANY, true>
                : nt == 64 ? gemm_fp8_small_kernel<64, 1, EPI_K_ANY, true>
                           : gemm_fp8_small_kernel<32, 1, EPI_K_ANY, true>, rows, nt, 512);
    if (f32)
      return go(nt == 128  ? gemm_fp8_small_kernel<128, 2, EPI_K_ANY, true>
                : nt == 64 ? gemm_fp8_small_kernel<64, 2, EPI_K_ANY, true>
                           : gemm_fp8_small_kernel<32, 2, EPI_K_ANY, true>, rows, nt, 512);
    if (one)
      return go(nt == 128  ? gemm_fp8_small_kernel<128, 1, EPI_K_ANY, false>
                : nt == 64 ? gemm_fp8_small_kernel<64, 1, EPI_K_ANY, false>
                           : gemm_fp8_small_kernel<32, 1, EPI_K_ANY, false>, rows, nt, 512);
    return go(nt == 64 ? gemm_fp8_small_kernel<64, 2, EPI_K_ANY, false> : gemm_fp8_small_kernel<32, 2, EPI_K_ANY, false>,
              rows, nt, 512);
  }
  // Rounds of the chip times a tile's time, which is 4 us and some per slice of 128 of K
  // (fitted to each kernel alone over the sizes below).  In us, 64 x 128, 128 x 128, 256 x 128 and 256 x 256 tiles:
  //   512 x 10240 x 5120  45 44 36 56    1024 x 10240 x 5120 75 81 76 55    512 x 5120 x 5120  29 39 37 56
  //   2048 x 4096 x 4096  50 40 36 51    4096 x 4096 x 1024  39 32 32 23    1333 x 1000 x 2320 13 25 27 37
  // and f32 outputs on 64 x 128 and 128 x 128 tiles:
  //   4096 x 4096 x 4096 147 122   32760 x 5120 x 2048 794 668   512 x 10240 x 5120 66 68   32760 x 64 x 5120 54 64
  struct Tile { int bm, bn, per_cu; double slice_us; };
  auto cost = [&](const Tile& c) {
    const int64_t slots = (int64_t)n_cu * c.per_cu;
    return (double)((tiles(c.bm, c.bn) + slots - 1) / slots) * ((g.K + 127) / 128 * c.slice_us + 4);
  };
  if (f32) {
    // One work-group per CU: two groups of waves, one's widening beside the other's
    // products, where either has some slices.  256 x 5120 x 5120 31.5 -> 24.6 us,
    // 1333 x 1000 x 2320 18.6 -> 16.8 (512 x 4096 x 528: 10.1 and 10.3).  It gives bf16 outputs nothing
    // (256 x 5120 x 5120 18.6 and 18.4 us, 1333 x 1000 x 2320 12.8 and 13.5).
    if (tiles(64, 128) <= n_cu && g.K > 1024) return go(gemm_fp8_tile_kernel<64, EPI_K_ANY, true, 2>, 64, 128, 512);
    if (cost({64, 128, 2, 1.02}) <= cost({128, 128, 2, 1.78}))
      return go(gemm_fp8_tile_kernel<64, EPI_K_ANY, true>, 64, 128, 256);
    return go(gemm_fp8_tile_kernel<128, EPI_K_ANY, true>, 128, 128, 256);
  }
  const Tile cfg[] = {{64, 128, 2, 0.62}, {128, 128, 2, 1.0}, {256, 128, 1, 0.95}, {256, 256, 1, 1.5}};
  int best = 0;
  for (int c = 1; c < 4; ++c)
    if (cost(cfg[c]) < cost(cfg[best])) best = c;
  if (best == 3)
    return go(fp8 ? gemm_fp8_ring_kernel<EPI_K_FP8> : store ? gemm_fp8_ring_kernel<EPI_K_STORE>
              : only_gate ? gemm_fp8_ring_kernel<EPI_K_GATED> : gemm_fp8_ring_kernel<EPI_K_ANY>, 256, 256, 512);
  if (best == 2)
    return go(fp8 ? gemm_fp8_tile_kernel<256, EPI_K_FP8, false> : store ? gemm_fp8_tile_kernel<256, EPI_K_STORE, false>
              : gemm_fp8_tile_kernel<256, EPI_K_ANY, false>, 256, 128, 512);
  if (best == 1)
    return go(fp8 ? gemm_fp8_tile_kernel<128, EPI_K_FP8, false> : store ? gemm_fp8_tile_kernel<128, EPI_K_STORE, false>
              : gemm_fp8_tile_kernel<128, EPI_K_ANY, false>, 128, 128, 256);
  return go(fp8 ? gemm_fp8_tile_kernel<64, EPI_K_FP8, false> : store ? gemm_fp8_tile_kernel<64, EPI_K_STORE, false>
              : gemm_fp8_tile_kernel<64, EPI_K_ANY, false>, 64, 128, 256);
}

}  // namespace dit
