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
// with their scale in registers (exact) and multiplied by bf16 MFMAs (WIDE).
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
// row.  One pass: bound by the copy rate.
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
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
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

// The 128 x 128-deep step of one 16 x 16 block.  A lane holds row lr's 16-byte
// chunks lq and lq + 4 of the block of 128 (the sum over k does not mind their
// order, and these are the chunks that a swizzled LDS row serves without bank
// conflicts).  sa and sw: scale bytes of the lane's rows in bits 0..7.
__device__ __forceinline__ f32x4_t mfma_scaled(const i32x8_t& a, const i32x8_t& w, const f32x4_t& c, int sa, int sw) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, w, c, 0, 0, 0, sa, 0, sw);
#else
  return c;
#endif
}

__device__ __forceinline__ i32x8_t frag8(const uint4& lo, const uint4& hi) {
  return i32x8_t{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

// The fragment widened to bf16, times its row's scale: four 32-deep operands.
// (The conversion reads the scale's exponent bits only: byte << 23 is 2^(byte - 127)
// at either end of the range, too.)
__device__ __forceinline__ void widen(const i32x8_t& f, int scale, bf16x8_t (&w)[4]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const float s = __uint_as_float((uint32_t)(scale & 255) << 23);
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
// XOR-swizzled by ((row >> 1) & 7)).
//
// A slice is one MFMA step: eight groups of four MFMAs, group j with W
// fragment j and the wave's four A fragments.  W fragments are read two
// groups ahead, each A fragment of the next slice right after its last MFMA.
// The work-groups' waves meet before group 6, where the next slice's first
// reads begin: by then every read of this slice is done, so its two units take
// A slice kt + 2 and W slice kt + 3.  Slices past the last one are copied as
// zeros (no memory traffic), which keeps every iteration and wait the same.
template <int KIND>
__global__ __launch_bounds__(512) void gemm_fp8_ring_kernel(Fp8Prob P) {
  constexpr int UNIT = 256 * 128, INS = 4, TM = 4, TN = 8;
  __shared__ __attribute__((aligned(1024))) char smem[5 * UNIT];
  int tm, tn;
  tile_at(P, xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n), tm, tn);
  const int m0 = tm * 256, n0 = tn * 256;
  const int nk = (P.K + 127) >> 7;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int lr = lane & 15, lq = lane >> 4;

  // copy j of this wave moves rows 8 (4 wave + j) .. + 7 of an operand's slice
  const uint8_t* Ab = P.A + (int64_t)m0 * P.lda;
  const uint8_t* Wb = P.W + (int64_t)n0 * P.ldw;
  uint32_t aoff[INS], woff[INS];
#pragma unroll
  for (int j = 0; j < INS; ++j) {
    const int row = 8 * (wave * INS + j) + (lane >> 3);
    const int c = (lane & 7) ^ ((row >> 1) & 7);
    aoff[j] = (uint32_t)min(row, P.M - 1 - m0) * (uint32_t)P.lda + c * 16;
    woff[j] = (uint32_t)min(row, P.N - 1 - n0) * (uint32_t)P.ldw + c * 16;
  }
  auto issue = [&](const uint8_t* base, const uint32_t (&off)[INS], int u, int s) {
    char* d = smem + u;
    const int left = P.K - 128 * s;
#pragma unroll
    for (int j = 0; j < INS; ++j) {
      const int c = (lane & 7) ^ (((4 * j + (lane >> 4))) & 7);  // chunk of copy j (4 wave INS is a multiple of 8)
      copy16_oob(base, (lds_void_t*)(d + (wave * INS + j) * 1024), 16 * c < left ? off[j] : OOB, (uint32_t)s * 128);
    }
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
    for (int i = 0; i < TM; ++i) sa[i] = __builtin_amdgcn_ds_bpermute(4 * (16 * i + lr), sna);
#pragma unroll
    for (int j = 0; j < TN; ++j) sw[j] = __builtin_amdgcn_ds_bpermute(4 * (16 * (j & 3) + lr), j < 4 ? snw0 : snw1);
  };

  int loff[2];  // this lane's two chunks inside 16 rows of a unit
#pragma unroll
  for (int h = 0; h < 2; ++h) loff[h] = lr * 128 + (((4 * h + lq) ^ ((lr >> 1) & 7)) << 4);
  auto rd = [&](int at) {
    return frag8(*(const uint4*)(smem + at + loff[0]), *(const uint4*)(smem + at + loff[1]));
  };
  f32x4_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // W slice kt in unit kt % 3, A slice kt in unit 3 + kt % 2
  int wu = 0, au = 3 * UNIT;
  auto next_w = [](int u) { return u == 2 * UNIT ? 0 : u + UNIT; };
  load_scales(0);
  issue(Wb, woff, 0, 0);
  issue(Ab, aoff, 3 * UNIT, 0);
  issue(Wb, woff, UNIT, 1);
  issue(Ab, aoff, 4 * UNIT, 1);
  issue(Wb, woff, 2 * UNIT, 2);
  wait_vmcnt<3 * INS>();  // scales and slice 0 have landed
  barrier_no_fence();
  i32x8_t a[TM], w[4];
  const int wa = wm * 64 * 128, ww = wn * 128 * 128;
#pragma unroll
  for (int i = 0; i < TM; ++i) a[i] = rd(au + wa + i * 2048);
  w[0] = rd(wu + ww);
  w[1] = rd(wu + ww + 2048);
  for (int kt = 0; kt < nk; ++kt) {
    if ((kt & 3) == 0) {
      spread_scales();
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = (int)((uint32_t)sa[i] >> 8);
#pragma unroll
      for (int j = 0; j < TN; ++j) sw[j] = (int)((uint32_t)sw[j] >> 8);
    }
    const int wn_ = next_w(wu), an_ = 7 * UNIT - au;
#pragma unroll
    for (int j = 0; j < 6; ++j) {
      w[(j + 2) & 3] = rd(wu + ww + (j + 2) * 2048);
#pragma unroll
      for (int i = 0; i < TM; ++i) acc[i][j] = mfma_scaled(a[i], w[j & 3], acc[i][j], sa[i], sw[j]);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    // this wave's reads of slice kt and its copies of slice kt + 1 are done (W
    // slice kt + 2 may stay in flight); then everyone's are
    wait_vmcnt_lgkm0<INS>();
    barrier_no_fence();
    issue(Ab, aoff, au, kt + 2);
    if ((kt & 3) == 0) load_scales((kt >> 2) + 1);
    issue(Wb, woff, wu, kt + 3);
    __builtin_amdgcn_sched_barrier(0);
    w[0] = rd(wn_ + ww);
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[i][6] = mfma_scaled(a[i], w[2], acc[i][6], sa[i], sw[6]);
    __builtin_amdgcn_sched_barrier(0);
    w[1] = rd(wn_ + ww + 2048);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      acc[i][7] = mfma_scaled(a[i], w[3], acc[i][7], sa[i], sw[7]);
      __builtin_amdgcn_sched_barrier(0);
      a[i] = rd(an_ + wa + i * 2048);
      __builtin_amdgcn_sched_barrier(0);
    }
    wu = wn_;
    au = an_;
  }
  __builtin_amdgcn_s_waitcnt(0);  // the copies past the end have landed
  __syncthreads();
  EpiLds<KIND> epi(P, m0 + 64 * wm, n0 + 128 * wn, lane & 31, lane >> 5, (float*)smem + wave * (32 * 128));
  epi.prep();
  uint2 old[2][8][2];
  if (epi.gated) { epi.load_old(0, old[0]); epi.load_old(1, old[1]); }
  epi.slab_pass16(acc[0], acc[1], 0, old[0], lr, lq);
  epi.slab_pass16(acc[2], acc[3], 1, old[1], lr, lq);
}

// BM x 128 tiles, four waves of BM / 2 x 64, two work-groups per CU, ST slices
// of 128 of K in LDS.  For launches that 256 x 256 tiles would not fill, short
// K, and (WIDE) f32 outputs.
template <int BM, int ST, int KIND, bool WIDE>
__global__ __launch_bounds__(256, 2) void gemm_fp8_tile_kernel(Fp8Prob P) {
  constexpr int TM = BM / 32, TN = 4, NW = 4;
  constexpr int SLICE = (BM + 128) * 128;
  constexpr int A_INS = BM / 8 / NW, W_INS = 128 / 8 / NW;
  constexpr int EPI = BM * 128 * 4;
  __shared__ __attribute__((aligned(1024))) char smem[ST * SLICE > EPI ? ST * SLICE : EPI];
  int tm, tn;
  tile_at(P, xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n), tm, tn);
  const int m0 = tm * BM, n0 = tn * 128;
  const int nk = (P.K + 127) >> 7;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int lr = lane & 15, lq = lane >> 4;

  const uint8_t* Ab = P.A + (int64_t)m0 * P.lda;
  const uint8_t* Wb = P.W + (int64_t)n0 * P.ldw;
  uint32_t aoff[A_INS], woff[W_INS];
  int ac[A_INS], wc[W_INS];
#pragma unroll
  for (int j = 0; j < A_INS; ++j) {
    const int row = 8 * (wave * A_INS + j) + (lane >> 3);
    ac[j] = 16 * ((lane & 7) ^ ((row >> 1) & 7));
    aoff[j] = (uint32_t)min(row, P.M - 1 - m0) * (uint32_t)P.lda + ac[j];
  }
#pragma unroll
  for (int j = 0; j < W_INS; ++j) {
    const int row = 8 * (wave * W_INS + j) + (lane >> 3);
    wc[j] = 16 * ((lane & 7) ^ ((row >> 1) & 7));
    woff[j] = (uint32_t)min(row, P.N - 1 - n0) * (uint32_t)P.ldw + wc[j];
  }
  auto issue = [&](int s) {
    char* d = smem + (s % ST) * SLICE;
    const int left = P.K - 128 * s;
#pragma unroll
    for (int j = 0; j < A_INS; ++j)
      copy16_oob(Ab, (lds_void_t*)(d + (wave * A_INS + j) * 1024), ac[j] < left ? aoff[j] : OOB, (uint32_t)s * 128);
#pragma unroll
    for (int j = 0; j < W_INS; ++j)
      copy16_oob(Wb, (lds_void_t*)(d + BM * 128 + (wave * W_INS + j) * 1024), wc[j] < left ? woff[j] : OOB,
                 (uint32_t)s * 128);
  };
  const uint8_t *sap[TM], *swp[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) sap[i] = P.As + (int64_t)min(m0 + wm * (BM / 2) + 16 * i + lr, P.M - 1) * P.ldas;
#pragma unroll
  for (int j = 0; j < TN; ++j) swp[j] = P.Ws + (int64_t)min(n0 + 64 * wn + 16 * j + lr, P.N - 1) * P.ldws;
  int sa[TM], sw[TN], sna[TM], snw[TN];
  auto load_scales = [&](int g) {
    const int at = 4 * min(g, (nk - 1) >> 2);
#pragma unroll
    for (int i = 0; i < TM; ++i) sna[i] = *(const int*)(sap[i] + at);
#pragma unroll
    for (int j = 0; j < TN; ++j) snw[j] = *(const int*)(swp[j] + at);
  };
  int loff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) loff[h] = lr * 128 + (((4 * h + lq) ^ ((lr >> 1) & 7)) << 4);
  f32x4_t acc[TM][TN] = {};

  load_scales(0);
#pragma unroll
  for (int s = 0; s < ST - 1; ++s) issue(s);
  for (int kt = 0; kt < nk; ++kt) {
    // slice kt has landed and this wave's reads of slice kt - 1 are done; then everyone's
    wait_vmcnt_lgkm0<(ST - 2) * (A_INS + W_INS)>();
    barrier_no_fence();
    if ((kt & 3) == 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = sna[i];
#pragma unroll
      for (int j = 0; j < TN; ++j) sw[j] = snw[j];
      load_scales((kt >> 2) + 1);
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = (int)((uint32_t)sa[i] >> 8);
#pragma unroll
      for (int j = 0; j < TN; ++j) sw[j] = (int)((uint32_t)sw[j] >> 8);
    }
    issue(kt + ST - 1);
    const char* sA = smem + (kt % ST) * SLICE + wm * (BM / 2) * 128;
    const char* sW = smem + (kt % ST) * SLICE + BM * 128 + wn * 64 * 128;
    i32x8_t a[TM], w[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
      a[i] = frag8(*(const uint4*)(sA + i * 2048 + loff[0]), *(const uint4*)(sA + i * 2048 + loff[1]));
#pragma unroll
    for (int j = 0; j < TN; ++j)
      w[j] = frag8(*(const uint4*)(sW + j * 2048 + loff[0]), *(const uint4*)(sW + j * 2048 + loff[1]));
    if constexpr (WIDE) {
      bf16x8_t aw[TM][4];
#pragma unroll
      for (int i = 0; i < TM; ++i) widen(a[i], sa[i], aw[i]);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        bf16x8_t wv[4];
        widen(w[j], sw[j], wv);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < TM; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aw[i][t], wv[t], acc[i][j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[i][j] = mfma_scaled(a[i], w[j], acc[i][j], sa[i], sw[j]);
    }
  }
  __builtin_amdgcn_s_waitcnt(0);  // the copies past the end have landed
  __syncthreads();
  // The tile in LDS as slabs of 32 (BM = 32: 8) rows x 128, one per wave, columns
  // XOR 16 ((row >> 2) & 3): then each wave has whole 128-column rows.
  float* tile = (float*)smem;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        tile[(wm * (BM / 2) + 16 * i + 4 * lq + r) * 128 + ((64 * wn + 16 * j + lr) ^ (lq << 4))] = acc[i][j][r];
  __syncthreads();
  constexpr int ROWS = BM / NW;
  EpiLds<KIND> epi(P, m0 + ROWS * wave, n0, lane & 31, lane >> 5, tile + ROWS * wave * 128);
  epi.prep();
  uint2 old[8][2];
  if (epi.gated) epi.load_old(0, old);
  epi.template slab_rows<3, 4, ROWS>(0, old);
}

// Few rows or few tiles: 16 RB x NT outputs per work-group, operands straight
// from global memory into the fragments, K shared by its eight waves (NT = 128:
// by four, the other four take the second 64 columns).
template <int NT, int RB, int KIND, bool WIDE>
__global__ __launch_bounds__(512) void gemm_fp8_small_kernel(Fp8Prob P) {
  constexpr int NH = NT / 64, KS = 8 / NH, LD = 68;
  __shared__ __attribute__((aligned(16))) float part[8][16 * RB][LD];
  const int lt = xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n);
  const int m0 = lt % P.tiles_m * (16 * RB), n0 = lt / P.tiles_m * NT;  // neighbours share the weights
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int ks = wave % KS, nh = wave / KS;
  const uint8_t *ap[RB], *wp[4], *sap[RB], *swp[4];
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const int64_t r = min(m0 + 16 * i + lr, P.M - 1);
    ap[i] = P.A + r * P.lda;
    sap[i] = P.As + r * P.ldas;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = min(n0 + 64 * nh + 16 * j + lr, P.N - 1);
    wp[j] = P.W + r * P.ldw;
    swp[j] = P.Ws + r * P.ldws;
  }
  const int steps = (P.K + 127) >> 7, per = (steps + KS - 1) / KS;
  const int s0 = ks * per, s1 = min(steps, s0 + per);
  f32x4_t acc[RB][4] = {};
  auto load16 = [&](const uint8_t* p, int k) {
    const uint4 v = *(const uint4*)(p + min(k, P.K - 16));
    return k < P.K ? v : make_uint4(0, 0, 0, 0);
  };
  auto load = [&](const uint8_t* p, int s) { return frag8(load16(p, 128 * s + 16 * lq), load16(p, 128 * s + 64 + 16 * lq)); };
  constexpr int U = 2;  // steps whose loads are in flight together
  for (int s = s0; s < s1; s += U) {
    i32x8_t a[U][RB], w[U][4];
    int sa[U][RB], sw[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= s1) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) { w[u][j] = load(wp[j], s + u); sw[u][j] = swp[j][s + u]; }
#pragma unroll
      for (int i = 0; i < RB; ++i) { a[u][i] = load(ap[i], s + u); sa[u][i] = sap[i][s + u]; }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= s1) break;
      if constexpr (WIDE) {
        bf16x8_t aw[RB][4];
#pragma unroll
        for (int i = 0; i < RB; ++i) widen(a[u][i], sa[u][i], aw[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bf16x8_t wv[4];
          widen(w[u][j], sw[u][j], wv);
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < RB; ++i)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aw[i][t], wv[t], acc[i][j], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < RB; ++i) acc[i][j] = mfma_scaled(a[u][i], w[u][j], acc[i][j], sa[u][i], sw[u][j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[wave][16 * i + 4 * lq + r][16 * j + lr] = acc[i][j][r];
  __syncthreads();

  // 16 threads per row: columns 4 c .. + 3 of each half, added in wave order
  const int row = tid >> 4, c = tid & 15, m = m0 + row;
  if (row >= 16 * RB) return;  // whole waves
  float v[NH][4];
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    const int n = n0 + 64 * h + 4 * c;
    f32x4_t t = {};
#pragma unroll
    for (int w = 0; w < KS; ++w) t += *(const f32x4_t*)&part[KS * h + w][row][4 * c];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[h][e] = t[e] + (P.bias && n < P.N ? bf16_to_f32(P.bias[n + e]) : 0.f);
  }
  if constexpr (NT == 128) {
    if (n0 < P.rms_cols) {  // one 128-wide head per tile
      float ss = 0.f;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) ss += v[h][e] * v[h][e];
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) ss += __shfl_xor(ss, o, 64);
      const float sc = rsqrtf(ss * (1.f / 128.f) + DIT_RMS_EPS);
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[h][e] *= sc;
    }
  }
  uint32_t top = 0;
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    const int n = n0 + 64 * h + 4 * c;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (n >= P.gelu_from) v[h][e] = gelu_tanh_f(v[h][e]);
      if (P.flags & DIT_EPI_SILU) v[h][e] = silu_f(v[h][e]);
      top = max(top, __float_as_uint(v[h][e]) & 0x7fffffffu);
    }
  }
  uint32_t byte = 127;
  float inv = 1.f;
  if constexpr (KIND == EPI_K_FP8) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    byte = e8m0_of(top);
    inv = e8m0_inverse(byte);
  }
  if (m >= P.M) return;
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    const int n = n0 + 64 * h + 4 * c;
    if (n >= P.N) continue;
    if constexpr (KIND == EPI_K_FP8) {
      *(uint32_t*)((uint8_t*)P.C + (int64_t)m * P.ldc + n) =
          pack_fp8x4(v[h][0] * inv, v[h][1] * inv, v[h][2] * inv, v[h][3] * inv);
      if (n % 128 == 0) P.Cs[(int64_t)m * P.ldcs + (n >> 7)] = (uint8_t)byte;
      continue;
    }
    const int64_t at = (int64_t)m * P.ldc + n + (n >= P.gap_at ? P.gap : 0);
    if constexpr (WIDE) {
      *(float4*)((float*)P.C + at) = make_float4(v[h][0], v[h][1], v[h][2], v[h][3]);
      continue;
    }
    uint2* o = (uint2*)((bf16_t*)P.C + at);
    if (P.flags & DIT_EPI_GATED_RES) {
      const uint2 x = *o;
      const float4 g = *(const float4*)(P.gate + n);
      v[h][0] = __uint_as_float(x.x << 16) + g.x * v[h][0];
      v[h][1] = __uint_as_float(x.x & 0xffff0000u) + g.y * v[h][1];
      v[h][2] = __uint_as_float(x.y << 16) + g.z * v[h][2];
      v[h][3] = __uint_as_float(x.y & 0xffff0000u) + g.w * v[h][3];
    }
    *o = make_uint2(pack_bf16x2(v[h][0], v[h][1]), pack_bf16x2(v[h][2], v[h][3]));
  }
}

}  // namespace

hipError_t launch_quant_fp8(const void* x, bool bf16, int64_t ldx, void* q, int64_t ldq, void* scale, int64_t lds, int M,
                            int K, hipStream_t s) {
  if (M == 0 || K == 0) return hipSuccess;
  const int per_row = (K + 1023) / 1024;
  const int64_t groups = ((int64_t)M * per_row + 3) / 4;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
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
    const int64_t n = (int64_t)p.tiles_m * p.tiles_n;
    if (n > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL(fn, dim3((uint32_t)n), dim3(threads), 0, s, p);
    return hipGetLastError();
  };
  const int nt = groups ? 128 : 64;
  if (tiles(32, nt) <= n_cu) {
    const bool one = g.M <= 16;
    if (fp8) return one ? go(gemm_fp8_small_kernel<128, 1, EPI_K_FP8, false>, 16, 128, 512)
                        : go(gemm_fp8_small_kernel<128, 2, EPI_K_FP8, false>, 32, 128, 512);
    if (f32) {
      if (groups) return one ? go(gemm_fp8_small_kernel<128, 1, EPI_K_ANY, true>, 16, 128, 512)
                             : go(gemm_fp8_small_kernel<128, 2, EPI_K_ANY, true>, 32, 128, 512);
      return one ? go(gemm_fp8_small_kernel<64, 1, EPI_K_ANY, true>, 16, 64, 512)
                 : go(gemm_fp8_small_kernel<64, 2, EPI_K_ANY, true>, 32, 64, 512);
    }
    if (groups) return one ? go(gemm_fp8_small_kernel<128, 1, EPI_K_ANY, false>, 16, 128, 512)
                           : go(gemm_fp8_small_kernel<128, 2, EPI_K_ANY, false>, 32, 128, 512);
    return one ? go(gemm_fp8_small_kernel<64, 1, EPI_K_ANY, false>, 16, 64, 512)
               : go(gemm_fp8_small_kernel<64, 2, EPI_K_ANY, false>, 32, 64, 512);
  }
  const bool half = tiles(128, 128) < 2 * n_cu;
  if (f32) return half ? go(gemm_fp8_tile_kernel<64, 3, EPI_K_ANY, true>, 64, 128, 256)
                       : go(gemm_fp8_tile_kernel<128, 2, EPI_K_ANY, true>, 128, 128, 256);
  const bool plain = !(g.flags & DIT_EPI_SILU);
  const bool store = plain && !gated && !fp8 && (g.gelu_from >= g.N || g.gelu_from % 128 == 0) &&
                     (g.gap == 0 || g.gap_at % 128 == 0);
  const bool only_gate = plain && gated && g.rms_cols == 0 && g.gelu_from >= g.N && g.gap == 0;
  if (tiles(256, 256) >= n_cu)
    return go(fp8 ? gemm_fp8_ring_kernel<EPI_K_FP8> : store ? gemm_fp8_ring_kernel<EPI_K_STORE>
              : only_gate ? gemm_fp8_ring_kernel<EPI_K_GATED> : gemm_fp8_ring_kernel<EPI_K_ANY>, 256, 256, 512);
  if (half) return go(fp8 ? gemm_fp8_tile_kernel<64, 3, EPI_K_FP8, false> : gemm_fp8_tile_kernel<64, 3, EPI_K_ANY, false>,
                      64, 128, 256);
  return go(fp8 ? gemm_fp8_tile_kernel<128, 2, EPI_K_FP8, false> : gemm_fp8_tile_kernel<128, 2, EPI_K_ANY, false>, 128, 128,
            256);
}

}  // namespace dit
