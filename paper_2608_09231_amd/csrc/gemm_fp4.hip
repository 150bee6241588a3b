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
// One pass, bound by memory.
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

// Eight values a lane.  e2m1 as a bf16 or f32 number, then times the scale: two
// factors, so that neither is subnormal where the product is not.
template <typename T>
__global__ __launch_bounds__(256) void dequant_fp4_kernel(const uint8_t* __restrict__ q, int64_t ldq,
                                                          const uint8_t* __restrict__ scale, int64_t lds,
                                                          T* __restrict__ y, int64_t ldy, int M, int K, int per_row) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t m = unit / per_row;
  if (m >= M) return;
  const int k0 = (int)(unit - m * per_row) * 1024 + 8 * lane;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int k = k0 + 512 * h;
    if (k >= K) return;
    const uint32_t w = *(const uint32_t*)(q + m * ldq + (k >> 1));
    const int byte = scale[m * lds + (k >> 5)];
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t c = w >> (4 * i);
      // 0, 1/2, then 1.m * 2^(e - 1)
      const uint32_t mag = (c & 7) < 2 ? (c & 1) * 0x3f000000u : 0x3f800000u + (((c & 7) - 2) << 22);
      const float f = __uint_as_float(mag | (c & 8) << 28);
      v[i] = byte == 255 ? __uint_as_float(0x7fc00000u) : ldexpf(f, byte - 127);
    }
    if constexpr (sizeof(T) == 2) {
      *(uint4*)(y + m * ldy + k) = pack8(v);
    } else {
      *(float4*)(y + m * ldy + k) = make_float4(v[0], v[1], v[2], v[3]);
      *(float4*)(y + m * ldy + k + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
#endif
}

// ---------------------------------------------------------------- products

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
          const float inv = e8m0_inverse(byte);
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

// 64 x 128 tiles, four waves of 32 x 64, operands straight from memory to
// registers: the simplest form.
template <int KIND>
__global__ __launch_bounds__(256) void gemm_fp4_tile_kernel(Fp4Prob P) {
  constexpr int BM = 64, WM = 32, TM = 2, TN = 4;
  __shared__ __attribute__((aligned(1024))) char smem[BM * 128 * 4];
  int tm, tn;
  tile_at(P, xcd_remap(blockIdx.x, P.tiles_m * P.tiles_n), tm, tn);
  const int m0 = tm * BM, n0 = tn * 128;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int lr = lane & 15, lq = lane >> 4;
  const uint8_t *row[TM + TN], *sc[TM + TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = min(m0 + WM * wm + 16 * i + lr, P.M - 1);
    row[i] = P.A + m * P.lda;
    sc[i] = P.As + m * P.ldas;
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int64_t n = min(n0 + 64 * wn + 16 * j + lr, P.N - 1);
    row[TM + j] = P.W + n * P.ldw;
    sc[TM + j] = P.Ws + n * P.ldws;
  }
  f32x4_t acc[TM][TN] = {};
  for (int k = 0; k < P.K; k += 128) {
    const int at = k + 32 * lq;
    const bool in = at < P.K;  // K % 32 == 0: a block is inside or not
    i32x4_t f[TM + TN];
    int s[TM + TN];
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) {
      f[i] = in ? *(const i32x4_t*)(row[i] + (at >> 1)) : i32x4_t{0, 0, 0, 0};
      s[i] = in ? sc[i][at >> 5] : 127;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = mfma_fp4(f[i], f[TM + j], acc[i][j], s[i], s[TM + j]);
  }
  float* tile = (float*)smem;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        tile[(wm * WM + 16 * i + 4 * lq + r) * 128 + ((64 * wn + 16 * j + lr) ^ (lq << 4))] = acc[i][j][r];
  __syncthreads();
  constexpr int ROWS = BM / 4;
  Epi<KIND> epi(P, m0 + ROWS * wave, n0, lane & 31, lane >> 5, tile + ROWS * wave * 128);
  epi.prep();
  uint2 old[8][2];
  if (epi.gated) epi.load_old(0, old);
  epi.template rows<3, 4, ROWS>(0, old);
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
  const int per_row = (K + 1023) / 1024;
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
  return go(g.flags & DIT_EPI_FP4 ? gemm_fp4_tile_kernel<EPI_K_FP4> : gemm_fp4_tile_kernel<EPI_K_ANY>, 64, 128, 256);
}

}  // namespace dit
