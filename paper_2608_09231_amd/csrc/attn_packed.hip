// Attention over packed sequences, o = softmax(q k^T / sqrt(128)) v in each of them,
// causal or not, heads grouped over key heads.
//
// The queries of a sequence and of the `group` heads that share a key head are one
// matrix of rows for that head's keys: row r is query r / group of head r % group of
// them.  So a tile of K and V serves every head that reads it, single tokens of
// grouped heads fill rows that would be empty, and a causal tile spans group times
// fewer keys that it masks.
#include <math.h>

#include <algorithm>

#include "attention_tile.h"
#include "common.h"
#include "gemm_tile.h"
#include "kernels.h"

namespace dit {
namespace {

struct PackedArgs {
  const bf16_t* q; int64_t ldq;
  const bf16_t* k; int64_t ldk;
  const bf16_t* v; int64_t ldv;
  bf16_t* o; int64_t ldo;
  const int32_t *qoff, *koff, *klen;
  int batch, Tq, Tk, kv_heads, group;
  float* ws;
  float scale_log2;
};

// A sequence: its first rows and lengths, clamped to what the caller's matrices hold.
struct Seq {
  int q0, lq, k0, lk;
};
__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }
__device__ __forceinline__ int queries_of(const PackedArgs& P, int z) {
  const int a = clamp_to(P.qoff[z], 0, P.Tq);
  return clamp_to(P.qoff[z + 1], a, P.Tq) - a;
}
__device__ __forceinline__ Seq seq_of(const PackedArgs& P, int z) {
  Seq s;
  s.q0 = clamp_to(P.qoff[z], 0, P.Tq);
  s.lq = clamp_to(P.qoff[z + 1], s.q0, P.Tq) - s.q0;
  s.k0 = clamp_to(P.koff[z], 0, P.Tk);
  s.lk = clamp_to(P.koff[z + 1], s.k0, P.Tk) - s.k0;
  if (P.klen) s.lk = clamp_to(P.klen[z], 0, s.lk);
  return s;
}

// Sum of v over the lanes up to this one.
__device__ __forceinline__ int scan_lanes(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    v += lane >= o ? u : 0;
  }
  return v;
}

// The sequence that tile t of `rows` rows falls in, 64 sequences at a time, and the
// tile's number in it; false past the last one.
__device__ __forceinline__ bool find_tile(const PackedArgs& P, int t, int rows, int& z, int& tile) {
  const int lane = threadIdx.x & 63;
  for (int z0 = 0; z0 < P.batch; z0 += 64) {
    const int n = z0 + lane < P.batch ? (queries_of(P, z0 + lane) * P.group + rows - 1) / rows : 0;
    const int end = scan_lanes(n);
    const uint64_t past = __ballot(end > t);
    if (past) {
      const int l = __ffsll((unsigned long long)past) - 1;
      z = z0 + l;
      tile = t - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(n, l));
      return true;
    }
    t -= __builtin_amdgcn_readlane(end, 63);
  }
  return false;
}

// 16 bytes per lane from base + off (valid up to `bytes`; zeros past it) to LDS at
// dst + 16 lane, as an instruction that the compiler does not see through: it
// would have every transposing read of LDS wait for all copies in flight.  The
// kernel's own waits and barriers order them.  (No registers come back; the
// address escapes, so that the barriers' memory clobbers cover what is written.)
__device__ __forceinline__ void copy16_unseen(const void* base, uint32_t bytes, const void* dst, uint32_t off) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const uint64_t b = (uint64_t)base;
  const u32x4 r = {(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, bytes, 0x00020000u};
  const uint32_t l = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)dst;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(l), "v"(off), "s"(r));
#endif
}

// Largest of three in one instruction (a NaN gives way to a number, as with fmaxf).
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

__device__ __forceinline__ bool not_finite(const bf16x8_t& f) {
  const uint4 u = __builtin_bit_cast(uint4, f);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
    bad |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
  }
  return bad;
}

constexpr int ROWS = 128;

// 128 rows of a sequence and key head: four waves of 32, tiles of 64 keys of K and V in
// XOR-swizzled LDS rows of 256 bytes, two of each; S^T = K Q^T, O^T = V^T P^T,
// probabilities from one to the other in registers, V^T read from the row-major
// tile by transposing LDS reads.  Probabilities are rounded to bf16, the type that
// the second product takes beside V; the sum takes the rounded values, so that the weights add up to one.
template <bool BOUNDED, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void attn_packed_kernel(PackedArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int TILE = KT * D * 2, STAGE = 2 * TILE;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];  // [stage][K | V]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int unit = blockIdx.x, kh = unit % P.kv_heads;
  int z, tile;
  if (!find_tile(P, unit / P.kv_heads, ROWS, z, tile)) return;
  z = __builtin_amdgcn_readfirstlane(z);
  tile = __builtin_amdgcn_readfirstlane(tile);
  const Seq s_ = seq_of(P, z);
  const int nrows = s_.lq * P.group;
  if (CAUSAL) tile = (nrows + ROWS - 1) / ROWS - 1 - tile;  // the longest first
  // keys that query i sees: past + i, at most all; not causal: all
  const int past = s_.lk - s_.lq + 1;
  auto seen = [&](int row) { return CAUSAL ? max(past + row / P.group, 0) : s_.lk; };
  const int wrow = tile * ROWS + 32 * wave;
  const int nkeys = seen(min(tile * ROWS + ROWS, nrows) - 1);        // of the work-group
  const bool active = wrow < nrows;  // wave-uniform; idle waves copy and meet the others
  const int wkeys = active ? seen(min(wrow + 32, nrows) - 1) : 0;    // of the wave
  const int common = active ? seen(wrow) : 0;                        // of all its rows
  int lim[2];
  bf16x8_t qf[2][4];
  bf16_t* op[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = min(wrow + 16 * g + lr, nrows - 1), qi = row / P.group, h = kh * P.group + row - qi * P.group;
    lim[g] = seen(row);
    const bf16_t* qp = P.q + (int64_t)(s_.q0 + qi) * P.ldq + (int64_t)h * D + 8 * lq;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[g][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 32 * s));
    op[g] = wrow + 16 * g + lr < nrows ? P.o + (int64_t)(s_.q0 + qi) * P.ldo + (int64_t)h * D + 4 * lq : nullptr;
  }
  const bf16_t* kbase = P.k + (int64_t)s_.k0 * P.ldk + (int64_t)kh * D;
  const bf16_t* vbase = P.v + (int64_t)s_.k0 * P.ldv + (int64_t)kh * D;
  // copy c of this wave: rows 4 (4 wave + c) .. + 3 of a tile
  uint32_t ko[4], vo[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int row = 4 * (4 * wave + c) + (lane >> 4);
    const uint32_t ch = ((lane & 15) ^ (row & 15)) << 4;
    ko[c] = (uint32_t)row * (uint32_t)P.ldk * 2u + ch;
    vo[c] = (uint32_t)row * (uint32_t)P.ldv * 2u + ch;
  }
  // rows past the last key are zeros
  auto issue = [&](int key, int at) {
    const int n = min(nkeys - key, KT);
    const uint32_t kn = n <= 0 ? 0u : (uint32_t)(n - 1) * (uint32_t)P.ldk * 2u + 2u * D;
    const uint32_t vn = n <= 0 ? 0u : (uint32_t)(n - 1) * (uint32_t)P.ldv * 2u + 2u * D;
    const int64_t row = n <= 0 ? 0 : key;
    char* d = smem + at + wave * 4096;
#pragma unroll
    for (int c = 0; c < 4; ++c) copy16_unseen(kbase + row * P.ldk, kn, d + c * 1024, ko[c]);
#pragma unroll
    for (int c = 0; c < 4; ++c) copy16_unseen(vbase + row * P.ldv, vn, d + TILE + c * 1024, vo[c]);
  };
  // (queries waited for later would wait for the copies, too)
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int s = 0; s < 4; ++s) asm volatile("" : "+v"(qf[g][s]));
  int koff[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) koff[s] = k_off(lr, 4 * s + lq);
  // V^T fragment (d = 16 dt + lr; keys 4 lq .. + 3 of a 16-key block): lane 4 k + j of a
  // quarter addresses row 4 lq + k, columns 16 dt + 4 j, and receives column lr.  The
  // chunk 2 dt + (j >> 1) enters the swizzled address by XOR.
  const int voff = k_off(4 * lq + (lr >> 2), (lr & 3) >> 1) + 8 * (lr & 1);
  f32x4_t acc[8][2];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) acc[dt][0] = acc[dt][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m[2], l[2] = {0.f, 0.f};
  m[0] = m[1] = BOUNDED ? BOUNDED_SHIFT_LOG2 : -INFINITY;
  const bf16x2_t ones = {(__bf16)1.f, (__bf16)1.f};

  issue(0, 0);
  int at = 0;
  for (int key = 0; key < nkeys; key += KT) {
    // this tile has landed and everyone is done with the one before it
    __builtin_amdgcn_s_waitcnt(0);
    barrier_no_fence();
    issue(key + KT, at ^ STAGE);
    if (key < wkeys) {
      const char* sk = smem + at;
      f32x4_t s[4][2];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        s[kb][0] = s[kb][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4) {
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *(const uint4*)(sk + koff[t4] + kb * 16 * 256));
#pragma unroll
          for (int g = 0; g < 2; ++g) s[kb][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][t4], s[kb][g], 0, 0, 0);
        }
      }
      const bool masked = key + KT > common;  // wave-uniform
      if (masked) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int g = 0; g < 2; ++g)
              if (key + 16 * kb + 4 * lq + r >= lim[g]) s[kb][g][r] = -INFINITY;
      }
      bf16x8_t pf[2][2];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        if constexpr (!BOUNDED) {
          float mx = s[0][g][0];
#pragma unroll
          for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int r = 0; r < 4; r += 2) mx = max3(mx, s[kb][g][r], s[kb][g][r + 1]);
          mx = max_quarters(mx) * P.scale_log2;
          // (kept unless the new one is well above it: softmax is shift invariant)
          const bool up = mx > m[g] + RESCALE_SLACK;
          if (__builtin_amdgcn_ballot_w64(up)) {
            const float mn = up ? mx : m[g];
            const float a = up ? __builtin_amdgcn_exp2f(m[g] - mn) : 1.f;
            l[g] *= a;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[dt][g][r] *= a;
            m[g] = mn;
          }
        }
        const float mneg = BOUNDED ? -BOUNDED_SHIFT_LOG2 : neg_shift(m[g]);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f32x4_t& x = s[2 * ks + (e >> 1)][g];
            w[e] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * (e & 1)], P.scale_log2, mneg)),
                               __builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * (e & 1) + 1], P.scale_log2, mneg)));
            l[g] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[e]), ones, l[g], false);
          }
          pf[ks][g] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
        }
      }
      auto v_frag = [&](int dt, int ks) { return vt_frag(sk + TILE + (voff ^ (dt << 5)) + ks * 32 * 256); };
      // 0 times a value that is not finite would reach the rows that do not see its key
      bool spoilt = false;
      if (masked) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) spoilt |= not_finite(v_frag(dt, 0)) || not_finite(v_frag(dt, 1));
        spoilt = __builtin_amdgcn_ballot_w64(spoilt) != 0;
      }
      if (!spoilt) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) {
            const bf16x8_t vf = v_frag(dt, ks);
#pragma unroll
            for (int g = 0; g < 2; ++g) acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[ks][g], acc[dt][g], 0, 0, 0);
          }
      } else {
        // key by key: a lane keeps the product only if its row sees the key
#pragma unroll 1
        for (int j = 0; j < KT; ++j) {
          const bool second = j & 32, mine = ((j >> 2) & 3) == lq;
          const int e0 = 4 * ((j >> 4) & 1) + (j & 3);
          bf16x8_t pj[2];
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              pj[g][e] = mine && e == e0 ? (second ? pf[1][g][e] : pf[0][g][e]) : (__bf16)0.f;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) {
            bf16x8_t vj = v_frag(dt, second);
#pragma unroll
            for (int e = 0; e < 8; ++e) vj[e] = mine && e == e0 ? vj[e] : (__bf16)0.f;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const f32x4_t y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vj, pj[g], acc[dt][g], 0, 0, 0);
              if (key + j < lim[g]) acc[dt][g] = y;
            }
          }
        }
      }
    }
    at ^= STAGE;
  }
  __builtin_amdgcn_s_waitcnt(0);  // no copy outlives its work-group
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float ls = sum_quarters(l[g]);
    const float inv = ls == 0.f ? 0.f : 1.f / ls;  // no key: zeros
    if (!op[g]) continue;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      *(uint2*)(op[g] + 16 * dt) = make_uint2(pack_bf16x2(acc[dt][g][0] * inv, acc[dt][g][1] * inv),
                                              pack_bf16x2(acc[dt][g][2] * inv, acc[dt][g][3] * inv));
  }
#endif
}

}  // namespace

size_t attention_packed_ws_bytes(const dit_packed_shape&) { return 0; }

hipError_t launch_attention_packed(const dit_packed_shape& s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                   const void* v, int64_t ldv, void* o, int64_t ldo, bool bounded, bool causal, void* ws,
                                   hipStream_t st) {
  if (s.batch == 0 || s.Tq == 0) return hipSuccess;
  PackedArgs P{};
  P.q = (const bf16_t*)q; P.ldq = ldq; P.k = (const bf16_t*)k; P.ldk = ldk;
  P.v = (const bf16_t*)v; P.ldv = ldv; P.o = (bf16_t*)o; P.ldo = ldo;
  P.qoff = s.qoff; P.koff = s.koff; P.klen = s.klen;
  P.batch = s.batch; P.Tq = s.Tq; P.Tk = s.Tk; P.kv_heads = s.kv_heads; P.group = s.heads / s.kv_heads;
  P.ws = (float*)ws;
  P.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  // tiles of a key head, at most: whole ones and one begun by each sequence
  const int64_t tiles = (int64_t)s.Tq * P.group / ROWS + std::min(s.batch, s.Tq);
  void (*fn)(PackedArgs) = causal ? (bounded ? attn_packed_kernel<true, true> : attn_packed_kernel<false, true>)
                                  : (bounded ? attn_packed_kernel<true, false> : attn_packed_kernel<false, false>);
  hipLaunchKernelGGL(fn, dim3((uint32_t)(tiles * s.kv_heads)), dim3(256), 0, st, P);
  return hipGetLastError();
}

}  // namespace dit
