// Attention over chosen key blocks: which blocks of 64 keys a block of 128
// queries attends (the largest products of the blocks' means), and the
// attention over the chosen ones.
//
//   score[i, j] = mean(q rows of block i) . mean(k rows of block j)        (float64)
//   o[r] = sum over listed blocks j, keys c in j: exp(q_r.k_c / sqrt(128)) v_c / (the same sum without v_c)
#include <algorithm>
#include <type_traits>

#include "attention_tile.h"
#include "common.h"
#include "gemm_tile.h"
#include "kernels.h"

namespace dit {
namespace {

constexpr int QBLK = DIT_SPARSE_QB;  // queries that share a list
constexpr int KBLK = DIT_SPARSE_KB;  // keys of a block
static_assert(QBLK == 128 && KBLK == KT, "block sizes");

typedef double f64x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int keys_of(const int32_t* klen, int z, int Lk) {
  return klen ? min(max(klen[z], 0), Lk) : Lk;
}

// ---------------------------------------------------------------- selection

// Means of the rows of one block and head, float64: a bf16 has 8 bits, so these
// sums are exact for any sane range, whatever their order, and the choice of
// blocks does not hang on rounding.  256 threads: 16 rows at a time, 8 columns
// a thread.  Rows past the sequence's keys do not count.
template <int BLK>
__global__ __launch_bounds__(256) void block_mean_kernel(const bf16_t* __restrict__ x, int64_t ldx,
                                                         double* __restrict__ out, int L, const int32_t* klen) {
  __shared__ double part[16][D];
  const int blk = blockIdx.x, h = blockIdx.y, z = blockIdx.z, nb = gridDim.x, H = gridDim.y;
  const int c = threadIdx.x & 15, r0 = threadIdx.x >> 4;
  const int n = min(keys_of(klen, z, L) - blk * BLK, BLK);
  const bf16_t* p = x + ((int64_t)z * L + (int64_t)blk * BLK) * ldx + h * D + 8 * c;
  uint4 u[BLK / 16];
#pragma unroll
  for (int i = 0; i < BLK / 16; ++i) {
    const int r = r0 + 16 * i;
    u[i] = r < n ? *(const uint4*)(p + (int64_t)r * ldx) : make_uint4(0, 0, 0, 0);
  }
  double s[8] = {};
#pragma unroll
  for (int i = 0; i < BLK / 16; ++i) {
    float v[8];
    unpack8(u[i], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += (double)v[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part[r0][8 * c + e] = s[e];
  __syncthreads();
  if (threadIdx.x < D) {
    double t = 0.;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += part[i][threadIdx.x];
    out[(((int64_t)z * H + h) * nb + blk) * D + threadIdx.x] = t / (double)max(n, 1);
  }
}

// Order-preserving integer of a score: NaN counts as -inf, and no score gives 0
// (a block without keys) or all ones (a block that is always taken).
__device__ __forceinline__ uint64_t score_key(double s) {
  s = s != s ? -(double)INFINITY : s + 0.0;  // + 0: one zero
  const uint64_t u = __builtin_bit_cast(uint64_t, s);
  return u >> 63 ? ~u : u | (1ull << 63);
}

// Keys of 16 NI query blocks x 64 key blocks per wave on f64 MFMAs (16x16x4; lane
// (lr, lq) holds d = 16 t + 4 lq + e of its row for step 4 t + e).
template <int NI>
__global__ __launch_bounds__(256) void block_score_kernel(const double* __restrict__ qm, const double* __restrict__ km,
                                                          uint64_t* __restrict__ keys, int nqb, int nkb, int heads,
                                                          int kv_heads, int Lk, int first, const int32_t* klen) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int hz = blockIdx.z, z = hz / heads, h = hz - z * heads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
  const int q0 = (blockIdx.y * 4 + wave) * 16 * NI, k0 = blockIdx.x * 64;
  if (q0 >= nqb) return;
  const double* qp[NI];
  const double* kp[4];
#pragma unroll
  for (int i = 0; i < NI; ++i) qp[i] = qm + ((int64_t)hz * nqb + min(q0 + 16 * i + lr, nqb - 1)) * D + 4 * lq;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    kp[j] = km + (((int64_t)z * kv_heads + h / (heads / kv_heads)) * nkb + min(k0 + 16 * j + lr, nkb - 1)) * D + 4 * lq;
  f64x4_t acc[NI][4] = {};
#pragma unroll 2
  for (int t = 0; t < D / 16; ++t) {
    f64x4_t a[NI], b[4];
#pragma unroll
    for (int i = 0; i < NI; ++i) a[i] = *(const f64x4_t*)(qp[i] + 16 * t);
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = *(const f64x4_t*)(kp[j] + 16 * t);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f64_16x16x4f64(a[i][e], b[j][e], acc[i][j], 0, 0, 0);
  }
  const int nvalid = (keys_of(klen, z, Lk) + KBLK - 1) / KBLK;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int q = q0 + 16 * i + 4 * r + lq;  // f64 accumulators: row 4 r + lq
      if (q >= nqb) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k0 + 16 * j + lr;
        if (k < nkb)
          keys[((int64_t)hz * nqb + q) * nkb + k] = k >= nvalid ? 0 : k < first ? ~0ull : score_key(acc[i][j][r]);
      }
    }
#endif
}

// The topk largest keys of each row, in the order of their blocks; equal keys go to
// the lowest block.  A work-group of NW waves per row, R keys a lane.  The
// threshold is found bit by bit from the top: a bit stays set while at least
// topk keys reach it, and the search ends as soon as exactly topk do.
template <int NW, int R>
__global__ __launch_bounds__(64 * NW) void block_topk_kernel(const uint64_t* __restrict__ keys, int32_t* __restrict__ idx,
                                                             int nkb, int topk) {
  __shared__ int red[2][NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  uint64_t key[R];  // wave w holds keys w 64 R ..: block index = base + 64 r + lane
  const int base = wave * 64 * R;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int j = base + 64 * r + lane;
    key[r] = j < nkb ? keys[row * nkb + j] : 0;
  }
  int flip = 0;
  // sum over the work-group of a wave-uniform count; `before`: that of the waves before this one
  auto total = [&](int c, int& before) {
    if constexpr (NW == 1) {
      before = 0;
      return c;
    } else {
      if (lane == 0) red[flip][wave] = c;
      __syncthreads();
      int t = 0;
      before = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const int x = red[flip][w];
        if (w < wave) before += x;
        t += x;
      }
      flip ^= 1;
      return t;
    }
  };
  auto count = [&](uint64_t t) {  // keys >= t
    int c = 0, b;
#pragma unroll
    for (int r = 0; r < R; ++r) c += __popcll(__ballot(key[r] >= t));
    return total(c, b);
  };
  const int want = min(topk, count(1));
  uint64_t T = 1;
  bool exact = false;
  if (want > 0) {
    for (int b = 63; b >= 0; --b) {
      const uint64_t cand = (T & ~1ull) | (1ull << b);
      const int c = count(cand);
      if (c >= want) T = cand;
      if (c == want) { exact = true; break; }
    }
  }
  // keys above T, and of those equal to it the first `ties`
  int ties = 0, eq_before = 0;
  if (want > 0 && !exact) {
    int c = 0, e = 0, b;
#pragma unroll
    for (int r = 0; r < R; ++r) { c += __popcll(__ballot(key[r] > T)); e += __popcll(__ballot(key[r] == T)); }
    ties = want - total(c, b);
    total(e, eq_before);
  }
  const uint64_t below = (1ull << lane) - 1;
  uint64_t sel[R];
  int mine = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (want == 0) {
      sel[r] = 0;
    } else if (exact) {
      sel[r] = __ballot(key[r] >= T);
    } else {
      const uint64_t eq = __ballot(key[r] == T);
      sel[r] = __ballot(key[r] > T || (key[r] == T && eq_before + __popcll(eq & below) < ties));
      eq_before += __popcll(eq);
    }
    mine += __popcll(sel[r]);
  }
  int at;
  total(mine, at);
  int32_t* o = idx + row * topk;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (sel[r] >> lane & 1) o[at + __popcll(sel[r] & below)] = base + 64 * r + lane;
    at += __popcll(sel[r]);
  }
  for (int j = want + tid; j < topk; j += 64 * NW) o[j] = -1;
}

// ---------------------------------------------------------------- attention

struct SparseArgs {
  const bf16_t* q; int64_t ldq;
  const bf16_t* k; int64_t ldk;
  const bf16_t* v; int64_t ldv;
  bf16_t* o; int64_t ldo;
  const int32_t* idx;
  const int32_t* klen;
  int Lq, Lk, heads, kv_heads, nqb, nkb, topk;
  int items, parts;   // the list of an item is shared by `parts` work-groups
  int rows;           // query rows of a piece in ws
  float* ws;
  float scale_log2;
};

// A piece of an item: its unnormalised outputs [rows][128], row sums and running maxima.
__host__ __device__ __forceinline__ int64_t piece_floats(int rows) { return (int64_t)rows * (D + 2); }

// The valid entries of one list, in their order; every wave walks it alike.
struct ListCursor {
  const int32_t* p;
  int n, base, v, nkb;
  uint64_t left;
  __device__ __forceinline__ ListCursor(const int32_t* p_, int n_, int nkb_) : p(p_), n(n_), base(-64), v(0), nkb(nkb_), left(0) {}
  __device__ __forceinline__ int next() {  // -1: none left
    while (left == 0) {
      base += 64;
      if (base >= n) return -1;
      const int lane = threadIdx.x & 63;
      v = base + lane < n ? p[base + lane] : -1;
      left = __ballot((uint32_t)v < (uint32_t)nkb);
    }
    const int b = __ffsll((unsigned long long)left) - 1;
    left &= left - 1;
    return __builtin_amdgcn_readlane(v, b);
  }
};

// Four waves of 32 queries on one list, two work-groups per CU; K and V tiles of
// 64 keys in XOR-swizzled LDS rows of 256 bytes, two of each.  The products
// and the softmax are those of the dense kernel (S^T = K Q^T, O^T = V^T P^T);
// V^T fragments are read from the row-major tile by transposing LDS reads, so no
// transposed copy of V is made.
template <bool BOUNDED>
__global__ __launch_bounds__(256, 2) void attn_sparse_kernel(SparseArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int TILE = KT * D * 2;
  __shared__ __attribute__((aligned(1024))) char smem[4 * TILE];  // K, V of even tiles, then of odd ones
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int unit = xcd_remap(blockIdx.x, P.items * P.parts);
  const int item = unit / P.parts, part = unit - item * P.parts;
  const int hz = item / P.nqb, qb = item - hz * P.nqb;
  const int z = hz / P.heads, h = hz - z * P.heads, g_ = h / (P.heads / P.kv_heads);
  const int nkeys = keys_of(P.klen, z, P.Lk), nkb = (nkeys + KBLK - 1) / KBLK;
  const int p0 = (int)((int64_t)P.topk * part / P.parts), p1 = (int)((int64_t)P.topk * (part + 1) / P.parts);
  ListCursor list(P.idx + (int64_t)item * P.topk + p0, p1 - p0, nkb);

  const int q0 = qb * QBLK + 32 * wave;
  const bool active = q0 < P.Lq;  // wave-uniform; idle waves copy and meet the others
  const bf16_t* kbase = P.k + (int64_t)z * P.Lk * P.ldk + g_ * D;
  const bf16_t* vbase = P.v + (int64_t)z * P.Lk * P.ldv + g_ * D;
  // copy c of this wave: rows 4 (4 wave + c) .. + 3 of a tile
  uint32_t ko[4], vo[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int row = 4 * (4 * wave + c) + (lane >> 4);
    const uint32_t ch = ((lane & 15) ^ (row & 15)) << 4;
    ko[c] = (uint32_t)row * (uint32_t)P.ldk * 2u + ch;
    vo[c] = (uint32_t)row * (uint32_t)P.ldv * 2u + ch;
  }
  auto issue = [&](int kb, int st) {  // rows past the last key read zeros
    const uint32_t last = min(nkeys - kb * KBLK, KBLK) - 1;
    const bf16_t* kp = kbase + (int64_t)kb * KBLK * P.ldk;
    const bf16_t* vp = vbase + (int64_t)kb * KBLK * P.ldv;
    char* d = smem + st * 2 * TILE + wave * 4096;
#pragma unroll
    for (int c = 0; c < 4; ++c) copy16(kp, last * (uint32_t)P.ldk * 2u + 2u * D, (lds_void_t*)(d + c * 1024), ko[c]);
#pragma unroll
    for (int c = 0; c < 4; ++c) copy16(vp, last * (uint32_t)P.ldv * 2u + 2u * D, (lds_void_t*)(d + TILE + c * 1024), vo[c]);
  };

  bf16x8_t qf[2][4];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const bf16_t* qp = P.q + ((int64_t)z * P.Lq + min(q0 + 16 * g + lr, P.Lq - 1)) * P.ldq + h * D + 8 * lq;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[g][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 32 * s));
  }
  int koff[4], voff[8];
#pragma unroll
  for (int s = 0; s < 4; ++s) koff[s] = k_off(lr, 4 * s + lq);
  // V^T fragment (d = 16 dt + lr; keys 4 lq .. + 3 of a 16-key block): lane 4 k + j of a
  // quarter addresses row 4 lq + k, columns 16 dt + 4 j, and receives column lr
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) {
    const int row = 4 * lq + (lr >> 2);
    voff[dt] = TILE + k_off(row, 2 * dt + ((lr & 3) >> 1)) + 8 * (lr & 1);
  }
  f32x4_t acc[8][2];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) acc[dt][0] = acc[dt][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m[2], l[2] = {0.f, 0.f};
  m[0] = m[1] = BOUNDED ? BOUNDED_SHIFT_LOG2 : -INFINITY;
  const bf16x2_t ones = {(__bf16)1.f, (__bf16)1.f};

  int cur = list.next();
  if (cur >= 0) issue(cur, 0);
  int st = 0;
  while (cur >= 0) {
    const int nxt = list.next();
    // this tile has landed and everyone is done with the one before it
    __builtin_amdgcn_s_waitcnt(0);
    barrier_no_fence();
    if (nxt >= 0) issue(nxt, st ^ 1);
    if (active) {
      const char* sk = smem + st * 2 * TILE;
      f32x4_t s[4][2];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        s[kb][0] = s[kb][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *(const uint4*)(sk + koff[t] + kb * 16 * 256));
#pragma unroll
          for (int g = 0; g < 2; ++g) s[kb][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][t], s[kb][g], 0, 0, 0);
        }
      }
      if ((cur + 1) * KBLK > nkeys) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (cur * KBLK + 16 * kb + 4 * lq + r >= nkeys) s[kb][0][r] = s[kb][1][r] = -INFINITY;
      }
      bf16x8_t pf[2][2];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        if constexpr (!BOUNDED) {
          float mx = -INFINITY;
#pragma unroll
          for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[kb][g][r]);
          mx = max_quarters(mx) * P.scale_log2;
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
            // the sum takes exactly the rounded values that the second product uses
            l[g] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[e]), ones, l[g], false);
          }
          pf[ks][g] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
        }
      }
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          typedef short s4 __attribute__((ext_vector_type(4)));
          typedef __attribute__((address_space(3))) s4* lds_s4;
          const char* p = sk + voff[dt] + ks * 32 * 256;
          const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)p);
          const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(p + 16 * 256));
          const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
          const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(a.x, a.y, b.x, b.y));
#pragma unroll
          for (int g = 0; g < 2; ++g) acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[ks][g], acc[dt][g], 0, 0, 0);
        }
    }
    st ^= 1;
    cur = nxt;
  }
  if (!active) return;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = 32 * wave + 16 * g + lr, qi = qb * QBLK + row;
    const float ls = sum_quarters(l[g]);
    if (qi >= P.Lq) continue;
    if (P.parts == 1) {
      const float inv = ls == 0.f ? 0.f : 1.f / ls;  // no key: zeros
      bf16_t* op = P.o + ((int64_t)z * P.Lq + qi) * P.ldo + h * D + 4 * lq;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
        *(uint2*)(op + 16 * dt) = make_uint2(pack_bf16x2(acc[dt][g][0] * inv, acc[dt][g][1] * inv),
                                             pack_bf16x2(acc[dt][g][2] * inv, acc[dt][g][3] * inv));
    } else {
      float* w = P.ws + unit * piece_floats(P.rows);
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *(f32x4_t*)(w + row * D + 16 * dt + 4 * lq) = acc[dt][g];
      if (lq == 0) {
        w[P.rows * D + row] = ls;
        w[P.rows * D + P.rows + row] = m[g];
      }
    }
  }
#endif
}

// Adds the pieces of an item in the order of its list and stores the normalised
// output.  32 threads a row, 4 columns each.
__global__ __launch_bounds__(256) void sparse_combine_kernel(SparseArgs P) {
  const int item = blockIdx.x, row = blockIdx.y * 8 + (threadIdx.x >> 5), c = 4 * (threadIdx.x & 31);
  const int hz = item / P.nqb, qb = item - hz * P.nqb;
  const int z = hz / P.heads, h = hz - z * P.heads, qi = qb * QBLK + row;
  if (row >= P.rows || qi >= P.Lq) return;
  const int64_t pf = piece_floats(P.rows);
  const float* w = P.ws + (int64_t)item * P.parts * pf;
  float mx = -INFINITY;
  for (int p = 0; p < P.parts; ++p) mx = fmaxf(mx, w[p * pf + P.rows * D + P.rows + row]);
  const float shift = neg_shift(mx);
  float den = 0.f;
  f32x4_t y = {};
  for (int p = 0; p < P.parts; ++p) {
    const float* x = w + p * pf;
    const float f = __builtin_amdgcn_exp2f(x[P.rows * D + P.rows + row] + shift);
    const f32x4_t t = *(const f32x4_t*)(x + row * D + c);
    den += f * x[P.rows * D + row];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += f * t[e];
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;
  *(uint2*)(P.o + ((int64_t)z * P.Lq + qi) * P.ldo + h * D + c) =
      make_uint2(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv));
}

int blocks_of(int n, int b) { return n / b + (n % b != 0); }

}  // namespace

// Means of the query blocks and of the key blocks (f64), then one key per pair.
size_t select_blocks_ws_bytes(const dit_sparse_shape& s) {
  const size_t nqb = blocks_of(s.Lq, QBLK), nkb = blocks_of(s.Lk, KBLK), b = s.batch;
  return 8 * (b * s.heads * nqb * D + b * s.kv_heads * nkb * D + b * s.heads * nqb * nkb);
}

hipError_t launch_select_blocks(const dit_sparse_shape& s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                int first, int32_t* idx, void* ws, hipStream_t st) {
  const int nqb = blocks_of(s.Lq, QBLK), nkb = blocks_of(s.Lk, KBLK);
  const int64_t rows = (int64_t)s.batch * s.heads * nqb;
  if (rows == 0) return hipSuccess;
  double* qm = (double*)ws;
  double* km = qm + rows * D;
  uint64_t* keys = (uint64_t*)(km + (int64_t)s.batch * s.kv_heads * nkb * D);
  if (nkb > 0) {
    hipLaunchKernelGGL(block_mean_kernel<QBLK>, dim3(nqb, s.heads, s.batch), dim3(256), 0, st, (const bf16_t*)q, ldq, qm,
                       s.Lq, (const int32_t*)nullptr);
    hipLaunchKernelGGL(block_mean_kernel<KBLK>, dim3(nkb, s.kv_heads, s.batch), dim3(256), 0, st, (const bf16_t*)k, ldk,
                       km, s.Lk, s.klen);
    hipLaunchKernelGGL(block_score_kernel<2>, dim3((nkb + 63) / 64, (nqb + 127) / 128, s.batch * s.heads), dim3(256), 0,
                       st, qm, km, keys, nqb, nkb, s.heads, s.kv_heads, s.Lk, first, s.klen);
  }
  const dim3 grid((uint32_t)rows);
#define DIT_TOPK(NW, R) \
  hipLaunchKernelGGL((block_topk_kernel<NW, R>), grid, dim3(64 * NW), 0, st, keys, idx, nkb, s.topk)
  if (nkb <= 64) DIT_TOPK(1, 1);
  else if (nkb <= 256) DIT_TOPK(1, 4);
  else if (nkb <= 512) DIT_TOPK(1, 8);
  else if (nkb <= 1024) DIT_TOPK(1, 16);
  else if (nkb <= 4096) DIT_TOPK(4, 16);
  else DIT_TOPK(16, 16);
#undef DIT_TOPK
  return hipGetLastError();
}

// Work-groups that share one list: enough for two per CU of the chip.
int sparse_parts(const dit_sparse_shape& s) {
  const int64_t items = (int64_t)s.batch * s.heads * blocks_of(s.Lq, QBLK);
  if (items == 0) return 1;
  const int64_t p = 512 / items;
  return (int)std::max<int64_t>(1, std::min<int64_t>(p, s.topk));
}
int sparse_rows(const dit_sparse_shape& s) { return std::min(QBLK, (s.Lq + 31) / 32 * 32); }

size_t attention_sparse_ws_bytes(const dit_sparse_shape& s) {
  const int parts = sparse_parts(s);
  if (parts == 1) return 0;
  return (size_t)s.batch * s.heads * blocks_of(s.Lq, QBLK) * parts * piece_floats(sparse_rows(s)) * sizeof(float);
}

hipError_t launch_attention_sparse(const dit_sparse_shape& s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                   const void* v, int64_t ldv, void* o, int64_t ldo, const int32_t* idx, bool bounded,
                                   void* ws, hipStream_t st) {
  SparseArgs P{};
  P.q = (const bf16_t*)q; P.ldq = ldq; P.k = (const bf16_t*)k; P.ldk = ldk;
  P.v = (const bf16_t*)v; P.ldv = ldv; P.o = (bf16_t*)o; P.ldo = ldo;
  P.idx = idx; P.klen = s.klen;
  P.Lq = s.Lq; P.Lk = s.Lk; P.heads = s.heads; P.kv_heads = s.kv_heads; P.topk = s.topk;
  P.nqb = blocks_of(s.Lq, QBLK);
  P.nkb = blocks_of(s.Lk, KBLK);
  P.items = s.batch * s.heads * P.nqb;
  if (P.items == 0) return hipSuccess;
  P.parts = sparse_parts(s);
  P.rows = sparse_rows(s);
  P.ws = (float*)ws;
  P.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  hipLaunchKernelGGL((bounded ? attn_sparse_kernel<true> : attn_sparse_kernel<false>), dim3(P.items * P.parts), dim3(256),
                     0, st, P);
  if (P.parts > 1)
    hipLaunchKernelGGL(sparse_combine_kernel, dim3(P.items, (P.rows + 7) / 8), dim3(256), 0, st, P);
  return hipGetLastError();
}

}  // namespace dit
