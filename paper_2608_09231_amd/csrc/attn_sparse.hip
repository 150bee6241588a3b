// Attention over chosen key blocks: which blocks of 64 keys a block of 128
// queries attends (the largest products of the blocks' means), and the
// attention over the chosen ones.
//
//   score[i, j] = mean(q rows of block i) . mean(k rows of block j)        (float64)
//   o[r] = sum over listed blocks j, keys c in j: exp(q_r.k_c / sqrt(128)) v_c / (the same sum without v_c)
#include <algorithm>
#include <type_traits>

#include "attention_copy.h"
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
// blocks does not hang on rounding.  256 threads: 16 rows at a time, 8 columns a
// thread, all loads in flight together.  One launch for the query blocks and the
// key blocks behind them.  Rows past the sequence's keys do not count.
//
// Means are laid out in groups of 16 blocks as the score products read them:
// lane (b, lq) of a wave holds d = 8 t + 2 lq + e of block b for step 2 t + e, one
// 16-byte load per t that is contiguous over the wave.  Work-groups run over the
// heads first, so that those in flight together read whole rows; where 8 divides
// the heads, a head's blocks then share an XCD, whose L2 puts the lines of their
// 16-byte pieces together (the rows pass it by).  Bound by the copy rate: 32760
// tokens, 40 heads (674 MB) 129 us, 5.2 TB/s; rows through L2 139 us, blocks first 154 us.
__host__ __device__ __forceinline__ int64_t mean_doubles(int blocks) { return (int64_t)((blocks + 15) / 16) * 16 * D; }
struct MeanArgs {
  const bf16_t* x[2]; int64_t ld[2];
  double* out[2];
  int L[2], heads[2], blocks[2];
  int queries;  // work-groups (block, head, sequence) of queries; those of keys follow
  const int32_t* klen;
};
template <int BLK>
__device__ __forceinline__ void block_mean(const MeanArgs& P, int kind, int unit, double (&part)[16][D]) {
  const int H = P.heads[kind], h = unit % H, bz = unit / H, z = bz / P.blocks[kind], blk = bz - z * P.blocks[kind];
  const int tid = threadIdx.x, c = tid & 15, r0 = tid >> 4, L = P.L[kind];
  const int n = min((kind ? keys_of(P.klen, z, L) : L) - blk * BLK, BLK);
  const int64_t ld = P.ld[kind];
  const bf16_t* p = P.x[kind] + ((int64_t)z * L + (int64_t)blk * BLK) * ld + h * D + 8 * c;
  uint4 u[BLK / 16];
#pragma unroll
  for (int i = 0; i < BLK / 16; ++i) {
    const int r = r0 + 16 * i;
    u[i] = r < n ? ld_stream(p + (int64_t)r * ld) : make_uint4(0, 0, 0, 0);
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
  if (tid < D) {
    double t = 0.;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += part[i][tid];
    double* o = P.out[kind] + (z * H + h) * mean_doubles(P.blocks[kind]) + (blk >> 4) * 16 * D;
    o[(tid >> 3) * 128 + (((tid >> 1) & 3) * 16 + (blk & 15)) * 2 + (tid & 1)] = t / (double)max(n, 1);
  }
}
__global__ __launch_bounds__(256) void block_mean_kernel(MeanArgs P) {
  __shared__ double part[16][D];
  const int unit = blockIdx.x;
  if (unit < P.queries) block_mean<QBLK>(P, 0, unit, part);
  else block_mean<KBLK>(P, 1, unit - P.queries, part);
}

// Order-preserving integer of a score: NaN counts as -inf, and no score gives 0
// (a block without keys) or all ones (a block that is always taken).
__device__ __forceinline__ uint64_t score_key(double s) {
  s = s != s ? -(double)INFINITY : s + 0.0;  // + 0: one zero
  const uint64_t u = __builtin_bit_cast(uint64_t, s);
  return u >> 63 ? ~u : u | (1ull << 63);
}

typedef double f64x2_t __attribute__((ext_vector_type(2)));

// Keys of 16 NI query blocks x 64 key blocks per wave on f64 MFMAs.
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
  for (int i = 0; i < NI; ++i) qp[i] = qm + hz * mean_doubles(nqb) + min(q0 / 16 + i, (nqb - 1) / 16) * 16 * D + 2 * lane;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    kp[j] = km + ((int64_t)z * kv_heads + h / (heads / kv_heads)) * mean_doubles(nkb) +
            min(k0 / 16 + j, (nkb - 1) / 16) * 16 * D + 2 * lane;
  f64x4_t acc[NI][4] = {};
#pragma unroll 4
  for (int t = 0; t < D / 8; ++t) {
    f64x2_t a[NI], b[4];
#pragma unroll
    for (int i = 0; i < NI; ++i) a[i] = *(const f64x2_t*)(qp[i] + 128 * t);
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = *(const f64x2_t*)(kp[j] + 128 * t);
#pragma unroll
    for (int e = 0; e < 2; ++e)
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

// Largest of a wave's values, the same in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_over<16>(v);
  return max(max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16)),
             max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
}

// The topk largest keys of a row, in the order of their blocks; equal keys go to the
// lowest block.  NW waves, R keys a lane (wave w holds blocks 64 R w + 64 r + lane).
// The threshold is found bit by bit from the top: a bit stays set while at least
// topk keys reach it, and the search ends as soon as exactly topk do.  red: 2 NW
// ints of LDS (NW > 1).
template <int NW, int R>
__device__ __forceinline__ void topk_row(const uint64_t (&key)[R], int32_t* __restrict__ o, int topk, int* red) {
  const int tid = threadIdx.x % (64 * NW), lane = tid & 63, wave = tid >> 6;
  const int base = wave * 64 * R;
  int flip = 0;
  // sum over the waves of a wave-uniform count; `before`: that of the waves before this one
  auto total = [&](int c, int& before) {
    before = 0;
    if constexpr (NW == 1) {
      return c;
    } else {
      if (lane == 0) red[flip * NW + wave] = c;
      __syncthreads();
      int t = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const int x = red[flip * NW + w];
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
  auto count_high = [&](uint32_t t) {  // keys whose upper half is >= t
    int c = 0, b;
#pragma unroll
    for (int r = 0; r < R; ++r) c += __popcll(__ballot((uint32_t)(key[r] >> 32) >= t));
    return total(c, b);
  };
  // (every key of a block is at least 2^32: that of -inf is 0x000fffffffffffff)
  const int have = count_high(1), want = min(topk, have);
  uint64_t T = 1;
  bool exact = want == have;  // every block that there is
  if (want > 0 && !exact) {
    // on the upper halves first, from the highest bit in which they differ
    uint32_t t = 0;
    int b = 31;
    if constexpr (NW == 1) {
      uint32_t hi = 0, lo = ~0u;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint32_t x = (uint32_t)(key[r] >> 32);
        hi = max(hi, x);
        lo = min(lo, x ? x : ~0u);
      }
      hi = wave_max(hi);
      lo = ~wave_max(~lo);
      b = hi == lo ? -1 : 31 - __builtin_clz(hi ^ lo);
      t = b < 0 ? hi : b == 31 ? 0 : hi & (~0u << (b + 1));
    }
#pragma unroll 1
    for (; b >= 0; --b) {
      const uint32_t cand = t | (1u << b);
      const int c = count_high(cand);
      if (c >= want) t = cand;
      if (c == want) { exact = true; break; }
    }
    T = (uint64_t)t << 32;
    if (!exact) {
#pragma unroll 1
      for (b = 31; b >= 0; --b) {
        const uint64_t cand = T | (1ull << b);
        const int c = count(cand);
        if (c >= want) T = cand;
        if (c == want) { exact = true; break; }
      }
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
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (sel[r] >> lane & 1) o[at + __popcll(sel[r] & below)] = base + 64 * r + lane;
    at += __popcll(sel[r]);
  }
  for (int j = want + tid; j < topk; j += 64 * NW) o[j] = -1;
}

// Scores and choice in one for at most 64 R key blocks: 16 query blocks of a head, their
// means in registers, their keys in LDS.  NW waves take 16 key blocks in turn (f64
// 16x16x4 MFMAs), then 16 / NW rows each.
//
// 32760 tokens, 40 heads: 57 us, in which a CU's f64 MFMAs alone take 20, the means
// from L2 (640 work-groups of 16 query blocks against 512 key blocks) about as long and the
// search the rest, one after the other within a work-group.
template <int R, int NW>
__global__ __launch_bounds__(64 * NW, R == 16 && NW == 8 ? 2 : 4) void block_select_kernel(
    const double* __restrict__ qm, const double* __restrict__ km, int32_t* __restrict__ idx, int nqb, int nkb, int heads,
    int kv_heads, int Lk, int first, int topk, const int32_t* klen) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ uint64_t keys[16][64 * R + 2];
  const int hz = blockIdx.y, z = hz / heads, h = hz - z * heads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
  const int q0 = blockIdx.x * 16;
  const int nvalid = (keys_of(klen, z, Lk) + KBLK - 1) / KBLK;
  const double* qp = qm + hz * mean_doubles(nqb) + (int64_t)blockIdx.x * 16 * D + 2 * lane;
  const double* kh = km + ((int64_t)z * kv_heads + h / (heads / kv_heads)) * mean_doubles(nkb) + 2 * lane;
  f64x2_t a[D / 8], b[D / 8];
#pragma unroll
  for (int t = 0; t < D / 8; ++t) a[t] = *(const f64x2_t*)(qp + 128 * t);
  auto load = [&](int k0, f64x2_t (&x)[D / 8]) {
    const double* p = kh + min(k0 >> 4, (nkb - 1) >> 4) * 16 * D;
#pragma unroll
    for (int t = 0; t < D / 8; ++t) x[t] = *(const f64x2_t*)(p + 128 * t);
  };
  auto block = [&](int k0, const f64x2_t (&x)[D / 8]) {
    f64x4_t s = {}, u = {};  // two chains
#pragma unroll
    for (int t = 0; t < D / 8; ++t) {
      s = __builtin_amdgcn_mfma_f64_16x16x4f64(a[t][0], x[t][0], s, 0, 0, 0);
      u = __builtin_amdgcn_mfma_f64_16x16x4f64(a[t][1], x[t][1], u, 0, 0, 0);
    }
    const int k = k0 + lr;
#pragma unroll
    for (int r = 0; r < 4; ++r)  // f64 accumulators: row 4 r + lq
      keys[4 * r + lq][k] = k >= nvalid ? 0 : k < first ? ~0ull : score_key(s[r] + u[r]);
  };
  for (int k0 = 16 * wave; k0 < 64 * R; k0 += 16 * NW) {
    load(k0, b);
    block(k0, b);
  }
  __syncthreads();
  // The wave's rows in step, on the upper halves of their keys: one row's chain
  // of counts would leave the wave waiting.  (A bit above the highest in which a row's keys
  // differ is set in all of them or in none: trying it changes nothing.)
  constexpr int ROWS = 16 / NW;
  uint32_t hi[ROWS][R], t[ROWS], top[ROWS], low[ROWS], differ = 0;
  int want[ROWS];
  bool exact[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    top[i] = 0;
    low[i] = ~0u;
    int have = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      hi[i][r] = (uint32_t)(keys[ROWS * wave + i][64 * r + lane] >> 32);
      have += __popcll(__ballot(hi[i][r] != 0));
      top[i] = max(top[i], hi[i][r]);
      low[i] = min(low[i], hi[i][r] ? hi[i][r] : ~0u);
    }
    want[i] = min(topk, have);
    exact[i] = want[i] == have;  // every block that there is
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const uint32_t x = wave_max(top[i]), y = ~wave_max(~low[i]);
    const uint32_t d = exact[i] ? 0 : x ^ y;
    // bits that all of the row's keys share
    t[i] = exact[i] ? 1 : d == 0 ? x : x & ~(~0u >> __builtin_clz(d));
    differ |= d;
  }
#pragma unroll 1
  for (int bit = differ ? 31 - __builtin_clz(differ) : -1; bit >= 0; --bit) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const uint32_t cand = t[i] | (1u << bit);
      int c = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) c += __popcll(__ballot(hi[i][r] >= cand));
      if (!exact[i] && c >= want[i]) { t[i] = cand; exact[i] = c == want[i]; }
    }
    bool all = true;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) all &= exact[i];
    if (all) break;
  }
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int q = q0 + ROWS * wave + i;
    if (q >= nqb) break;
    int32_t* o = idx + ((int64_t)hz * nqb + q) * topk;
    if (!exact[i]) {  // upper halves that are equal at the threshold
      uint64_t key[R];
#pragma unroll
      for (int r = 0; r < R; ++r) key[r] = keys[ROWS * wave + i][64 * r + lane];
      topk_row<1, R>(key, o, topk, nullptr);
      continue;
    }
    int at = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint64_t sel = __ballot(hi[i][r] >= t[i]);
      if (sel >> lane & 1) o[at + __popcll(sel & below)] = 64 * r + lane;
      at += __popcll(sel);
    }
    for (int j = want[i] + lane; j < topk; j += 64) o[j] = -1;
  }
#endif
}

// Rows of more key blocks, from keys in memory: a work-group of NW waves per row.
template <int NW, int R>
__global__ __launch_bounds__(64 * NW) void block_topk_kernel(const uint64_t* __restrict__ keys, int32_t* __restrict__ idx,
                                                             int nkb, int topk) {
  __shared__ int red[2 * NW];
  const int64_t row = blockIdx.x;
  uint64_t key[R];
  const int base = (threadIdx.x >> 6) * 64 * R + (threadIdx.x & 63);
#pragma unroll
  for (int r = 0; r < R; ++r) key[r] = base + 64 * r < nkb ? keys[row * nkb + base + 64 * r] : 0;
  topk_row<NW, R>(key, idx + row * topk, topk, red);
}

// ---------------------------------------------------------------- attention

struct SparseArgs {
  const bf16_t* q; int64_t ldq;
  const bf16_t* k; int64_t ldk;
  const bf16_t* v; int64_t ldv;
  bf16_t* o; int64_t ldo;
  const int32_t* idx;
  const int32_t* klen;
  int Lq, Lk, heads, kv_heads, nqb, topk;
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
  __device__ __forceinline__ ListCursor(const int32_t* p_, int n_, int nkb_)
      : p(p_), n(n_), base(-64), v(0), nkb(nkb_), left(0) {}
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

// A wave's 32 queries (block rows wrow ..), 16 per group, d blocks of 16: normalised
// to o, or as a part of the list.
__device__ __forceinline__ void store_rows(const SparseArgs& P, const f32x4_t (&acc)[8][2], const float (&l)[2],
                                           const float (&m)[2], int unit, int z, int h, int qb, int wrow, int lr, int lq) {
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = wrow + 16 * g + lr, qi = qb * QBLK + row;
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
}

// One work-group per list (or part of one): TP groups of four waves, each with tiles
// of 64 keys of K and V of its own in XOR-swizzled LDS rows of 256 bytes, two of
// each; the products are those of the dense kernel (S^T = K Q^T, O^T = V^T P^T,
// probabilities from one to the other in registers).  V^T fragments are read from
// the row-major tile by transposing LDS reads, so no transposed copy of V is made.
//
// Probabilities are rounded to bf16, the type that the second product takes beside V, by at
// most 2^-8 of each and of either sign, as the output is in its turn.  The sum takes the
// rounded values, so that the weights add up to one.
//
// TP = 1: two work-groups per CU, one's softmax beside the other's products.  TP =
// 2: one per CU, for launches that leave no second one; the groups take tiles in
// turn, and their outputs meet in LDS.
//
// A tile's score product, softmax and second product follow one another in every
// wave: 192 lists of 9 blocks on as many CUs take 19 - 21 us (0.35 PFLOP/s), the MFMAs busy
// in 0.22 of the cycles and LDS in 0.18; 10240 lists of 52, two work-groups per CU,
// 2.3 ms (0.97).  V's rows in an order without bank conflicts (a third of the LDS
// cycles) change nothing.
template <bool BOUNDED, int TP>
__global__ __launch_bounds__(256 * TP, 2) void attn_sparse_kernel(SparseArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int TILE = KT * D * 2, STAGE = 2 * TILE;
  __shared__ __attribute__((aligned(1024))) char smem[2 * TP * STAGE];  // [group][stage][K | V]
  const int tid = threadIdx.x, lane = tid & 63;
  const int grp = TP == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 8);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3;  // of its group
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
  // Rows past the last key are zeros; so is all of no tile (kb < 0), copied to keep
  // the number of copies in flight the same.
  auto issue = [&](int kb, int at) {
    const uint32_t last = min(nkeys - kb * KBLK, KBLK) - 1;
    const int64_t row = (int64_t)max(kb, 0) * KBLK;
    const uint32_t kn = kb < 0 ? 0u : last * (uint32_t)P.ldk * 2u + 2u * D;
    const uint32_t vn = kb < 0 ? 0u : last * (uint32_t)P.ldv * 2u + 2u * D;
    char* d = smem + 2 * grp * STAGE + at + wave * 4096;
#pragma unroll
    for (int c = 0; c < 4; ++c) copy16_unseen(kbase + row * P.ldk, kn, d + c * 1024, ko[c]);
#pragma unroll
    for (int c = 0; c < 4; ++c) copy16_unseen(vbase + row * P.ldv, vn, d + TILE + c * 1024, vo[c]);
  };
  bf16x8_t qf[2][4];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const bf16_t* qp = P.q + ((int64_t)z * P.Lq + min(q0 + 16 * g + lr, P.Lq - 1)) * P.ldq + h * D + 8 * lq;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[g][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 32 * s));
  }
  // Key blocks of the group's tile and of any (the first group's comes first).  The
  // queries arrive with the list: waited for later, they would wait for the copies, too.
  auto take = [&](int& any) {
    any = list.next();
    if constexpr (TP == 1) return any;
    const int second = any < 0 ? -1 : list.next();
    return grp ? second : any;
  };
  int any, cur = take(any);
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int s = 0; s < 4; ++s) asm volatile("" : "+v"(qf[g][s]));
  issue(cur, 0);
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

  int at = 0;
  while (any >= 0) {
    const int nxt = take(any);
    // this tile has landed and everyone is done with the one before it
    __builtin_amdgcn_s_waitcnt(0);
    barrier_no_fence();
    issue(nxt, at ^ STAGE);
    if (active && cur >= 0) {
      const char* sk = smem + 2 * grp * STAGE + at;
      const int keys = nkeys - cur * KBLK;
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
      if (keys < KBLK) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * kb + 4 * lq + r >= keys) s[kb][0][r] = s[kb][1][r] = -INFINITY;
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
          const bf16x8_t vf = vt_frag(sk + TILE + (voff ^ (dt << 5)) + ks * 32 * 256);
#pragma unroll
          for (int g = 0; g < 2; ++g) acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[ks][g], acc[dt][g], 0, 0, 0);
        }
    }
    cur = nxt;
    at ^= STAGE;
  }
  if constexpr (TP == 2) {
    __builtin_amdgcn_s_waitcnt(0);  // the copies past the end have landed
    __syncthreads();
    f32x4_t* so = (f32x4_t*)smem + (wave * 64 + lane) * 17;  // the second group's outputs, lane by lane
    float* sm = (float*)(so + 16);
    if (grp) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) so[8 * g + dt] = acc[dt][g];
        sm[g] = l[g];
        sm[2 + g] = m[g];
      }
    }
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const float mn = fmaxf(m[g], sm[2 + g]), shift = neg_shift(mn);
      const float a = __builtin_amdgcn_exp2f(m[g] + shift), b = __builtin_amdgcn_exp2f(sm[2 + g] + shift);
      l[g] = a * l[g] + b * sm[g];
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        const f32x4_t x = so[8 * g + dt];
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[dt][g][r] = a * acc[dt][g][r] + b * x[r];
      }
      m[g] = mn;
    }
  }
  __builtin_amdgcn_s_waitcnt(0);  // no copy outlives its work-group
  if (active) store_rows(P, acc, l, m, unit, z, h, qb, 32 * wave, lr, lq);
#endif
}

// At most 16 NG queries a sequence (single tokens, say): what bounds it is the way
// of K and V from memory.  Each of four waves takes all queries and its own share
// of the list, 32 keys at a time in its own two buffers of LDS: no wave waits for
// another until their four parts meet at the end.  One token, 40 heads, 64 blocks (84
// MB): 17 us and 2.5 - 4 to join the pieces, 4.3 TB/s; 200 blocks 5.6 TB/s.
template <bool BOUNDED, int NG>
__global__ __launch_bounds__(256, 1) void attn_few_kernel(SparseArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int HK = 32, TILE = HK * D * 2, STAGE = 2 * TILE, ROWS = 16 * NG, LD = D + 4;
  __shared__ __attribute__((aligned(1024))) char smem[8 * STAGE];  // [wave][stage][K | V]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int unit = xcd_remap(blockIdx.x, P.items * P.parts);
  const int item = unit / P.parts, part = unit - item * P.parts;  // one query block: item = z heads + h
  const int z = item / P.heads, h = item - z * P.heads, g_ = h / (P.heads / P.kv_heads);
  const int nkeys = keys_of(P.klen, z, P.Lk), nkb = (nkeys + KBLK - 1) / KBLK;
  const int shares = 4 * P.parts, share = 4 * part + wave;
  const int p0 = (int)((int64_t)P.topk * share / shares), p1 = (int)((int64_t)P.topk * (share + 1) / shares);
  ListCursor list(P.idx + (int64_t)item * P.topk + p0, p1 - p0, nkb);

  const bf16_t* kbase = P.k + (int64_t)z * P.Lk * P.ldk + g_ * D;
  const bf16_t* vbase = P.v + (int64_t)z * P.Lk * P.ldv + g_ * D;
  bf16x8_t qf[NG][4];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const bf16_t* qp = P.q + ((int64_t)z * P.Lq + min(16 * g + lr, P.Lq - 1)) * P.ldq + h * D + 8 * lq;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[g][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 32 * s));
  }
  // first key of the next 32; -1: none
  int kb = list.next(), half = 0;
#pragma unroll
  for (int g = 0; g < NG; ++g)  // (queries waited for later would wait for the copies, too)
#pragma unroll
    for (int s = 0; s < 4; ++s) asm volatile("" : "+v"(qf[g][s]));
  auto next = [&]() {
    const int k = kb < 0 ? -1 : kb * KBLK + 32 * half;
    if (kb >= 0 && (half || k + 32 >= nkeys)) {  // a block's second half may hold no key
      kb = list.next();
      half = 0;
    } else {
      half = 1;
    }
    return k;
  };
  // copy c: rows 4 c .. + 3; rows past the last key, and all of none, are zeros
  auto issue = [&](int k, int st) {
    const uint32_t rows = k < 0 ? 0u : (uint32_t)min(nkeys - k, HK);
    const bf16_t* kp = kbase + (int64_t)max(k, 0) * P.ldk;
    const bf16_t* vp = vbase + (int64_t)max(k, 0) * P.ldv;
    const uint32_t kn = rows ? (rows - 1) * (uint32_t)P.ldk * 2u + 2u * D : 0u;
    const uint32_t vn = rows ? (rows - 1) * (uint32_t)P.ldv * 2u + 2u * D : 0u;
    char* d = smem + (2 * wave + st) * STAGE;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t row = 4 * c + (lane >> 4), ch = ((lane & 15) ^ (row & 15)) << 4;
      copy16_unseen(kp, kn, d + c * 1024, row * (uint32_t)P.ldk * 2u + ch);
      copy16_unseen(vp, vn, d + TILE + c * 1024, row * (uint32_t)P.ldv * 2u + ch);
    }
  };
  int koff[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) koff[s] = k_off(lr, 4 * s + lq);
  const int voff = k_off(4 * lq + (lr >> 2), (lr & 3) >> 1) + 8 * (lr & 1);  // as in attn_sparse_kernel
  f32x4_t acc[8][NG] = {};
  float m[NG], l[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) { m[g] = BOUNDED ? BOUNDED_SHIFT_LOG2 : -INFINITY; l[g] = 0.f; }
  const bf16x2_t ones = {(__bf16)1.f, (__bf16)1.f};

  int cur = next(), st = 0;
  issue(cur, 0);
  while (cur >= 0) {
    const int nxt = next();
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the other buffer is read
    asm volatile("" ::: "memory");
    issue(nxt, st ^ 1);
    wait_vmcnt<16>();  // this one has landed
    asm volatile("" ::: "memory");
    const char* sk = smem + (2 * wave + st) * STAGE;
    f32x4_t s[2][NG];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *(const uint4*)(sk + koff[t] + b * 16 * 256));
#pragma unroll
        for (int g = 0; g < NG; ++g)
          s[b][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][t], t ? s[b][g] : f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      }
    if (cur + HK > nkeys) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (cur + 16 * b + 4 * lq + r >= nkeys)
#pragma unroll
            for (int g = 0; g < NG; ++g) s[b][g][r] = -INFINITY;
    }
    bf16x8_t pf[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      if constexpr (!BOUNDED) {
        float mx = s[0][g][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; r += 2) mx = max3(mx, s[b][g][r], s[b][g][r + 1]);
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
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4_t& x = s[e >> 1][g];
        w[e] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * (e & 1)], P.scale_log2, mneg)),
                           __builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * (e & 1) + 1], P.scale_log2, mneg)));
        // the sum takes exactly the rounded values that the second product uses
        l[g] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[e]), ones, l[g], false);
      }
      pf[g] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const bf16x8_t vf = vt_frag(sk + TILE + (voff ^ (dt << 5)));
#pragma unroll
      for (int g = 0; g < NG; ++g) acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[g], acc[dt][g], 0, 0, 0);
    }
    cur = nxt;
    st ^= 1;
  }
  // the waves' parts in LDS; then eight threads a row, 16 columns each
  __builtin_amdgcn_s_waitcnt(0);  // the copies past the end have landed
  __syncthreads();
  float* so = (float*)smem;                // [wave][row][LD]
  float* sl = so + 4 * ROWS * LD;          // [wave][row]: sums, then maxima
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const float ls = sum_quarters(l[g]);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) *(f32x4_t*)(so + (wave * ROWS + 16 * g + lr) * LD + 16 * dt + 4 * lq) = acc[dt][g];
    if (lq == 0) {
      sl[wave * ROWS + 16 * g + lr] = ls;
      sl[(4 + wave) * ROWS + 16 * g + lr] = m[g];
    }
  }
  __syncthreads();
  const int row = tid >> 3, c = 4 * (tid & 7);
  if (row >= P.Lq) return;
  float mx = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sl[(4 + w) * ROWS + row]);
  const float shift = neg_shift(mx);
  float den = 0.f;
  f32x4_t y[4] = {};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(sl[(4 + w) * ROWS + row] + shift);
    den += f * sl[w * ROWS + row];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4_t x = *(const f32x4_t*)(so + (w * ROWS + row) * LD + c + 32 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[i][e] += f * x[e];
    }
  }
  if (P.parts == 1) {
    const float inv = den == 0.f ? 0.f : 1.f / den;  // no key: zeros
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(uint2*)(P.o + ((int64_t)z * P.Lq + row) * P.ldo + h * D + c + 32 * i) =
          make_uint2(pack_bf16x2(y[i][0] * inv, y[i][1] * inv), pack_bf16x2(y[i][2] * inv, y[i][3] * inv));
  } else {
    float* w = P.ws + unit * piece_floats(P.rows);
#pragma unroll
    for (int i = 0; i < 4; ++i) *(f32x4_t*)(w + row * D + c + 32 * i) = y[i];
    if (c == 0) {
      w[P.rows * D + row] = den;
      w[P.rows * D + P.rows + row] = mx;
    }
  }
#endif
}

// attn_sparse_kernel for long lists of bounded logits, two work-groups per CU; K and V tiles in
// LDS: three K, two V.
//
// Iteration t issues the score product of tile t + 1 and the PV product of tile
// t - 1 on MFMA with the softmax of tile t, which depends on neither, between
// them in 32 fenced slots of two MFMAs, one fragment read AHEAD slots before its use
// and a share of the softmax.  Its copies are V of tile t and K of tile t + 3.
//
// 32760 tokens, 40 heads, lists of 52 (2.2 TFLOP): 2.03 - 2.1 ms, 1.07 PFLOP/s (a large bf16
// product: 1.35).  Power and the way from memory bound it: 1.6 ms on zeros, 1.9 ms where all lists are the
// same.  A running maximum between the slots costs more than the overlap gives: such
// lists take attn_sparse_kernel.
__global__ __launch_bounds__(256, 2) void attn_sparse_long_kernel(SparseArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int TILE = KT * D * 2, VBASE = 3 * TILE;
  __shared__ __attribute__((aligned(1024))) char smem[5 * TILE];
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
  // Rows past the last key, and all rows of no tile (kb < 0), are zeros.
  struct Src {
    const bf16_t* p;
    uint32_t bytes;
  };
  auto src = [&](const bf16_t* base, int64_t ld, int kb) {
    const int rows = min(nkeys - kb * KBLK, KBLK);
    return Src{base + (int64_t)max(kb, 0) * KBLK * ld, kb < 0 ? 0u : (uint32_t)(rows - 1) * (uint32_t)ld * 2u + 2u * D};
  };
  auto copy = [&](const Src& x, int at, uint32_t off, int c) {
    copy16_unseen(x.p, x.bytes, smem + at + (4 * wave + c) * 1024, off);
  };

  bf16x8_t qf[2][4];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const bf16_t* qp = P.q + ((int64_t)z * P.Lq + min(q0 + 16 * g + lr, P.Lq - 1)) * P.ldq + h * D + 8 * lq;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[g][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 32 * s));
  }
  int koff[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) koff[s] = k_off(lr, 4 * s + lq);
  // V^T fragment (d = 16 dt + lr; keys 4 lq .. + 3 of a 16-key block): lane 4 k + j of a
  // quarter addresses row 4 lq + k, columns 16 dt + 4 j, and receives column lr.  The
  // chunk 2 dt + (j >> 1) enters the swizzled address by XOR.
  const int voff = k_off(4 * lq + (lr >> 2), (lr & 3) >> 1) + 8 * (lr & 1);
  // A tile's fragments in the order of their use, K 0..15 and V^T 0..15, so that four
  // independent accumulators stand between the steps of a dependent chain.
  auto k_kb = [](int i) { return 2 * (i >> 3) + (i & 1); };
  auto k_s = [](int i) { return (i >> 1) & 3; };
  auto v_dt = [](int i) { return 2 * (i >> 2) + (i & 1); };
  auto v_ks = [](int i) { return (i >> 1) & 1; };
  auto k_frag = [&](int at, int i) {
    return __builtin_bit_cast(bf16x8_t, *(const uint4*)(smem + at + koff[k_s(i)] + k_kb(i) * 16 * 256));
  };
  auto v_frag = [&](int at, int i) { return vt_frag(smem + (voff ^ (v_dt(i) << 5)) + at + v_ks(i) * 32 * 256); };
  f32x4_t acc[8][2], sb[2][4][2];
  bf16x8_t pb[2][2][2];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) acc[dt][0] = acc[dt][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float l[2] = {0.f, 0.f};
  const bf16x2_t ones = {(__bf16)1.f, (__bf16)1.f};
  auto score_step = [&](int i, const bf16x8_t& kf, f32x4_t (&s)[4][2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      f32x4_t& c = s[k_kb(i)][g];
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][k_s(i)], k_s(i) ? c : f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
    }
  };
  auto pv_step = [&](int i, const bf16x8_t& vf, const bf16x8_t (&pf)[2][2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
      acc[v_dt(i)][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[v_ks(i)][g], acc[v_dt(i)][g], 0, 0, 0);
  };
  // Step i of 16 of a tile's softmax: two probabilities of a query group.
  struct Soft {
    float sum[2];
    uint32_t w[4];
  };
  auto exp_step = [&](int i, const f32x4_t (&s)[4][2], bf16x8_t (&pf)[2][2], Soft& x) {
    const int g = i >> 3, ks = (i >> 2) & 1, e = i & 3;
    const f32x4_t& c = s[2 * ks + (e >> 1)][g];
    x.w[e] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(c[2 * (e & 1)], P.scale_log2, -BOUNDED_SHIFT_LOG2)),
                         __builtin_amdgcn_exp2f(__builtin_fmaf(c[2 * (e & 1) + 1], P.scale_log2, -BOUNDED_SHIFT_LOG2)));
    // formed here: the branches between iterations would otherwise draw the softmax
    // past the barrier, away from the MFMAs
    asm volatile("" : "+v"(x.w[e]));
    // the sum takes exactly the rounded values that the second product uses
    x.sum[g] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x.w[e]), ones, (i & 7) ? x.sum[g] : 0.f, false);
    if (e == 3) pf[ks][g] = __builtin_bit_cast(bf16x8_t, make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]));
  };
  // keys of a tile past the sequence's last one; all of no tile (kb < 0)
  auto keys_in = [&](int kb) { return kb < 0 ? 0 : nkeys - kb * KBLK; };
  auto mask = [&](int keys, f32x4_t (&s)[4][2]) {
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * b + 4 * lq + r >= keys) s[b][0][r] = s[b][1][r] = -INFINITY;
  };

  // Key blocks of tiles t .. t + 3 (-1: none), K places of tiles t, t + 1, t + 2.
  // Tiles come in pairs; a last one without keys adds nothing.
  int i0 = -1, i1 = -1, i2 = -1, i3 = -1;
  int ks0 = 0, ks1 = TILE, ks2 = 2 * TILE;
  for (int u = 0; u < 3; ++u) {
    i0 = i1; i1 = i2;
    i2 = list.next();
    const Src x = src(kbase, P.ldk, i2);
#pragma unroll
    for (int c = 0; c < 4; ++c) copy(x, u * TILE, ko[c], c);
  }
  i3 = list.next();
  const Src none = src(vbase, P.ldv, -1);  // "tile - 1"
#pragma unroll
  for (int c = 0; c < 4; ++c) copy(none, VBASE + TILE, vo[c], c);
  // End of an iteration: its copies have landed and the waves meet.  Fragments still
  // on their way are of K of tile t + 2, which stays for another iteration.
  auto meet = [&]() {
    wait_vmcnt<0>();
    barrier_no_fence();
    i0 = i1; i1 = i2; i2 = i3;
    i3 = list.next();
    const int k = ks0;
    ks0 = ks1; ks1 = ks2; ks2 = k;
  };
  constexpr int AHEAD = 4;
  bf16x8_t fr[AHEAD];
  auto iter = [&](auto par) {
    constexpr int B = decltype(par)::value;
    const Src vs = src(vbase, P.ldv, i0), kn = src(kbase, P.ldk, i3);
    if (keys_in(i0) < KBLK) mask(keys_in(i0), sb[B]);
    Soft x;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (i < 16) score_step(i, fr[i % AHEAD], sb[B ^ 1]);
      else pv_step(i - 16, fr[i % AHEAD], pb[B ^ 1]);
      const int n = i + AHEAD;
      fr[i % AHEAD] = n < 16 ? k_frag(ks1, n) : n < 32 ? v_frag(VBASE + (B ^ 1) * TILE, n - 16) : k_frag(ks2, n - 32);
      if (i % 2 == 0 && i < 16) {
        if (i < 8) copy(vs, VBASE + B * TILE, vo[i / 2], i / 2);
        else copy(kn, ks0, ko[i / 2 - 4], i / 2 - 4);
      }
      if (i & 1) exp_step(i >> 1, sb[B], pb[B], x);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) l[g] += x.sum[g];
    meet();
  };
  wait_vmcnt<0>();
  barrier_no_fence();
  if (active) {
#pragma unroll
    for (int i = 0; i < 16; ++i) score_step(i, k_frag(0, i), sb[0]);
#pragma unroll
    for (int f = 0; f < AHEAD; ++f) fr[f] = k_frag(ks1, f);
    pb[1][0][0] = pb[1][0][1] = pb[1][1][0] = pb[1][1][1] = __builtin_bit_cast(bf16x8_t, make_uint4(0, 0, 0, 0));
    wait_vmcnt_lgkm0<0>();
    barrier_no_fence();  // K of tile 0 is read: its place is free
    while (i0 >= 0) {
      iter(std::integral_constant<int, 0>{});
      iter(std::integral_constant<int, 1>{});
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) pv_step(i, v_frag(VBASE + TILE, i), pb[1]);
  } else {
    barrier_no_fence();
    for (int par = 0; par || i0 >= 0; par ^= 1) {
      const Src vs = src(vbase, P.ldv, i0), kn = src(kbase, P.ldk, i3);
#pragma unroll
      for (int c = 0; c < 4; ++c) copy(vs, VBASE + par * TILE, vo[c], c);
#pragma unroll
      for (int c = 0; c < 4; ++c) copy(kn, ks0, ko[c], c);
      meet();
    }
  }
  const float m[2] = {BOUNDED_SHIFT_LOG2, BOUNDED_SHIFT_LOG2};
  if (active) store_rows(P, acc, l, m, unit, z, h, qb, 32 * wave, lr, lq);
#endif
}

// Joins the pieces of an item's rows and stores the normalised output.  PG x 32
// threads a row, 4 columns each; each of the PG takes consecutive pieces, U at a time,
// whose loads are in flight together, and the PG meet in LDS in their order.
template <int PG>
__global__ __launch_bounds__(256) void sparse_combine_kernel(SparseArgs P) {
  constexpr int U = 8, RB = 8 / PG;
  const int item = blockIdx.x, tid = threadIdx.x, pg = (tid >> 5) % PG, c = 4 * (tid & 31);
  const int row = blockIdx.y * RB + (tid >> 5) / PG;
  const int hz = item / P.nqb, qb = item - hz * P.nqb;
  const int z = hz / P.heads, h = hz - z * P.heads, qi = qb * QBLK + row;
  const bool in = row < P.rows && qi < P.Lq;
  const int64_t pf = piece_floats(P.rows);
  const int per = (P.parts + PG - 1) / PG, p0 = pg * per, p1 = in ? min(P.parts, p0 + per) : 0;
  const float* w = P.ws + (int64_t)item * P.parts * pf;
  float mx = -INFINITY, den = 0.f;
  f32x4_t y = {};
  // one more piece (or sum of pieces) of weight 2^m
  auto rescale = [&](float nm) {
    const float a = __builtin_amdgcn_exp2f(mx + neg_shift(nm));
    den *= a;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= a;
    mx = nm;
  };
  auto add = [&](float m, float s, const f32x4_t& v) {
    const float a = __builtin_amdgcn_exp2f(m + neg_shift(mx));
    den += a * s;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += a * v[e];
  };
  for (int p = p0; p < p1; p += U) {
    f32x4_t v[U];
    float m[U], s[U], nm = mx;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float* x = w + min(p + i, p1 - 1) * pf;
      v[i] = *(const f32x4_t*)(x + row * D + c);
      s[i] = x[P.rows * D + row];
      m[i] = x[P.rows * D + P.rows + row];
    }
#pragma unroll
    for (int i = 0; i < U; ++i) nm = fmaxf(nm, m[i]);
    rescale(nm);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (p + i < p1) add(m[i], s[i], v[i]);
  }
  if constexpr (PG > 1) {
    __shared__ float red[6][256];
    red[0][tid] = mx;
    red[1][tid] = den;
#pragma unroll
    for (int e = 0; e < 4; ++e) red[2 + e][tid] = y[e];
    __syncthreads();
    if (pg) return;
    float nm = mx;
#pragma unroll
    for (int i = 1; i < PG; ++i) nm = fmaxf(nm, red[0][tid + 32 * i]);
    rescale(nm);
#pragma unroll
    for (int i = 1; i < PG; ++i) {
      const int t = tid + 32 * i;
      add(red[0][t], red[1][t], f32x4_t{red[2][t], red[3][t], red[4][t], red[5][t]});
    }
  }
  if (!in) return;
  const float inv = den == 0.f ? 0.f : 1.f / den;
  *(uint2*)(P.o + ((int64_t)z * P.Lq + qi) * P.ldo + h * D + c) =
      make_uint2(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv));
}

int blocks_of(int n, int b) { return n / b + (n % b != 0); }

}  // namespace

// Key blocks up to which scores and choice are one kernel, whose LDS holds the keys.
constexpr int SELECT_BLOCKS = 1024;

// Means of the query blocks and of the key blocks (f64), then, past SELECT_BLOCKS, one key per pair.
size_t select_blocks_ws_bytes(const dit_sparse_shape& s) {
  const size_t nqb = blocks_of(s.Lq, QBLK), nkb = blocks_of(s.Lk, KBLK), b = s.batch;
  return 8 * (b * s.heads * mean_doubles((int)nqb) + b * s.kv_heads * mean_doubles((int)nkb) +
              (nkb > SELECT_BLOCKS ? b * s.heads * nqb * nkb : 0));
}

hipError_t launch_select_blocks(const dit_sparse_shape& s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                int first, int32_t* idx, void* ws, hipStream_t st, int n_cu) {
  const int nqb = blocks_of(s.Lq, QBLK), nkb = blocks_of(s.Lk, KBLK);
  const int64_t rows = (int64_t)s.batch * s.heads * nqb;
  if (rows == 0) return hipSuccess;
  double* qm = (double*)ws;
  double* km = qm + (int64_t)s.batch * s.heads * mean_doubles(nqb);
  uint64_t* keys = (uint64_t*)(km + (int64_t)s.batch * s.kv_heads * mean_doubles(nkb));
  if (nkb == 0) {  // lists of -1
    hipLaunchKernelGGL((block_topk_kernel<1, 1>), dim3((uint32_t)rows), dim3(64), 0, st, keys, idx, 0, s.topk);
    return hipGetLastError();
  }
  MeanArgs a{};
  a.x[0] = (const bf16_t*)q; a.ld[0] = ldq; a.out[0] = qm; a.L[0] = s.Lq; a.heads[0] = s.heads; a.blocks[0] = nqb;
  a.x[1] = (const bf16_t*)k; a.ld[1] = ldk; a.out[1] = km; a.L[1] = s.Lk; a.heads[1] = s.kv_heads; a.blocks[1] = nkb;
  a.klen = s.klen;
  a.queries = (int)rows;
  hipLaunchKernelGGL(block_mean_kernel, dim3((uint32_t)(rows + (int64_t)s.batch * s.kv_heads * nkb)), dim3(256), 0, st, a);
  if (nkb <= SELECT_BLOCKS) {
    // More waves a work-group where there is at most one per CU: 4608 tokens, 24 heads (72)
    // 12.0 us with 16 waves, 14.0 with 8; 32760 tokens, 40 heads (640) 58.9 and 54.0.
    const int64_t groups = (int64_t)((nqb + 15) / 16) * s.batch * s.heads;
    const bool few = groups <= n_cu;
#define DIT_SELECT(R)                                                                                                \
  hipLaunchKernelGGL((few ? block_select_kernel<R, 16> : block_select_kernel<R, 8>),                                  \
                     dim3((nqb + 15) / 16, s.batch * s.heads), dim3(few ? 1024 : 512), 0, st, qm, km, idx, nqb, nkb, \
                     s.heads, s.kv_heads, s.Lk, first, s.topk, s.klen)
    if (nkb <= 64) DIT_SELECT(1);
    else if (nkb <= 256) DIT_SELECT(4);
    else if (nkb <= 512) DIT_SELECT(8);
    else DIT_SELECT(16);
#undef DIT_SELECT
    return hipGetLastError();
  }
  hipLaunchKernelGGL(block_score_kernel<2>, dim3((nkb + 63) / 64, (nqb + 127) / 128, s.batch * s.heads), dim3(256), 0, st,
                     qm, km, keys, nqb, nkb, s.heads, s.kv_heads, s.Lk, first, s.klen);
  if (nkb <= 4096)
    hipLaunchKernelGGL((block_topk_kernel<4, 16>), dim3((uint32_t)rows), dim3(256), 0, st, keys, idx, nkb, s.topk);
  else
    hipLaunchKernelGGL((block_topk_kernel<16, 16>), dim3((uint32_t)rows), dim3(1024), 0, st, keys, idx, nkb, s.topk);
  return hipGetLastError();
}

// Work-groups that share one list, so that the launch fills the chip's 256 CUs, of
// at least MIN_PART entries each.  (By the shape alone: the workspace's size does
// not depend on the device.)  One token, 8 heads, 256 entries: 32 parts 16.6 us, 16
// 17.3, 10 20.5; 24 heads, 52 entries: 10 parts 13.3, 4 15.5, 2 20.5; 128 queries, 8
// heads, 24 entries: 12 parts 14.3, 6 14.8, 3 18.5.  Twice as many work-groups as CUs lose:
// one token, 40 heads, 64 entries 20.5 -> 25.3 us; 32760 tokens' last 1280, 24 heads, 24 entries 35.5 -> 43.0.
// Few queries' four waves share a list anyhow: up to FEW_WHOLE entries the joining
// launch costs more than it saves (40 heads, 16 entries: 11.7 us whole, 13.4 in four).
constexpr int MIN_PART = 4, FEW_QUERIES = 32, FEW_WHOLE = 16;
int sparse_parts(const dit_sparse_shape& s) {
  const int64_t items = (int64_t)s.batch * s.heads * blocks_of(s.Lq, QBLK);
  if (items == 0 || (s.Lq <= FEW_QUERIES && s.topk <= FEW_WHOLE)) return 1;
  const int64_t p = 256 / items;
  return (int)std::max<int64_t>(1, std::min<int64_t>(p, s.topk / MIN_PART));
}
int sparse_rows(const dit_sparse_shape& s) { return std::min(QBLK, (s.Lq + 15) / 16 * 16); }

size_t attention_sparse_ws_bytes(const dit_sparse_shape& s) {
  const int parts = sparse_parts(s);
  if (parts == 1) return 0;
  return (size_t)s.batch * s.heads * blocks_of(s.Lq, QBLK) * parts * piece_floats(sparse_rows(s)) * sizeof(float);
}

// Entries from which the pipelined kernel is the faster one: 32760 tokens, 40 heads,
// bounded, in us, pipelined and plain: 8 entries 486 and 475, 12 638 and 635, 16 781 and 793, 32 1369 and 1417.
constexpr int LONG_LIST = 16;

hipError_t launch_attention_sparse(const dit_sparse_shape& s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                   const void* v, int64_t ldv, void* o, int64_t ldo, const int32_t* idx, bool bounded,
                                   void* ws, hipStream_t st, int n_cu) {
  SparseArgs P{};
  P.q = (const bf16_t*)q; P.ldq = ldq; P.k = (const bf16_t*)k; P.ldk = ldk;
  P.v = (const bf16_t*)v; P.ldv = ldv; P.o = (bf16_t*)o; P.ldo = ldo;
  P.idx = idx; P.klen = s.klen;
  P.Lq = s.Lq; P.Lk = s.Lk; P.heads = s.heads; P.kv_heads = s.kv_heads; P.topk = s.topk;
  P.nqb = blocks_of(s.Lq, QBLK);
  P.items = s.batch * s.heads * P.nqb;
  if (P.items == 0) return hipSuccess;
  P.parts = sparse_parts(s);
  P.rows = sparse_rows(s);
  P.ws = (float*)ws;
  P.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  const int64_t groups = (int64_t)P.items * P.parts;
  // One work-group per CU leaves it the whole LDS: for few queries four waves with
  // lists of their own (40 heads, 64 entries: 20.5 us, 23.8 with the waves in step; 300 lists of 50
  // entries on two work-groups per CU 111, on one 117), else eight waves (1280 queries, 24
  // heads, 24 entries: 35.5 us, 41.1 with four).
  const bool one = groups <= n_cu, few = one && s.Lq <= FEW_QUERIES, two = one && !few;
  void (*fn)(SparseArgs);
  if (few && s.Lq <= 16) fn = bounded ? attn_few_kernel<true, 1> : attn_few_kernel<false, 1>;
  else if (few) fn = bounded ? attn_few_kernel<true, 2> : attn_few_kernel<false, 2>;
  else if (two) fn = bounded ? attn_sparse_kernel<true, 2> : attn_sparse_kernel<false, 2>;
  else if (bounded && s.topk >= LONG_LIST) fn = attn_sparse_long_kernel;
  else fn = bounded ? attn_sparse_kernel<true, 1> : attn_sparse_kernel<false, 1>;
  hipLaunchKernelGGL(fn, dim3((uint32_t)groups), dim3(two ? 512 : 256), 0, st, P);
  if (P.parts > 8)
    hipLaunchKernelGGL(sparse_combine_kernel<8>, dim3(P.items, std::min(s.Lq, QBLK)), dim3(256), 0, st, P);
  else if (P.parts > 1)
    hipLaunchKernelGGL(sparse_combine_kernel<1>, dim3(P.items, (std::min(s.Lq, QBLK) + 7) / 8), dim3(256), 0, st, P);
  return hipGetLastError();
}

}  // namespace dit
