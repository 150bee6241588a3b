// Attention kernels of the DiT blocks.
//
// bf16 flash attention (head_dim 128) on gfx950 MFMA 16x16x32.  The score
// tile is computed transposed, S^T = K Q^T, so each lane holds one query's
// scores: row statistics need one exchange over the four lanes of a query and
// the running rescale of the output is a per-lane scalar.  The output is
// accumulated transposed as well, O^T = V^T P^T, which lets the probabilities
// feed the second MFMA straight from the score accumulators (same lane, same
// registers); V is therefore read from a per-head transposed copy [128][keys]
// whose keys are permuted inside 32-key groups so each operand is one 16-byte
// LDS read.  K and V^T tiles of 64 keys are copied into XOR-swizzled LDS.
// With bounded logits (unit-gain RMS-normalised q and k) a fixed shift
// replaces the running max; the row sum takes the bf16-rounded P with a
// packed dot product.  Exact-softmax semantics (non-causal), f32 statistics,
// output normalised once at the end.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "attention_tile.h"
#include "common.h"
#include "kernels.h"

namespace dit {
namespace {

// Position of key k (0..31) inside its 32-key group of the transposed V: the
// two 4-key runs a lane quarter needs for one MFMA k-step become adjacent.
__host__ __device__ constexpr int vt_slot(int k) { return 8 * ((k >> 2) & 3) + 4 * (k >> 4) + (k & 3); }

// LDS tiles (bf16, no padding): K [64 keys][128 d], 16-byte chunk c of row r
// stored at chunk c ^ (r & 15); V^T [128 d][64 keys], chunk c of row d at
// c ^ ((d >> 1) & 7).  Both make the MFMA operand reads of 16 consecutive
// rows hit 16 distinct 16-byte bank groups.
__device__ __forceinline__ int v_off(int d, int c) { return d * 128 + ((c ^ ((d >> 1) & 7)) << 4); }

// Rows of one joint sequence that lies in two pieces (the text rows of a
// sequence, then its image rows further down a buffer of several stacked
// sequences): row r is stored at base + r, plus gap once r >= split.
// split = INT_MAX: one piece.
struct RowMap {
  int split;
  int64_t gap, base;
  __device__ __forceinline__ int64_t operator()(int r) const { return base + r + (r >= split ? gap : 0); }
};

// Sequence z of a launch (blockIdx.z): base z * zs, gap gap0 + z * gz.
struct SeqMap {
  int split;
  int64_t gap0, gz, zs;
  __host__ __device__ __forceinline__ RowMap at(int z) const { return RowMap{split, gap0 + z * gz, z * zs}; }
};

constexpr int TILE_BYTES = 2 * KT * D * 2;

// What bounds it: at many keys the board's power (the clock sits near 2.05 GHz)
// and the softmax beside the products (VALU and MFMA each about 0.6 busy); at
// 512 keys the queries and outputs on their way from and to HBM; at few items
// the last, partly filled round of the chip.  Measured in turn on one card
// through the entry point (transpose included) against one work-group per item
// on 32x32x16 MFMAs: 32760 x 32760, 40 heads 18.1 -> 17.4 ms; 16896^2, 24 heads
// (6.2 rounds) 3200 -> 2752 us; 4352^2, 48 heads (3.2 rounds) 517 -> 436 us;
// 4608^2, 24 heads (1.7 rounds) 275 -> 260 us; 1536^2, 96 heads 170 -> 148 us;
// 32760 x 512, 40 heads 483 -> 410 us; 5000^2, 3 heads 133 -> 72 us.
//
// One launch runs at most one work-group per CU (all of LDS) over a list of
// (sequence, head, 256-query block) items; see Plan.  Per key tile t of an
// item, one iteration issues the PV product of tile t - 1 and the score
// product of tile t + 1 on MFMA together with the softmax of tile t (VALU),
// which depends on neither.  Five LDS stages: tiles t - 1 (V), t, t + 1 (K),
// t + 2 and t + 3 (in flight).  The copies run on through the list, so an
// item starts on tiles that the previous one's last iterations fetched.
constexpr int PSTAGE = 5;
// The last round is shared out when that shortens the longest work-group by
// this many tiles (about 1.7 us each): the second launch and the pieces' round
// trip take 12-17 us at the shapes above.
constexpr int SPLIT_MIN_TILES = 8;
constexpr int SMALL_MAX_KEYS = 1280;
constexpr int NW = 8;          // waves per work-group, 32 queries each
constexpr int QB = 32 * NW;    // queries per item
constexpr int CPW = 16 / NW;   // 1 KB copies per wave for each of K and V^T

// Items are numbered sequence-major, then head, then query block.  Work-groups
// are dispatched to the 8 XCDs round-robin (block b to XCD b % 8); XCD x takes
// one contiguous range of items, so that the work-groups that stream one
// head's K and V at a time share an L2.  Its W work-groups take whole items in
// rounds.  The last, partial round (rem items) is either one item each for rem
// of them, or (split) its rem x ntiles key tiles in W contiguous shares: each
// share covers a part of one item or of two, whose unnormalised outputs go to
// the workspace for attn_combine_kernel.
struct Plan {
  int items, nqb, heads, ntiles;
  int shares;  // most shares of an XCD's last round; 0: whole items
};

struct Range {  // items of one XCD
  int start, full, rem;
  __host__ __device__ Range(int items, int x, int W) {
    const int q = items >> 3, r = items & 7, cnt = q + (x < r ? 1 : 0);
    start = x * q + (x < r ? x : r);
    full = cnt / W;
    rem = cnt % W;
  }
};
// First key tile (over the rem items) of share j.  A share has at least
// SHARE_MIN_TILES tiles, so that writing and adding its piece (133 KB) stays
// below the time of its products, and at most ntiles.
constexpr int SHARE_MIN_TILES = 4;
struct Shares {
  int n;  // shares
  int64_t units;
  __host__ __device__ Shares(int rem, const Plan& p) {
    units = (int64_t)rem * p.ntiles;
    const int64_t most = units / SHARE_MIN_TILES;
    n = most < rem ? rem : most < p.shares ? (int)most : p.shares;
  }
  __host__ __device__ int at(int j) const { return (int)(units * (j < n ? j : n) / n); }
};

// Partial output of a piece: O^T in register order (wave, 16 blocks of 16 d x
// 16 queries, lane, 4 d), then the queries' row sums and running maxima.
constexpr int PIECE_FLOATS = QB * D + 2 * QB;

template <bool BOUNDED>
__global__ __launch_bounds__(64 * NW) void flash_attn_kernel(
    const bf16_t* __restrict__ q, int64_t ldq, const bf16_t* __restrict__ k, int64_t ldk,
    const bf16_t* __restrict__ vt, int ldvt, bf16_t* __restrict__ o, int64_t ldo, int Lq, int Lk,
    float scale_log2, SeqMap sm, Plan pl, float* __restrict__ ws) {
  __shared__ __attribute__((aligned(1024))) char smem[PSTAGE * TILE_BYTES];  // [stage][K | V^T]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;

  // this work-group's items: nfull whole ones, then its share of the rest
  const int W = gridDim.x >> 3, j = blockIdx.x >> 3;
  const Range rg(pl.items, blockIdx.x & 7, W);
  const bool split = pl.shares && rg.rem;
  const Shares sh(rg.rem, pl);
  const int u0 = split ? sh.at(j) : 0, u1 = split ? sh.at(j + 1) : 0;
  const int nfull = rg.full + (!split && j < rg.rem ? 1 : 0);
  const int first_rest = u0 / pl.ntiles;  // of the rest
  const int nseg = nfull + (u1 > u0 ? (u1 - 1) / pl.ntiles - first_rest + 1 : 0);
  if (nseg == 0) return;

  struct Seg {
    int z, h, q0, t0, n, piece;  // key tiles t0 .. t0 + n - 1; piece: workspace slot or -1
  };
  auto segment = [&](int i) {
    Seg s;
    int item;
    if (i < nfull) {
      item = rg.start + i * W + j;
      s.t0 = 0;
      s.n = pl.ntiles;
      s.piece = -1;
    } else {
      const int r = first_rest + i - nfull;
      item = rg.start + rg.full * W + r;
      s.t0 = max(u0 - r * pl.ntiles, 0);
      s.n = min(u1 - r * pl.ntiles, pl.ntiles) - s.t0;
      s.piece = s.n == pl.ntiles ? -1 : 2 * (int)blockIdx.x + i - nfull;
    }
    const int hb = item / pl.nqb;
    s.q0 = (item - hb * pl.nqb) * QB;
    s.z = hb / pl.heads;
    s.h = hb - s.z * pl.heads;
    return s;
  };

  // copies of a key tile: K rows 4 ii .. 4 ii + 3 and V^T rows 8 ii .. 8 ii + 7
  // for ii = CPW wave + c.  A tile on one side of the split takes one uniform
  // base and these per-lane byte offsets (32 bits: ldk, ldvt < 2^24); rows past
  // the last key read zeros.
  const bool narrow = ldk < (1 << 24) && ldvt < (1 << 24) && (sm.split >= Lk || sm.split % KT == 0);
  uint32_t kvo[CPW], vvo[CPW];
#pragma unroll
  for (int c = 0; c < CPW; ++c) {
    const int ii = wave * CPW + c;
    const int row = 4 * ii + (lane >> 4), d = 8 * ii + (lane >> 3);
    kvo[c] = ((uint32_t)row * (narrow ? (uint32_t)ldk : 0) + (((lane & 15) ^ (row & 15)) << 3)) * 2u;
    vvo[c] = ((uint32_t)d * (narrow ? (uint32_t)ldvt : 0) + (((lane & 7) ^ ((d >> 1) & 7)) << 3)) * 2u;
  }
  // The copies' own place in the list, three tiles ahead of the products: tile
  // ct of segment cs, its bases and bytes worked out an iteration ahead.  Past
  // the end of the list (ci == nseg) the narrow form copies the last tile
  // again, so that every iteration waits for the same number of copies.
  int ci = 0, ct = 0;
  Seg cs = segment(0);
  struct {
    uint32_t k_lo, k_hi, k_bytes, v_lo, v_hi;
  } cp;
  auto uniform = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
  auto find_copy = [&](const Seg& s, int tile) {
    const int kb0 = tile * KT;
    const uint64_t kp = (uint64_t)(k + sm.at(s.z)(kb0)*ldk + s.h * D);
    const uint64_t vp = (uint64_t)(vt + (int64_t)(s.z * pl.heads + s.h) * D * ldvt + kb0);
    cp.k_lo = uniform((uint32_t)kp);
    cp.k_hi = uniform((uint32_t)(kp >> 32));
    cp.v_lo = uniform((uint32_t)vp);
    cp.v_hi = uniform((uint32_t)(vp >> 32));
    cp.k_bytes = uniform((uint32_t)(min(Lk - kb0, KT) - 1) * (uint32_t)ldk * 2u + 2u * D);
  };
  // NARROW: known to be.  (The middle iterations hold no global_load_lds: the
  // compiler counts one as an LDS event that may return out of order, and
  // then waits for every LDS read instead of the oldest.)
  auto issue = [&](int so, auto narrow_) {
    constexpr bool NARROW = decltype(narrow_)::value;
    char* sk = smem + so + wave * CPW * 1024;
    char* sv = sk + KT * D * 2;
    if (NARROW || narrow) {
      const void* kt = (const void*)(((uint64_t)cp.k_hi << 32) | cp.k_lo);
      const void* vh = (const void*)(((uint64_t)cp.v_hi << 32) | cp.v_lo);
#pragma unroll
      for (int c = 0; c < CPW; ++c) {
        copy16(kt, cp.k_bytes, (lds_void_t*)(sk + c * 1024), kvo[c]);
        copy16(vh, 0xffffffffu, (lds_void_t*)(sv + c * 1024), vvo[c]);
      }
    } else if (ci < nseg) {
      const RowMap rm = sm.at(cs.z);
      const int kb0 = (cs.t0 + ct) * KT;
      const bf16_t* kh = k + cs.h * D;
      const bf16_t* vh = vt + (int64_t)(cs.z * pl.heads + cs.h) * D * ldvt + kb0;
#pragma unroll
      for (int c = 0; c < CPW; ++c) {
        const int ii = wave * CPW + c;
        const int row = 4 * ii + (lane >> 4), d = 8 * ii + (lane >> 3);
        __builtin_amdgcn_global_load_lds(
            (glb_void_t*)(kh + rm(min(kb0 + row, Lk - 1)) * ldk + (((lane & 15) ^ (row & 15)) << 3)),
            (lds_void_t*)(sk + c * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((glb_void_t*)(vh + (int64_t)d * ldvt + (((lane & 7) ^ ((d >> 1) & 7)) << 3)),
                                         (lds_void_t*)(sv + c * 1024), 16, 0, 0);
      }
    }
  };
  auto issued = [&]() {  // on to the next tile
    if (ci == nseg) return;
    if (ct + 1 < cs.n) {
      ++ct;
    } else if (++ci < nseg) {
      cs = segment(ci);
      ct = 0;
    }
    find_copy(cs, cs.t0 + ct);
  };
  find_copy(cs, cs.t0);

  // Fragments (16x16x32).  Q^T (B operand): d = 32 s + 8 lq + [0, 8) of query
  // 16 g + lr.  K (A): key 16 kb + lr, the same d.  S^T: query lr, keys 4 lq +
  // [0, 4) of block kb.  P^T (B): blocks 2 ks and 2 ks + 1 of a lane side by
  // side, so slot 8 lq + e of a 32-key group is key 16 (e >> 2) + 4 lq + (e & 3):
  // the key order of V^T (A: row d = 16 dt + lr, slots 32 ks + 8 lq + [0, 8)).
  bf16x8_t qf[2][4];
  auto load_q = [&](const Seg& s) {
    const RowMap rm = sm.at(s.z);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const bf16_t* qp = q + rm(min(s.q0 + 32 * wave + 16 * g + lr, Lq - 1)) * ldq + s.h * D + 8 * lq;
#pragma unroll
      for (int t = 0; t < 4; ++t) qf[g][t] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 32 * t));
    }
  };
  int koff[4], voff[2];
#pragma unroll
  for (int s = 0; s < 4; ++s) koff[s] = k_off(lr, 4 * s + lq);
#pragma unroll
  for (int s = 0; s < 2; ++s) voff[s] = KT * D * 2 + v_off(lr, 4 * s + lq);
  // A tile's fragments in the order of their use: V^T 0..15 (two d blocks, then
  // their k-steps) and K 0..15 (two key blocks, then their d steps), so that
  // four independent accumulators stand between the steps of a dependent chain.
  auto v_dt = [](int i) { return 2 * (i >> 2) + (i & 1); };
  auto v_ks = [](int i) { return (i >> 1) & 1; };
  auto k_kb = [](int i) { return 2 * (i >> 3) + (i & 1); };
  auto k_s = [](int i) { return (i >> 1) & 3; };
  auto v_frag = [&](int so, int i) {
    return __builtin_bit_cast(bf16x8_t, *(const uint4*)(smem + so + voff[v_ks(i)] + v_dt(i) * 16 * 128));
  };
  auto k_frag = [&](int so, int i) {
    return __builtin_bit_cast(bf16x8_t, *(const uint4*)(smem + so + koff[k_s(i)] + k_kb(i) * 16 * 256));
  };
  auto scores_step = [&](int i, const bf16x8_t& kf, f32x4_t (&sacc)[4][2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      f32x4_t& c = sacc[k_kb(i)][g];
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][k_s(i)], k_s(i) ? c : f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
    }
  };
  auto scores = [&](int so, f32x4_t (&sacc)[4][2]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) scores_step(i, k_frag(so, i), sacc);
  };
  f32x4_t oacc[8][2];
  float m_run[2], l_run[2];
  const bf16x2_t ones = {(__bf16)1.f, (__bf16)1.f};
  auto mask = [&](int t, f32x4_t (&sacc)[4][2]) {  // keys past the last one
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (t * KT + kb * 16 + 4 * lq + r >= Lk) sacc[kb][0][r] = sacc[kb][1][r] = -INFINITY;
  };
  // running maximum (kept unless the new one is more than RESCALE_SLACK above
  // it: softmax is shift invariant); rescales what has been accumulated
  auto tile_max = [&](const f32x4_t (&sacc)[4][2], int i, float (&mx)[2]) {  // its step i of 16
    const f32x4_t& c = sacc[i & 3][i >> 3];
    mx[i >> 3] = fmaxf(mx[i >> 3], fmaxf(c[2 * ((i >> 2) & 1)], c[2 * ((i >> 2) & 1) + 1]));
  };
  auto raise_max = [&](float (&mx)[2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) mx[g] = max_quarters(mx[g]) * scale_log2;
    const bool need = mx[0] > m_run[0] + RESCALE_SLACK || mx[1] > m_run[1] + RESCALE_SLACK;
    if (__builtin_amdgcn_ballot_w64(need)) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const bool up = mx[g] > m_run[g] + RESCALE_SLACK;
        const float m_new = up ? mx[g] : m_run[g];
        const float alpha = up ? __builtin_amdgcn_exp2f(m_run[g] - m_new) : 1.f;
        l_run[g] *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) oacc[dt][g][r] *= alpha;
        m_run[g] = m_new;
      }
    }
  };
  // probability e of a lane's 32; the row sum takes exactly the rounded values
  // that the second product uses
  struct Soft {
    float p0, ls, sum[2];
    uint32_t w[4];
  };
  auto softmax_step = [&](int e, const f32x4_t (&sacc)[4][2], bf16x8_t (&pf)[2][2], Soft& x) {
    const int g = e >> 4, ks = (e >> 3) & 1, i = e & 7;
    const float mneg = BOUNDED ? -BOUNDED_SHIFT_LOG2 : neg_shift(m_run[g]);
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[2 * ks + (i >> 2)][g][i & 3], scale_log2, mneg));
    if (!(e & 1)) {
      x.p0 = p;
      return;
    }
    x.w[i >> 1] = pack_bf16x2(x.p0, p);
    // formed here: the branches at an iteration's end would otherwise draw the
    // whole softmax past the barrier, away from the MFMAs
    asm volatile("" : "+v"(x.w[i >> 1]));
    x.ls = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x.w[i >> 1]), ones, (e & 15) == 1 ? 0.f : x.ls,
                                           false);
    if (i == 7) pf[ks][g] = __builtin_bit_cast(bf16x8_t, make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]));
    if (i == 7 && ks == 1) x.sum[g] = x.ls;
  };
  auto pv_step = [&](int i, const bf16x8_t& vf, const bf16x8_t (&pf)[2][2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
      oacc[v_dt(i)][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[v_ks(i)][g], oacc[v_dt(i)][g], 0, 0, 0);
  };
  auto pv = [&](int so, const bf16x8_t (&pf)[2][2]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) pv_step(i, v_frag(so, i), pf);
  };

  f32x4_t sb[2][4][2];
  bf16x8_t pb[2][2][2];
  // stage byte offsets of tiles t - 1 (PV), t (this one), t + 1 (scores) and
  // t + 3 (copies), advanced once per iteration
  constexpr int RING = PSTAGE * TILE_BYTES;
  int so_pv = (PSTAGE - 1) * TILE_BYTES, so_sc = TILE_BYTES, so_is = 3 * TILE_BYTES;
  auto next = [](int so) { return so + TILE_BYTES == RING ? 0 : so + TILE_BYTES; };
  auto advance = [&]() {
    so_pv = next(so_pv);
    so_sc = next(so_sc);
    so_is = next(so_is);
  };
  auto store_out = [&](const Seg& s) {
    if (s.piece < 0) {
      const RowMap rm = sm.at(s.z);
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int qi = s.q0 + 32 * wave + 16 * g + lr;
        const float inv = 1.f / sum_quarters(l_run[g]);
        if (qi < Lq) {
          bf16_t* op = o + rm(qi) * ldo + s.h * D + 4 * lq;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt)
            *(uint2*)(op + 16 * dt) = make_uint2(pack_bf16x2(oacc[dt][g][0] * inv, oacc[dt][g][1] * inv),
                                                 pack_bf16x2(oacc[dt][g][2] * inv, oacc[dt][g][3] * inv));
        }
      }
    } else {
      float* w = ws + (int64_t)s.piece * PIECE_FLOATS;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
          *(f32x4_t*)(w + ((wave * 16 + 8 * g + dt) * 64 + lane) * 4) = oacc[dt][g];
        const float l = sum_quarters(l_run[g]);
        if (lq == 0) {
          w[QB * D + 32 * wave + 16 * g + lr] = l;
          w[QB * D + QB + 32 * wave + 16 * g + lr] = m_run[g];
        }
      }
    }
  };

  // End of an iteration: the copies before this one's have landed (vmcnt(4), or
  // vmcnt(20) while the 16 stores of an output stand between the two), LDS
  // reads are down to LGKM, and the work-groups' waves meet.
  int stores = 0;  // iterations in which the copies waited for are older than the stores
  auto meet = [&](auto lgkm_, auto narrow_) {
    constexpr int LGKM = decltype(lgkm_)::value;
    if (!decltype(narrow_)::value && !narrow) {
      __builtin_amdgcn_s_waitcnt(0);
    } else if (stores > 0) {
      __builtin_amdgcn_s_waitcnt((20 & 15) | (7 << 4) | (LGKM << 8) | ((20 >> 4) << 14));
      --stores;
    } else {
      __builtin_amdgcn_s_waitcnt((2 * CPW) | (7 << 4) | (LGKM << 8));
    }
    asm volatile("s_barrier" ::: "memory");
    advance();
    issued();
  };
  // Iteration over tile t of the n of segment s.  In: its scores in sb[0], the
  // probabilities of the tile before it in pb[0]; out: the same for the next
  // tile.  At its end tile t + 2 has landed (tile t + 3 may stay in flight) and
  // every wave is done with tile t - 1.
  int si = 0;  // this segment's place in the list
  Seg s = cs;
  int t = 0;
  // Any tile, one product after the other.  Before tile 0 stands the last
  // segment's PV product, whose output then leaves; after tile n - 1 the next
  // segment's first scores.
  Seg prev{};
  auto iter_edge = [&]() {
    const bool last = t + 1 == s.n, end = last && si + 1 == nseg;
    Seg nxt = s;
    if (last && !end) {
      nxt = segment(si + 1);
      load_q(nxt);
    }
    issue(so_is, std::false_type{});
    if (t > 0 || si > 0) pv(so_pv, pb[0]);
    if (t == 0) {
      if (si > 0) {
        store_out(prev);
        // both query groups of the wave stored: 16 or 20 instructions
        stores = prev.piece >= 0 || prev.q0 + 32 * wave + 16 < Lq ? 2 : 0;
      }
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) oacc[dt][0] = oacc[dt][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        m_run[g] = BOUNDED ? BOUNDED_SHIFT_LOG2 : -INFINITY;
        l_run[g] = 0.f;
      }
    }
    if ((s.t0 + t + 1) * KT > Lk) mask(s.t0 + t, sb[0]);
    if constexpr (!BOUNDED) {
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < 16; ++i) tile_max(sb[0], i, mx);
      raise_max(mx);
    }
    Soft x;
#pragma unroll
    for (int e = 0; e < 32; ++e) softmax_step(e, sb[0], pb[0], x);
#pragma unroll
    for (int g = 0; g < 2; ++g) l_run[g] += x.sum[g];
    if (!end) scores(so_sc, sb[0]);
    meet(std::integral_constant<int, 0>{}, std::false_type{});
    ++t;
    if (last) {
      prev = s;
      s = nxt;
      t = 0;
      ++si;
    }
  };
  // 1 <= t, t + 1 < n (so t is full), bounded logits: with the two buffers of
  // each kind in turn (P), in 32 fenced steps of two MFMAs, one
  // fragment read AHEAD steps before its use (the last ones for the next
  // iteration: V^T of tile t, across the barrier) and 1/32 of the softmax; the
  // fences keep the reads ahead (left to the scheduler each read stood right
  // before its MFMAs).
  constexpr int AHEAD = 4;
  bf16x8_t fr[AHEAD];
  auto iter_mid = [&](auto par_) {
    constexpr int P = decltype(par_)::value;
    issue(so_is, std::true_type{});
    const int so_t = next(so_pv);
    Soft x;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (i < 16) pv_step(i, fr[i % AHEAD], pb[P]);
      else scores_step(i - 16, fr[i % AHEAD], sb[P ^ 1]);
      const int n = i + AHEAD;
      fr[i % AHEAD] = n < 16 ? v_frag(so_pv, n) : n < 32 ? k_frag(so_sc, n - 16) : v_frag(so_t, n - 32);
      softmax_step(i, sb[P], pb[P ^ 1], x);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) l_run[g] += x.sum[g];
    // the fragment reads still in flight are of tile t, which stays for another iteration
    meet(std::integral_constant<int, 15>{}, std::true_type{});
    ++t;
  };
  // The same tiles without a bound, one product after the other: the running
  // maximum stands between them, and a second set of buffers would spill.
  auto iter_mid_max = [&]() {
    issue(so_is, std::true_type{});
    pv(so_pv, pb[0]);
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < 16; ++i) tile_max(sb[0], i, mx);
    raise_max(mx);
    Soft x;
#pragma unroll
    for (int e = 0; e < 32; ++e) softmax_step(e, sb[0], pb[0], x);
#pragma unroll
    for (int g = 0; g < 2; ++g) l_run[g] += x.sum[g];
    scores(so_sc, sb[0]);
    meet(std::integral_constant<int, 0>{}, std::true_type{});
    ++t;
  };
  load_q(s);
  for (int u = 0; u < 3; ++u) {
    issue(u * TILE_BYTES, std::false_type{});
    issued();
  }
  // tiles 0 and 1 have landed (tile 2 may stay in flight)
  if (narrow) __builtin_amdgcn_s_waitcnt((2 * CPW) | (7 << 4) | (0 << 8));
  else __builtin_amdgcn_s_waitcnt(0);
  asm volatile("s_barrier" ::: "memory");
  scores(0, sb[0]);
  while (si < nseg) {
    if constexpr (BOUNDED) {
      if (narrow && t > 0 && t + 2 < s.n) {  // two tiles inside the segment
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) fr[f] = v_frag(so_pv, f);
        do {
          iter_mid(std::integral_constant<int, 0>{});
          iter_mid(std::integral_constant<int, 1>{});
        } while (t + 2 < s.n);
      }
    } else if (narrow && t > 0) {
      while (t + 1 < s.n) iter_mid_max();
    }
    iter_edge();
  }
  pv(so_pv, pb[0]);
  store_out(prev);
}

// Adds the pieces of the shared items in the order of their keys and stores
// the normalised output.  blockIdx.x: XCD (8) x shared item; blockIdx.y: the
// item's 16-query group; each of the four waves takes two of its 16-wide d blocks.
__global__ __launch_bounds__(256) void attn_combine_kernel(bf16_t* __restrict__ o, int64_t ldo, int Lq, SeqMap sm,
                                                           Plan pl, int W, const float* __restrict__ ws) {
  const int x = blockIdx.x & 7, r = blockIdx.x >> 3;
  const Range rg(pl.items, x, W);
  if (r >= rg.rem) return;
  const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4, dt0 = 2 * (threadIdx.x >> 6);
  const Shares sh(rg.rem, pl);
  // shares j0 .. j1 - 1 hold this item's tiles [r ntiles, (r + 1) ntiles)
  const int ub = r * pl.ntiles, ue = ub + pl.ntiles;
  int j0 = (int)((int64_t)ub * sh.n / sh.units);
  while (sh.at(j0 + 1) <= ub) ++j0;
  if (sh.at(j0) <= ub && sh.at(j0 + 1) >= ue) return;  // one share's whole item: stored already
  int j1 = j0 + 1;
  while (sh.at(j1) < ue) ++j1;
  auto piece = [&](int j) {
    return ws + (int64_t)(2 * (8 * j + x) + r - sh.at(j) / pl.ntiles) * PIECE_FLOATS;
  };
  const int wg = blockIdx.y, qw = 16 * wg + lr;
  float m = -INFINITY, l = 0.f;
  for (int j = j0; j < j1; ++j) m = fmaxf(m, piece(j)[QB * D + QB + qw]);
  f32x4_t acc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
  constexpr int U = 4;  // pieces whose loads are in flight together
  for (int j = j0; j < j1; j += U) {
    f32x4_t v[U][2];
    float a[U], lv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* w = piece(min(j + u, j1 - 1));
      a[u] = w[QB * D + QB + qw];
      lv[u] = w[QB * D + qw];
#pragma unroll
      for (int d = 0; d < 2; ++d) v[u][d] = *(const f32x4_t*)(w + ((wg * 8 + dt0 + d) * 64 + lane) * 4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j + u >= j1) break;
      const float f = __builtin_amdgcn_exp2f(a[u] - m);
      l += f * lv[u];
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[d][e] += f * v[u][d][e];
    }
  }
  const int item = rg.start + rg.full * W + r, hb = item / pl.nqb;
  const int z = hb / pl.heads, h = hb - z * pl.heads;
  const int qi = (item - hb * pl.nqb) * QB + qw;
  if (qi >= Lq) return;
  const float inv = 1.f / l;
  bf16_t* op = o + sm.at(z)(qi)*ldo + h * D + 16 * dt0 + 4 * lq;
#pragma unroll
  for (int d = 0; d < 2; ++d)
    *(uint2*)(op + 16 * d) = make_uint2(pack_bf16x2(acc[d][0] * inv, acc[d][1] * inv),
                                        pack_bf16x2(acc[d][2] * inv, acc[d][3] * inv));
}

// Few, short sequences: 32 queries of a head per work-group, the 32-key blocks
// dealt out to its eight waves, operands straight from global memory (V too:
// no transposed copy, no launch for one).  What bounds such a launch is its
// chain of latencies: the kernel above fills and drains a five-stage pipeline
// on a work-group per 256 queries.  The same products, roundings and f32
// statistics; the eight waves' outputs meet in LDS.  Through the entry point
// (about 11 us of it launch and wait), one work-group per 256 queries -> now:
// 1 x 1 18.9 -> 14.8 us, 240 x 240, 2 heads 31.2 -> 19.5, 1000 x 1000, 8 heads 48.0
// -> 29.3, 256 x 1000, 32 heads without a bound 55.4 -> 37.4.
template <bool BOUNDED>
__global__ __launch_bounds__(512) void flash_attn_small_kernel(
    const bf16_t* __restrict__ q, int64_t ldq, const bf16_t* __restrict__ k, int64_t ldk,
    const bf16_t* __restrict__ v, int64_t ldv, bf16_t* __restrict__ o, int64_t ldo, int Lq, int Lk,
    float scale_log2, SeqMap sm) {
  constexpr int LD = D + 4;
  __shared__ __attribute__((aligned(16))) float so[8][32][LD];
  __shared__ float sl[8][32], smax[8][32];
  const RowMap rm = sm.at(blockIdx.z);
  const int h = blockIdx.y, q0 = blockIdx.x * 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  bf16x8_t qf[2][4];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const bf16_t* p = q + rm(min(q0 + 16 * g + lr, Lq - 1)) * ldq + h * D + 8 * lq;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[g][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(p + 32 * s));
  }
  f32x4_t acc[8][2] = {};
  float m[2], l[2] = {0.f, 0.f};
  m[0] = m[1] = BOUNDED ? BOUNDED_SHIFT_LOG2 : -INFINITY;
  const bf16x2_t ones = {(__bf16)1.f, (__bf16)1.f};
  const int blocks = (Lk + 31) / 32;
  for (int b = wave; b < blocks; b += 8) {
    const int k0 = 32 * b;
    bf16x8_t kf[2][4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const bf16_t* p = k + rm(min(k0 + 16 * kb + lr, Lk - 1)) * ldk + h * D + 8 * lq;
#pragma unroll
      for (int s = 0; s < 4; ++s) kf[kb][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(p + 32 * s));
    }
    // V^T fragment dt: d = 16 dt + lr, slot 8 lq + e of the block is key 16 (e >> 2) + 4 lq + (e & 3)
    uint32_t vw[8][4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const int key = k0 + 16 * (e >> 2) + 4 * lq + (e & 3);
      const bf16_t* p0 = v + rm(min(key, Lk - 1)) * ldv + h * D + lr;
      const bf16_t* p1 = v + rm(min(key + 1, Lk - 1)) * ldv + h * D + lr;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) vw[dt][e >> 1] = p0[16 * dt] | ((uint32_t)p1[16 * dt] << 16);
    }
    f32x4_t s[2][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        s[kb][g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 4; ++t)
          s[kb][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kb][t], qf[g][t], s[kb][g], 0, 0, 0);
      }
    // keys past the last one: no probability, and zeros for V (0 times what lies there may be a NaN)
    const bool ragged = k0 + 32 > Lk;
    if (ragged) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (k0 + 16 * kb + 4 * lq + r >= Lk) s[kb][0][r] = s[kb][1][r] = -INFINITY;
    }
    bf16x8_t pf[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      if constexpr (!BOUNDED) {
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[kb][g][r]);
        mx = max_quarters(mx) * scale_log2;
        const float mn = mx > m[g] + RESCALE_SLACK ? mx : m[g];
        const float a = __builtin_amdgcn_exp2f(m[g] - mn);
        if (mn != m[g]) {
          l[g] *= a;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[dt][g][r] *= a;
        }
        m[g] = mn;
      }
      const float mneg = BOUNDED ? -BOUNDED_SHIFT_LOG2 : neg_shift(m[g]);
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 1][g][2 * (e & 1)], scale_log2, mneg));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 1][g][2 * (e & 1) + 1], scale_log2, mneg));
        w[e] = pack_bf16x2(p0, p1);
        l[g] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[e]), ones, l[g], false);
      }
      pf[g] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      if (ragged) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = k0 + 16 * (e >> 1) + 4 * lq + 2 * (e & 1);
          if (key >= Lk) vw[dt][e] = 0;
          else if (key + 1 >= Lk) vw[dt][e] &= 0xffffu;
        }
      }
      const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(vw[dt][0], vw[dt][1], vw[dt][2], vw[dt][3]));
#pragma unroll
      for (int g = 0; g < 2; ++g) acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[g], acc[dt][g], 0, 0, 0);
    }
  }
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float ls = sum_quarters(l[g]);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) *(f32x4_t*)&so[wave][16 * g + lr][16 * dt + 4 * lq] = acc[dt][g];
    if (lq == 0) {
      sl[wave][16 * g + lr] = ls;
      smax[wave][16 * g + lr] = m[g];
    }
  }
  __syncthreads();
  const int row = tid >> 4, c = 8 * (tid & 15), nw = min(8, blocks);
  if (q0 + row >= Lq) return;
  float mx = smax[0][row];
  for (int w = 1; w < nw; ++w) mx = fmaxf(mx, smax[w][row]);
  float den = 0.f, y[8] = {};
  for (int w = 0; w < nw; ++w) {
    const float a = BOUNDED ? 1.f : __builtin_amdgcn_exp2f(smax[w][row] - mx);
    den += a * sl[w][row];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] += a * so[w][row][c + e];
  }
  const float inv = 1.f / den;
  uint2* op = (uint2*)(o + rm(q0 + row) * ldo + h * D + c);
  op[0] = make_uint2(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv));
  op[1] = make_uint2(pack_bf16x2(y[4] * inv, y[5] * inv), pack_bf16x2(y[6] * inv, y[7] * inv));
}

// vt[h][d][32 g + vt_slot(k)] = v[32 g + k][h*128 + d] for keys < Lk, 0 up to ldvt.
// 16-byte reads of a 64 x 128 tile into LDS rows of 65 words, then eight
// halves down a column per 16-byte write: 8 x 8 (key run, d) lanes read 8
// different banks' words in each of the steps.
__global__ __launch_bounds__(256) void transpose_v_kernel(const bf16_t* __restrict__ v, int64_t ldv,
                                                          bf16_t* __restrict__ vt, int Lk, int ldvt, SeqMap sm) {
  __shared__ uint32_t tile[64][D / 2 + 1];
  const RowMap rm = sm.at(blockIdx.z);
  vt += (int64_t)blockIdx.z * gridDim.y * D * ldvt;
  const int l0 = blockIdx.x * 64, h = blockIdx.y, tid = threadIdx.x;
  const bool wide = !(((uintptr_t)v | (uintptr_t)(2 * ldv)) & 15);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = tid + 256 * j, r = i / 16, c = i % 16;
    uint32_t w[4] = {0, 0, 0, 0};
    if (l0 + r < Lk) {
      const bf16_t* p = v + rm(l0 + r) * ldv + h * D + 8 * c;
      if (wide) {
        const uint4 u = *(const uint4*)p;
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = p[2 * e] | ((uint32_t)p[2 * e + 1] << 16);
      }
    }
    const int rs = (r & ~31) | vt_slot(r & 31);
#pragma unroll
    for (int e = 0; e < 4; ++e) tile[rs][4 * c + e] = w[e];
  }
  __syncthreads();
  bf16_t* out = vt + (int64_t)h * D * ldvt + l0;
  const int run = tid & 7;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int d = (tid >> 3) + 32 * j, sh = 16 * (d & 1);
    uint32_t x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (tile[8 * run + e][d / 2] >> sh) & 0xffffu;
    *(uint4*)(out + (int64_t)d * ldvt + 8 * run) =
        make_uint4(x[0] | (x[1] << 16), x[2] | (x[3] << 16), x[4] | (x[5] << 16), x[6] | (x[7] << 16));
  }
}

// ------------------------------------------------------------------ f32 path
// The small f32 workloads (tens to about a thousand tokens): latency bounds
// them, so a work-group takes only 16 queries of a head and its four waves a
// quarter of the key blocks each, on v_mfma_f32_16x16x4_f32 with operands
// straight from global memory.  As in the bf16 kernel the products are
// transposed (S^T = K Q^T, O^T = V^T P^T): lane (lr, lq) holds query lr, keys
// 4 lq .. 4 lq + 3 of a 16-key block, which is the second product's operand.
// The four (maximum, sum, output) triples meet in LDS.  VEC: 16-byte aligned
// rows of q and k (not so when the MLP beside them has an odd width).
// Measured (80 tokens, 4 heads of 32) against one thread per query: 64.3 -> 5.1 us.
template <int HD, bool VEC>
__global__ __launch_bounds__(256) void attn_f32_kernel(const float* __restrict__ q, int64_t ldq,
                                                       const float* __restrict__ k, int64_t ldk,
                                                       const float* __restrict__ v, int64_t ldv,
                                                       float* __restrict__ o, int64_t ldo, int Lq,
                                                       int Lk, float scale) {
  __shared__ float so[4][16][HD + 1], sm[4][16], sl[4][16];
  const int h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lr = lane & 15, lq = lane >> 4;
  const int q0 = blockIdx.x * 16;
  constexpr int ND = HD / 16;
  auto load4 = [](const float* p) {
    if constexpr (VEC) return *(const f32x4_t*)p;
    return f32x4_t{p[0], p[1], p[2], p[3]};
  };
  // MFMA j of step t takes d = 16 t + 4 lq + j from each lane (both operands)
  f32x4_t qf[ND];
  const float* qp = q + (int64_t)min(q0 + lr, Lq - 1) * ldq + h * HD + 4 * lq;
#pragma unroll
  for (int t = 0; t < ND; ++t) {
    qf[t] = load4(qp + 16 * t);
#pragma unroll
    for (int e = 0; e < 4; ++e) qf[t][e] *= scale;
  }
  f32x4_t acc[ND] = {};
  float m = -INFINITY, l = 0.f;
  const int blocks = (Lk + 15) / 16, per = (blocks + 3) / 4;
  const int b1 = min(blocks, (wave + 1) * per);
  for (int b = wave * per; b < b1; ++b) {
    const int k0 = 16 * b;
    const float* kp = k + (int64_t)min(k0 + lr, Lk - 1) * ldk + h * HD + 4 * lq;
    f32x4_t kf[ND];
#pragma unroll
    for (int t = 0; t < ND; ++t) kf[t] = load4(kp + 16 * t);
    float vf[4][ND];  // V[key k0 + 4 lq + i][16 t + lr]
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < ND; ++t)
        vf[i][t] = v[(int64_t)min(k0 + 4 * lq + i, Lk - 1) * ldv + h * HD + 16 * t + lr];
    f32x4_t s = {};
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[t][e], qf[t][e], s, 0, 0, 0);
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (k0 + 4 * lq + i >= Lk) s[i] = -INFINITY;
      mx = fmaxf(mx, s[i]);
    }
    const float mn = fmaxf(m, max_quarters(mx)), a = expf(m - mn);
    l *= a;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t][e] *= a;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = expf(s[i] - mn);
      l += p;
#pragma unroll
      for (int t = 0; t < ND; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][t], p, acc[t], 0, 0, 0);
    }
    m = mn;
  }
  // acc[t][r]: d = 16 t + 4 lq + r of query lr
  l = sum_quarters(l);
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) so[wave][lr][16 * t + 4 * lq + r] = acc[t][r];
  if (lq == 0) {
    sm[wave][lr] = m;
    sl[wave][lr] = l;
  }
  __syncthreads();
  for (int i = tid; i < 16 * HD; i += 256) {
    const int r = i / HD, d = i % HD;
    if (q0 + r >= Lq) continue;
    const float mx = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
    float num = 0.f, den = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a = w * per < blocks ? expf(sm[w][r] - mx) : 0.f;  // a wave without keys holds zeros
      num += a * so[w][r][d];
      den += a * sl[w][r];
    }
    o[(int64_t)(q0 + r) * ldo + h * HD + d] = num / den;
  }
}

}  // namespace

hipError_t launch_transpose_v_bf16(const void* v, int64_t ldv, void* vt, int Lk, int heads,
                                   hipStream_t s, int split, int64_t gap, int nseq, int64_t zs, int64_t gz) {
  if (nseq < 1 || Lk < 1) return hipErrorInvalidValue;
  const int ldvt = (Lk + 63) / 64 * 64;
  hipLaunchKernelGGL(transpose_v_kernel, dim3(ldvt / 64, heads, nseq), dim3(256), 0, s,
                     (const bf16_t*)v, ldv, (bf16_t*)vt, Lk, ldvt, SeqMap{split, gap, gz, zs});
  return hipGetLastError();
}

namespace {
// Work-groups per XCD: one per CU.
int attn_width(int n_cu) { return std::max(1, n_cu / 8); }

Plan attn_plan(int Lq, int Lk, int heads, int nseq, int W) {
  Plan p;
  p.nqb = (Lq + QB - 1) / QB;
  p.heads = heads;
  p.items = nseq * heads * p.nqb;
  p.ntiles = (Lk + KT - 1) / KT;
  p.shares = W;
  // key tiles that the longest work-group saves by sharing the last round
  const int most = (p.items + 7) / 8, rem = most % W;
  const int64_t longest = rem ? (Shares(rem, p).units + Shares(rem, p).n - 1) / Shares(rem, p).n : 0;
  if (!rem || p.ntiles - longest < SPLIT_MIN_TILES) p.shares = 0;
  return p;
}
}  // namespace

// Whether launch_flash_attn_small_bf16 takes these shapes: rounds of the chip
// times keys.  Against the list kernel, through the entry point (us, list / small):
// one round of 1500 keys 35.4 / 34.0, of 2000 39.9 / 40.8 (half a chip) and 44.7 /
// 40.6 (all of it), of 3000 42.0 / 52.1, of 4000 47.8 / 62.9; two rounds of 200 keys
// 31.8 / 25.6, of 512 37.6 / 33.4, of 1024 40.8 / 44.5.  More rounds pay the fixed
// part of a work-group (query loads, 135 KB of LDS, the sum of the waves) each time:
// eight of 5 keys 27.4 / 34.3, twelve of 20 keys 35.1 / 45.1.
bool flash_attn_small_fits(int Lq, int Lk, int heads, int nseq, int n_cu) {
  const int64_t rounds = ((int64_t)((Lq + 31) / 32) * heads * nseq + n_cu - 1) / n_cu;
  return rounds <= 2 && rounds * Lk <= SMALL_MAX_KEYS;
}

hipError_t launch_flash_attn_small_bf16(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                                        int64_t ldv, void* o, int64_t ldo, int Lq, int Lk, int heads,
                                        bool bounded_logits, hipStream_t s, int split, int64_t gap, int nseq,
                                        int64_t zs, int64_t gz) {
  if (nseq < 1 || Lq < 1 || Lk < 1) return hipErrorInvalidValue;
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  hipLaunchKernelGGL(bounded_logits ? flash_attn_small_kernel<true> : flash_attn_small_kernel<false>,
                     dim3((Lq + 31) / 32, heads, nseq), dim3(512), 0, s, (const bf16_t*)q, ldq, (const bf16_t*)k, ldk,
                     (const bf16_t*)v, ldv, (bf16_t*)o, ldo, Lq, Lk, scale_log2, SeqMap{split, gap, gz, zs});
  return hipGetLastError();
}

bool flash_attn_uses_ws(int Lq, int Lk, int heads, int nseq, int n_cu) {
  return attn_plan(Lq, Lk, heads, nseq, attn_width(n_cu)).shares > 0;
}

size_t flash_attn_ws_bytes(int n_cu) { return (size_t)16 * attn_width(n_cu) * PIECE_FLOATS * sizeof(float); }

hipError_t launch_flash_attn_bf16(const void* q, int64_t ldq, const void* k, int64_t ldk,
                                  const void* vt, int ldvt, void* o, int64_t ldo, int Lq, int Lk,
                                  int heads, bool bounded_logits, hipStream_t s, int n_cu, float* ws, int split,
                                  int64_t gap, int nseq, int64_t zs, int64_t gz) {
  if (nseq < 1 || Lq < 1 || Lk < 1) return hipErrorInvalidValue;
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  const SeqMap sm{split, gap, gz, zs};
  int W = attn_width(n_cu);
  Plan p = attn_plan(Lq, Lk, heads, nseq, W);
  if (!ws) p.shares = 0;
  if (!p.shares) W = std::min(W, (p.items + 7) / 8);
  hipLaunchKernelGGL(bounded_logits ? flash_attn_kernel<true> : flash_attn_kernel<false>, dim3(8 * W), dim3(64 * NW), 0,
                     s, (const bf16_t*)q, ldq, (const bf16_t*)k, ldk, (const bf16_t*)vt, ldvt, (bf16_t*)o, ldo, Lq, Lk,
                     scale_log2, sm, p, ws);
  if (p.shares) {
    const int rest = std::max(Range(p.items, 0, W).rem, Range(p.items, 7, W).rem);
    hipLaunchKernelGGL(attn_combine_kernel, dim3(8 * rest, 2 * NW), dim3(256), 0, s, (bf16_t*)o, ldo, Lq, sm, p, W, ws);
  }
  return hipGetLastError();
}

hipError_t launch_attn_f32(const float* q, int64_t ldq, const float* k, int64_t ldk,
                           const float* v, int64_t ldv, float* o, int64_t ldo, int Lq, int Lk,
                           int heads, int head_dim, hipStream_t s) {
  const float scale = 1.f / sqrtf((float)head_dim);
  dim3 grid((Lq + 15) / 16, heads);
  const bool vec = ldq % 4 == 0 && ldk % 4 == 0 && !(((uintptr_t)q | (uintptr_t)k) & 15);
#define DIT_ATTN_F32(HD_)                                                                        \
  case HD_:                                                                                      \
    hipLaunchKernelGGL((vec ? attn_f32_kernel<HD_, true> : attn_f32_kernel<HD_, false>), grid,   \
                       dim3(256), 0, s, q, ldq, k, ldk, v, ldv, o, ldo, Lq, Lk, scale);          \
    break;
  switch (head_dim) {
    DIT_ATTN_F32(16)
    DIT_ATTN_F32(32)
    DIT_ATTN_F32(64)
    DIT_ATTN_F32(128)
    default:
      return hipErrorInvalidValue;
  }
#undef DIT_ATTN_F32
  return hipGetLastError();
}

}  // namespace dit
