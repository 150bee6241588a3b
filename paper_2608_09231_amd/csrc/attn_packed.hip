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
#include <type_traits>

#include "attention_copy.h"
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
  int ranked;          // tiles in the order of their keys, most first
  int workers, least;  // workers that share the units, and units that each takes at least
  float* ws;
  float scale_log2;
};

// Sum or maximum (of what is not negative) of v over the lanes up to this one, on the VALU (rows of 16 lanes, then
// their last lanes' to the rows behind).
template <typename F>
__device__ __forceinline__ int over_lanes(int v, F op) {
#if defined(__HIP_DEVICE_COMPILE__)
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));  // 1, 2, 4 and 8 lanes before, in a row
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));  // lane 15 of a row to the next, 31 to the upper half
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
#endif
  return v;
}
__device__ __forceinline__ int scan_lanes(int v) {
  return over_lanes(v, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int max_scan_lanes(int v) {
  return over_lanes(v, [](int a, int b) { return max(a, b); });
}

// A sequence: its first rows and lengths.
struct Seq {
  int q0, lq, k0, lk;
};
__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }
__device__ __forceinline__ Seq seq_of_lane(const Seq& s, int l) {
  return Seq{__builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.lq, l), __builtin_amdgcn_readlane(s.k0, l),
             __builtin_amdgcn_readlane(s.lk, l)};
}
// 64 sequences at a time, one a lane (past the last one: empty).  Offsets are clamped to what the caller's
// matrices hold, and one below an earlier one counts as that one, so that no two sequences share a row: their tiles
// are no more than the host counts, and no two work-groups write the same.  qat, kat: the largest offsets before.
struct Seqs {
  Seq s;
  int qat = 0, kat = 0;
  __device__ __forceinline__ void load(const PackedArgs& P, int z0) {
    const int z = z0 + (threadIdx.x & 63);
    int q0 = 0, q1 = 0, k0 = 0, k1 = 0, n = 0;
    if (z < P.batch) {
      q0 = clamp_to(P.qoff[z], 0, P.Tq); q1 = clamp_to(P.qoff[z + 1], 0, P.Tq);
      k0 = clamp_to(P.koff[z], 0, P.Tk); k1 = clamp_to(P.koff[z + 1], 0, P.Tk);
      n = P.klen ? P.klen[z] : 0x7fffffff;
    }
    // (200 tokens of 500 keys each 31.0 us, 32.1 with the scans in every call)
    if (__builtin_amdgcn_ballot_w64(z < P.batch && (q0 > q1 || k0 > k1 || q0 < qat || k0 < kat))) {
      q0 = max(max_scan_lanes(q0), qat);
      k0 = max(max_scan_lanes(k0), kat);
    }
    s = Seq{q0, max(q1 - q0, 0), k0, clamp_to(n, 0, max(k1 - k0, 0))};
    qat = __builtin_amdgcn_readlane(s.q0, 63);
    kat = __builtin_amdgcn_readlane(s.k0, 63);
  }
};

// The same of 64-bit values, halves moved alike.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int64_t lanes_before(int64_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int lo = __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROW_MASK, 0xf, false);
  return (int64_t)((uint64_t)(uint32_t)lo | (uint64_t)(uint32_t)hi << 32);
#else
  return 0;
#endif
}
__device__ __forceinline__ int64_t scan_lanes64(int64_t v) {
  v += lanes_before<0x111, 0xf>(v);
  v += lanes_before<0x112, 0xf>(v);
  v += lanes_before<0x114, 0xf>(v);
  v += lanes_before<0x118, 0xf>(v);
  v += lanes_before<0x142, 0xa>(v);
  return v + lanes_before<0x143, 0xc>(v);
}
__device__ __forceinline__ int sum_lanes(int v) { return __builtin_amdgcn_readlane(scan_lanes(v), 63); }

// The sequence that tile t of `rows` rows falls in, 64 sequences at a time, and the
// tile's number in it, its last one first; false past the last one.
__device__ __forceinline__ bool find_tile(const PackedArgs& P, int t, int rows, Seq& seq, int& tile) {
  Seqs all;
  for (int z0 = 0; z0 < P.batch; z0 += 64) {
    all.load(P, z0);
    const Seq& s = all.s;
    const int n = (s.lq * P.group + rows - 1) / rows;
    const int end = scan_lanes(n);
    const uint64_t past = __ballot(end > t);
    if (past) {
      const int l = __ffsll((unsigned long long)past) - 1;
      seq = seq_of_lane(s, l);
      tile = __builtin_amdgcn_readlane(end, l) - 1 - t;
      return true;
    }
    t -= __builtin_amdgcn_readlane(end, 63);
  }
  return false;
}

// Waits until the products in s are written: the compiler knows when its own instructions may
// read a matrix instruction's result, but not when max3 may.
template <int N, int NG>
__device__ __forceinline__ void settle(f32x4_t (&s)[N][NG]) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int b = 0; b < N; ++b)
#pragma unroll
    for (int g = 0; g < NG; ++g) asm volatile("" : "+v"(s[b][g]));
  asm volatile("s_nop 15" : "+v"(s[N - 1][NG - 1]));
#pragma unroll
  for (int b = 0; b < N; ++b)
#pragma unroll
    for (int g = 0; g < NG; ++g) asm volatile("" : "+v"(s[b][g]));
#endif
}

typedef uint16_t u16x8_t __attribute__((ext_vector_type(8)));

// Values for a careful product: finite ones as they are, and flags in place of the others, +inf 1, -inf 128 and
// NaN 16384, so that their product with whether a row sees the key (a tile has at most 64) counts each kind.
__device__ __forceinline__ void part_odd(const bf16x8_t& v, bf16x8_t& clean, bf16x8_t& flag) {
  const u16x8_t bits = __builtin_bit_cast(u16x8_t, v);
  u16x8_t c, f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool odd = (bits[e] & 0x7f80) == 0x7f80;
    c[e] = odd ? 0 : bits[e];
    f[e] = !odd ? 0 : bits[e] == 0x7f80 ? 0x3f80 : bits[e] == 0xff80 ? 0x4300 : 0x4680;
  }
  clean = __builtin_bit_cast(bf16x8_t, c);
  flag = __builtin_bit_cast(bf16x8_t, f);
}
// What the counted values add to a sum.
__device__ __forceinline__ float odd_sum(float count) {
  const int c = (int)count;
  const float up = c & 127 ? INFINITY : 0.f, down = c & 0x3f80 ? -INFINITY : 0.f;
  return (up + down) + (c >> 14 ? __uint_as_float(0x7fc00000u) : 0.f);
}

// A launch's work as one line of units: sequence by sequence, tile of R rows by tile and key head
// by key head (an item), KEYS keys of it each (one unit at least).  Workers take `per`
// consecutive units each, so that sequences of any lengths fill the chip evenly; where an item is
// shared its parts are joined from the workspace.  Worker w's part that begins where its units do
// lies in slot 2 w there, one that begins later (and is cut off by the worker's end) in slot 2 w + 1.
struct Place {
  int z, tile, kh, unit, n;  // unit of n
  int64_t item;
};
__device__ __forceinline__ int64_t readlane64(int64_t v, int l) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)v, l) |
                   (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32);
}
template <int R, int KEYS>
struct Line {
  const PackedArgs& P;
  Seqs all;                   // 64 sequences from z0 on, one a lane:
  int z0, n;                  // units of an item,
  int64_t items, cost;        // items and units of the sequence,
  int64_t items_end, cost_end;  // and up to its end from z0 on
  int64_t items_base, cost_base;  // those before z0

  __device__ __forceinline__ explicit Line(const PackedArgs& P_) : P(P_), items_base(0), cost_base(0) { load(0); }
  __device__ __forceinline__ void load(int z) {
    z0 = z;
    all.load(P, z0);
    const Seq& s = all.s;
    n = max(1, (s.lk + KEYS - 1) / KEYS);
    items = (int64_t)((s.lq * P.group + R - 1) / R) * P.kv_heads;
    cost = items * n;
    items_end = scan_lanes64(items);
    cost_end = scan_lanes64(cost);
  }
  __device__ __forceinline__ void next() {
    items_base += readlane64(items_end, 63);
    cost_base += readlane64(cost_end, 63);
    load(z0 + 64);
  }
  __device__ __forceinline__ int64_t total() const {
    if (P.batch <= 64) return readlane64(cost_end, 63);
    Line l(P);
    while (l.z0 + 64 < P.batch) l.next();
    return l.cost_base + readlane64(l.cost_end, 63);
  }
  // The sequence of the place that was asked for last.
  __device__ __forceinline__ Seq seq(const Place& p) const { return seq_of_lane(all.s, p.z - z0); }
  // Place of unit u (below the total, not before the last one asked for).  Offsets that
  // change under a running call may find none: then a place of no rows.
  __device__ __forceinline__ Place at(int64_t u) {
    while (u >= cost_base + readlane64(cost_end, 63) && z0 + 64 < P.batch) next();
    const uint64_t here = __ballot(cost_base + cost_end > u);
    Place p;
    if (!here) {
      p.z = -1;
      return p;
    }
    const int l = __ffsll((unsigned long long)here) - 1;
    p.z = z0 + l;
    p.n = __builtin_amdgcn_readlane(n, l);
    const int64_t rest = u - cost_base - (readlane64(cost_end, l) - readlane64(cost, l));
    const int64_t i = readlane64(rest / p.n, 0);
    p.unit = __builtin_amdgcn_readfirstlane((int)(rest - i * p.n));
    p.item = items_base + readlane64(items_end, l) - readlane64(items, l) + i;
    p.tile = __builtin_amdgcn_readfirstlane((int)(i / P.kv_heads));
    p.kh = __builtin_amdgcn_readfirstlane((int)(i - (int64_t)p.tile * P.kv_heads));
    return p;
  }
};
__device__ __forceinline__ int64_t units_each(int64_t total, int workers, int least) {
  return max((int64_t)least, (total + workers - 1) / workers);
}

// A part of an item: its unnormalised outputs [R][128], row sums and running maxima.
__host__ __device__ __forceinline__ int64_t part_floats(int rows) { return (int64_t)rows * (D + 2); }

// Joins the parts of an item's rows and stores the normalised output.  32 threads a
// row, 4 columns each; PG of them take consecutive parts, U at a time, whose loads are in flight
// together, and the PG meet in LDS in their order.
// A work-group takes `rows` rows, 8 / PG at a time.  Bound by memory: 44 MB of parts of 128 rows 13 us.
template <int R, int KEYS, int PG>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedArgs P, int rows) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int U = 8, RB = 8 / PG;
  __shared__ float red[6][256];
  const int64_t item = blockIdx.x;
  const int tid = threadIdx.x, pg = (tid >> 5) % PG, c = 4 * (tid & 31);
  Line<R, KEYS> line(P);
  const int64_t per = units_each(line.total(), P.workers, P.least);
  while (item >= line.items_base + readlane64(line.items_end, 63)) {
    if (line.z0 + 64 >= P.batch) return;
    line.next();
  }
  const int l = __ffsll((unsigned long long)__ballot(line.items_base + line.items_end > item)) - 1;
  const int n = __builtin_amdgcn_readlane(line.n, l);
  const int64_t i = item - line.items_base - (readlane64(line.items_end, l) - readlane64(line.items, l));
  const int64_t a = line.cost_base + readlane64(line.cost_end, l) - readlane64(line.cost, l) + i * n;
  const int64_t w0 = a / per, w1 = (a + n - 1) / per;  // the item's workers
  if (w0 == w1) return;  // one worker has stored it
  const Seq s = seq_of_lane(line.all.s, l);
  const int tile = (int)(i / P.kv_heads), kh = (int)(i - (int64_t)tile * P.kv_heads);
  const int parts = (int)(w1 - w0) + 1, each = (parts + PG - 1) / PG;
  const int64_t pf = part_floats(R);
  const int64_t late = a != w0 * per;  // the first worker's part is not its units' beginning
  auto part_of = [&](int p) { return P.ws + (2 * (w0 + p) + (p == 0 ? late : 0)) * pf; };
  for (int row0 = blockIdx.y * rows; row0 < min((int)(blockIdx.y + 1) * rows, s.lq * P.group - tile * R); row0 += RB) {
  const int row = row0 + (tid >> 5) / PG, r = tile * R + row, qi = r / P.group, h = kh * P.group + r - qi * P.group;
  const bool in = r < s.lq * P.group;
  const int p0 = pg * each, p1 = in ? min(parts, p0 + each) : 0;
  float mx = -INFINITY, den = 0.f;
  f32x4_t y = {};
  auto rescale = [&](float nm) {
    const float f = __builtin_amdgcn_exp2f(mx + neg_shift(nm));
    den *= f;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= f;
    mx = nm;
  };
  auto add = [&](float m, float ls, const f32x4_t& v) {  // one more part, of weight 2^m
    const float f = __builtin_amdgcn_exp2f(m + neg_shift(mx));
    den += f * ls;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += f * v[e];
  };
  for (int p = p0; p < p1; p += U) {
    f32x4_t v[U];
    float m[U], ls[U], nm = mx;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const float* x = part_of(min(p + j, p1 - 1));
      v[j] = *(const f32x4_t*)(x + row * D + c);
      ls[j] = x[R * D + row];
      m[j] = x[R * D + R + row];
    }
#pragma unroll
    for (int j = 0; j < U; ++j) nm = fmaxf(nm, m[j]);
    rescale(nm);
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (p + j < p1) add(m[j], ls[j], v[j]);
  }
  if constexpr (PG > 1) {
    __syncthreads();  // (the rows before are read)
    red[0][tid] = mx;
    red[1][tid] = den;
#pragma unroll
    for (int e = 0; e < 4; ++e) red[2 + e][tid] = y[e];
    __syncthreads();
    if (pg) continue;
    float nm = mx;
#pragma unroll
    for (int j = 1; j < PG; ++j) nm = fmaxf(nm, red[0][tid + 32 * j]);
    rescale(nm);
#pragma unroll
    for (int j = 1; j < PG; ++j) {
      const int t = tid + 32 * j;
      add(red[0][t], red[1][t], f32x4_t{red[2][t], red[3][t], red[4][t], red[5][t]});
    }
  }
  if (!in) continue;
  const float inv = den == 0.f ? 0.f : 1.f / den;
  *(uint2*)(P.o + (int64_t)(s.q0 + qi) * P.ldo + (int64_t)h * D + c) =
      make_uint2(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv));
  }
#endif
}

// Few rows a sequence (single tokens and their heads): what bounds it is the way of K
// and V from memory.  Every wave is a worker with units of 32 keys in two buffers
// of LDS of its own, and no wave waits for another.  With MFMAs to spare, probabilities
// enter the second product as two bf16 parts, so that only the output is rounded to 8 bits.
// An infinity among the values meets a second part of zero or of the other sign, and one that a row does not see a
// probability of zero: both give NaN. So where an item's sums are not finite, the wave goes through its units
// again, and adds what is not finite by product of flags.
// 16 tokens against up to 8192 keys each, 32 heads on 8: 45 us for 263 MB, 5.9 TB/s, and 6 for joining.
template <bool BOUNDED, bool CAUSAL, int NG>
__global__ __launch_bounds__(256, 1) void attn_packed_few_kernel(PackedArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int HK = 32, TILE = HK * D * 2, STAGE = 2 * TILE, R = 16 * NG;
  __shared__ __attribute__((aligned(1024))) char smem[8 * STAGE];  // [wave][stage][K | V]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int worker = blockIdx.x * 4 + wave;
  Line<R, HK> line(P);
  const int64_t total = line.total(), per = units_each(total, P.workers, P.least);
  const int64_t begin = worker * per, end = min(total, begin + per);
  if (begin >= end) return;

  // keys that row `row` of a sequence's sees, and those that the tile's last row, and so any of its rows, sees
  auto seen = [&](const Seq& s, int row) { return CAUSAL ? max(s.lk - s.lq + 1 + row / P.group, 0) : s.lk; };
  auto seen_by = [&](const Place& p, const Seq& s) { return seen(s, min(p.tile * R + R, s.lq * P.group) - 1); };
  // copy c: rows 4 c .. + 3; rows past the last of `keys` are zeros (what none of the tile's rows sees may
  // hold infinities or NaN, and 0 times those is NaN)
  auto issue = [&](const Place& p, const Seq& s, int keys, int st) {
    const int key = p.unit * HK;
    const int rows = min(keys - key, HK);
    const int64_t at = s.k0 + (rows > 0 ? key : 0);
    const bf16_t* kp = P.k + at * P.ldk + (int64_t)p.kh * D;
    const bf16_t* vp = P.v + at * P.ldv + (int64_t)p.kh * D;
    const uint32_t kn = rows > 0 ? (uint32_t)(rows - 1) * (uint32_t)P.ldk * 2u + 2u * D : 0u;
    const uint32_t vn = rows > 0 ? (uint32_t)(rows - 1) * (uint32_t)P.ldv * 2u + 2u * D : 0u;
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
  const int voff = k_off(4 * lq + (lr >> 2), (lr & 3) >> 1) + 8 * (lr & 1);  // as in attn_packed_kernel

  bf16x8_t qf[NG][4];
  f32x4_t acc[8][NG];
  float m[NG], l[NG];
  int lim[NG], common = 0, first = 0;  // first unit of this worker's part of the item
  auto enter = [&](const Place& p, const Seq& s) {  // an item: its queries
    const int nrows = s.lq * P.group;
    common = seen(s, p.tile * R);
    first = p.unit;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int row = min(p.tile * R + 16 * g + lr, nrows - 1), qi = row / P.group, h = p.kh * P.group + row - qi * P.group;
      lim[g] = seen(s, row);
      const bf16_t* qp = P.q + (int64_t)(s.q0 + qi) * P.ldq + (int64_t)h * D + 8 * lq;
#pragma unroll
      for (int t = 0; t < 4; ++t) qf[g][t] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 32 * t));
      m[g] = BOUNDED ? BOUNDED_SHIFT_LOG2 : -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) acc[dt][g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int g = 0; g < NG; ++g)  // (queries waited for later would wait for the copies, too)
#pragma unroll
      for (int t = 0; t < 4; ++t) asm volatile("" : "+v"(qf[g][t]));
  };
  // logits of the keys from `key` on; -inf where a row does not see them
  auto scores = [&](const char* sk, int key, f32x4_t(&s)[2][NG]) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *(const uint4*)(sk + koff[t] + b * 16 * 256));
#pragma unroll
        for (int g = 0; g < NG; ++g)
          s[b][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][t], t ? s[b][g] : f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      }
    if (key + HK > common) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int g = 0; g < NG; ++g)
            if (key + 16 * b + 4 * lq + r >= lim[g]) s[b][g][r] = -INFINITY;
    }
  };
  // probabilities of a query group, bf16 and what it leaves; their sum
  auto weights = [&](const f32x4_t(&s)[2][NG], int g, bf16x8_t& ph, bf16x8_t& pl) {
    const float mneg = BOUNDED ? -BOUNDED_SHIFT_LOG2 : neg_shift(m[g]);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][g][e & 3], P.scale_log2, mneg));
      ph[e] = (__bf16)p;
      pl[e] = (__bf16)(p - (float)ph[e]);
      sum += p;
    }
    return sum;
  };
  // An item's sums anew, unit by unit through the buffer of the last one, with the maxima that are known by now.
  auto again = [&](Place p, const Seq& s, int st) {
    const int keys = seen_by(p, s), last = p.unit;
    const char* sk = smem + (2 * wave + st) * STAGE;
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) acc[dt][g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (p.unit = first; p.unit <= last; ++p.unit) {
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the buffer is read
      asm volatile("" ::: "memory");
      issue(p, s, keys, st);
      wait_vmcnt<0>();
      asm volatile("" ::: "memory");
      const int key = p.unit * HK;
      f32x4_t t[2][NG];
      scores(sk, key, t);
      bf16x8_t ph[NG], pl[NG], sees[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        weights(t, g, ph[g], pl[g]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sees[g][e] = key + 16 * (e >> 2) + 4 * lq + (e & 3) < lim[g] ? (__bf16)1.f : (__bf16)0.f;
      }
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        bf16x8_t clean, flag;
        part_odd(vt_frag(sk + TILE + (voff ^ (dt << 5))), clean, flag);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(clean, ph[g], acc[dt][g], 0, 0, 0);
          acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(clean, pl[g], acc[dt][g], 0, 0, 0);
          const f32x4_t n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(flag, sees[g], f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[dt][g][r] += odd_sum(n[r]);
        }
      }
    }
  };
  auto leave = [&](const Place& p, const Seq& s, int late) {
    const int nrows = s.lq * P.group;
    const bool whole = first == 0 && p.unit == p.n - 1;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int at = 16 * g + lr, row = p.tile * R + at;
      const float ls = sum_quarters(l[g]);
      if (row >= nrows) continue;
      if (whole) {
        const int qi = row / P.group, h = p.kh * P.group + row - qi * P.group;
        const float inv = ls == 0.f ? 0.f : 1.f / ls;  // no key: zeros
        bf16_t* op = P.o + (int64_t)(s.q0 + qi) * P.ldo + (int64_t)h * D + 4 * lq;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
          *(uint2*)(op + 16 * dt) = make_uint2(pack_bf16x2(acc[dt][g][0] * inv, acc[dt][g][1] * inv),
                                               pack_bf16x2(acc[dt][g][2] * inv, acc[dt][g][3] * inv));
      } else {
        float* w = P.ws + (2 * (int64_t)worker + late) * part_floats(R);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *(f32x4_t*)(w + at * D + 16 * dt + 4 * lq) = acc[dt][g];
        if (lq == 0) {
          w[R * D + at] = ls;
          w[R * D + R + at] = m[g];
        }
      }
    }
  };

  Place cur = line.at(begin);
  if (cur.z < 0) return;
  Seq seq = line.seq(cur);
  int late = 0, keys = seen_by(cur, seq);
  issue(cur, seq, keys, 0);
  enter(cur, seq);
  int st = 0;
  for (int64_t u = begin; u < end; ++u) {
    Place nxt = cur;
    Seq nseq = seq;
    bool more = u + 1 < end;
    const bool change = more && cur.unit + 1 == cur.n;
    if (change) {
      nxt = line.at(u + 1);
      if (nxt.z < 0) more = false;
      else {
        nseq = line.seq(nxt);
        keys = seen_by(nxt, nseq);
      }
    } else {
      ++nxt.unit;
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the other buffer is read
    asm volatile("" ::: "memory");
    issue(nxt, nseq, more ? keys : 0, st ^ 1);
    wait_vmcnt<16>();  // this one has landed
    asm volatile("" ::: "memory");
    const char* sk = smem + (2 * wave + st) * STAGE;
    f32x4_t s[2][NG];
    scores(sk, cur.unit * HK, s);
    bf16x8_t ph[NG], pl[NG];
    if constexpr (!BOUNDED) settle(s);
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
      l[g] += weights(s, g, ph[g], pl[g]);
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const bf16x8_t vf = vt_frag(sk + TILE + (voff ^ (dt << 5)));
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, ph[g], acc[dt][g], 0, 0, 0);
        acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[g], acc[dt][g], 0, 0, 0);
      }
    }
    if (change || !more) {
      float zero = 0.f;  // NaN where a sum is not finite
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r) zero = __builtin_fmaf(acc[dt][g][r], 0.f, zero);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(zero != 0.f) != 0, 0)) again(cur, seq, st);
      leave(cur, seq, late);
      late = 1;
      if (more) enter(nxt, nseq);
    }
    if (!more) break;
    cur = nxt;
    seq = nseq;
    st ^= 1;
  }
  __builtin_amdgcn_s_waitcnt(0);  // no copy outlives its work-group
#endif
}

constexpr int ROWS = 128;

// Tile of rank t among the tiles of a key head in the order of their keys, most first, so that
// a launch ends with short ones: up to 64 sequences, one a lane; false past the last tile.
// Of a sequence with T tiles those from first(c) on have c key blocks of 64 or more.
template <bool CAUSAL>
__device__ __forceinline__ bool ranked_tile(const PackedArgs& P, int t, Seq& seq, int& tile) {
  Seqs all;
  all.load(P, 0);
  const Seq& s = all.s;
  const int T = (s.lq * P.group + ROWS - 1) / ROWS, past = s.lk - s.lq + 1;
  const int top = (s.lk + KT - 1) / KT;  // key blocks of the last tile
  auto first = [&](int c) {
    if (c <= 0) return 0;
    if (c > top) return T;
    if (!CAUSAL) return 0;
    // the tile's last query, (128 j + 127) / group, sees past + query > 64 (c - 1) keys
    const int64_t need = (int64_t)(KT * (c - 1) - past + 1) * P.group - (ROWS - 1);
    return need <= 0 ? 0 : (int)min((int64_t)T - 1, (need + ROWS - 1) / ROWS);  // (the last one sees all)
  };
  auto count = [&](int c) {  // tiles with c blocks or more
    return sum_lanes(T - first(c));
  };
  if (t >= count(0)) return false;
  int lo = 0, hi = T ? top : 0;  // count(lo) > t >= count(hi)
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) hi = max(hi, __shfl_xor(hi, o, 64));
  hi = __builtin_amdgcn_readfirstlane(hi) + 1;
  while (hi - lo > 1) {
    const int c = (lo + hi) >> 1;
    if (count(c) > t) lo = c;
    else hi = c;
  }
  t -= count(hi);
  const int here = first(hi) - first(lo), end = scan_lanes(here);
  const int l = __ffsll((unsigned long long)__ballot(end > t)) - 1;
  seq = seq_of_lane(s, l);
  tile = __builtin_amdgcn_readlane(first(lo) + here, l) - 1 -
         (t - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(here, l)));
  return true;
}

// 128 rows of a sequence and key head: four waves of 32, tiles of 64 keys of K and V in
// XOR-swizzled LDS rows of 256 bytes, two of each; S^T = K Q^T, O^T = V^T P^T,
// probabilities from one to the other in registers, V^T read from the row-major
// tile by transposing LDS reads.  Probabilities are rounded to bf16, the type that
// the second product takes beside V; the sum takes the rounded values, so that the weights add up to one.
// (Errors of 0.0020 in the 2-norm where outputs rounded from f32 have 0.0016; a second part of the probabilities
// would add half of the matrix instructions again.)
//
// SPLIT: launches whose tiles are fewer than the chip's places for work-groups share the units
// of the whole launch out (Line); a work-group may go through parts of several items.
//
// 16384 tokens, 16 heads on 4, causal: 0.96 ms, 1.15 PFLOP/s, MFMAs busy 0.53 at a power-limited 2.02 GHz.  8 prompts
// of up to 512, 28 on 4: 25 us, one round of eight tiles of keys one after the other.  5 of up to 701 x 5003, 12 on
// 4: 65 us and 13 for joining, bound by the memory side: 20 tiles of keys a worker, but 264 MB fetched for 37 of inputs and
// outputs, as a sequence's tiles read the same keys at different times on different XCDs.  Workers in the order of the
// XCDs, key heads first, so that neighbours share keys in L2: 5 % less there, but up to 10 more elsewhere (256 x 16384 98
// to 109, 1000 x 1500 35 to 37).
template <bool BOUNDED, bool CAUSAL, bool SPLIT, bool PIPE>
__global__ __launch_bounds__(256, 2) void attn_packed_kernel(PackedArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int TILE = KT * D * 2, STAGE = 2 * TILE, VBASE = 3 * TILE;
  // [stage][K | V], or three tiles of K and two of V
  __shared__ __attribute__((aligned(1024))) char smem[PIPE ? 5 * TILE : 2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int worker = blockIdx.x;
  int64_t u = 0, end = 1;
  Place p{};
  Seq s_;
  [[maybe_unused]] int late = 0;
  if constexpr (SPLIT) {
    Line<ROWS, KT> line(P);
    const int64_t total = line.total(), per = units_each(total, P.workers, P.least);
    u = worker * per;
    end = min(total, u + per);
    if (u >= end) return;
  } else {
    p.kh = worker % P.kv_heads;
    const int t = worker / P.kv_heads;
    // (the order matters where work-groups wait for their turn)
    const bool any = P.ranked ? ranked_tile<CAUSAL>(P, t, s_, p.tile) : find_tile(P, t, ROWS, s_, p.tile);
    if (!any) return;
  }
#pragma unroll 1
  do {
  if constexpr (SPLIT) {
    Line<ROWS, KT> line(P);  // (anew for each item: few, and the registers are the loop's)
    p = line.at(u);
    if (p.z < 0) return;
    s_ = line.seq(p);
  }
  const int tile = p.tile, kh = p.kh;
  const int nrows = s_.lq * P.group;
  // keys that query i sees: past + i, at most all; not causal: all
  const int past = s_.lk - s_.lq + 1;
  auto seen = [&](int row) { return CAUSAL ? max(past + row / P.group, 0) : s_.lk; };
  const int wrow = tile * ROWS + 32 * wave;
  int nkeys = seen(min(tile * ROWS + ROWS, nrows) - 1);        // of the work-group
  int key0 = 0;
  bool whole = true;
  if constexpr (SPLIT) {  // units of the item
    const int units = (int)min((int64_t)(p.n - p.unit), end - u);
    whole = units == p.n;
    key0 = p.unit * KT;
    nkeys = min(nkeys, key0 + units * KT);
    u += units;
  }
  const bool active = wrow < nrows;  // wave-uniform; idle waves copy and meet the others
  const int wkeys = active ? min(nkeys, seen(min(wrow + 32, nrows) - 1)) : 0;    // of the wave
  const int common = active ? seen(wrow) : 0;                        // of all its rows
  int lim[2];
  bf16x8_t qf[2][4];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = min(wrow + 16 * g + lr, nrows - 1), qi = row / P.group, h = kh * P.group + row - qi * P.group;
    lim[g] = seen(row);
    const bf16_t* qp = P.q + (int64_t)(s_.q0 + qi) * P.ldq + (int64_t)h * D + 8 * lq;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[g][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 32 * s));
  }
  const bf16_t* kbase = P.k + (int64_t)s_.k0 * P.ldk + (int64_t)kh * D;
  const bf16_t* vbase = P.v + (int64_t)s_.k0 * P.ldv + (int64_t)kh * D;
  // copy c of this wave: rows 4 (4 wave + c) .. + 3 of a tile, chunks swizzled by the row's lowest four bits
  const int crow = 16 * wave + (lane >> 4);
  const uint32_t kr = (uint32_t)crow * (uint32_t)P.ldk * 2u, vr = (uint32_t)crow * (uint32_t)P.ldv * 2u;
  const uint32_t chunk = ((lane & 15) ^ (lane >> 4)) << 4;
  auto ko = [&](int c) { return kr + (uint32_t)(8 * c) * (uint32_t)P.ldk + (chunk ^ (uint32_t)(c << 6)); };
  auto vo = [&](int c) { return vr + (uint32_t)(8 * c) * (uint32_t)P.ldv + (chunk ^ (uint32_t)(c << 6)); };
  // rows past the last key are zeros
  auto issue = [&](int key, int at) {
    const int n = min(nkeys - key, KT);
    const uint32_t kn = n <= 0 ? 0u : (uint32_t)(n - 1) * (uint32_t)P.ldk * 2u + 2u * D;
    const uint32_t vn = n <= 0 ? 0u : (uint32_t)(n - 1) * (uint32_t)P.ldv * 2u + 2u * D;
    const int64_t row = n <= 0 ? 0 : key;
    char* d = smem + at + wave * 4096;
#pragma unroll
    for (int c = 0; c < 4; ++c) copy16_unseen(kbase + row * P.ldk, kn, d + c * 1024, ko(c));
#pragma unroll
    for (int c = 0; c < 4; ++c) copy16_unseen(vbase + row * P.ldv, vn, d + TILE + c * 1024, vo(c));
  };
  struct Src {
    const bf16_t* p;
    uint32_t bytes;
  };
  auto src = [&](const bf16_t* base, int64_t ld, int key) {
    const int n = min(nkeys - key, KT);
    return Src{base + (n <= 0 ? 0 : key) * ld, n <= 0 ? 0u : (uint32_t)(n - 1) * (uint32_t)ld * 2u + 2u * D};
  };
  auto copy = [&](const Src& x, int at, uint32_t off, int c) {
    copy16_unseen(x.p, x.bytes, smem + at + (4 * wave + c) * 1024, off);
  };
  const bool piped = PIPE && nkeys - key0 > 2 * KT;
  if (piped) {
#pragma unroll
    for (int u_ = 0; u_ < 3; ++u_) {
      const Src x = src(kbase, P.ldk, key0 + u_ * KT);
#pragma unroll
      for (int c = 0; c < 4; ++c) copy(x, u_ * TILE, ko(c), c);
    }
    const Src none{vbase, 0u};  // values of the tile before the first
#pragma unroll
    for (int c = 0; c < 4; ++c) copy(none, VBASE + TILE, vo(c), c);
  } else {
    issue(key0, 0);
  }
  const int koff0 = k_off(lr, lq);  // chunk 4 s + lq of the row: XOR 64 s
  // V^T fragment (d = 16 dt + lr; keys 4 lq .. + 3 of a 16-key block): lane 4 k + j of a
  // quarter addresses row 4 lq + k, columns 16 dt + 4 j, and receives column lr.  The
  // chunk 2 dt + (j >> 1) enters the swizzled address by XOR.
  const int voff = k_off(4 * lq + (lr >> 2), (lr & 3) >> 1) + 8 * (lr & 1);
  f32x4_t acc[8][2];
  float m[2], l[2];
  const bf16x2_t ones = {(__bf16)1.f, (__bf16)1.f};
  // 0 times a value that is not finite reaches the rows of a tile that do not see its key.  Rather
  // than look for such values in every masked tile, the work-group looks at its sums, and
  // where one is not finite it goes through its keys again, carefully.
  bool careful = false;
  while (true) {
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) acc[dt][0] = acc[dt][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  l[0] = l[1] = 0.f;
  m[0] = m[1] = BOUNDED ? BOUNDED_SHIFT_LOG2 : -INFINITY;
  // the first tile lands with the queries (waited for later, they would wait for later copies)
  __builtin_amdgcn_s_waitcnt(0);
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int s = 0; s < 4; ++s) asm volatile("" : "+v"(qf[g][s]));
  bool done = false;
  if constexpr (PIPE) if (piped && !careful) {
    done = true;
    barrier_no_fence();  // the first three tiles of K have landed
    // Iteration t issues the score product of tile t + 1 and the PV product of tile t - 1
    // on MFMA with the softmax of tile t, which depends on neither, between them in 32 fenced slots of
    // two MFMAs, a fragment read AHEAD slots before its use and a share of the softmax.  Its copies
    // are V of tile t and K of tile t + 3.  Tiles come in pairs; a last one without keys adds nothing.
    // A tile's fragments in the order of their use, K 0..15 and V^T 0..15, so that four
    // independent accumulators stand between the steps of a dependent chain.
    auto k_kb = [](int i) { return 2 * (i >> 3) + (i & 1); };
    auto k_s = [](int i) { return (i >> 1) & 3; };
    auto v_dt = [](int i) { return 2 * (i >> 2) + (i & 1); };
    auto v_ks = [](int i) { return (i >> 1) & 1; };
    auto k_frag = [&](int at, int i) {
      return __builtin_bit_cast(bf16x8_t, *(const uint4*)(smem + at + (koff0 ^ (k_s(i) << 6)) + k_kb(i) * 16 * 256));
    };
    auto v_frag = [&](int at, int i) { return vt_frag(smem + (voff ^ (v_dt(i) << 5)) + at + v_ks(i) * 32 * 256); };
    f32x4_t sb[2][4][2];
    bf16x8_t pb[2][2][2];
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
      x.w[e] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(c[2 * (e & 1)], P.scale_log2, -m[g])),
                           __builtin_amdgcn_exp2f(__builtin_fmaf(c[2 * (e & 1) + 1], P.scale_log2, -m[g])));
      // formed here: the branches between iterations would otherwise draw the softmax
      // past the barrier, away from the MFMAs
      asm volatile("" : "+v"(x.w[e]));
      x.sum[g] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x.w[e]), ones, (i & 7) ? x.sum[g] : 0.f, false);
      if (e == 3) pf[ks][g] = __builtin_bit_cast(bf16x8_t, make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]));
    };
    auto mask = [&](int key, f32x4_t (&s)[4][2]) {
#pragma unroll
      for (int b_ = 0; b_ < 4; ++b_)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int g = 0; g < 2; ++g)
            if (key + 16 * b_ + 4 * lq + r >= min(lim[g], nkeys)) s[b_][g][r] = -INFINITY;
    };
    const int clear = min(common, nkeys);  // keys that every row of the wave sees
    // places of K of tiles t, t + 1, t + 2
    int ks0 = 0, ks1 = TILE, ks2 = 2 * TILE;
    // End of an iteration: its copies have landed and the waves meet.  Fragments still
    // on their way are of K of tile t + 2, which stays for another iteration.
    auto meet = [&]() {
      wait_vmcnt<0>();
      barrier_no_fence();
      const int k = ks0;
      ks0 = ks1; ks1 = ks2; ks2 = k;
    };
    constexpr int AHEAD = 4;
    bf16x8_t fr[AHEAD];
    auto iter = [&](int key, auto par) {
      constexpr int B = decltype(par)::value;
      const Src vs = src(vbase, P.ldv, key), kn = src(kbase, P.ldk, key + 3 * KT);
      if (key + KT > clear) mask(key, sb[B]);
      Soft x;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i_ = 0; i_ < 32; ++i_) {
        if (i_ < 16) score_step(i_, fr[i_ % AHEAD], sb[B ^ 1]);
        else pv_step(i_ - 16, fr[i_ % AHEAD], pb[B ^ 1]);
        const int n = i_ + AHEAD;
        fr[i_ % AHEAD] = n < 16 ? k_frag(ks1, n) : n < 32 ? v_frag(VBASE + (B ^ 1) * TILE, n - 16) : k_frag(ks2, n - 32);
        if (i_ % 2 == 0 && i_ < 16) {
          if (i_ < 8) copy(vs, VBASE + B * TILE, vo(i_ / 2), i_ / 2);
          else copy(kn, ks0, ko(i_ / 2 - 4), i_ / 2 - 4);
        }
        if (i_ & 1) exp_step(i_ >> 1, sb[B], pb[B], x);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int g = 0; g < 2; ++g) l[g] += x.sum[g];
      meet();
    };
    if (active) {
#pragma unroll
      for (int i_ = 0; i_ < 16; ++i_) score_step(i_, k_frag(0, i_), sb[0]);
#pragma unroll
      for (int f = 0; f < AHEAD; ++f) fr[f] = k_frag(ks1, f);
      pb[1][0][0] = pb[1][0][1] = pb[1][1][0] = pb[1][1][1] = __builtin_bit_cast(bf16x8_t, make_uint4(0, 0, 0, 0));
      if constexpr (!BOUNDED) {
        // The shift is the first tile's maximum.  Later logits may be larger: probabilities
        // and sums are floating point numbers and lose nothing up to 2^100, where the
        // work-group goes through its keys again.  (Of no key: finite, so that -inf logits stay zeros.)
        if (key0 + KT > clear) mask(key0, sb[0]);
        settle(sb[0]);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          float mx = sb[0][0][g][0];
#pragma unroll
          for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int r = 0; r < 4; r += 2) mx = max3(mx, sb[0][kb][g][r], sb[0][kb][g][r + 1]);
          m[g] = fmaxf(max_quarters(mx) * P.scale_log2, -1e30f);
        }
      }
      wait_vmcnt_lgkm0<0>();
      barrier_no_fence();  // K of tile 0 is read: its place is free
#pragma unroll 1
      for (int key = key0; key < nkeys; key += 2 * KT) {
        iter(key, std::integral_constant<int, 0>{});
        iter(key + KT, std::integral_constant<int, 1>{});
      }
#pragma unroll
      for (int i_ = 0; i_ < 16; ++i_) pv_step(i_, v_frag(VBASE + TILE, i_), pb[1]);
    } else {
      barrier_no_fence();
      for (int key = key0; key < nkeys; key += 2 * KT)
        for (int par = 0; par < 2; ++par) {
          const Src vs = src(vbase, P.ldv, key + par * KT), kn = src(kbase, P.ldk, key + par * KT + 3 * KT);
#pragma unroll
          for (int c = 0; c < 4; ++c) copy(vs, VBASE + par * TILE, vo(c), c);
#pragma unroll
          for (int c = 0; c < 4; ++c) copy(kn, ks0, ko(c), c);
          meet();
        }
    }
  }
  if (!PIPE || !done) {
  int at = 0;
  for (int key = key0; key < nkeys; key += KT) {
    // this tile has landed and everyone is done with the one before it
    __builtin_amdgcn_s_waitcnt(0);
    barrier_no_fence();
    issue(key + KT, at ^ STAGE);
    if (key < wkeys) {
      const char* sk = smem + at;
      // the wave in its products goes before the one in its softmax (8 prompts of up to 512, 28 / 4 heads: 26.0 us for 26.7;
      // with long shares 2 % slower, so whole tiles alone)
      if constexpr (!SPLIT) __builtin_amdgcn_s_setprio(1);
      f32x4_t s[4][2];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        s[kb][0] = s[kb][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4) {
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *(const uint4*)(sk + (koff0 ^ (t4 << 6)) + kb * 16 * 256));
#pragma unroll
          for (int g = 0; g < 2; ++g) s[kb][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][t4], s[kb][g], 0, 0, 0);
        }
      }
      if constexpr (!SPLIT) __builtin_amdgcn_s_setprio(0);
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
      if constexpr (!BOUNDED) settle(s);
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
      if constexpr (!SPLIT) __builtin_amdgcn_s_setprio(1);
      const bool spoilt = CAUSAL && careful && masked;
      if (__builtin_expect(!spoilt, 1)) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) {
            const bf16x8_t vf = v_frag(dt, ks);
#pragma unroll
            for (int g = 0; g < 2; ++g) acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[ks][g], acc[dt][g], 0, 0, 0);
          }
      } else {
        // finite values as ever; of the others the rows that see their keys are told by a product of flags
        bf16x8_t sees[2][2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              sees[ks][g][e] = key + 32 * ks + 16 * (e >> 2) + 4 * lq + (e & 3) < lim[g] ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          f32x4_t n[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) {
            bf16x8_t clean, flag;
            part_odd(v_frag(dt, ks), clean, flag);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              acc[dt][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(clean, pf[ks][g], acc[dt][g], 0, 0, 0);
              n[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(flag, sees[ks][g], n[g], 0, 0, 0);
            }
          }
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[dt][g][r] += odd_sum(n[g][r]);
        }
      }
    }
    if constexpr (!SPLIT) __builtin_amdgcn_s_setprio(0);
    at ^= STAGE;
  }
  }
  __builtin_amdgcn_s_waitcnt(0);  // no copy outlives its work-group
  if ((!CAUSAL && (BOUNDED || !piped)) || careful) break;
  float zero = 0.f;  // NaN where a sum is not finite or passes 2^100
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    zero = __builtin_fmaf(l[g] * 0x1p28f, 0.f, zero);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) zero = __builtin_fmaf(acc[dt][g][r] * 0x1p28f, 0.f, zero);
  }
  int* bad = (int*)smem;
  lds_barrier();  // everyone has read the last tiles
  bad[wave] = active && __builtin_amdgcn_ballot_w64(zero != 0.f) != 0;
  lds_barrier();
  if (!(bad[0] | bad[1] | bad[2] | bad[3])) break;
  careful = true;
  lds_barrier();  // everyone has read the flags
  issue(key0, 0);
  }
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float ls = sum_quarters(l[g]);
    const int row = wrow + 16 * g + lr;
    if (row >= nrows) continue;
    if (!SPLIT || whole) {
      const int qi = row / P.group, h = kh * P.group + row - qi * P.group;
      bf16_t* op = P.o + (int64_t)(s_.q0 + qi) * P.ldo + (int64_t)h * D + 4 * lq;
      const float inv = ls == 0.f ? 0.f : 1.f / ls;  // no key: zeros
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
        *(uint2*)(op + 16 * dt) = make_uint2(pack_bf16x2(acc[dt][g][0] * inv, acc[dt][g][1] * inv),
                                             pack_bf16x2(acc[dt][g][2] * inv, acc[dt][g][3] * inv));
    } else {
      const int in = 32 * wave + 16 * g + lr;
      float* w = P.ws + (2 * (int64_t)worker + late) * part_floats(ROWS);
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *(f32x4_t*)(w + in * D + 16 * dt + 4 * lq) = acc[dt][g];
      if (lq == 0) {
        w[ROWS * D + in] = ls;
        w[ROWS * D + ROWS + in] = m[g];
      }
    }
  }
  if constexpr (SPLIT) {
    late = 1;
    if (u < end) lds_barrier();  // everyone is done with the last tile: its place takes the next item's
  }
  } while (SPLIT && u < end);
#endif
}

}  // namespace

// Few rows a sequence, on average: the memory-bound kernel, a wave of which takes 16 or 32.  In us, against tiles of
// 128 rows, shared out: 16 tokens with 8192 keys, 32 / 8 heads 50 56; 4 x 8192 19 22; 16 of 4 x 4096 35 37; 1 x 16384
// 25 23; 64 tokens with 1024 keys 32 31 (and half the error: the probabilities stay unrounded).
int few_rows(const dit_packed_shape& s) {
  const int64_t rows = (int64_t)s.Tq * (s.heads / s.kv_heads);
  return rows <= 16 * (int64_t)s.batch ? 16 : rows <= 32 * (int64_t)s.batch ? 32 : 0;
}
// tiles of r rows of a key head, at most: whole ones and one begun by each sequence
int64_t tiles_of(const dit_packed_shape& s, int r) {
  return (int64_t)s.Tq * (s.heads / s.kv_heads) / r + std::min(s.batch, s.Tq);
}
// Waves of 256 CUs (by the shape alone: the workspace's size does not depend on the device).
constexpr int FEW_WORKERS = 1024, FEW_LEAST = 4;
// Whether the tiles are fewer than the places for work-groups of 256 CUs (two each) and sharing their
// keys out is worth the joining: in us, whole tiles take 1.6 for 64 keys (2.1 beside
// another work-group, and less where causal tiles of few keys stand beside those of many), shared ones 2.1 times their
// share of all, masked or not, and 20 for parts and joining (fitted; shares of what causal tiles see alone begin and
// end inside items: 2/2 16384 x 16384 183, but 16/4 2048 x 8192 177).  By the average
// length of the slots, which is all that the host knows: the constants are fitted to them, and a cache that is nearly
// empty costs less than the rule counts.  Measured, shared and whole:
//   heads / key heads, queries x keys   32/8 256 x 16384 101 386   16/16 77 x 4096 23 92   32/8 8 of 64 x 4096 42 101
//   8/8 2048 x 2048 causal 43 47, 2 of up to 4096 x 4096 106 89, 3 of up to 2048 x 2048 65 47   12/12 1000 x 1500 34 40
//   28/4 2048 x 2048 causal 93 63   28/4 512 x 512 causal 24 19   16/4 2048 x 8192 causal 141 165   2/2 16384 x 16384 causal 230 308
constexpr int SPLIT_WORKERS = 512, SPLIT_LEAST = 8;
bool split_tiles(const dit_packed_shape& s, bool causal) {
  const int64_t items = tiles_of(s, ROWS) * s.kv_heads;
  const double units = (double)s.Tk / s.batch / KT;
  const double seen = causal ? 1 - 0.5 * std::min(s.Tq, s.Tk) / std::max(s.Tk, 1) : 1;  // of the keys, by the average tile
  const double whole = std::max(1.6, items > SPLIT_WORKERS / 2 ? 2.1 * seen : 0);
  return items < SPLIT_WORKERS && 20 + 2.1 * units * items / SPLIT_WORKERS < units * whole;
}

// Whether the pipelined loop is the faster one: it fills and drains over some tiles.  In us, pipelined and
// not, whole tiles: 8 of 512 x 512 causal, 28 / 4 heads 29.8 26.7; 1024 x 1024 29.0 31.8; 4096 x 4096, 16 / 4 99 114;
// 16384 x 16384 983 1107.  Shares of 33 tiles by the slots, 20 as they are filled (5 of up to 701 x 5003 in a cache, 12 / 4,
// bounded) 86 75, of 36 (256 x 16384, 32 / 8) 90 96, of 128 (1024 x 16384) 265 304.
bool pipelined(const dit_packed_shape& s, bool split) {
  const double units = (double)s.Tk / s.batch / KT;
  return split ? units * (double)(tiles_of(s, ROWS) * s.kv_heads) >= 64.0 * SPLIT_WORKERS : units >= 12;
}

size_t attention_packed_ws_bytes(const dit_packed_shape& s) {
  if (s.batch == 0 || s.Tq == 0) return 0;
  const int few = few_rows(s);
  if (few) return 2 * FEW_WORKERS * part_floats(few) * sizeof(float);
  // (a causal launch shares out only where another would: seen <= 1)
  if (split_tiles(s, false)) return 2 * SPLIT_WORKERS * part_floats(ROWS) * sizeof(float);
  return 0;
}

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
  void (*fn)(PackedArgs);
#define DIT_PICK(kernel, ...)                                                                              \
  (causal ? (bounded ? kernel<true, true __VA_ARGS__> : kernel<false, true __VA_ARGS__>)                   \
          : (bounded ? kernel<true, false __VA_ARGS__> : kernel<false, false __VA_ARGS__>))
#define DIT_COMMA ,
  if (const int few = few_rows(s)) {
    P.workers = FEW_WORKERS;
    P.least = FEW_LEAST;
    fn = few == 16 ? DIT_PICK(attn_packed_few_kernel, DIT_COMMA 1) : DIT_PICK(attn_packed_few_kernel, DIT_COMMA 2);
    hipLaunchKernelGGL(fn, dim3(FEW_WORKERS / 4), dim3(256), 0, st, P);
    const uint32_t items = (uint32_t)(tiles_of(s, few) * s.kv_heads);
    // (few items: more work-groups for each, since they have many parts)
    const int rows = items <= 256 ? 2 : few / 4;
    if (few == 16) hipLaunchKernelGGL((packed_join_kernel<16, 32, 4>), dim3(items, few / rows), dim3(256), 0, st, P, rows);
    else hipLaunchKernelGGL((packed_join_kernel<32, 32, 4>), dim3(items, few / rows), dim3(256), 0, st, P, rows);
    return hipGetLastError();
  }
  const bool split = split_tiles(s, causal), pipe = pipelined(s, split);
  if (split) {
    P.workers = SPLIT_WORKERS;
    P.least = SPLIT_LEAST;
    fn = pipe ? DIT_PICK(attn_packed_kernel, DIT_COMMA true DIT_COMMA true)
              : DIT_PICK(attn_packed_kernel, DIT_COMMA true DIT_COMMA false);
    hipLaunchKernelGGL(fn, dim3(SPLIT_WORKERS), dim3(256), 0, st, P);
    const uint32_t items = (uint32_t)(tiles_of(s, ROWS) * s.kv_heads);
    const int rows = items <= 128 ? 8 : 32;
    if (items <= 64) hipLaunchKernelGGL((packed_join_kernel<ROWS, KT, 4>), dim3(items, ROWS / 2), dim3(256), 0, st, P, 2);
    else hipLaunchKernelGGL((packed_join_kernel<ROWS, KT, 1>), dim3(items, ROWS / rows), dim3(256), 0, st, P, rows);
    return hipGetLastError();
  }
  P.ranked = s.batch > 1 && s.batch <= 64 && tiles_of(s, ROWS) * s.kv_heads > SPLIT_WORKERS / 2;
  fn = pipe ? DIT_PICK(attn_packed_kernel, DIT_COMMA false DIT_COMMA true)
            : DIT_PICK(attn_packed_kernel, DIT_COMMA false DIT_COMMA false);
  hipLaunchKernelGGL(fn, dim3((uint32_t)(tiles_of(s, ROWS) * s.kv_heads)), dim3(256), 0, st, P);
  return hipGetLastError();
}

}  // namespace dit
