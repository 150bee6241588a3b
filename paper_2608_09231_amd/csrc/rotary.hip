// Rotary positions: the pairs (a, b) of each head's first `rot` values become
//   scale * (a cos t - b sin t, b cos t + a sin t),  t = pos[axis(i)][row] * freq[i],
// pair i being the values i and i + rot / 2 (half) or 2 i and 2 i + 1 (interleaved).
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace dit {
namespace {

struct RotaryArgs {
  const void* x; int64_t ldx;
  void* y; int64_t ldy;
  const int32_t* pos; int64_t ldpos;
  const double* freq;
  int rows, heads, head_dim, rot;
  int end[DIT_ROTARY_AXES];  // pairs up to each axis's end
  float scale;
  int rows_wg;               // rows of a work-group
};

// cos and sin of p * f radians.  The angle is formed in double and reduced there to
// quarter turns r in [-1/2, 1/2] (a position of 2^31 leaves 2^-22 of a turn's bits), which
// f32 holds to 2^-26; then Taylor's series of sine and cosine up to y^9 and y^10 for |y| <= pi / 4,
// whose rests are below 2e-9 and 2e-10.
__device__ __forceinline__ float2 cos_sin(int p, double f) {
  const double q = (double)p * (f * 0.63661977236758134308);  // quarter turns: 2 / pi
  const double n = rint(q);
  const float y = (float)(q - n) * 1.57079632679489661923f, z = y * y;
  const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const int k = (int)(n - 4.0 * rint(n * 0.25)) & 3;
  const float cc = k & 1 ? s : c, ss = k & 1 ? c : s;
  return make_float2((k + 1) & 2 ? -cc : cc, k & 2 ? -ss : ss);
}

// Eight values from any element's address: bits as they are, and as f32 numbers.
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
  uint4 raw;
  __device__ __forceinline__ void load(const bf16_t* p) {
    const vec v = *(const vec*)p;
    raw = make_uint4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { unpack8(raw, v); }
  __device__ __forceinline__ void set(const float (&v)[8]) { raw = pack8(v); }
  __device__ __forceinline__ void keep(const Eight& x, int pair) {  // a pair of neighbours as in x
    if (pair == 0) raw.x = x.raw.x;
    if (pair == 1) raw.y = x.raw.y;
    if (pair == 2) raw.z = x.raw.z;
    if (pair == 3) raw.w = x.raw.w;
  }
  __device__ __forceinline__ void store(bf16_t* p) const { *(vec*)p = vec{raw.x, raw.y, raw.z, raw.w}; }
};
template <> struct Eight<float> {
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  float raw[8];
  __device__ __forceinline__ void load(const float* p) {
    const vec a = *(const vec*)p, b = *(const vec*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { raw[i] = a[i]; raw[4 + i] = b[i]; }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = raw[i];
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = v[i];
  }
  __device__ __forceinline__ void keep(const Eight& x, int pair) {
    raw[2 * pair] = x.raw[2 * pair];
    raw[2 * pair + 1] = x.raw[2 * pair + 1];
  }
  __device__ __forceinline__ void store(float* p) const {
    *(vec*)p = vec{raw[0], raw[1], raw[2], raw[3]};
    *(vec*)(p + 4) = vec{raw[4], raw[5], raw[6], raw[7]};
  }
};

// A work-group takes rows_wg rows: first the cosines and sines of their pairs, one a
// thread, to LDS; then every thread walks over the rows' units, at a stride of all threads.
// One pass over x, bound by memory: 32760 x 40 heads of 128 (671 MB) 128 us, 5.2 TB/s.
//
// A unit is two runs of eight values.  Half: eight pairs' first and second values; then, where y
// is not x, two runs of what lies past rot.  Interleaved: runs of the head's two halves, a pair past rot as it is.  All
// lanes load, turn and store alike, whichever they have (each kind in a branch of its own: rot 96 of 128 166 us,
// so 139).  A last unit with fewer values begins earlier and repeats some of the one before it; only in
// place, where those may be turned already, and of less than eight values it goes value by value.
template <typename T, bool HALF>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs P) {
  extern __shared__ float2 cs[];  // [rows_wg][pairs]
  const int tid = threadIdx.x, pairs = P.rot >> 1, last = max(pairs - 1, 0);
  const int64_t r0 = (int64_t)blockIdx.x * P.rows_wg;
  const int rows = (int)min((int64_t)P.rows_wg, P.rows - r0);
  for (int e = tid; e < rows * pairs; e += 256) {
    const int r = e / pairs, i = e - r * pairs;
    int axis = 0;
#pragma unroll
    for (int a = 0; a < DIT_ROTARY_AXES - 1; ++a) axis += i >= P.end[a];
    const float2 v = cos_sin(P.pos[axis * P.ldpos + r0 + r], P.freq[i]);
    cs[e] = make_float2(v.x * P.scale, v.y * P.scale);
  }
  __syncthreads();
  const T* x = (const T*)P.x + r0 * P.ldx;
  T* y = (T*)P.y + r0 * P.ldy;
  const bool in_place = (const void*)P.x == (const void*)P.y;
  // values of a head that are walked over: those that change (interleaved: whole units of them), or all
  const int width = !in_place ? P.head_dim : HALF ? P.rot : (P.rot + 7) & ~7;
  const int turned = HALF ? (pairs + 7) >> 3 : 0;
  const int units = HALF ? turned + ((width - P.rot + 15) >> 4) : (width + 15) >> 4;
  const int per_row = units * P.heads;
  for (int e = tid; e < rows * per_row; e += 256) {
    const int r = e / per_row, w = e - r * per_row;
    const int h = w / units, u = w - h * units;
    const T* px = x + r * P.ldx + (int64_t)h * P.head_dim;
    T* py = y + r * P.ldy + (int64_t)h * P.head_dim;
    const float2* t = cs + r * pairs;
    const bool turn = HALF && u < turned;
    // the runs' places, where they end, and how many values they have
    int at, bt, na = 8, nb = 8;
    if (HALF) {
      at = turn ? 8 * u : P.rot + 16 * (u - turned);
      const int begin = turn ? 0 : P.rot, end = turn ? pairs : width;
      if (!in_place) at = max(begin, min(at, end - (turn ? 8 : 16)));
      bt = turn ? at + pairs : max(begin, min(at + 8, end - 8));  // (runs that are copied may overlap)
      na = min(8, end - at);
      nb = turn ? na : min(8, end - bt);
    } else {
      at = 8 * u;
      bt = 8 * (u + units);
      if (bt >= width) nb = 0;  // an odd number of runs
    }
    if (!HALF || (na == 8 && nb == 8)) {
      Eight<T> a, b, ya, yb;
      float p[8], q[8];
      a.load(px + at);
      b = a;
      if (HALF || nb) b.load(px + bt);
      a.get(p);
      b.get(q);
      if (HALF) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 c = t[min(at + i, last)];
          const float f = p[i], g = q[i];
          p[i] = f * c.x - g * c.y;
          q[i] = g * c.x + f * c.y;
        }
        ya.set(p);
        yb.set(q);
        if (!turn) { ya = a; yb = b; }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float* v = i < 4 ? p + 2 * i : q + 2 * (i - 4);
          const float2 c = t[min((i < 4 ? at >> 1 : (bt >> 1) - 4) + i, last)];
          const float f = v[0], g = v[1];
          v[0] = f * c.x - g * c.y;
          v[1] = g * c.x + f * c.y;
        }
        ya.set(p);
        yb.set(q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if ((at >> 1) + i >= pairs) ya.keep(a, i);
          if ((bt >> 1) + i >= pairs) yb.keep(b, i);
        }
      }
      ya.store(py + at);
      if (HALF || nb) yb.store(py + bt);
    } else {
      T p[8], q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i < na) p[i] = px[at + i];
        if (i < nb) q[i] = px[bt + i];
      }
      if (turn) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < na) {
            const float2 c = t[at + i];
            const float f = St<T>::ld(p + i), g = St<T>::ld(q + i);
            St<T>::st(p + i, f * c.x - g * c.y);
            St<T>::st(q + i, g * c.x + f * c.y);
          }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i < na) py[at + i] = p[i];
        if (i < nb) py[bt + i] = q[i];
      }
    }
  }
}

}  // namespace

hipError_t launch_rotary(const dit_rotary_desc& d, hipStream_t s) {
  if (d.rows == 0 || d.heads == 0) return hipSuccess;
  const bool in_place = d.x == d.y;
  if (in_place && d.rot == 0) return hipSuccess;
  RotaryArgs P{};
  P.x = d.x; P.ldx = d.ldx; P.y = d.y; P.ldy = d.ldy;
  P.pos = d.pos; P.ldpos = d.axes > 1 ? d.ldpos : 0; P.freq = d.freq;
  P.rows = d.rows; P.heads = d.heads; P.head_dim = d.head_dim; P.rot = d.rot; P.scale = d.scale;
  int end = 0;
  for (int a = 0; a < DIT_ROTARY_AXES; ++a) {
    end += a < d.axes ? d.pairs[a] : 0;
    P.end[a] = a < d.axes ? end : 0x7fffffff;
  }
  // (pairs of the last axis end at rot / 2; no pair lies past it)
  // Rows of a work-group: as many as have a pair for each of its 256 threads, which take 2 KB of LDS.
  const int pairs = std::max(1, d.rot / 2);
  P.rows_wg = std::max(1, 256 / pairs);
  // (a work-group's chunks fit 32 bits: width <= 2^30, and more rows only of narrow heads)
  while (P.rows_wg > 1 && (int64_t)P.rows_wg * d.heads * d.head_dim > ((int64_t)1 << 30)) P.rows_wg /= 2;
  const int64_t groups = ((int64_t)d.rows + P.rows_wg - 1) / P.rows_wg;
  const size_t lds = (size_t)P.rows_wg * pairs * sizeof(float2);
  const bool half = d.layout == DIT_ROTARY_HALF;
  void (*fn)(RotaryArgs) = d.dtype == DIT_DTYPE_BF16 ? (half ? rotary_kernel<bf16_t, true> : rotary_kernel<bf16_t, false>)
                                                     : (half ? rotary_kernel<float, true> : rotary_kernel<float, false>);
  hipLaunchKernelGGL(fn, dim3((uint32_t)groups), dim3(256), lds, s, P);
  return hipGetLastError();
}

}  // namespace dit
