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

// A work-group takes rows_wg rows: first the cosines and sines of their pairs, one a
// thread, to LDS; then every thread walks over the rows' chunks of 8 values
// (interleaved: 4 pairs; half: the chunk and its partner rot / 2 further on).
// One pass over x, bound by memory.
//
// VEC: chunks of 8 (half: rot / 2 a multiple of 8); else a pair, or a value past rot, a thread.
template <typename T, bool HALF, bool VEC>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs P) {
  extern __shared__ float2 cs[];  // [rows_wg][pairs]
  const int tid = threadIdx.x, pairs = P.rot >> 1;
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
  const bool in_place = (const void*)x == (const void*)y;
  if constexpr (VEC) {
    // units of a head: pairs of chunks (half) or chunks, then the chunks past rot
    const int turned = HALF ? P.rot >> 4 : (P.rot + 7) >> 3;
    const int units = turned + (in_place ? 0 : (P.head_dim >> 3) - (HALF ? 2 * turned : turned));
    const int per_row = units * P.heads;
    auto load = [](const T* p, float (&v)[8]) {
      if constexpr (sizeof(T) == 2) unpack8(*(const uint4*)p, v);
      else load_f8(p, v);
    };
    auto store = [](T* p, const float (&v)[8]) {
      if constexpr (sizeof(T) == 2) {
        *(uint4*)p = pack8(v);
      } else {
        *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
        *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
      }
    };
    for (int e = tid; e < rows * per_row; e += 256) {
      const int r = e / per_row, w = e - r * per_row;
      const int h = w / units, u = w - h * units;
      const T* px = x + r * P.ldx + (int64_t)h * P.head_dim;
      T* py = y + r * P.ldy + (int64_t)h * P.head_dim;
      const float2* t = cs + r * pairs;
      float a[8], b[8];
      if (u >= turned) {
        const int at = 8 * (HALF ? u + turned : u);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4*)(py + at))[i] = ((const uint4*)(px + at))[i];
      } else if (HALF) {
        load(px + 8 * u, a);
        load(px + 8 * u + pairs, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 c = t[8 * u + i];
          const float p = a[i], q = b[i];
          a[i] = p * c.x - q * c.y;
          b[i] = q * c.x + p * c.y;
        }
        store(py + 8 * u, a);
        store(py + 8 * u + pairs, b);
      } else {
        load(px + 8 * u, a);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (4 * u + i >= pairs) break;  // (the last chunk's values past rot)
          const float2 c = t[4 * u + i];
          const float p = a[2 * i], q = a[2 * i + 1];
          a[2 * i] = p * c.x - q * c.y;
          a[2 * i + 1] = q * c.x + p * c.y;
        }
        store(py + 8 * u, a);
      }
    }
  } else {
    const int units = pairs + (in_place ? 0 : P.head_dim - P.rot), per_row = units * P.heads;
    for (int e = tid; e < rows * per_row; e += 256) {
      const int r = e / per_row, w = e - r * per_row;
      const int h = w / units, u = w - h * units;
      const T* px = x + r * P.ldx + (int64_t)h * P.head_dim;
      T* py = y + r * P.ldy + (int64_t)h * P.head_dim;
      if (u >= pairs) {
        py[pairs + u] = px[pairs + u];
      } else {
        const int i = HALF ? u : 2 * u, j = HALF ? u + pairs : 2 * u + 1;
        const float2 c = cs[r * pairs + u];
        const float p = St<T>::ld(px + i), q = St<T>::ld(px + j);
        St<T>::st(py + i, p * c.x - q * c.y);
        St<T>::st(py + j, q * c.x + p * c.y);
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
  // Rows of a work-group: enough pairs for its 256 threads, at most 16384 of them in LDS.
  const int pairs = std::max(1, d.rot / 2);
  P.rows_wg = std::max(1, 256 / pairs);
  // (a work-group's chunks fit 32 bits: width <= 2^30, and more rows only of narrow heads)
  while (P.rows_wg > 1 && (int64_t)P.rows_wg * d.heads * d.head_dim > ((int64_t)1 << 30)) P.rows_wg /= 2;
  const int64_t groups = ((int64_t)d.rows + P.rows_wg - 1) / P.rows_wg;
  const size_t lds = (size_t)P.rows_wg * pairs * sizeof(float2);
  const bool half = d.layout == DIT_ROTARY_HALF, vec = !half || d.rot % 16 == 0;
  const bool bf16 = d.dtype == DIT_DTYPE_BF16;
  void (*fn)(RotaryArgs);
  if (bf16) fn = half ? (vec ? rotary_kernel<bf16_t, true, true> : rotary_kernel<bf16_t, true, false>)
                      : rotary_kernel<bf16_t, false, true>;
  else fn = half ? (vec ? rotary_kernel<float, true, true> : rotary_kernel<float, true, false>)
                 : rotary_kernel<float, false, true>;
  hipLaunchKernelGGL(fn, dim3((uint32_t)groups), dim3(256), lds, s, P);
  return hipGetLastError();
}

}  // namespace dit
