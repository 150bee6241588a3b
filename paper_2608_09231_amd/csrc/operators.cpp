// C entry points of the low-precision products, the rotary positions and the sparse
// and packed attention: argument checks, then one launcher.  Nothing here waits,
// allocates or throws.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "../../include/dit_kernels.h"
#include "kernels.h"

namespace {

using dit::component_fail;

bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Compute units of the current device, asked for once per device.
int compute_units() {
  static std::atomic<int> known[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) dev = 0;
  const bool kept = dev >= 0 && dev < 64;
  int n = kept ? known[dev].load(std::memory_order_relaxed) : 0;
  if (n > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
  if (kept) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

dit_status launched(hipError_t e) {
  if (e == hipSuccess) return DIT_OK;
  return component_fail(DIT_EHIP, hipGetErrorString(e));
}

// Strides and alignment of the scale bytes of rows of K values.
bool scale_ok(const void* p, int64_t ld, int32_t K) { return aligned(p, 4) && ld % 4 == 0 && ld >= DIT_FP8_SCALE_LD(K); }

bool scale4_ok(const void* p, int64_t ld, int32_t K) { return aligned(p, 4) && ld % 4 == 0 && ld >= DIT_FP4_SCALE_LD(K); }

// A launch has fewer than 2^32 threads: work-groups of 1024, 512 and 256.
constexpr int64_t kMaxGroups1024 = ((int64_t)1 << 22) - 1, kMaxGroups512 = ((int64_t)1 << 23) - 1,
                  kMaxGroups256 = ((int64_t)1 << 24) - 1;
int64_t blocks_of(int64_t n, int64_t b) { return (n + b - 1) / b; }

constexpr int64_t kMaxStride = (int64_t)1 << 22;  // a tile's rows lie below 2^31 bytes from its first one

dit_status check_shape(const dit_sparse_shape* s) {
  if (!s) return component_fail(DIT_EINVAL, "null argument");
  if (s->batch < 0 || s->Lq < 0 || s->Lk < 0 || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads)
    return component_fail(DIT_ESHAPE, "bad attention shape");
  // (rounded up to whole tiles, key positions stay inside 32 bits)
  if (s->Lk > (1 << 30)) return component_fail(DIT_ESHAPE, "Lk must not pass 2^30");
  if (s->topk < 1 || s->topk > (1 << 30)) return component_fail(DIT_ESHAPE, "topk must lie in [1, 2^30]");
  const int64_t heads = (int64_t)s->batch * s->heads;  // (times 2^24 query blocks at most: inside 64 bits)
  if (s->heads > (1 << 20) || heads > 0x7fffffff || heads * blocks_of(s->Lq, DIT_SPARSE_QB) > (1 << 22))
    return component_fail(DIT_ESHAPE, "too many lists");
  return DIT_OK;
}

// (past 4096 key blocks a list takes 1024 threads)
dit_status check_select(const dit_sparse_shape* s) {
  const dit_status st = check_shape(s);
  if (st != DIT_OK) return st;
  const int64_t heads = (int64_t)s->batch * s->heads, nkb = blocks_of(s->Lk, DIT_SPARSE_KB);
  const int64_t lists = heads * blocks_of(s->Lq, DIT_SPARSE_QB);
  if (nkb > 16384 || heads > 65535 || lists + (int64_t)s->batch * s->kv_heads * nkb > kMaxGroups256 ||
      (nkb > 4096 && lists > kMaxGroups1024))
    return component_fail(DIT_ESHAPE, "too many blocks or heads");
  return DIT_OK;
}

// (empty: no rows, so that nothing is read or written at p)
dit_status check_rows(const void* p, int64_t ld, int64_t width, int64_t most, bool empty) {
  if (!p && !empty) return component_fail(DIT_EINVAL, "null argument");
  if (!aligned(p, 16)) return component_fail(DIT_EINVAL, "rows must be 16-byte aligned");
  if (ld < width || ld % 8 || ld > most) return component_fail(DIT_ESHAPE, "bad row stride");
  return DIT_OK;
}

dit_status check_packed(const dit_packed_shape* s) {
  if (!s) return component_fail(DIT_EINVAL, "null argument");
  if (s->batch < 0 || s->Tq < 0 || s->Tk < 0 || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads)
    return component_fail(DIT_ESHAPE, "bad attention shape");
  const int64_t rows = (int64_t)s->Tq * (s->heads / s->kv_heads);  // of a key head
  if (rows > (1 << 30) || s->Tk > (1 << 30)) return component_fail(DIT_ESHAPE, "more than 2^30 rows");
  if (s->heads > (1 << 20) || ((int64_t)s->batch + blocks_of(rows, 16)) * s->kv_heads > (1 << 22))
    return component_fail(DIT_ESHAPE, "too many sequences, heads or queries");
  return DIT_OK;
}

// The values of 4-bit rows that are written or read (the other side of the rows).
dit_status check_fp4(const void* x, int32_t dtype, int64_t ldx, const void* q, int64_t ldq, const void* scale, int64_t lds,
                     int32_t M, int32_t K) {
  if (M != 0 && K != 0 && (!x || !q || !scale)) return component_fail(DIT_EINVAL, "null argument");
  if (dtype != DIT_DTYPE_BF16 && dtype != DIT_DTYPE_F32) return component_fail(DIT_EINVAL, "bad type");
  if (!aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 4))
    return component_fail(DIT_EINVAL, "values and 4-bit rows must be 16-byte, scale 4-byte aligned");
  if (M < 0 || K < 0 || K % 32) return component_fail(DIT_ESHAPE, "K must be a multiple of 32");
  if (ldx < K || ldx % (dtype == DIT_DTYPE_BF16 ? 8 : 4) || ldq < K / 2 || ldq % 16 || !scale4_ok(scale, lds, K))
    return component_fail(DIT_ESHAPE, "bad row stride");
  if (K > (1 << 30) || blocks_of((int64_t)M * blocks_of(K, 1024), 4) > kMaxGroups256)
    return component_fail(DIT_ESHAPE, "too many values");
  return DIT_OK;
}

}  // namespace

#define TRY(expr)                \
  do {                           \
    dit_status s_ = (expr);      \
    if (s_ != DIT_OK) return s_; \
  } while (0)

extern "C" {

dit_status dit_quant_fp8(const void* x, int32_t x_dtype, int64_t ldx, void* q, int64_t ldq, void* scale, int64_t lds,
                         int32_t M, int32_t K, void* hip_stream) {
  if (M != 0 && K != 0 && (!x || !q || !scale)) return component_fail(DIT_EINVAL, "null argument");
  if (x_dtype != DIT_DTYPE_BF16 && x_dtype != DIT_DTYPE_F32) return component_fail(DIT_EINVAL, "bad input type");
  if (!aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 4))
    return component_fail(DIT_EINVAL, "x and q must be 16-byte, scale 4-byte aligned");
  if (M < 0 || K < 0 || K % 16) return component_fail(DIT_ESHAPE, "K must be a multiple of 16");
  if (ldx < K || ldx % (x_dtype == DIT_DTYPE_BF16 ? 8 : 4) || ldq < K || ldq % 16 || !scale_ok(scale, lds, K))
    return component_fail(DIT_ESHAPE, "bad row stride");
  if (K > (1 << 30) || blocks_of((int64_t)M * blocks_of(K, 1024), 4) > kMaxGroups256)
    return component_fail(DIT_ESHAPE, "too many values");
  return launched(dit::launch_quant_fp8(x, x_dtype == DIT_DTYPE_BF16, ldx, q, ldq, scale, lds, M, K,
                                        (hipStream_t)hip_stream));
}

dit_status dit_gemm_fp8(const dit_gemm_fp8_desc* d, void* hip_stream) {
  if (!d) return component_fail(DIT_EINVAL, "null argument");
  const bool empty = d->M == 0 || d->N == 0;
  if (!empty && (!d->A || !d->W || !d->a_scale || !d->w_scale || !d->C)) return component_fail(DIT_EINVAL, "null argument");
  const bool f32 = d->flags & DIT_EPI_F32, fp8 = d->flags & DIT_EPI_FP8, gated = d->flags & DIT_EPI_GATED_RES;
  if ((d->flags & ~(DIT_EPI_F32 | DIT_EPI_GATED_RES | DIT_EPI_SILU | DIT_EPI_FP8)) || f32 + fp8 + gated > 1)
    return component_fail(DIT_EINVAL, "bad flags");
  if (gated && !d->gate && !empty) return component_fail(DIT_EINVAL, "the gated residual needs a gate");
  if (fp8 && !d->c_scale && !empty) return component_fail(DIT_EINVAL, "the 8-bit output needs c_scale");
  if (!aligned(d->A, 16) || !aligned(d->W, 16) || !aligned(d->C, 16) || !aligned(d->bias, 2) ||
      (gated && !aligned(d->gate, 16)))
    return component_fail(DIT_EINVAL, "A, W, C and gate must be 16-byte aligned");
  if (!aligned(d->a_scale, 4) || !aligned(d->w_scale, 4) || (fp8 && !aligned(d->c_scale, 4)))
    return component_fail(DIT_EINVAL, "scales must be 4-byte aligned");
  if (d->M < 0 || d->N < 0 || d->K < 1 || d->K % 16 || d->N % 8)
    return component_fail(DIT_ESHAPE, "K must be a multiple of 16, N of 8");
  if (d->lda < d->K || d->ldw < d->K || d->lda % 16 || d->ldw % 16 || d->lda > kMaxStride || d->ldw > kMaxStride)
    return component_fail(DIT_ESHAPE, "bad operand stride");
  if (!scale_ok(d->a_scale, d->ld_as, d->K) || !scale_ok(d->w_scale, d->ld_ws, d->K))
    return component_fail(DIT_ESHAPE, "bad scale stride");
  const bool gap = d->gap != 0, gelu = d->gelu_from < d->N;
  if (d->gap < 0 || d->gap % 4 || (gap && (d->gap_at < 0 || d->gap_at % 4)))
    return component_fail(DIT_ESHAPE, "gap and gap_at must be multiples of 4");
  if (gelu && (d->gelu_from < 0 || d->gelu_from % 4)) return component_fail(DIT_ESHAPE, "gelu_from must be a multiple of 4");
  if (d->rms_cols < 0 || d->rms_cols % 128 || d->rms_cols > d->N || (d->rms_cols && d->N % 128))
    return component_fail(DIT_ESHAPE, "rms_cols and N must be multiples of 128");
  const int64_t width = (int64_t)d->N + (gap && d->gap_at < d->N ? d->gap : 0);
  if (gap && width > dit::kMaxGapWidth) return component_fail(DIT_ESHAPE, "output row too wide");
  if (d->ldc < width || d->ldc % 8) return component_fail(DIT_ESHAPE, "bad output stride");
  if (fp8 && (d->N % 128 || (gelu && d->gelu_from % 128) || gap || d->ldc % 16 || !scale_ok(d->c_scale, d->ld_cs, d->N)))
    return component_fail(DIT_ESHAPE, "bad shape of the 8-bit output");
  if (blocks_of(d->M, 64) * blocks_of(d->N, 128) > kMaxGroups512) return component_fail(DIT_ESHAPE, "too many outputs");
  dit::GemmFp8Args g{};
  g.A = d->A; g.lda = d->lda; g.W = d->W; g.ldw = d->ldw;
  g.As = d->a_scale; g.ldas = d->ld_as; g.Ws = d->w_scale; g.ldws = d->ld_ws;
  g.bias = d->bias; g.C = d->C; g.ldc = d->ldc; g.Cs = d->c_scale; g.ldcs = d->ld_cs; g.gate = d->gate;
  g.M = d->M; g.N = d->N; g.K = d->K;
  g.flags = d->flags; g.rms_cols = d->rms_cols; g.gelu_from = d->gelu_from;
  g.gap_at = gap ? d->gap_at : 0x7fffffff; g.gap = d->gap;
  return launched(dit::launch_gemm_fp8(g, (hipStream_t)hip_stream, compute_units()));
}

size_t dit_select_blocks_ws_bytes(const dit_sparse_shape* s) {
  return check_select(s) == DIT_OK ? dit::select_blocks_ws_bytes(*s) : 0;
}

dit_status dit_select_blocks_bf16(const dit_sparse_shape* s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                  int32_t first, int32_t* idx, void* ws, void* hip_stream) {
  TRY(check_select(s));
  const bool no_q = s->batch == 0 || s->Lq == 0, no_k = no_q || s->Lk == 0;
  if (!no_q && (!idx || !ws)) return component_fail(DIT_EINVAL, "null argument");
  if (!aligned(ws, 16) || !aligned(idx, 4) || !aligned(s->klen, 4))
    return component_fail(DIT_EINVAL, "the workspace must be 16-byte, idx and klen 4-byte aligned");
  TRY(check_rows(q, ldq, (int64_t)s->heads * 128, (int64_t)1 << 40, no_q));
  TRY(check_rows(k, ldk, (int64_t)s->kv_heads * 128, (int64_t)1 << 40, no_k));
  if (first < 0 || first > s->topk) return component_fail(DIT_EINVAL, "first must lie in [0, topk]");
  return launched(dit::launch_select_blocks(*s, q, ldq, k, ldk, first, idx, ws, (hipStream_t)hip_stream, compute_units()));
}

size_t dit_attention_sparse_ws_bytes(const dit_sparse_shape* s) {
  return check_shape(s) == DIT_OK ? dit::attention_sparse_ws_bytes(*s) : 0;
}

dit_status dit_attention_sparse_bf16(const dit_sparse_shape* s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                     const void* v, int64_t ldv, void* o, int64_t ldo, const int32_t* idx, int32_t flags,
                                     void* ws, void* hip_stream) {
  TRY(check_shape(s));
  const bool no_q = s->batch == 0 || s->Lq == 0, no_k = no_q || s->Lk == 0;
  if (!idx && !no_q) return component_fail(DIT_EINVAL, "null argument");
  if (flags & ~DIT_ATTN_BOUNDED_LOGITS) return component_fail(DIT_EINVAL, "bad attention flags");
  if (!aligned(idx, 4) || !aligned(s->klen, 4)) return component_fail(DIT_EINVAL, "idx and klen must be 4-byte aligned");
  TRY(check_rows(q, ldq, (int64_t)s->heads * 128, kMaxStride - 1, no_q));
  TRY(check_rows(k, ldk, (int64_t)s->kv_heads * 128, kMaxStride - 1, no_k));
  TRY(check_rows(v, ldv, (int64_t)s->kv_heads * 128, kMaxStride - 1, no_k));
  TRY(check_rows(o, ldo, (int64_t)s->heads * 128, kMaxStride - 1, no_q));
  if (dit::attention_sparse_ws_bytes(*s) && (!ws || !aligned(ws, 16)))
    return component_fail(DIT_EINVAL, "needs a 16-byte aligned workspace");
  return launched(dit::launch_attention_sparse(*s, q, ldq, k, ldk, v, ldv, o, ldo, idx,
                                               (flags & DIT_ATTN_BOUNDED_LOGITS) != 0, ws, (hipStream_t)hip_stream,
                                               compute_units()));
}

dit_status dit_quant_fp4(const void* x, int32_t x_dtype, int64_t ldx, void* q, int64_t ldq, void* scale, int64_t lds,
                         int32_t M, int32_t K, void* hip_stream) {
  TRY(check_fp4(x, x_dtype, ldx, q, ldq, scale, lds, M, K));
  return launched(dit::launch_quant_fp4(x, x_dtype == DIT_DTYPE_BF16, ldx, q, ldq, scale, lds, M, K,
                                        (hipStream_t)hip_stream));
}

dit_status dit_dequant_fp4(const void* q, int64_t ldq, const void* scale, int64_t lds, void* y, int32_t y_dtype,
                           int64_t ldy, int32_t M, int32_t K, void* hip_stream) {
  TRY(check_fp4(y, y_dtype, ldy, q, ldq, scale, lds, M, K));
  return launched(dit::launch_dequant_fp4(q, ldq, scale, lds, y, y_dtype == DIT_DTYPE_BF16, ldy, M, K,
                                          (hipStream_t)hip_stream));
}

dit_status dit_gemm_fp4(const dit_gemm_fp4_desc* d, void* hip_stream) {
  if (!d) return component_fail(DIT_EINVAL, "null argument");
  const bool empty = d->M == 0 || d->N == 0;
  if (!empty && (!d->A || !d->W || !d->a_scale || !d->w_scale || !d->C)) return component_fail(DIT_EINVAL, "null argument");
  const bool f32 = d->flags & DIT_EPI_F32, fp4 = d->flags & DIT_EPI_FP4, gated = d->flags & DIT_EPI_GATED_RES;
  if ((d->flags & ~(DIT_EPI_F32 | DIT_EPI_GATED_RES | DIT_EPI_SILU | DIT_EPI_FP4)) || f32 + fp4 + gated > 1)
    return component_fail(DIT_EINVAL, "bad flags");
  if (gated && !d->gate && !empty) return component_fail(DIT_EINVAL, "the gated residual needs a gate");
  if (fp4 && !d->c_scale && !empty) return component_fail(DIT_EINVAL, "the 4-bit output needs c_scale");
  if (!aligned(d->A, 16) || !aligned(d->W, 16) || !aligned(d->C, 16) || !aligned(d->bias, 2) ||
      (gated && !aligned(d->gate, 16)))
    return component_fail(DIT_EINVAL, "A, W, C and gate must be 16-byte aligned");
  if (!aligned(d->a_scale, 4) || !aligned(d->w_scale, 4) || (fp4 && !aligned(d->c_scale, 4)))
    return component_fail(DIT_EINVAL, "scales must be 4-byte aligned");
  if (d->M < 0 || d->N < 0 || d->K < 1 || d->K % 32 || d->N % 8)
    return component_fail(DIT_ESHAPE, "K must be a multiple of 32, N of 8");
  if (d->lda < d->K / 2 || d->ldw < d->K / 2 || d->lda % 16 || d->ldw % 16 || d->lda > kMaxStride || d->ldw > kMaxStride)
    return component_fail(DIT_ESHAPE, "bad operand stride");
  if (!scale4_ok(d->a_scale, d->ld_as, d->K) || !scale4_ok(d->w_scale, d->ld_ws, d->K) || d->ld_as > kMaxStride ||
      d->ld_ws > kMaxStride)
    return component_fail(DIT_ESHAPE, "bad scale stride");
  const bool gap = d->gap != 0, gelu = d->gelu_from < d->N;
  if (d->gap < 0 || d->gap % 4 || (gap && (d->gap_at < 0 || d->gap_at % 4)))
    return component_fail(DIT_ESHAPE, "gap and gap_at must be multiples of 4");
  if (gelu && (d->gelu_from < 0 || d->gelu_from % 4)) return component_fail(DIT_ESHAPE, "gelu_from must be a multiple of 4");
  if (d->rms_cols < 0 || d->rms_cols % 128 || d->rms_cols > d->N || (d->rms_cols && d->N % 128))
    return component_fail(DIT_ESHAPE, "rms_cols and N must be multiples of 128");
  const int64_t width = (int64_t)d->N + (gap && d->gap_at < d->N ? d->gap : 0);
  if (gap && width > dit::kMaxGapWidth) return component_fail(DIT_ESHAPE, "output row too wide");
  if (d->ldc < (fp4 ? d->N / 2 : width) || d->ldc % 8) return component_fail(DIT_ESHAPE, "bad output stride");
  if (fp4 && (d->N % 32 || (gelu && d->gelu_from % 128) || gap || d->ldc % 16 || !scale4_ok(d->c_scale, d->ld_cs, d->N)))
    return component_fail(DIT_ESHAPE, "bad shape of the 4-bit output");
  if (blocks_of(d->M, 64) * blocks_of(d->N, 128) > kMaxGroups512) return component_fail(DIT_ESHAPE, "too many outputs");
  dit::GemmFp4Args g{};
  g.A = d->A; g.lda = d->lda; g.W = d->W; g.ldw = d->ldw;
  g.As = d->a_scale; g.ldas = d->ld_as; g.Ws = d->w_scale; g.ldws = d->ld_ws;
  g.bias = d->bias; g.C = d->C; g.ldc = d->ldc; g.Cs = d->c_scale; g.ldcs = d->ld_cs; g.gate = d->gate;
  g.M = d->M; g.N = d->N; g.K = d->K;
  g.flags = d->flags; g.rms_cols = d->rms_cols; g.gelu_from = d->gelu_from;
  g.gap_at = gap ? d->gap_at : 0x7fffffff; g.gap = d->gap;
  return launched(dit::launch_gemm_fp4(g, (hipStream_t)hip_stream, compute_units()));
}

dit_status dit_rotary_freqs(int32_t pairs, double base, int32_t method, double factor, double context, double* freq,
                            double* scale) {
  if (pairs < 0) return component_fail(DIT_ESHAPE, "pairs must not be negative");
  if ((!freq && pairs) || !scale) return component_fail(DIT_EINVAL, "null argument");
  if (method < DIT_ROTARY_PLAIN || method > DIT_ROTARY_PARTS) return component_fail(DIT_EINVAL, "bad method");
  auto positive = [](double v) { return v > 0 && isfinite(v); };
  if (!positive(base) || (method != DIT_ROTARY_PLAIN && !positive(factor)) ||
      (method == DIT_ROTARY_PARTS && !positive(context)))
    return component_fail(DIT_EINVAL, "base, factor and context must be positive and finite");
  if (method == DIT_ROTARY_BASE && pairs == 1) return component_fail(DIT_ESHAPE, "a single pair has no base to change");
  if (method == DIT_ROTARY_BASE) base *= pow(factor, (double)pairs / (pairs - 1));
  for (int32_t i = 0; i < pairs; ++i) {
    double f = pow(base, -(double)i / pairs);
    if (method == DIT_ROTARY_LINEAR) f /= factor;
    if (method == DIT_ROTARY_PARTS) {
      constexpr double kTwoPi = 6.283185307179586477, kSlow = 1, kFast = 32;
      const double keep = fmin(1.0, fmax(0.0, (context * f / kTwoPi - kSlow) / (kFast - kSlow)));
      f = f * keep + f / factor * (1 - keep);
    }
    freq[i] = f;
  }
  *scale = method == DIT_ROTARY_PARTS ? 0.1 * log(factor) + 1 : 1;
  return DIT_OK;
}

dit_status dit_rotary(const dit_rotary_desc* d, void* hip_stream) {
  if (!d) return component_fail(DIT_EINVAL, "null argument");
  if (d->rows < 0 || d->heads < 0 || d->head_dim < 8 || d->head_dim % 8 || d->head_dim > 512)
    return component_fail(DIT_ESHAPE, "bad sizes");
  if (d->rows > kMaxGroups256) return component_fail(DIT_ESHAPE, "too many rows");
  if (d->rot < 0 || d->rot % 2 || d->rot > d->head_dim) return component_fail(DIT_ESHAPE, "bad rotated width");
  if (d->axes < 1 || d->axes > DIT_ROTARY_AXES) return component_fail(DIT_ESHAPE, "bad number of axes");
  int64_t pairs = 0;
  for (int a = 0; a < d->axes; ++a) {
    if (d->pairs[a] < 0) return component_fail(DIT_ESHAPE, "negative pairs");
    pairs += d->pairs[a];
  }
  if (pairs != d->rot / 2) return component_fail(DIT_ESHAPE, "the axes' pairs must make rot / 2");
  const bool empty = d->rows == 0 || d->heads == 0;
  if (!empty && (!d->x || !d->y || (d->rot && (!d->pos || !d->freq)))) return component_fail(DIT_EINVAL, "null argument");
  if (d->dtype != DIT_DTYPE_BF16 && d->dtype != DIT_DTYPE_F32) return component_fail(DIT_EINVAL, "bad type");
  if (d->layout != DIT_ROTARY_HALF && d->layout != DIT_ROTARY_INTERLEAVED) return component_fail(DIT_EINVAL, "bad layout");
  if (!isfinite(d->scale)) return component_fail(DIT_EINVAL, "scale must be finite");
  if (!aligned(d->x, 16) || !aligned(d->y, 16) || !aligned(d->pos, 4) || !aligned(d->freq, 8))
    return component_fail(DIT_EINVAL, "x and y must be 16-byte, freq 8-byte, pos 4-byte aligned");
  const int64_t width = (int64_t)d->heads * d->head_dim, esize = d->dtype == DIT_DTYPE_BF16 ? 2 : 4;
  if (width > (1 << 30)) return component_fail(DIT_ESHAPE, "rows too wide");
  for (const int64_t ld : {d->ldx, d->ldy})
    if (ld < width || ld % (16 / esize) || ld > ((int64_t)1 << 40)) return component_fail(DIT_ESHAPE, "bad row stride");
  if (d->axes > 1 && (d->ldpos < d->rows || d->ldpos > ((int64_t)1 << 40)))
    return component_fail(DIT_ESHAPE, "bad stride of the positions");
  if (!empty && (d->x != d->y || d->ldx != d->ldy)) {
    const uintptr_t x = (uintptr_t)d->x, y = (uintptr_t)d->y, w = (uintptr_t)(width * esize);
    const uintptr_t xe = x + (uintptr_t)((d->rows - 1) * d->ldx * esize) + w, ye = y + (uintptr_t)((d->rows - 1) * d->ldy * esize) + w;
    if (x < ye && y < xe) {  // the ranges cross: only columns of one matrix beside each other may
      const uintptr_t step = (uintptr_t)(d->ldx * esize), apart = (y > x ? y - x : x - y) % step;
      if (d->ldx != d->ldy || apart < w || step - apart < w) return component_fail(DIT_EINVAL, "x and y overlap");
    }
  }
  return launched(dit::launch_rotary(*d, (hipStream_t)hip_stream));
}

size_t dit_attention_packed_ws_bytes(const dit_packed_shape* s) {
  return check_packed(s) == DIT_OK ? dit::attention_packed_ws_bytes(*s) : 0;
}

dit_status dit_attention_packed_bf16(const dit_packed_shape* s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                     const void* v, int64_t ldv, void* o, int64_t ldo, int32_t flags, void* ws,
                                     void* hip_stream) {
  TRY(check_packed(s));
  const bool no_q = s->batch == 0 || s->Tq == 0, no_k = no_q || s->Tk == 0;
  if (!no_q && (!s->qoff || !s->koff)) return component_fail(DIT_EINVAL, "null argument");
  if (flags & ~(DIT_ATTN_BOUNDED_LOGITS | DIT_ATTN_CAUSAL)) return component_fail(DIT_EINVAL, "bad attention flags");
  if (!aligned(s->qoff, 4) || !aligned(s->koff, 4) || !aligned(s->klen, 4))
    return component_fail(DIT_EINVAL, "qoff, koff and klen must be 4-byte aligned");
  TRY(check_rows(q, ldq, (int64_t)s->heads * 128, kMaxStride - 1, no_q));
  TRY(check_rows(k, ldk, (int64_t)s->kv_heads * 128, kMaxStride - 1, no_k));
  TRY(check_rows(v, ldv, (int64_t)s->kv_heads * 128, kMaxStride - 1, no_k));
  TRY(check_rows(o, ldo, (int64_t)s->heads * 128, kMaxStride - 1, no_q));
  if (dit::attention_packed_ws_bytes(*s) && (!ws || !aligned(ws, 16)))
    return component_fail(DIT_EINVAL, "needs a 16-byte aligned workspace");
  return launched(dit::launch_attention_packed(*s, q, ldq, k, ldk, v, ldv, o, ldo, (flags & DIT_ATTN_BOUNDED_LOGITS) != 0,
                                               (flags & DIT_ATTN_CAUSAL) != 0, ws, (hipStream_t)hip_stream));
}

}  // extern "C"
