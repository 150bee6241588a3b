/*
 * dit_kernels.h -- component entry points of the cached DiT sampler's
 * full-step kernels (gfx950), for callers that drive single operations:
 * parity tests at full workload shapes and kernel microbenchmarks.
 * Same conventions as dit_cache.h (status codes, caller-owned device
 * buffers, the call returns after the stream has drained).
 */
#ifndef DIT_KERNELS_H
#define DIT_KERNELS_H

#include <stddef.h>
#include <stdint.h>

#include "dit_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Epilogue flags of the bf16 GEMM. */
enum {
  DIT_EPI_STORE = 0,      /* C = S(acc + bias)                                   */
  DIT_EPI_F32 = 1,        /* C (f32) = acc + bias                                */
  DIT_EPI_GATED_RES = 2,  /* C = S(C + gate[n] * (acc + bias)), in place         */
  DIT_EPI_SILU = 4        /* C = S(SiLU(acc + bias))                             */
};

/* C = epilogue(A . W^T + bias): the linear layers of the blocks (QKV with
 * per-head RMS norm of q and k, out-projection and MLP-down with the
 * adaLN-gated residual, MLP-up with GELU-tanh).  bf16 operands, f32
 * accumulation on MFMA, S = round to bf16 (nearest even).
 *   A    device bf16 [M, K], row stride lda elements (lda >= K, K % 8 == 0)
 *   W    device bf16 [N, K], row stride ldw (torch nn.Linear layout)
 *   bias device bf16 [N] or NULL
 *   C    device bf16 (f32 with DIT_EPI_F32) [M, *], row stride ldc (>= N,
 *        plus gap when gap_at < N; else DIT_ESHAPE)
 *   gate device f32 [N], DIT_EPI_GATED_RES only
 *   rms_cols  columns n < rms_cols are normalised per 128-wide head
 *             (RMS, eps 1e-6, unit gain) before rounding; 0 = none;
 *             must be a multiple of 128
 *   gelu_from columns n >= gelu_from get GELU-tanh; >= N = none
 *   gap_at, gap  output column = n + gap for n >= gap_at (writes the MLP
 *             half of a fused projection next to a hole for the attention
 *             output); gap = 0 = none
 * Where few 256 x 256 output tiles are left past the chip's last whole round,
 * they are shared out over K and the parts added from f32 sums in device
 * memory of the library: 65 MiB per call in flight that does so, allocated on
 * first use, at most four such buffers per GPU kept for further calls.  Whether
 * a call does depends on its shape alone, so that the result's bits do not
 * depend on other calls; only with no device memory left does it run whole
 * tiles instead (the same result up to the rounding of f32 sums).
 * Errors: DIT_EINVAL (null pointers, bad flags), DIT_ESHAPE (K % 8, lda or
 * ldw < K, ldc too small, gap < 0, an output row of more than 2^30 columns with
 * its gap, rms_cols not a multiple of 128), DIT_EHIP. */
typedef struct dit_gemm_desc {
  const void* A; int64_t lda;
  const void* W; int64_t ldw;
  const void* bias;
  void* C; int64_t ldc;
  int32_t M, N, K;
  int32_t flags;
  const float* gate;
  int32_t rms_cols;
  int32_t gelu_from;
  int32_t gap_at, gap;
} dit_gemm_desc;

dit_status dit_gemm_bf16(const dit_gemm_desc* d, void* hip_stream);

/* Attention flags. */
enum {
  /* The caller guarantees |q . k| <= 128 per head (e.g. q and k RMS-normalised
   * with unit gain), so every logit is at most sqrt(128) and a fixed shift
   * replaces the running maximum of the softmax (same result). */
  DIT_ATTN_BOUNDED_LOGITS = 1
};

/* o = softmax(q k^T / sqrt(128)) v per head (non-causal), bf16 in and out,
 * f32 softmax and accumulation on MFMA.  q [Lq, heads*128] (row stride
 * ldq), k and v [Lk, heads*128] (ldk, ldv), o [Lq, heads*128] (ldo);
 * head h occupies columns [128h, 128h + 128).  flags: 0 or
 * DIT_ATTN_BOUNDED_LOGITS.  vt_ws is a device workspace of heads * 128 *
 * round_up(Lk, 64) bf16 elements for v transposed per head.  Where the work
 * fills the chip's CUs only partly in its last round, the key ranges are
 * shared out and the parts added from f32 sums in device memory of the library
 * (see dit_gemm_bf16): by the shapes alone, so that the result's bits do not
 * depend on other calls.
 * Errors: DIT_EINVAL, DIT_ESHAPE (Lq, Lk < 1), DIT_EHIP. */
dit_status dit_attention_bf16(const void* q, int64_t ldq, const void* k, int64_t ldk,
                              const void* v, int64_t ldv, void* o, int64_t ldo,
                              int32_t Lq, int32_t Lk, int32_t heads, int32_t flags, void* vt_ws,
                              void* hip_stream);

/* Largest v-transpose the allocation-free attention holds: heads * 128 *
 * round_up(Lk, 64) bf16 elements (32 MiB; e.g. 24 heads at up to 5440 keys). */
#define DIT_NOALLOC_VT_MAX_ELEMS (16 * 1024 * 1024)

/* dit_attention_bf16 without the vt_ws workspace argument, for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc).  The transposed values and the f32
 * sums of a shared last round go to fixed device arrays inside the library
 * (DIT_NOALLOC_VT_MAX_ELEMS bf16 elements, 32 MiB, and 65 MiB), one of each per
 * GPU, held until the process ends; the call allocates nothing (no hipMalloc /
 * hipFree, no allocating library routine).  The arrays' device addresses are
 * looked up once per device, on the first call made with that device
 * current.  Same arguments, kernels and result bits as dit_attention_bf16.
 * Every call on one GPU shares that GPU's arrays:
 * calls that overlap on one GPU (other streams or host threads) race and
 * must be serialised by the caller.  Errors: as dit_attention_bf16, plus
 * DIT_ESHAPE when heads * 128 * round_up(Lk, 64) > DIT_NOALLOC_VT_MAX_ELEMS
 * (nothing is launched). */
dit_status dit_attention_bf16_noalloc(const void* q, int64_t ldq, const void* k, int64_t ldk,
                                      const void* v, int64_t ldv, void* o, int64_t ldo,
                                      int32_t Lq, int32_t Lk, int32_t heads, int32_t flags,
                                      void* hip_stream);

/* ---- a full step in 8-bit products and sparse attention ---------------
 *
 * The calls below only enqueue their work: they return before it has run,
 * wait for nothing, allocate nothing and can be captured into a HIP graph.
 * Their workspaces belong to the caller, and a workspace serves one call at
 * a time: two calls (or graphs) that may run at the same time need two.  The
 * current device is the stream's.  Nothing is launched where a status other
 * than DIT_OK is returned for an argument.  A size of zero is no error (K = 0
 * of a product is), and the pointers to what is empty then may be NULL; where
 * nothing is to be written nothing is launched.
 *
 * 8-bit rows.  A row of K values is held as K bytes of e4m3 (OCP, largest
 * value 448) and one scale byte (E8M0: 2^(byte - 127)) for each 128 of them,
 * the last of which may be partial: x = e4m3 * scale.  Scale bytes of row m
 * start at scale + m * lds; lds is a multiple of 4 and at least
 * DIT_FP8_SCALE_LD(K), scale is 4-byte aligned (bytes past the last block's
 * are read with their neighbours, and not used). */
#define DIT_FP8_SCALE_LD(K) ((((int64_t)(K) + 511) / 512) * 4)

/* q, scale = 8-bit rows of x: per block the least scale with
 * max |x| <= 448 * scale, e4m3(x / scale) rounded to nearest even.  A block of
 * zeros gets scale byte 0; one that holds a NaN or an infinity gets scale
 * byte 255 (NaN) and NaNs.
 *   x      device, x_dtype DIT_DTYPE_BF16 or DIT_DTYPE_F32 [M, K], row stride ldx
 *   q      device e4m3 [M, K], row stride ldq bytes
 * Errors: DIT_EINVAL (null pointers, bad type, x or q not 16-byte or scale not
 * 4-byte aligned), DIT_ESHAPE (negative sizes, K % 16, a stride below the row
 * or, in bytes, no multiple of 16, lds, K above 2^30, M * ceil(K / 1024) above 2^26 - 4), DIT_EHIP. */
dit_status dit_quant_fp8(const void* x, int32_t x_dtype, int64_t ldx, void* q, int64_t ldq, void* scale,
                         int64_t lds, int32_t M, int32_t K, void* hip_stream);

/* Epilogue flag of dit_gemm_fp8 beside those of dit_gemm_bf16: C and c_scale =
 * the 8-bit rows of acc + bias (after norm, GELU, SiLU), each row's 128
 * columns a block. */
enum { DIT_EPI_FP8 = 8 };

/* C = epilogue(A . W^T + bias) on 8-bit rows, with the epilogues of
 * dit_gemm_bf16 (same meaning of bias, gate, rms_cols, gelu_from, gap_at, gap).
 *   A, a_scale  8-bit rows [M, K], row strides lda, ld_as bytes
 *   W, w_scale  8-bit rows [N, K], row strides ldw, ld_ws bytes
 *   C           bf16, f32 (DIT_EPI_F32) or e4m3 (DIT_EPI_FP8), row stride ldc elements
 *   c_scale     DIT_EPI_FP8 only: scale bytes of C, row stride ld_cs
 * Accumulation is f32.  bf16 and e4m3 outputs come from the 8-bit matrix cores,
 * which add a few neighbouring products in about 14 bits before they enter the
 * f32 sum (2e-5 in the 2-norm on normal data); f32 outputs are computed from
 * operands widened to bf16, at half that rate.  Every scale byte is good for
 * every output; f32 outputs of rows with bytes above 236, or whose sums pass 2^108,
 * take up to ten times as long.
 * Errors: DIT_EINVAL (null pointers; bad flags: one of F32, FP8 and GATED_RES
 * at most; A, W, C, gate not 16-byte, scales not 4-byte, bias not 2-byte
 * aligned), DIT_ESHAPE (negative sizes, K < 1, K % 16, N % 8, lda or ldw below
 * K, above 2^22 or no multiple of 16, the scale strides, ldc below the written
 * row or no multiple of 8, rms_cols no multiple of 128 or above N, gelu_from < N
 * no multiple of 4, gap or gap_at no multiple of 4 or negative, an output row of
 * more than 2^30 columns with its gap; with DIT_EPI_FP8: N or gelu_from < N no
 * multiple of 128, ldc no multiple of 16, a gap; with rms_cols: N no multiple of
 * 128; ceil(M / 64) * ceil(N / 128) of 2^23 or more), DIT_EHIP. */
typedef struct dit_gemm_fp8_desc {
  const void* A; int64_t lda;
  const void* a_scale; int64_t ld_as;
  const void* W; int64_t ldw;
  const void* w_scale; int64_t ld_ws;
  const void* bias;
  void* C; int64_t ldc;
  void* c_scale; int64_t ld_cs;
  const float* gate;
  int32_t M, N, K;
  int32_t flags;
  int32_t rms_cols;
  int32_t gelu_from;
  int32_t gap_at, gap;
} dit_gemm_fp8_desc;

dit_status dit_gemm_fp8(const dit_gemm_fp8_desc* d, void* hip_stream);

/* Sparse attention: DIT_SPARSE_QB consecutive queries of a head share a list of
 * blocks of DIT_SPARSE_KB consecutive keys (the last block of either may be
 * partial), head_dim 128, bf16.
 * `batch` sequences are stacked by rows: sequence z's queries are rows z Lq ..
 * of q and o, its keys rows z Lk .. of k and v.  Query head h reads key head
 * h / (heads / kv_heads).  klen: keys of each sequence (device, clamped to [0,
 * Lk]); rows past them are not read for their values, whatever they hold.
 * Lists: device int32 [batch, heads, ceil(Lq / DIT_SPARSE_QB), topk]. */
enum { DIT_SPARSE_QB = 128, DIT_SPARSE_KB = 64 };
typedef struct dit_sparse_shape {
  int32_t batch, Lq, Lk;
  int32_t heads, kv_heads;
  int32_t topk;            /* entries of a list */
  const int32_t* klen;     /* device [batch], or NULL: Lk each */
} dit_sparse_shape;

/* idx = for each query block the topk key blocks with the largest product of
 * the blocks' mean query and mean key (means over the rows that exist, in
 * float64; equal products go to the lowest block, NaN counts as -inf), in
 * ascending order.  Blocks 0 .. first - 1 are taken whatever their product.
 * Where a sequence has fewer blocks than topk, the rest of the list is -1.
 *   q [batch Lq, heads 128] (row stride ldq), k [batch Lk, kv_heads 128] (ldk)
 *   ws  device, dit_select_blocks_ws_bytes(s) (0 for shapes that are refused), 16-byte aligned
 * Errors: DIT_EINVAL (null pointers, alignment of 16 bytes, first outside [0,
 * topk]), DIT_ESHAPE (negative sizes; heads no multiple of kv_heads; topk < 1; topk or Lk above 2^30;
 * strides below the row or no multiple of 8; more than 2^22 lists; more than
 * 16384 key blocks a sequence, 65535 batch * heads, 2^24 - 1 lists and key
 * blocks of all key heads together, or 2^22 - 1 lists where a sequence has more than
 * 4096 key blocks), DIT_EHIP. */
size_t dit_select_blocks_ws_bytes(const dit_sparse_shape* s);
dit_status dit_select_blocks_bf16(const dit_sparse_shape* s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                  int32_t first, int32_t* idx, void* ws, void* hip_stream);

/* o = softmax(q k^T / sqrt(128)) v over the listed key blocks.  Entries outside
 * the sequence's key blocks (-1, say) are passed over; a block listed twice
 * counts twice; a query without a key gets zeros.  flags: 0 or
 * DIT_ATTN_BOUNDED_LOGITS.  Probabilities are rounded to bf16 (both in the sum
 * and in the product), sums and outputs are f32 until the one rounding of o.
 *   ws  device, dit_attention_sparse_ws_bytes(s) (may be 0: then NULL will do),
 *       16-byte aligned
 * Errors: as dit_select_blocks_bf16 (without `first` and the last four
 * limits), strides of 2^22 or more, bad flags. */
size_t dit_attention_sparse_ws_bytes(const dit_sparse_shape* s);
dit_status dit_attention_sparse_bf16(const dit_sparse_shape* s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                     const void* v, int64_t ldv, void* o, int64_t ldo, const int32_t* idx,
                                     int32_t flags, void* ws, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DIT_KERNELS_H */
