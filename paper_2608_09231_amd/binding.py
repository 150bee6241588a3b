"""ctypes binding of libdit_cache.so (argument marshalling only).

Every tensor operation of the sampler runs in the library's HIP kernels;
this module converts Python / torch arguments into the C structs and
pointers of ``include/dit_cache.h`` and ``include/dit_kernels.h``.  Loading
fails loudly when the library has not been built: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdit_cache.so")

DIT_OK, DIT_EINVAL, DIT_ENOMEM, DIT_EHIP, DIT_ESHAPE, DIT_EBUDGET, DIT_ENONFINITE = 0, -1, -2, -3, -4, -5, -6
STATUS_NAMES = {0: "DIT_OK", -1: "DIT_EINVAL", -2: "DIT_ENOMEM", -3: "DIT_EHIP", -4: "DIT_ESHAPE",
                -5: "DIT_EBUDGET", -6: "DIT_ENONFINITE"}
DTYPE_F32, DTYPE_BF16 = 0, 1
INDICATOR_MODULATED, INDICATOR_PATCH = 0, 1
EPI_STORE, EPI_F32, EPI_GATED_RES, EPI_SILU, EPI_FP8, EPI_FP4 = 0, 1, 2, 4, 8, 16
ABI_VERSION = 4
POLICIES = {"gate": 0, "static": 1, "threshold": 2}
SOLVERS = {"euler": 0, "unipc": 1}
N_FEATURES = 8
K_CLASSES = ["gemm", "attn", "indicator", "reuse", "full_other", "once"]

# Every symbol the headers declare.
EXPORTS = ["dit_cache_create", "dit_cache_sample", "dit_cache_sample_ex", "dit_cache_sample_batch",
           "dit_gate_logit", "dit_cache_destroy",
           "dit_cache_last_error", "dit_cache_set_profiling", "dit_cache_get_stats",
           "dit_cache_reset_stats", "dit_gemm_bf16", "dit_attention_bf16", "dit_attention_bf16_noalloc",
           "dit_quant_fp8", "dit_gemm_fp8", "dit_select_blocks_ws_bytes", "dit_select_blocks_bf16",
           "dit_attention_sparse_ws_bytes", "dit_attention_sparse_bf16",
           "dit_quant_fp4", "dit_dequant_fp4", "dit_gemm_fp4", "dit_rotary_freqs", "dit_rotary",
           "dit_attention_packed_ws_bytes", "dit_attention_packed_bf16"]


class ModelConfigC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "abi_version", "dtype", "n_double", "n_single", "n_cross", "hidden", "heads", "head_dim",
        "mlp_hidden", "in_channels", "ctx_dim", "time_dim", "n_img", "n_txt", "batch", "pooled_text")]


class SampleParamsC(C.Structure):
    _fields_ = [("T", C.c_int32), ("B", C.c_int32), ("sigmas", C.POINTER(C.c_double)),
                ("shift", C.c_double), ("tau", C.c_double), ("guidance", C.c_double),
                ("forced_mask", C.POINTER(C.c_uint8)), ("indicator", C.c_int32),
                ("policy", C.c_int32), ("delta", C.c_double), ("solver", C.c_int32)]


class ScheduleC(C.Structure):
    _fields_ = [("full", C.POINTER(C.c_uint8)), ("logit", C.POINTER(C.c_float)),
                ("forced", C.POINTER(C.c_uint8)), ("features", C.POINTER(C.c_double)),
                ("sums", C.POINTER(C.c_double)), ("nfe", C.c_int32), ("steps_done", C.c_int32)]


class StatsC(C.Structure):
    _fields_ = [("ms", C.c_double * 6), ("work", C.c_double * 6), ("launches", C.c_int64 * 6),
                ("host_gate_ms", C.c_double), ("sample_ms", C.c_double), ("samples", C.c_int64),
                ("full_steps", C.c_int64), ("reuse_steps", C.c_int64)]


class GemmDescC(C.Structure):
    _fields_ = [("A", C.c_void_p), ("lda", C.c_int64), ("W", C.c_void_p), ("ldw", C.c_int64),
                ("bias", C.c_void_p), ("C", C.c_void_p), ("ldc", C.c_int64),
                ("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("flags", C.c_int32),
                ("gate", C.c_void_p), ("rms_cols", C.c_int32), ("gelu_from", C.c_int32),
                ("gap_at", C.c_int32), ("gap", C.c_int32)]


class GemmFp8DescC(C.Structure):
    _fields_ = [("A", C.c_void_p), ("lda", C.c_int64), ("a_scale", C.c_void_p), ("ld_as", C.c_int64),
                ("W", C.c_void_p), ("ldw", C.c_int64), ("w_scale", C.c_void_p), ("ld_ws", C.c_int64),
                ("bias", C.c_void_p), ("C", C.c_void_p), ("ldc", C.c_int64), ("c_scale", C.c_void_p),
                ("ld_cs", C.c_int64), ("gate", C.c_void_p), ("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32),
                ("flags", C.c_int32), ("rms_cols", C.c_int32), ("gelu_from", C.c_int32), ("gap_at", C.c_int32),
                ("gap", C.c_int32)]


class SparseShapeC(C.Structure):
    _fields_ = [("batch", C.c_int32), ("Lq", C.c_int32), ("Lk", C.c_int32), ("heads", C.c_int32),
                ("kv_heads", C.c_int32), ("topk", C.c_int32), ("klen", C.c_void_p)]


class GemmFp4DescC(C.Structure):
    _fields_ = list(GemmFp8DescC._fields_)


class RotaryDescC(C.Structure):
    _fields_ = [("x", C.c_void_p), ("ldx", C.c_int64), ("y", C.c_void_p), ("ldy", C.c_int64),
                ("pos", C.c_void_p), ("ldpos", C.c_int64), ("freq", C.c_void_p)] \
        + [(n, C.c_int32) for n in ("dtype", "rows", "heads", "head_dim", "rot", "layout", "axes")] \
        + [("pairs", C.c_int32 * 4), ("scale", C.c_float)]


class PackedShapeC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "Tq", "Tk", "heads", "kv_heads")] \
        + [(n, C.c_void_p) for n in ("qoff", "koff", "klen")]


class DitError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


_lib = None


def load(path: str = LIB_PATH):
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} is missing: build it with `python -m paper_2608_09231_amd.build`")
    lib = C.CDLL(path)
    vp, sz = C.c_void_p, C.c_size_t
    lib.dit_cache_create.argtypes = [C.POINTER(ModelConfigC), vp, sz, vp, C.POINTER(vp)]
    lib.dit_cache_sample.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, vp, sz, C.POINTER(ScheduleC)]
    lib.dit_cache_sample_ex.argtypes = [vp, vp, vp, vp, sz, C.POINTER(SampleParamsC), C.POINTER(ScheduleC)]
    lib.dit_cache_sample_batch.argtypes = [vp, C.c_int32, vp, vp, vp, sz, C.POINTER(SampleParamsC),
                                           C.POINTER(ScheduleC)]
    lib.dit_gate_logit.argtypes = [vp, sz, vp, vp]
    lib.dit_cache_destroy.argtypes = [vp]
    lib.dit_cache_destroy.restype = None
    lib.dit_cache_last_error.argtypes = [vp]
    lib.dit_cache_last_error.restype = C.c_char_p
    lib.dit_cache_set_profiling.argtypes = [vp, C.c_int32]
    lib.dit_cache_get_stats.argtypes = [vp, C.POINTER(StatsC)]
    lib.dit_cache_reset_stats.argtypes = [vp]
    lib.dit_gemm_bf16.argtypes = [C.POINTER(GemmDescC), vp]
    lib.dit_attention_bf16.argtypes = [vp, C.c_int64, vp, C.c_int64, vp, C.c_int64, vp, C.c_int64,
                                       C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp, vp]
    lib.dit_attention_bf16_noalloc.argtypes = [vp, C.c_int64, vp, C.c_int64, vp, C.c_int64, vp, C.c_int64,
                                               C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp]
    i32, i64 = C.c_int32, C.c_int64
    lib.dit_quant_fp8.argtypes = [vp, i32, i64, vp, i64, vp, i64, i32, i32, vp]
    lib.dit_gemm_fp8.argtypes = [C.POINTER(GemmFp8DescC), vp]
    shape = C.POINTER(SparseShapeC)
    lib.dit_select_blocks_ws_bytes.argtypes = lib.dit_attention_sparse_ws_bytes.argtypes = [shape]
    lib.dit_select_blocks_bf16.argtypes = [shape, vp, i64, vp, i64, i32, vp, vp, vp]
    lib.dit_attention_sparse_bf16.argtypes = [shape, vp, i64, vp, i64, vp, i64, vp, i64, vp, i32, vp, vp]
    lib.dit_quant_fp4.argtypes = [vp, i32, i64, vp, i64, vp, i64, i32, i32, vp]
    lib.dit_dequant_fp4.argtypes = [vp, i64, vp, i64, vp, i32, i64, i32, i32, vp]
    lib.dit_gemm_fp4.argtypes = [C.POINTER(GemmFp4DescC), vp]
    lib.dit_rotary_freqs.argtypes = [i32, C.c_double, i32, C.c_double, C.c_double, vp, vp]
    lib.dit_rotary.argtypes = [C.POINTER(RotaryDescC), vp]
    packed = C.POINTER(PackedShapeC)
    lib.dit_attention_packed_ws_bytes.argtypes = [packed]
    lib.dit_attention_packed_bf16.argtypes = [packed, vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, vp]
    for n in EXPORTS:
        f = getattr(lib, n)
        if n not in ("dit_cache_destroy", "dit_cache_last_error"):
            f.restype = C.c_size_t if n.endswith("_ws_bytes") else C.c_int
    _lib = lib
    return lib


def _check(status, handle=None):
    if status != DIT_OK:
        msg = _lib.dit_cache_last_error(handle).decode()
        raise DitError(status, msg)


def _stream_ptr(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def model_config_c(cfg) -> ModelConfigC:
    return ModelConfigC(ABI_VERSION, DTYPE_BF16 if cfg.dtype == "bf16" else DTYPE_F32,
                        cfg.n_double, cfg.n_single, cfg.n_cross, cfg.hidden, cfg.heads, cfg.head_dim,
                        cfg.mlp_hidden, cfg.in_channels, cfg.ctx_dim, cfg.time_dim, cfg.n_img,
                        cfg.n_txt, cfg.batch, int(cfg.pooled_text))


@dataclass
class Schedule:
    full: np.ndarray
    logit: np.ndarray
    forced: np.ndarray
    features: np.ndarray
    sums: np.ndarray
    nfe: int
    steps_done: int


class DitCache:
    """Handle of dit_cache_create; ``sample`` wraps dit_cache_sample_ex."""

    def __init__(self, cfg, weights_blob: np.ndarray, stream=None):
        lib = load()
        self.cfg = cfg
        self._stream = stream
        blob = np.ascontiguousarray(weights_blob)
        h = C.c_void_p()
        c = model_config_c(cfg)
        st = lib.dit_cache_create(C.byref(c), blob.ctypes.data_as(C.c_void_p), blob.nbytes,
                                  _stream_ptr(stream), C.byref(h))
        if st != DIT_OK:
            raise DitError(st, lib.dit_cache_last_error(None).decode())
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            _lib.dit_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check_io(self, latents, text_embs, S):
        """The library reads S x [N, C] f32 latents and S x [batch, N_t, ctx]
        text embeddings in the storage dtype through raw device pointers:
        check that the tensors hold exactly that."""
        cfg = self.cfg
        esz = 2 if cfg.dtype == "bf16" else 4
        for t, name, n, size in ((latents, "latent", S * cfg.n_img * cfg.in_channels, 4),
                                 (text_embs, "text_emb", S * cfg.batch * cfg.n_txt * cfg.ctx_dim, esz)):
            if not getattr(t, "is_cuda", False):
                raise ValueError(f"{name} must be a device tensor")
            if not t.is_contiguous() or t.numel() != n or t.element_size() != size:
                raise ValueError(f"{name} must be contiguous with {n} elements of {size} bytes")
        if not latents.is_floating_point():
            raise ValueError("latent must be float32")

    @staticmethod
    def _params(T, B, sigmas, shift, tau, guidance, forced_mask, indicator, policy, delta, solver, S=1):
        sig = None if sigmas is None else np.ascontiguousarray(sigmas, np.float64)
        fm = None if forced_mask is None else np.ascontiguousarray(forced_mask, np.uint8)
        # the library reads T + 1 sigmas and T mask entries per sample
        if sig is not None and sig.size != int(T) + 1:
            raise ValueError(f"sigmas must hold T + 1 = {int(T) + 1} values")
        if fm is not None and fm.size != S * int(T):
            raise ValueError(f"forced mask must hold {S} x T = {S * int(T)} entries")
        p = SampleParamsC(int(T), int(B),
                          sig.ctypes.data_as(C.POINTER(C.c_double)) if sig is not None else None,
                          float(shift), float(tau), float(guidance),
                          fm.ctypes.data_as(C.POINTER(C.c_uint8)) if fm is not None else None,
                          INDICATOR_PATCH if indicator == "patch" else INDICATOR_MODULATED,
                          POLICIES[policy], float(delta), SOLVERS[solver])
        return p, (sig, fm)  # the arrays stay alive with the struct

    @staticmethod
    def _schedules(S, T):
        arrs = [(np.zeros(T, np.uint8), np.zeros(T, np.float32), np.zeros(T, np.uint8),
                 np.zeros(T * N_FEATURES, np.float64), np.zeros(T * 4, np.float64)) for _ in range(S)]
        cs = (ScheduleC * S)()
        for j, (full, logit, forced, feats, sums) in enumerate(arrs):
            cs[j] = ScheduleC(full.ctypes.data_as(C.POINTER(C.c_uint8)),
                              logit.ctypes.data_as(C.POINTER(C.c_float)),
                              forced.ctypes.data_as(C.POINTER(C.c_uint8)),
                              feats.ctypes.data_as(C.POINTER(C.c_double)),
                              sums.ctypes.data_as(C.POINTER(C.c_double)), 0, 0)
        return arrs, cs

    @staticmethod
    def _results(arrs, cs, T):
        return [Schedule(full, logit, forced, feats.reshape(T, N_FEATURES), sums.reshape(T, 4),
                         cs[j].nfe, cs[j].steps_done)
                for j, (full, logit, forced, feats, sums) in enumerate(arrs)]

    def _raise(self, st, res):
        err = DitError(st, _lib.dit_cache_last_error(self._h).decode())
        err.schedule = res
        raise err

    def sample(self, latent, text_emb, gate_blob, T, B, *, sigmas=None, shift=1.0, tau=0.5,
               guidance=1.0, forced_mask=None, indicator="modulated", policy="gate",
               delta=0.0, solver="euler") -> Schedule:
        """latent: torch f32 cuda [N, C] (in place); text_emb: torch cuda
        storage-dtype [batch, N_t, ctx] (bf16 workloads: int16/uint16 bits
        or torch.bfloat16); policy "gate" | "static" | "threshold" (the
        latter two do not read gate_blob, which may be None); solver
        "euler" | "unipc"."""
        self._check_io(latent, text_emb, 1)
        gate = np.ascontiguousarray(gate_blob if gate_blob is not None else [], np.float32)
        arrs, cs = self._schedules(1, T)
        p, keep = self._params(T, B, sigmas, shift, tau, guidance, forced_mask, indicator, policy, delta, solver)
        st = _lib.dit_cache_sample_ex(self._h, C.c_void_p(latent.data_ptr()),
                                      C.c_void_p(text_emb.data_ptr()),
                                      gate.ctypes.data_as(C.c_void_p) if gate.size else None, gate.size,
                                      C.byref(p), cs)
        res = self._results(arrs, cs, T)[0]
        if st != DIT_OK:
            self._raise(st, res)
        return res

    def sample_batch(self, latents, text_embs, gate_blob, T, B, *, sigmas=None, shift=1.0, tau=0.5,
                     guidance=1.0, forced_masks=None, indicator="modulated", policy="gate",
                     delta=0.0, solver="euler") -> list:
        """dit_cache_sample_batch: latents torch f32 cuda [S, N, C] (in
        place), text_embs [S, batch, N_t, ctx] in the storage dtype,
        forced_masks None or [S, T]; one Schedule per sample."""
        S = int(latents.shape[0])
        if S != int(text_embs.shape[0]):
            raise ValueError("latents and text_embs disagree on the number of samples")
        if forced_masks is not None and np.shape(forced_masks) != (S, T):
            raise ValueError("forced_masks must be [n_samples, T]")
        self._check_io(latents, text_embs, S)
        gate = np.ascontiguousarray(gate_blob if gate_blob is not None else [], np.float32)
        arrs, cs = self._schedules(S, T)
        p, keep = self._params(T, B, sigmas, shift, tau, guidance, forced_masks, indicator, policy, delta,
                               solver, S)
        st = _lib.dit_cache_sample_batch(self._h, S, C.c_void_p(latents.data_ptr()),
                                         C.c_void_p(text_embs.data_ptr()),
                                         gate.ctypes.data_as(C.c_void_p) if gate.size else None, gate.size,
                                         C.byref(p), cs)
        res = self._results(arrs, cs, T)
        if st != DIT_OK:
            self._raise(st, res)
        return res

    def set_profiling(self, on: bool):
        _check(_lib.dit_cache_set_profiling(self._h, int(on)), self._h)

    def reset_stats(self):
        _check(_lib.dit_cache_reset_stats(self._h), self._h)

    def stats(self) -> dict:
        s = StatsC()
        _check(_lib.dit_cache_get_stats(self._h, C.byref(s)), self._h)
        return {"ms": {k: s.ms[i] for i, k in enumerate(K_CLASSES)},
                "work": {k: s.work[i] for i, k in enumerate(K_CLASSES)},
                "launches": {k: s.launches[i] for i, k in enumerate(K_CLASSES)},
                "host_gate_ms": s.host_gate_ms, "sample_ms": s.sample_ms, "samples": s.samples,
                "full_steps": s.full_steps, "reuse_steps": s.reuse_steps}


def gemm_bf16(A, W, bias, Cout, *, M, N, K, lda=None, ldw=None, ldc=None, flags=EPI_STORE,
              gate=None, rms_cols=0, gelu_from=None, gap_at=0, gap=0, stream=None):
    """dit_gemm_bf16 on torch cuda tensors (bf16 data as torch.bfloat16 or int16)."""
    lib = load()
    d = GemmDescC(A.data_ptr(), lda if lda is not None else K, W.data_ptr(),
                  ldw if ldw is not None else K, bias.data_ptr() if bias is not None else None,
                  Cout.data_ptr(), ldc if ldc is not None else N, M, N, K, flags,
                  gate.data_ptr() if gate is not None else None, rms_cols,
                  gelu_from if gelu_from is not None else 0x7FFFFFFF, gap_at, gap)
    st = lib.dit_gemm_bf16(C.byref(d), _stream_ptr(stream))
    _check(st, None)


ATTN_BOUNDED_LOGITS = 1


def attention_bf16(q, k, v, o, *, Lq, Lk, heads, ldq, ldk, ldv, ldo, vt_ws, flags=0, stream=None):
    lib = load()
    st = lib.dit_attention_bf16(q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                                o.data_ptr(), ldo, Lq, Lk, heads, flags, vt_ws.data_ptr(), _stream_ptr(stream))
    _check(st, None)


NOALLOC_VT_MAX_ELEMS = 16 * 1024 * 1024


def attention_bf16_noalloc(q, k, v, o, *, Lq, Lk, heads, ldq, ldk, ldv, ldo, flags=0, stream=None):
    """dit_attention_bf16_noalloc: the library's own device array holds the
    transposed values (no workspace argument, nothing allocated)."""
    lib = load()
    st = lib.dit_attention_bf16_noalloc(q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                                        o.data_ptr(), ldo, Lq, Lk, heads, flags, _stream_ptr(stream))
    _check(st, None)


# ---- 8-bit products and sparse attention: these calls only enqueue their work

SPARSE_QB, SPARSE_KB = 128, 64


def fp8_scale_ld(K: int) -> int:
    """DIT_FP8_SCALE_LD: least row stride of the scale bytes of rows of K values."""
    return (K + 511) // 512 * 4


# what the library may read or write a type's elements as: 8-bit values and scales also as plain bytes, bf16 also as
# its bits
_E4M3, _E8M0, _BF16, _F32, _I32 = "e4m3 bytes", "E8M0 bytes", "bf16", "float32", "int32"
_MEANINGS = {"torch.uint8": (_E4M3, _E8M0), "torch.int8": (_E4M3, _E8M0), "torch.float8_e4m3fn": (_E4M3,),
             "torch.float8_e8m0fnu": (_E8M0,), "torch.bfloat16": (_BF16,), "torch.int16": (_BF16,),
             "torch.uint16": (_BF16,), "torch.float32": (_F32,), "torch.int32": (_I32,)}
_TYPES = {}  # by torch type: bytes of an element, meanings


def _type(t):
    known = _TYPES[t.dtype] = (t.element_size(), _MEANINGS.get(str(t.dtype), ()))
    return known


def _rows(t, name, rows, width, ld, esize, meaning=None):
    """Row stride of a device tensor that holds `rows` rows of `width` elements (None: a matrix's own; tensors of
    other dimensions hold them back to back): the library reads them through a raw pointer, and no further than the
    tensor's own last element."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    size, meanings = _TYPES.get(t.dtype) or _type(t)
    if size != esize or not (meaning or meanings):
        raise ValueError(f"{name} must have elements of {esize} bytes and not be {t.dtype}")
    if meaning and meaning not in meanings:
        raise ValueError(f"{name} must be {meaning} and not {t.dtype}")
    shape, strides, held = t.shape, t.stride(), 0
    if ld is None and len(shape) == 2:
        (have, wide), (ld, unit) = shape, strides
        if have <= 1:
            ld = max(ld, width)
        if unit == 1 and have >= rows and wide >= width:
            return ld
    else:
        if ld is None:
            if not t.is_contiguous():
                raise ValueError(f"{name} must be a matrix, or contiguous, or come with its row stride")
            ld = width
        if 0 not in shape:
            held = 1 + sum((n - 1) * step for n, step in zip(shape, strides))
    if len(shape) and shape[-1] > 1 and strides[-1] != 1:
        raise ValueError(f"{name} must have contiguous rows")
    if rows > 0 and (rows - 1) * ld + width > held:
        raise ValueError(f"{name} must hold {rows} rows of {width} elements with stride {ld}")
    return ld


class _Call:
    """Device and stream of one call: the tensors' device becomes the current one, the stream (default: that
    device's current one) must be its own."""

    __slots__ = ("stream", "ptr", "_dev", "_guard", "_torch")

    def __init__(self, stream, first, *more):
        import torch
        dev = first.device
        for t in more:
            if t is not None and t.device != dev:
                raise ValueError("all tensors of a call must be on one device")
        if stream is not None and stream.device != dev:
            raise ValueError("the stream belongs to another device than the tensors")
        self._torch, self._dev, self.stream = torch, dev, stream
        index = dev.index  # (of a tensor's device: the context is there, and its number needs no asking for it)
        self._guard = None if torch._C._cuda_getDevice() == index else torch.cuda.device(dev)
        self.ptr = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream

    def __enter__(self):
        if self._guard is not None:
            self._guard.__enter__()
        return self

    def __exit__(self, *exc):
        if self._guard is not None:
            self._guard.__exit__(*exc)

    def workspace(self, ws, nbytes, name):
        """The caller's workspace, or one of the caching allocator's, taken on the call's own stream."""
        if nbytes == 0:
            return None
        if ws is None:
            torch = self._torch
            if self.stream is None:
                return torch.empty(nbytes, dtype=torch.uint8, device=self._dev)
            with torch.cuda.stream(self.stream):
                return torch.empty(nbytes, dtype=torch.uint8, device=self._dev)
        if not ws.is_cuda or ws.device != self._dev or not ws.is_contiguous() or ws.numel() * ws.element_size() < nbytes:
            raise ValueError(f"{name} must be a contiguous tensor of {nbytes} bytes on the call's device")
        return ws


def quant_fp8(x, q, scale, *, M, K, ldx=None, ldq=None, lds=None, stream=None):
    """dit_quant_fp8: rows of x (torch.float32, else bf16 as torch.bfloat16 or int16) to e4m3 bytes q and
    E8M0 scale bytes (uint8 or torch's type of the format)."""
    lib = load()
    f32 = x.element_size() == 4
    if f32 and not x.is_floating_point():
        raise ValueError("x must be float32 or bf16")
    ldx = _rows(x, "x", M, K, ldx, 4, _F32) if f32 else _rows(x, "x", M, K, ldx, 2, _BF16)
    ldq = _rows(q, "q", M, K, ldq, 1, _E4M3)
    lds = _rows(scale, "scale", M, fp8_scale_ld(K), lds, 1, _E8M0)
    with _Call(stream, x, q, scale) as call:
        _check(lib.dit_quant_fp8(x.data_ptr(), DTYPE_F32 if f32 else DTYPE_BF16, ldx, q.data_ptr(), ldq,
                                 scale.data_ptr(), lds, M, K, call.ptr))


def gemm_fp8(A, a_scale, W, w_scale, bias, Cout, *, M, N, K, lda=None, ld_as=None, ldw=None, ld_ws=None, ldc=None,
             c_scale=None, ld_cs=None, flags=EPI_STORE, gate=None, rms_cols=0, gelu_from=None, gap_at=0, gap=0,
             stream=None):
    """dit_gemm_fp8 on torch cuda tensors: 8-bit rows as uint8 or torch's types of the formats, bias and Cout as in
    gemm_bf16 (Cout e4m3 with EPI_FP8, c_scale its scale bytes)."""
    lib = load()
    lda, ldw = _rows(A, "A", M, K, lda, 1, _E4M3), _rows(W, "W", N, K, ldw, 1, _E4M3)
    ld_as = _rows(a_scale, "a_scale", M, fp8_scale_ld(K), ld_as, 1, _E8M0)
    ld_ws = _rows(w_scale, "w_scale", N, fp8_scale_ld(K), ld_ws, 1, _E8M0)
    width = N + (gap if gap and gap_at < N else 0)
    ldc = _rows(Cout, "Cout", M, width, ldc, *((4, _F32) if flags & EPI_F32 else (1, _E4M3) if flags & EPI_FP8
                                               else (2, _BF16)))
    if bias is not None:
        _rows(bias, "bias", 1, N, None, 2, _BF16)
    if gate is not None:
        _rows(gate, "gate", 1, N, None, 4, _F32)
    if flags & EPI_FP8 and c_scale is not None:
        ld_cs = _rows(c_scale, "c_scale", M, fp8_scale_ld(N), ld_cs, 1, _E8M0)
    d = GemmFp8DescC(A.data_ptr(), lda, a_scale.data_ptr(), ld_as, W.data_ptr(), ldw, w_scale.data_ptr(), ld_ws,
                     bias.data_ptr() if bias is not None else None, Cout.data_ptr(), ldc,
                     c_scale.data_ptr() if c_scale is not None else None, ld_cs if ld_cs is not None else 0,
                     gate.data_ptr() if gate is not None else None, M, N, K, flags, rms_cols,
                     gelu_from if gelu_from is not None else 0x7FFFFFFF, gap_at, gap)
    with _Call(stream, A, a_scale, W, w_scale, bias, Cout, c_scale, gate) as call:
        _check(lib.dit_gemm_fp8(C.byref(d), call.ptr))


def sparse_shape(*, Lq, Lk, heads, topk, kv_heads=None, batch=1, klen=None) -> SparseShapeC:
    """dit_sparse_shape; klen: int32 cuda tensor [batch] or None."""
    if klen is not None:
        _rows(klen, "klen", 1, batch, None, 4, _I32)
    return SparseShapeC(batch, Lq, Lk, heads, kv_heads if kv_heads is not None else heads, topk,
                        klen.data_ptr() if klen is not None else None)


@functools.lru_cache(256)
def _ws_bytes(name, *sizes):
    """A workspace's size depends on the shape's numbers alone."""
    return getattr(load(), name)(C.byref(SparseShapeC(*sizes, None)))


def _ws_of(name, s):
    return _ws_bytes(name, s.batch, s.Lq, s.Lk, s.heads, s.kv_heads, s.topk)


def select_blocks_ws_bytes(**shape) -> int:
    return _ws_of("dit_select_blocks_ws_bytes", sparse_shape(**shape))


def attention_sparse_ws_bytes(**shape) -> int:
    return _ws_of("dit_attention_sparse_ws_bytes", sparse_shape(**shape))


def _lists(idx, s):
    if not idx.is_cuda:
        raise ValueError("idx must be a device tensor")
    if _I32 not in (_TYPES.get(idx.dtype) or _type(idx))[1]:
        raise ValueError("idx must be int32")
    if not idx.is_contiguous() or idx.numel() < s.batch * s.heads * -(-s.Lq // SPARSE_QB) * s.topk:
        raise ValueError("idx must be contiguous and hold every list")


def select_blocks_bf16(q, k, idx, *, first=0, ldq=None, ldk=None, ws=None, stream=None, **shape):
    """dit_select_blocks_bf16: idx int32 [batch, heads, ceil(Lq / 128), topk]; shape as in sparse_shape; ws None:
    a workspace of torch's caching allocator."""
    lib = load()
    s = sparse_shape(**shape)
    ldq = _rows(q, "q", s.batch * s.Lq, s.heads * 128, ldq, 2, _BF16)
    ldk = _rows(k, "k", s.batch * s.Lk, s.kv_heads * 128, ldk, 2, _BF16)
    _lists(idx, s)
    with _Call(stream, q, k, idx, shape.get("klen")) as call:
        w = call.workspace(ws, _ws_of("dit_select_blocks_ws_bytes", s) or 16, "ws")
        _check(lib.dit_select_blocks_bf16(C.byref(s), q.data_ptr(), ldq, k.data_ptr(), ldk, first, idx.data_ptr(),
                                          w.data_ptr(), call.ptr))


def attention_sparse_bf16(q, k, v, o, idx, *, flags=0, ldq=None, ldk=None, ldv=None, ldo=None, ws=None, stream=None,
                          **shape):
    """dit_attention_sparse_bf16; idx as select_blocks_bf16 writes it, shape as in sparse_shape."""
    lib = load()
    s = sparse_shape(**shape)
    ldq = _rows(q, "q", s.batch * s.Lq, s.heads * 128, ldq, 2, _BF16)
    ldk = _rows(k, "k", s.batch * s.Lk, s.kv_heads * 128, ldk, 2, _BF16)
    ldv = _rows(v, "v", s.batch * s.Lk, s.kv_heads * 128, ldv, 2, _BF16)
    ldo = _rows(o, "o", s.batch * s.Lq, s.heads * 128, ldo, 2, _BF16)
    _lists(idx, s)
    with _Call(stream, q, k, v, o, idx, shape.get("klen")) as call:
        w = call.workspace(ws, _ws_of("dit_attention_sparse_ws_bytes", s), "ws")
        _check(lib.dit_attention_sparse_bf16(C.byref(s), q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                                             o.data_ptr(), ldo, idx.data_ptr(), flags,
                                             w.data_ptr() if w is not None else None, call.ptr))


# ---- a prompt encoder's operators: 4-bit rows and products, rotary positions, packed attention; these calls only
# enqueue their work, too

ATTN_CAUSAL = 2
ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS = 0, 1, 2, 3
ROTARY_AXES = 4
_E2M1, _F64 = "pairs of e2m1", "float64"
_FOUR = C.c_int32 * 4
_MEANINGS["torch.float64"] = (_F64,)
_MEANINGS["torch.float4_e2m1fn_x2"] = (_E2M1,)
for _t in ("torch.uint8", "torch.int8"):
    _MEANINGS[_t] += (_E2M1,)


def fp4_scale_ld(K: int) -> int:
    """DIT_FP4_SCALE_LD: least row stride of the scale bytes of 4-bit rows of K values."""
    return (K + 127) // 128 * 4


def _values(x, name, M, K, ld):
    """Row stride and type of a matrix that is float32, or bf16 as torch.bfloat16 or int16."""
    size, meanings = _TYPES.get(x.dtype) or _type(x)
    if size != 4:
        return _rows(x, name, M, K, ld, 2, _BF16), DTYPE_BF16
    if _F32 not in meanings:
        raise ValueError(f"{name} must be float32 or bf16")
    return _rows(x, name, M, K, ld, 4, _F32), DTYPE_F32


def quant_fp4(x, q, scale, *, M, K, ldx=None, ldq=None, lds=None, stream=None):
    """dit_quant_fp4: rows of x (torch.float32, else bf16 as torch.bfloat16 or int16) to pairs of e2m1 q [M, K / 2]
    (uint8 or torch's type of the format) and E8M0 scale bytes (uint8 or torch's type of the format)."""
    lib = load()
    ldx, dtype = _values(x, "x", M, K, ldx)
    ldq = _rows(q, "q", M, K // 2, ldq, 1, _E2M1)
    lds = _rows(scale, "scale", M, fp4_scale_ld(K), lds, 1, _E8M0)
    with _Call(stream, x, q, scale) as call:
        _check(lib.dit_quant_fp4(x.data_ptr(), dtype, ldx, q.data_ptr(), ldq, scale.data_ptr(), lds, M, K, call.ptr))


def dequant_fp4(q, scale, y, *, M, K, ldq=None, lds=None, ldy=None, stream=None):
    """dit_dequant_fp4: the values of 4-bit rows (as quant_fp4 writes them) as float32 or bf16."""
    lib = load()
    ldy, dtype = _values(y, "y", M, K, ldy)
    ldq = _rows(q, "q", M, K // 2, ldq, 1, _E2M1)
    lds = _rows(scale, "scale", M, fp4_scale_ld(K), lds, 1, _E8M0)
    with _Call(stream, q, scale, y) as call:
        _check(lib.dit_dequant_fp4(q.data_ptr(), ldq, scale.data_ptr(), lds, y.data_ptr(), dtype, ldy, M, K, call.ptr))


def gemm_fp4(A, a_scale, W, w_scale, bias, Cout, *, M, N, K, lda=None, ld_as=None, ldw=None, ld_ws=None, ldc=None,
             c_scale=None, ld_cs=None, flags=EPI_STORE, gate=None, rms_cols=0, gelu_from=None, gap_at=0, gap=0,
             stream=None):
    """dit_gemm_fp4 on torch cuda tensors: 4-bit rows as quant_fp4 writes them, bias and Cout as in gemm_bf16 (Cout
    pairs of e2m1 [M, N / 2] with EPI_FP4, c_scale its scale bytes)."""
    lib = load()
    lda, ldw = _rows(A, "A", M, K // 2, lda, 1, _E2M1), _rows(W, "W", N, K // 2, ldw, 1, _E2M1)
    ld_as = _rows(a_scale, "a_scale", M, fp4_scale_ld(K), ld_as, 1, _E8M0)
    ld_ws = _rows(w_scale, "w_scale", N, fp4_scale_ld(K), ld_ws, 1, _E8M0)
    if flags & EPI_FP4:
        ldc = _rows(Cout, "Cout", M, N // 2, ldc, 1, _E2M1)
        if c_scale is not None:
            ld_cs = _rows(c_scale, "c_scale", M, fp4_scale_ld(N), ld_cs, 1, _E8M0)
    else:
        width = N + (gap if gap and gap_at < N else 0)
        ldc = _rows(Cout, "Cout", M, width, ldc, *((4, _F32) if flags & EPI_F32 else (2, _BF16)))
    if bias is not None:
        _rows(bias, "bias", 1, N, None, 2, _BF16)
    if gate is not None:
        _rows(gate, "gate", 1, N, None, 4, _F32)
    d = GemmFp4DescC(A.data_ptr(), lda, a_scale.data_ptr(), ld_as, W.data_ptr(), ldw, w_scale.data_ptr(), ld_ws,
                     bias.data_ptr() if bias is not None else None, Cout.data_ptr(), ldc,
                     c_scale.data_ptr() if c_scale is not None else None, ld_cs if ld_cs is not None else 0,
                     gate.data_ptr() if gate is not None else None, M, N, K, flags, rms_cols,
                     gelu_from if gelu_from is not None else 0x7FFFFFFF, gap_at, gap)
    with _Call(stream, A, a_scale, W, w_scale, bias, Cout, c_scale, gate) as call:
        _check(lib.dit_gemm_fp4(C.byref(d), call.ptr))


def rotary_freqs(pairs, *, base=10000.0, method=ROTARY_PLAIN, factor=1.0, context=0.0):
    """dit_rotary_freqs: (float64 array of radians per position, factor on cosine and sine); rotary takes the array
    as a device tensor."""
    lib = load()
    freq, scale = np.empty(max(pairs, 0)), C.c_double()
    _check(lib.dit_rotary_freqs(pairs, base, method, factor, context, freq.ctypes.data_as(C.c_void_p), C.byref(scale)))
    return freq, scale.value


def rotary(x, y, *, pos, freq, rows, heads, head_dim=128, pairs=None, layout=ROTARY_HALF, scale=1.0, ldx=None, ldy=None,
           ldpos=None, stream=None):
    """dit_rotary: rows of x to y (x itself: in place), both float32, or bf16 as torch.bfloat16 or int16.  pos: int32
    [rows] or [axes, rows]; freq: float64 cuda tensor, one per pair; pairs: those of each axis (None: one axis)."""
    lib = load()
    n = freq.numel()
    pairs = (n,) if pairs is None else tuple(pairs)
    axes = len(pairs)
    if not 1 <= axes <= ROTARY_AXES or sum(pairs) != n:
        raise ValueError(f"pairs must be those of 1 to {ROTARY_AXES} axes, {n} together")
    ldx, dtype = _values(x, "x", rows, heads * head_dim, ldx)
    ldy, out = _values(y, "y", rows, heads * head_dim, ldy)
    if dtype != out:
        raise ValueError("x and y must be of one type")
    _rows(freq, "freq", 1, n, None, 8, _F64)
    ldpos = _rows(pos, "pos", axes, rows, ldpos, 4, _I32) if axes > 1 or pos.dim() == 2 \
        else _rows(pos, "pos", 1, rows, rows, 4, _I32)
    d = RotaryDescC(x.data_ptr(), ldx, y.data_ptr(), ldy, pos.data_ptr(), ldpos, freq.data_ptr(), dtype, rows, heads,
                    head_dim, 2 * n, layout, axes, _FOUR(*pairs), scale)
    with _Call(stream, x, y, pos, freq) as call:
        _check(lib.dit_rotary(C.byref(d), call.ptr))


def packed_shape(*, qoff, koff, Tq, Tk, heads, kv_heads=None, klen=None) -> PackedShapeC:
    """dit_packed_shape; qoff, koff: int32 cuda tensors [batch + 1], klen: [batch] or None."""
    batch = qoff.numel() - 1
    if batch < 0 or koff.numel() != batch + 1 or (klen is not None and klen.numel() != batch):
        raise ValueError("qoff and koff must hold batch + 1 offsets, klen batch lengths")
    for t, name, n in ((qoff, "qoff", batch + 1), (koff, "koff", batch + 1), (klen, "klen", batch)):
        if t is not None:
            _rows(t, name, 1, n, None, 4, _I32)
    return PackedShapeC(batch, Tq, Tk, heads, kv_heads if kv_heads is not None else heads, qoff.data_ptr(),
                        koff.data_ptr(), klen.data_ptr() if klen is not None else None)


@functools.lru_cache(256)
def _packed_ws_bytes(*sizes):
    """A workspace's size depends on the shape's numbers alone."""
    return load().dit_attention_packed_ws_bytes(C.byref(PackedShapeC(*sizes, None, None, None)))


def attention_packed_ws_bytes(*, batch, Tq, Tk, heads, kv_heads=None) -> int:
    return _packed_ws_bytes(batch, Tq, Tk, heads, kv_heads if kv_heads is not None else heads)


def attention_packed_bf16(q, k, v, o, *, qoff, koff, heads, kv_heads=None, klen=None, Tq=None, Tk=None, flags=0, ldq=None,
                          ldk=None, ldv=None, ldo=None, ws=None, stream=None):
    """dit_attention_packed_bf16; shape as in packed_shape (Tq, Tk None: the rows of q and of k); ws None: a
    workspace of torch's caching allocator."""
    lib = load()
    s = packed_shape(qoff=qoff, koff=koff, Tq=q.shape[0] if Tq is None else Tq, Tk=k.shape[0] if Tk is None else Tk,
                     heads=heads, kv_heads=kv_heads, klen=klen)
    ldq = _rows(q, "q", s.Tq, s.heads * 128, ldq, 2, _BF16)
    ldk = _rows(k, "k", s.Tk, s.kv_heads * 128, ldk, 2, _BF16)
    ldv = _rows(v, "v", s.Tk, s.kv_heads * 128, ldv, 2, _BF16)
    ldo = _rows(o, "o", s.Tq, s.heads * 128, ldo, 2, _BF16)
    with _Call(stream, q, k, v, o, qoff, koff, klen) as call:
        w = call.workspace(ws, _packed_ws_bytes(s.batch, s.Tq, s.Tk, s.heads, s.kv_heads), "ws")
        _check(lib.dit_attention_packed_bf16(C.byref(s), q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                                             o.data_ptr(), ldo, flags, w.data_ptr() if w is not None else None, call.ptr))


def gate_logit(gate_blob, features) -> float:
    """dit_gate_logit: the library's host gate on one 8-feature state."""
    lib = load()
    gate = np.ascontiguousarray(gate_blob, np.float32)
    f = np.ascontiguousarray(np.asarray(features, np.float64).reshape(-1)[:N_FEATURES])
    if f.size < N_FEATURES:
        f = np.concatenate([f, np.zeros(N_FEATURES - f.size)])
    out = C.c_double()
    st = lib.dit_gate_logit(gate.ctypes.data_as(C.c_void_p) if gate.size else None, gate.size,
                            f.ctypes.data_as(C.c_void_p), C.byref(out))
    _check(st, None)
    return out.value
