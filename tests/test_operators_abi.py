"""Refusals and sizes of the 8-bit and sparse entry points: no GPU needed,
nothing is launched."""
import ctypes as C

import numpy as np
import pytest

from paper_2608_09231_amd import binding
from tests import _operators as ref

FAKE = 0x1000


def gemm_desc(**kw):
    d = dict(A=FAKE, lda=256, a_scale=FAKE, ld_as=4, W=FAKE, ldw=256, w_scale=FAKE, ld_ws=4, bias=None, C=FAKE,
             ldc=512, c_scale=None, ld_cs=0, gate=None, M=64, N=512, K=256, flags=0, rms_cols=0, gelu_from=512,
             gap_at=0, gap=0)
    d.update(kw)
    return binding.GemmFp8DescC(**d)


@pytest.mark.parametrize("kw", [
    {"K": 0}, {"K": 250}, {"K": -16}, {"M": -1}, {"N": -8}, {"N": 500}, {"lda": 128}, {"ldw": 240}, {"lda": 264},
    {"ldw": 1 << 23}, {"ld_as": 0}, {"ld_ws": 6}, {"K": 528, "lda": 528, "ldw": 528}, {"ldc": 504}, {"ldc": 516},
    {"gap": -4}, {"gap": 6, "gap_at": 8, "ldc": 600}, {"gap": 8, "gap_at": 6, "ldc": 600}, {"gap": 128, "gap_at": 256},
    {"gap": 8, "gap_at": -4, "ldc": 600}, {"gelu_from": 6}, {"gelu_from": -4}, {"rms_cols": 100}, {"rms_cols": 640},
    {"rms_cols": -128}, {"rms_cols": 128, "N": 200},
    {"flags": 8, "c_scale": FAKE, "ld_cs": 4, "N": 200}, {"flags": 8, "c_scale": FAKE, "ld_cs": 0},
    {"flags": 8, "c_scale": FAKE, "ld_cs": 4, "gelu_from": 64}, {"flags": 8, "c_scale": FAKE, "ld_cs": 4, "ldc": 520},
    {"flags": 8, "c_scale": FAKE, "ld_cs": 4, "gap": 128, "gap_at": 128, "ldc": 640}])
def test_gemm_fp8_refuses_shapes(kw):
    lib = binding.load()
    d = gemm_desc(**kw)
    assert lib.dit_gemm_fp8(C.byref(d), None) == binding.DIT_ESHAPE, kw
    assert lib.dit_cache_last_error(None)


@pytest.mark.parametrize("kw", [
    {"A": None}, {"W": None}, {"a_scale": None}, {"w_scale": None}, {"C": None}, {"flags": 16}, {"flags": 2},
    {"flags": 8}, {"flags": 3, "gate": FAKE}, {"flags": 9, "c_scale": FAKE}, {"A": FAKE + 8}, {"C": FAKE + 8},
    {"a_scale": FAKE + 2}, {"bias": FAKE + 1}, {"flags": 2, "gate": FAKE + 4},
    {"flags": 8, "c_scale": FAKE + 1, "ld_cs": 4}])
def test_gemm_fp8_refuses_pointers_and_flags(kw):
    lib = binding.load()
    d = gemm_desc(**kw)
    assert lib.dit_gemm_fp8(C.byref(d), None) == binding.DIT_EINVAL, kw
    assert lib.dit_gemm_fp8(None, None) == binding.DIT_EINVAL


def test_quant_fp8_refuses():
    lib = binding.load()
    good = dict(x=FAKE, t=1, ldx=256, q=FAKE, ldq=256, s=FAKE, lds=4, M=4, K=256)
    for st, kw in ((binding.DIT_EINVAL, {"x": None}), (binding.DIT_EINVAL, {"q": None}), (binding.DIT_EINVAL, {"s": None}),
                   (binding.DIT_EINVAL, {"t": 2}), (binding.DIT_EINVAL, {"x": FAKE + 8}),
                   (binding.DIT_EINVAL, {"q": FAKE + 4}), (binding.DIT_EINVAL, {"s": FAKE + 1}),
                   (binding.DIT_ESHAPE, {"K": 24}), (binding.DIT_ESHAPE, {"K": -16}), (binding.DIT_ESHAPE, {"M": -1}),
                   (binding.DIT_ESHAPE, {"ldx": 255}), (binding.DIT_ESHAPE, {"ldx": 260}), (binding.DIT_ESHAPE, {"ldq": 264}),
                   (binding.DIT_ESHAPE, {"ldq": 240}), (binding.DIT_ESHAPE, {"lds": 5}), (binding.DIT_ESHAPE, {"lds": 0}),
                   (binding.DIT_ESHAPE, {"K": 528, "ldx": 528, "ldq": 528})):
        a = dict(good, **kw)
        assert lib.dit_quant_fp8(a["x"], a["t"], a["ldx"], a["q"], a["ldq"], a["s"], a["lds"], a["M"], a["K"],
                                 None) == st, kw


SHAPE = dict(Lq=300, Lk=1000, heads=4, kv_heads=2, topk=5, batch=2)


@pytest.mark.parametrize("st,shape,kw", [
    (binding.DIT_ESHAPE, {"batch": -1}, {}), (binding.DIT_ESHAPE, {"Lq": -1}, {}), (binding.DIT_ESHAPE, {"Lk": -1}, {}),
    (binding.DIT_ESHAPE, {"heads": 0}, {}), (binding.DIT_ESHAPE, {"kv_heads": 3}, {}),
    (binding.DIT_ESHAPE, {"kv_heads": 0}, {}), (binding.DIT_ESHAPE, {"topk": 0}, {}),
    (binding.DIT_ESHAPE, {"topk": 2 ** 30 + 1}, {}),
    (binding.DIT_ESHAPE, {"batch": 2 ** 30, "heads": 2 ** 20}, {}),
    (binding.DIT_EINVAL, {}, {"q": None}), (binding.DIT_EINVAL, {}, {"k": None}), (binding.DIT_EINVAL, {}, {"idx": None}),
    (binding.DIT_EINVAL, {}, {"q": FAKE + 8}), (binding.DIT_EINVAL, {}, {"idx": FAKE + 2}),
    (binding.DIT_ESHAPE, {}, {"ldq": 504}), (binding.DIT_ESHAPE, {}, {"ldq": 516}), (binding.DIT_ESHAPE, {}, {"ldk": 128})])
def test_sparse_calls_refuse(st, shape, kw):
    lib = binding.load()
    s = binding.sparse_shape(**dict(SHAPE, **shape))
    a = dict(q=FAKE, ldq=512, k=FAKE, ldk=256, idx=FAKE)
    a.update(kw)
    assert lib.dit_select_blocks_bf16(C.byref(s), a["q"], a["ldq"], a["k"], a["ldk"], 0, a["idx"], FAKE, None) == st
    assert lib.dit_attention_sparse_bf16(C.byref(s), a["q"], a["ldq"], a["k"], a["ldk"], FAKE, 256, FAKE, 512, a["idx"], 0,
                                         FAKE, None) == st
    if shape:
        assert lib.dit_select_blocks_ws_bytes(C.byref(s)) == 0 and lib.dit_attention_sparse_ws_bytes(C.byref(s)) == 0


def test_sparse_calls_refuse_their_own():
    lib = binding.load()
    s = binding.sparse_shape(**SHAPE)

    def select(s=s, first=0, ws=FAKE):
        return lib.dit_select_blocks_bf16(C.byref(s), FAKE, 512, FAKE, 256, first, FAKE, ws, None)

    def attend(s=s, v=FAKE, ldv=256, o=FAKE, ldo=512, flags=0, ws=FAKE, ldk=256):
        return lib.dit_attention_sparse_bf16(C.byref(s), FAKE, 512, FAKE, ldk, v, ldv, o, ldo, FAKE, flags, ws, None)

    assert select(first=-1) == select(first=6) == select(ws=None) == select(ws=FAKE + 8) == binding.DIT_EINVAL
    big = binding.sparse_shape(**dict(SHAPE, Lk=16384 * 64 + 1))
    assert select(s=big) == binding.DIT_ESHAPE
    many = binding.sparse_shape(**dict(SHAPE, batch=20000))
    assert select(s=many) == binding.DIT_ESHAPE
    assert attend(v=None) == attend(o=None) == attend(flags=2) == binding.DIT_EINVAL
    split = binding.sparse_shape(**dict(SHAPE, topk=64))      # few lists that are shared
    assert lib.dit_attention_sparse_ws_bytes(C.byref(split)) > 0
    assert attend(s=split, ws=None) == attend(s=split, ws=FAKE + 4) == binding.DIT_EINVAL
    assert attend(ldv=128) == attend(ldo=256) == attend(ldk=1 << 22) == binding.DIT_ESHAPE
    assert lib.dit_select_blocks_bf16(None, FAKE, 512, FAKE, 256, 0, FAKE, FAKE, None) == binding.DIT_EINVAL
    assert lib.dit_attention_sparse_bf16(None, FAKE, 512, FAKE, 256, FAKE, 256, FAKE, 512, FAKE, 0, FAKE,
                                         None) == binding.DIT_EINVAL
    assert lib.dit_attention_sparse_ws_bytes(None) == 0


def test_launches_past_their_limits_are_refused():
    """Sizes whose grids would pass 2^32 threads, or whose indexes 32 bits; no rows or columns still do nothing."""
    lib = binding.load()
    top = 2 ** 31 - 1
    for kw in ({"M": top}, {"M": top, "N": 8}, {"M": 64, "N": top - 7, "ldc": 1 << 40},
               {"M": 1 << 20, "N": 1 << 17, "ldc": 1 << 20}):
        d = gemm_desc(**kw)
        assert lib.dit_gemm_fp8(C.byref(d), None) == binding.DIT_ESHAPE, kw
    d = gemm_desc(M=top, N=0)
    assert lib.dit_gemm_fp8(C.byref(d), None) == binding.DIT_OK
    for M, K in ((1 << 26, 16), (1, top - 15), (1 << 16, 1 << 21), (top, 1 << 30)):
        assert lib.dit_quant_fp8(FAKE, 1, 1 << 40, FAKE, 1 << 40, FAKE, 1 << 40, M, K, None) == binding.DIT_ESHAPE, (M, K)
    assert lib.dit_quant_fp8(FAKE, 1, 1 << 40, FAKE, 1 << 40, FAKE, 1 << 40, top, 0, None) == binding.DIT_OK
    for shape in (dict(Lq=top, heads=1, batch=1), dict(Lq=top, heads=1 << 20, batch=2047), dict(Lq=1, heads=2, batch=1 << 22),
                  dict(Lq=1, heads=(1 << 20) + 1, batch=1)):
        s = binding.sparse_shape(**dict(dict(Lk=64, topk=1, kv_heads=1), **shape))
        ld = 128 * shape["heads"]
        assert lib.dit_select_blocks_bf16(C.byref(s), FAKE, ld, FAKE, 128, 0, FAKE, FAKE, None) == binding.DIT_ESHAPE
        assert lib.dit_attention_sparse_bf16(C.byref(s), FAKE, ld, FAKE, 128, FAKE, 128, FAKE, ld, FAKE, 0, FAKE,
                                             None) == binding.DIT_ESHAPE
    s = binding.sparse_shape(Lq=1, Lk=16384 * 64, heads=8, kv_heads=8, batch=128, topk=1)
    assert lib.dit_select_blocks_bf16(C.byref(s), FAKE, 1024, FAKE, 1024, 0, FAKE, FAKE, None) == binding.DIT_ESHAPE


def test_output_columns_past_their_limit_are_refused():
    """A column index is 32 bits wide, its gap included."""
    lib = binding.load()
    for N, gap_at, gap in ((512, 0, 2 ** 31 - 8), (512, 508, 2 ** 30 - 508), (2 ** 20, 2 ** 19, 2 ** 30)):
        d = gemm_desc(M=1, N=N, ldc=1 << 40, gap_at=gap_at, gap=gap, gelu_from=N)
        assert lib.dit_gemm_fp8(C.byref(d), None) == binding.DIT_ESHAPE, (N, gap)
        b = binding.GemmDescC(A=FAKE, lda=256, W=FAKE, ldw=256, bias=None, C=FAKE, ldc=1 << 40, M=1, N=N, K=256, flags=0,
                              gate=None, rms_cols=0, gelu_from=N, gap_at=gap_at, gap=gap)
        assert lib.dit_gemm_bf16(C.byref(b), None) == binding.DIT_ESHAPE, (N, gap)
    # a gap that no column reaches is none
    d = gemm_desc(M=0, gap_at=512, gap=2 ** 31 - 8)
    assert lib.dit_gemm_fp8(C.byref(d), None) == binding.DIT_OK


def test_sequences_past_their_limit_are_refused():
    """Key counts whose rounding up to whole blocks would pass 32 bits."""
    lib = binding.load()
    for Lk in (2 ** 31 - 1, 2 ** 31 - 63, 2 ** 30 + 1):
        for klen in (None, FAKE):
            s = binding.SparseShapeC(2, 300, Lk, 4, 2, 5, klen)
            assert lib.dit_attention_sparse_bf16(C.byref(s), FAKE, 512, FAKE, 256, FAKE, 256, FAKE, 512, FAKE, 0, FAKE,
                                                 None) == binding.DIT_ESHAPE, Lk
            assert lib.dit_select_blocks_bf16(C.byref(s), FAKE, 512, FAKE, 256, 0, FAKE, FAKE, None) == binding.DIT_ESHAPE
            assert lib.dit_attention_sparse_ws_bytes(C.byref(s)) == 0 and lib.dit_select_blocks_ws_bytes(C.byref(s)) == 0
    s = binding.SparseShapeC(1, 300, 2 ** 30, 4, 2, 64, None)
    assert lib.dit_attention_sparse_ws_bytes(C.byref(s)) > 0


def test_selection_of_as_many_lists_as_threads_allow():
    """Past 4096 key blocks a list takes 1024 threads: 2^22 lists are one too many."""
    lib = binding.load()
    for heads, Lq, Lk, bad in ((32768, 128 * 128, 64 * 4097, True), (1024, 128 * 4096, 64 * 4097, True),
                               (32768, 128 * 128, 64 * 4096, False), (32768, 128 * 127, 64 * 4097, False)):
        s = binding.SparseShapeC(1, Lq, Lk, heads, 1, 1, None)
        st = lib.dit_select_blocks_bf16(C.byref(s), None, 128 * heads, None, 128, 0, FAKE, FAKE, None)
        assert st == (binding.DIT_ESHAPE if bad else binding.DIT_EINVAL), (heads, Lq, Lk)


def test_no_workspace_for_a_selection_that_is_refused():
    """Else its caller would first ask for gigabytes."""
    lib = binding.load()
    for shape in (dict(Lq=128, Lk=2 ** 30, heads=1, batch=1), dict(Lq=128, Lk=64, heads=65536, batch=1),
                  dict(Lq=1, Lk=16384 * 64, heads=8, batch=128)):
        s = binding.sparse_shape(topk=1, **shape)
        ld = 128 * shape["heads"]
        assert lib.dit_select_blocks_bf16(C.byref(s), FAKE, ld, FAKE, ld, 0, FAKE, FAKE, None) == binding.DIT_ESHAPE
        assert lib.dit_select_blocks_ws_bytes(C.byref(s)) == 0


def test_select_workspace_holds_means_and_keys():
    means = 2 * 4 * 16 * 128 + 2 * 2 * 16 * 128      # in groups of 16 blocks
    assert binding.select_blocks_ws_bytes(**SHAPE) == 8 * means
    nkb = 1025                                       # keys leave LDS
    means += 2 * 2 * (1040 - 16) * 128
    assert binding.select_blocks_ws_bytes(**dict(SHAPE, Lk=64 * nkb)) == 8 * (means + 2 * 4 * 3 * nkb)


def test_sparse_workspace_is_for_few_lists_only():
    assert binding.attention_sparse_ws_bytes(Lq=32760, Lk=32760, heads=40, topk=52) == 0
    assert binding.attention_sparse_ws_bytes(Lq=1, Lk=32760, heads=40, topk=1) == 0


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 128)
    b = torch.zeros(4, 128, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensor"):
        binding.quant_fp8(x, b, b, M=4, K=128)
    with pytest.raises(ValueError, match="device tensor"):
        binding.gemm_fp8(b, b, b, b, None, x, M=4, N=4, K=128)
    with pytest.raises(ValueError, match="device tensor"):
        binding.select_blocks_bf16(x, x, b, Lq=4, Lk=4, heads=1, topk=1)
    with pytest.raises(ValueError, match="device tensor"):
        binding.attention_sparse_bf16(x, x, x, x, b, Lq=4, Lk=4, heads=1, topk=1)


class _Device:
    """Stands in for a device tensor of one dimension or two."""

    def __init__(self, t, device="cuda:0"):
        self._t, self.is_cuda, self.device = t, True, device

    def __getattr__(self, name):
        return getattr(self._t, name)


def test_binding_checks_sizes_and_devices():
    torch = pytest.importorskip("torch")
    x = _Device(torch.zeros(4, 128, dtype=torch.bfloat16))
    q = _Device(torch.zeros(4, 128, dtype=torch.uint8))
    s = _Device(torch.zeros(4, 4, dtype=torch.uint8))
    for kw, match in ((dict(M=5, K=128), "must hold"), (dict(M=4, K=256), "must hold"), (dict(M=4, K=128, ldx=200), "must hold"),
                      (dict(M=4, K=128, ldq=130), "must hold")):
        with pytest.raises(ValueError, match=match):
            binding.quant_fp8(x, q, s, **kw)
    with pytest.raises(ValueError, match="elements of"):
        binding.quant_fp8(x, x, s, M=4, K=128)
    with pytest.raises(ValueError, match="contiguous rows"):
        binding.quant_fp8(_Device(torch.zeros(128, 128, dtype=torch.bfloat16).t()[:4]), q, s, M=4, K=128)
    with pytest.raises(ValueError, match="one device"):
        binding.quant_fp8(x, _Device(q._t, "cuda:1"), s, M=4, K=128)
    with pytest.raises(ValueError, match="another device"):
        binding.quant_fp8(x, q, s, M=4, K=128, stream=type("S", (), {"device": "cuda:1"})())


def test_binding_refuses_strided_tensors_of_other_dimensions():
    """A slice of a [batch, rows, 3, width] projection is no run of rows; with its row stride it is."""
    torch = pytest.importorskip("torch")
    qkv = torch.zeros(2, 5, 3, 256)
    part = _Device(qkv[:, :, 1])
    with pytest.raises(ValueError, match="row stride"):
        binding._rows(part, "q", 10, 256, None, 4)
    assert binding._rows(part, "q", 10, 256, 768, 4) == 768
    assert binding._rows(_Device(qkv.view(10, 768)[:, 256:512]), "q", 10, 256, None, 4) == 768
    assert binding._rows(_Device(torch.zeros(2, 5, 256)), "q", 10, 256, None, 4) == 256
    with pytest.raises(ValueError, match="row stride"):
        binding._rows(_Device(torch.zeros(20)[::2]), "klen", 1, 10, None, 4)


def test_binding_refuses_views_that_are_too_small():
    """What a view shows is what a call may touch, however large its storage is."""
    torch = pytest.importorskip("torch")
    buf = torch.zeros(12, 768, dtype=torch.uint8)
    for view, ld in ((buf[:10, :64], None), (buf[:3, :256], None), (buf[2:11, 256:512], None), (buf[:10, :64], 768),
                     (buf[:3, :256], 768), (buf[:3].view(-1), None), (buf[:3].view(-1), 256), (buf[:2].view(2, 3, 256), None),
                     (buf[:3, :256].view(3, 2, 128)[:, 0], None)):
        with pytest.raises(ValueError, match="must hold 10 rows"):
            binding._rows(_Device(view), "q", 10, 256, ld, 1)
    for view, ld, want in ((buf[:10, :256], None, 768), (buf[1:12, 512:], None, 768), (buf[:10, :256], 768, 768),
                           (buf[:4].view(-1)[:2560], None, 256), (buf[:4].view(12, 256)[:10], 256, 256),
                           (buf[:5].view(5, 3, 256), None, 256)):
        assert binding._rows(_Device(view), "q", 10, 256, ld, 1) == want
    x = _Device(torch.zeros(64, 768, dtype=torch.bfloat16)[:, :128])
    o = _Device(torch.zeros(64, 768, dtype=torch.bfloat16)[:, :64])
    idx = _Device(torch.zeros(1, 1, 1, 1, dtype=torch.int32))
    with pytest.raises(ValueError, match="o must hold 64 rows"):
        binding.attention_sparse_bf16(x, x, x, o, idx, Lq=64, Lk=64, heads=1, topk=1)


@pytest.mark.parametrize("dtype", ["float16", "float8_e5m2", "float8_e4m3fnuz", "bool"])
def test_binding_refuses_types_that_would_be_misread(dtype):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 128, dtype=getattr(torch, dtype))
    with pytest.raises(ValueError, match="not be torch"):
        binding._rows(_Device(x), "x", 4, 128, None, x.element_size())


@pytest.mark.filterwarnings("ignore:ComplexHalf")
def test_binding_refuses_types_of_another_meaning():
    """Same size, other values: whole numbers for floats, scale bytes for e4m3 and the reverse."""
    torch = pytest.importorskip("torch")

    def t(dtype, *shape):
        return _Device(torch.zeros(*shape, dtype=torch.uint8 if "float8" in dtype else getattr(torch, dtype)).view(
            getattr(torch, dtype)))

    good = dict(A="float8_e4m3fn", a_scale="float8_e8m0fnu", W="uint8", w_scale="int8", bias="bfloat16", Cout="float32",
                gate=None)
    sizes = dict(A=(16, 128), a_scale=(16, 4), W=(8, 128), w_scale=(8, 4), bias=(8,), Cout=(16, 8), gate=(8,))

    def gemm(flags, **kw):
        a = {n: d and t(d, *sizes[n]) for n, d in dict(good, **kw).items()}
        gate = a.pop("gate")
        binding.gemm_fp8(*a.values(), M=16, N=8, K=128, flags=flags, gate=gate)

    for flags, kw in ((1, dict(Cout="int32")), (1, dict(Cout="uint32")), (1, dict(A="float8_e8m0fnu")),
                      (1, dict(W="float8_e8m0fnu")), (1, dict(a_scale="float8_e4m3fn")), (1, dict(w_scale="float8_e4m3fn")),
                      (2, dict(Cout="bfloat16", gate="int32")), (0, dict(Cout="float16")), (1, dict(bias="float16"))):
        with pytest.raises(ValueError, match=next(iter(kw)) if len(kw) == 1 else "gate"):
            gemm(flags, **kw)
    x, q, s = t("bfloat16", 16, 128), t("uint8", 16, 128), t("uint8", 16, 4)
    with pytest.raises(ValueError, match="^q must"):
        binding.quant_fp8(x, t("float8_e8m0fnu", 16, 128), s, M=16, K=128)
    with pytest.raises(ValueError, match="^scale must"):
        binding.quant_fp8(x, q, t("float8_e4m3fn", 16, 4), M=16, K=128)
    for dtype in ("uint32", "complex32", "float32"):
        with pytest.raises(ValueError, match="idx must be int32"):
            binding.select_blocks_bf16(x, x, t(dtype, 1), Lq=16, Lk=16, heads=1, topk=1)
        with pytest.raises(ValueError, match="klen must be int32"):
            binding.select_blocks_bf16(x, x, t("int32", 1), Lq=16, Lk=16, heads=1, topk=1, klen=t(dtype, 1))


def test_nothing_to_write_needs_no_pointers():
    lib = binding.load()
    assert lib.dit_quant_fp8(None, 1, 256, None, 256, None, 4, 0, 256, None) == binding.DIT_OK
    for kw in ({"M": 0}, {"N": 0}):
        for flags in (0, 1, 2, 8):
            d = gemm_desc(A=None, W=None, a_scale=None, w_scale=None, C=None, flags=flags, ld_cs=4, **kw)
            assert lib.dit_gemm_fp8(C.byref(d), None) == binding.DIT_OK
    for shape in ({"Lq": 0}, {"batch": 0}):
        s = binding.sparse_shape(**dict(SHAPE, **shape))
        assert lib.dit_select_blocks_bf16(C.byref(s), None, 512, None, 256, 0, None, None, None) == binding.DIT_OK
        assert lib.dit_attention_sparse_bf16(C.byref(s), None, 512, None, 256, None, 256, None, 512, None, 0, None,
                                             None) == binding.DIT_OK
    # no keys: k and v may be empty, the lists and rows are written
    s = binding.sparse_shape(**dict(SHAPE, Lk=0))
    assert lib.dit_attention_sparse_bf16(C.byref(s), FAKE, 512, None, 256, None, 256, None, 512, FAKE, 0, None,
                                         None) == binding.DIT_EINVAL
    assert lib.dit_select_blocks_bf16(C.byref(s), FAKE, 512, None, 256, 0, None, FAKE, None) == binding.DIT_EINVAL


def test_oracle_rounds_to_nearest_even():
    """The oracle's quantiser against torch's conversion, which rounds to nearest even."""
    torch = pytest.importorskip("torch")
    x = np.random.default_rng(3).standard_normal((40, 128)) * 100
    x[:, 0] = 448.0                                  # scale 1
    x = np.clip(x, -448, 448)
    x[1, 1:120] = (ref.TABLE[1:120] + ref.TABLE[2:121]) / 2          # ties
    q, s = ref.quantise(x)
    assert (s == 127).all()
    t = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    ok = x == x.astype(np.float32)
    np.testing.assert_array_equal(ref.values(q, s)[ok], t[ok])
