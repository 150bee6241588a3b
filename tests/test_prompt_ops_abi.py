"""Refusals, sizes and host results of a prompt encoder's entry points: no GPU needed, nothing is launched."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2608_09231_amd import binding
from tests import _prompt_ops as ref

FAKE = 0x1000


def gemm_desc(**kw):
    d = dict(A=FAKE, lda=128, a_scale=FAKE, ld_as=8, W=FAKE, ldw=128, w_scale=FAKE, ld_ws=8, bias=None, C=FAKE,
             ldc=512, c_scale=None, ld_cs=0, gate=None, M=64, N=512, K=256, flags=0, rms_cols=0, gelu_from=512,
             gap_at=0, gap=0)
    d.update(kw)
    return binding.GemmFp4DescC(**d)


FP4 = {"flags": 16, "c_scale": FAKE, "ld_cs": 16, "ldc": 256}


@pytest.mark.parametrize("kw", [
    {"K": 0}, {"K": 250}, {"K": 240}, {"K": -32}, {"M": -1}, {"N": -8}, {"N": 500}, {"lda": 112}, {"ldw": 112}, {"lda": 136},
    {"ldw": 1 << 23}, {"ld_as": 4}, {"ld_ws": 10}, {"ld_as": 1 << 23}, {"K": 288, "lda": 144, "ldw": 144}, {"ldc": 504},
    {"ldc": 516}, {"gap": -4}, {"gap": 6, "gap_at": 8, "ldc": 600}, {"gap": 8, "gap_at": 6, "ldc": 600},
    {"gap": 128, "gap_at": 256}, {"gap": 8, "gap_at": -4, "ldc": 600}, {"gelu_from": 6}, {"gelu_from": -4}, {"rms_cols": 100},
    {"rms_cols": 640}, {"rms_cols": -128}, {"rms_cols": 128, "N": 200}, dict(FP4, N=200), dict(FP4, ld_cs=0),
    dict(FP4, ld_cs=12), dict(FP4, gelu_from=64), dict(FP4, ldc=264), dict(FP4, ldc=240), dict(FP4, gap=128, gap_at=128),
    {"M": 2 ** 31 - 1}, {"M": 64, "N": 2 ** 31 - 8, "ldc": 1 << 40}, {"gap_at": 0, "gap": 2 ** 31 - 8, "ldc": 1 << 40}])
def test_gemm_fp4_refuses_shapes(kw):
    lib = binding.load()
    d = gemm_desc(**kw)
    assert lib.dit_gemm_fp4(C.byref(d), None) == binding.DIT_ESHAPE, kw
    assert lib.dit_cache_last_error(None)


@pytest.mark.parametrize("kw", [
    {"A": None}, {"W": None}, {"a_scale": None}, {"w_scale": None}, {"C": None}, {"flags": 8}, {"flags": 32}, {"flags": 2},
    {"flags": 16}, {"flags": 3, "gate": FAKE}, {"flags": 17, "c_scale": FAKE}, {"A": FAKE + 8}, {"W": FAKE + 4}, {"C": FAKE + 8},
    {"a_scale": FAKE + 2}, {"w_scale": FAKE + 1}, {"bias": FAKE + 1}, {"flags": 2, "gate": FAKE + 4}, dict(FP4, c_scale=FAKE + 1)])
def test_gemm_fp4_refuses_pointers_and_flags(kw):
    lib = binding.load()
    d = gemm_desc(**kw)
    assert lib.dit_gemm_fp4(C.byref(d), None) == binding.DIT_EINVAL, kw
    assert lib.dit_gemm_fp4(None, None) == binding.DIT_EINVAL


def test_rows_of_4_bits_refuse():
    lib = binding.load()
    good = dict(x=FAKE, t=1, ldx=256, q=FAKE, ldq=128, s=FAKE, lds=8, M=4, K=256)
    for st, kw in ((binding.DIT_EINVAL, {"x": None}), (binding.DIT_EINVAL, {"q": None}), (binding.DIT_EINVAL, {"s": None}),
                   (binding.DIT_EINVAL, {"t": 2}), (binding.DIT_EINVAL, {"x": FAKE + 8}),
                   (binding.DIT_EINVAL, {"q": FAKE + 4}), (binding.DIT_EINVAL, {"s": FAKE + 1}),
                   (binding.DIT_ESHAPE, {"K": 48}), (binding.DIT_ESHAPE, {"K": -32}), (binding.DIT_ESHAPE, {"M": -1}),
                   (binding.DIT_ESHAPE, {"ldx": 255}), (binding.DIT_ESHAPE, {"ldx": 260}), (binding.DIT_ESHAPE, {"ldq": 136}),
                   (binding.DIT_ESHAPE, {"ldq": 112}), (binding.DIT_ESHAPE, {"lds": 9}), (binding.DIT_ESHAPE, {"lds": 4}),
                   (binding.DIT_ESHAPE, {"M": 1 << 26}), (binding.DIT_ESHAPE, {"K": 1 << 31 >> 1 << 1 & ~31, "M": 1}),
                   (binding.DIT_ESHAPE, {"M": 1 << 16, "K": 1 << 21, "ldx": 1 << 21, "ldq": 1 << 20, "lds": 1 << 16})):
        a = dict(good, **kw)
        if a["K"] >= 1 << 31:
            a["K"] = (1 << 31) - 32
        assert lib.dit_quant_fp4(a["x"], a["t"], a["ldx"], a["q"], a["ldq"], a["s"], a["lds"], a["M"], a["K"], None) == st, kw
        assert lib.dit_dequant_fp4(a["q"], a["ldq"], a["s"], a["lds"], a["x"], a["t"], a["ldx"], a["M"], a["K"], None) == st, kw


def rotary_desc(**kw):
    d = dict(x=FAKE, ldx=512, y=1 << 20, ldy=512, pos=FAKE, ldpos=16, freq=FAKE, dtype=1, rows=16, heads=4, head_dim=128,
             rot=128, layout=0, axes=1, pairs=(64, 0, 0, 0), scale=1.0)
    d.update(kw)
    d["pairs"] = (C.c_int32 * 4)(*d["pairs"])
    return binding.RotaryDescC(**d)


@pytest.mark.parametrize("kw", [
    {"rows": -1}, {"heads": -1}, {"rows": 1 << 24}, {"head_dim": 4}, {"head_dim": 132}, {"head_dim": 520, "ldx": 2080, "ldy": 2080},
    {"rot": 127}, {"rot": -2}, {"rot": 130}, {"rot": 126}, {"axes": 0}, {"axes": 5}, {"pairs": (63, 0, 0, 0)},
    {"axes": 2, "pairs": (65, -1, 0, 0)}, {"axes": 2, "pairs": (32, 32, 0, 0), "ldpos": 15}, {"ldx": 504}, {"ldy": 504},
    {"ldx": 516}, {"dtype": 0, "ldy": 514}, {"heads": (1 << 23) + 1, "ldx": 1 << 31, "ldy": 1 << 31}])
def test_rotary_refuses_shapes(kw):
    lib = binding.load()
    d = rotary_desc(**kw)
    assert lib.dit_rotary(C.byref(d), None) == binding.DIT_ESHAPE, kw


@pytest.mark.parametrize("kw", [
    {"x": None}, {"y": None}, {"pos": None}, {"freq": None}, {"dtype": 2}, {"layout": 2}, {"layout": -1}, {"x": FAKE + 8},
    {"y": FAKE + 8}, {"pos": FAKE + 2}, {"freq": FAKE + 4}, {"scale": math.inf}, {"scale": math.nan},
    # overlaps: shifted rows, other strides, columns that cross; a matrix's columns beside each other are none
    {"y": FAKE + 1024}, {"y": FAKE, "ldy": 520}, {"y": FAKE + 512, "ldx": 1024, "ldy": 1024},
    {"y": FAKE + 1024, "ldx": 1000, "ldy": 1000}, {"x": FAKE + 16, "y": FAKE}])
def test_rotary_refuses_pointers_and_overlaps(kw):
    lib = binding.load()
    d = rotary_desc(**kw)
    assert lib.dit_rotary(C.byref(d), None) == binding.DIT_EINVAL, kw
    assert lib.dit_rotary(None, None) == binding.DIT_EINVAL


def freqs(pairs, base, method, factor, context):
    i = np.arange(pairs)
    if method == binding.ROTARY_BASE:
        base = base * factor ** (pairs / (pairs - 1))
    f = base ** (-i / pairs)
    if method == binding.ROTARY_LINEAR:
        f = f / factor
    if method == binding.ROTARY_PARTS:
        keep = np.clip((context * f / (2 * np.pi) - 1) / 31, 0, 1)
        f = f * keep + f / factor * (1 - keep)
    return f


@pytest.mark.parametrize("pairs", [0, 1, 2, 22, 64, 256])
@pytest.mark.parametrize("method", [0, 1, 2, 3])
@pytest.mark.parametrize("base", [1e4, 5e5])
def test_rotary_frequencies(pairs, method, base):
    if method == binding.ROTARY_BASE and pairs == 1:
        with pytest.raises(binding.DitError):
            binding.rotary_freqs(pairs, base=base, method=method, factor=8.0)
        return
    f, scale = binding.rotary_freqs(pairs, base=base, method=method, factor=8.0, context=4096.0)
    np.testing.assert_allclose(f, freqs(pairs, base, method, 8.0, 4096.0) if pairs else np.empty(0), rtol=2.0 ** -48)
    assert scale == (0.1 * math.log(8.0) + 1 if method == binding.ROTARY_PARTS else 1.0)


def test_rotary_frequencies_at_their_ends():
    """The base's change leaves the fastest pair and slows the slowest by the factor; by parts, pairs of many turns in the
    trained range stay and those of less than one are slowed by the factor."""
    plain = binding.rotary_freqs(64)[0]
    f = binding.rotary_freqs(64, method=binding.ROTARY_BASE, factor=8.0)[0]
    assert f[0] == plain[0] == 1 and abs(plain[-1] / f[-1] - 8) < 1e-9
    f = binding.rotary_freqs(64, method=binding.ROTARY_PARTS, factor=8.0, context=4096.0)[0]
    turns = 4096 * plain / (2 * np.pi)
    assert (f[turns >= 32] == plain[turns >= 32]).all() and np.allclose(f[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    assert (np.diff(f) < 0).all()


def test_rotary_frequencies_refuse():
    lib = binding.load()
    out, scale = (C.c_double * 8)(), C.c_double()

    def call(pairs=8, base=1e4, method=0, factor=2.0, context=10.0, freq=out, s=C.byref(scale)):
        return lib.dit_rotary_freqs(pairs, base, method, factor, context, freq, s)

    assert call() == binding.DIT_OK
    assert call(pairs=-1) == binding.DIT_ESHAPE
    for kw in ({"base": 0.0}, {"base": -1.0}, {"base": math.inf}, {"base": math.nan}, {"method": 4}, {"method": -1}, {"freq": None},
               {"s": None}, {"method": 1, "factor": 0.0}, {"method": 2, "factor": math.nan}, {"method": 3, "context": 0.0},
               {"method": 3, "factor": math.inf}):
        assert call(**kw) == binding.DIT_EINVAL, kw
    assert call(factor=0.0, context=0.0) == binding.DIT_OK      # (not used)


def packed_shape(**kw):
    d = dict(batch=3, Tq=300, Tk=1000, heads=4, kv_heads=2, qoff=FAKE, koff=FAKE, klen=None)
    d.update(kw)
    return binding.PackedShapeC(*d.values())


def attend(s, q=FAKE, ldq=512, k=FAKE, ldk=256, v=FAKE, ldv=256, o=FAKE, ldo=512, flags=0, ws=FAKE):
    return binding.load().dit_attention_packed_bf16(C.byref(s) if s else None, q, ldq, k, ldk, v, ldv, o, ldo, flags, ws, None)


@pytest.mark.parametrize("st,shape,kw", [
    (binding.DIT_ESHAPE, {"batch": -1}, {}), (binding.DIT_ESHAPE, {"Tq": -1}, {}), (binding.DIT_ESHAPE, {"Tk": -1}, {}),
    (binding.DIT_ESHAPE, {"heads": 0}, {}), (binding.DIT_ESHAPE, {"kv_heads": 3}, {}), (binding.DIT_ESHAPE, {"kv_heads": 0}, {}),
    (binding.DIT_ESHAPE, {"Tq": 2 ** 30}, {}), (binding.DIT_ESHAPE, {"Tk": 2 ** 30 + 1}, {}),
    (binding.DIT_ESHAPE, {"batch": 2 ** 21}, {}), (binding.DIT_ESHAPE, {"Tq": 2 ** 26}, {}),
    (binding.DIT_ESHAPE, {"heads": 2 ** 21, "kv_heads": 2 ** 21}, {}),
    (binding.DIT_EINVAL, {"qoff": None}, {}), (binding.DIT_EINVAL, {"koff": None}, {}), (binding.DIT_EINVAL, {"qoff": FAKE + 2}, {}),
    (binding.DIT_EINVAL, {"koff": FAKE + 1}, {}), (binding.DIT_EINVAL, {"klen": FAKE + 2}, {}),
    (binding.DIT_EINVAL, {}, {"q": None}), (binding.DIT_EINVAL, {}, {"k": None}), (binding.DIT_EINVAL, {}, {"v": None}),
    (binding.DIT_EINVAL, {}, {"o": None}), (binding.DIT_EINVAL, {}, {"q": FAKE + 8}), (binding.DIT_EINVAL, {}, {"o": FAKE + 4}),
    (binding.DIT_EINVAL, {}, {"flags": 4}), (binding.DIT_EINVAL, {}, {"flags": -1}),
    (binding.DIT_ESHAPE, {}, {"ldq": 504}), (binding.DIT_ESHAPE, {}, {"ldq": 516}), (binding.DIT_ESHAPE, {}, {"ldk": 128}),
    (binding.DIT_ESHAPE, {}, {"ldv": 1 << 22}), (binding.DIT_ESHAPE, {}, {"ldo": 256})])
def test_packed_attention_refuses(st, shape, kw):
    s = packed_shape(**shape)
    assert attend(s, **kw) == st
    if shape and st == binding.DIT_ESHAPE:
        assert binding.load().dit_attention_packed_ws_bytes(C.byref(s)) == 0


def test_packed_attention_needs_its_workspace():
    lib = binding.load()
    assert attend(None) == binding.DIT_EINVAL and lib.dit_attention_packed_ws_bytes(None) == 0
    few = packed_shape(batch=300)                             # about one query a sequence
    assert lib.dit_attention_packed_ws_bytes(C.byref(few)) > 0
    assert attend(few, ws=None) == attend(few, ws=FAKE + 8) == binding.DIT_EINVAL
    shared = packed_shape(batch=1, Tk=20000)                  # few tiles of long keys
    assert lib.dit_attention_packed_ws_bytes(C.byref(shared)) > 0
    assert attend(shared, ws=None) == binding.DIT_EINVAL
    many = packed_shape(batch=1, Tq=40000, Tk=40000)
    assert lib.dit_attention_packed_ws_bytes(C.byref(many)) == 0


def test_nothing_to_write_needs_no_pointers():
    lib = binding.load()
    for kw in ({"batch": 0}, {"Tq": 0}):
        s = packed_shape(qoff=None, koff=None, **kw)
        assert attend(s, q=None, k=None, v=None, o=None, ws=None) == binding.DIT_OK
    for kw in ({"rows": 0}, {"heads": 0}):
        d = rotary_desc(x=None, y=None, pos=None, freq=None, **kw)
        assert lib.dit_rotary(C.byref(d), None) == binding.DIT_OK
    for kw in ({"M": 0}, {"N": 0}):
        d = gemm_desc(A=None, W=None, a_scale=None, w_scale=None, C=None, **kw)
        assert lib.dit_gemm_fp4(C.byref(d), None) == binding.DIT_OK
    for M, K in ((0, 256), (4, 0)):
        assert lib.dit_quant_fp4(None, 1, 256, None, 128, None, 8, M, K, None) == binding.DIT_OK
        assert lib.dit_dequant_fp4(None, 128, None, 8, None, 1, 256, M, K, None) == binding.DIT_OK


def test_binding_refuses_host_tensors():
    import torch
    t = torch.zeros(16, 512)
    u = torch.zeros(16, 256, dtype=torch.uint8)
    i = torch.zeros(16, dtype=torch.int32)
    for call in (lambda: binding.quant_fp4(t, u, u, M=16, K=512), lambda: binding.dequant_fp4(u, u, t, M=16, K=512),
                 lambda: binding.gemm_fp4(u, u, u, u, None, t, M=16, N=16, K=512),
                 lambda: binding.rotary(t, t, pos=i, freq=t, rows=16, heads=4),
                 lambda: binding.attention_packed_bf16(t, t, t, t, qoff=i, koff=i, heads=4)):
        with pytest.raises(ValueError):
            call()


def test_oracle_rounds_to_nearest_even():
    """The plain 4-bit form at its ties and borders."""
    x = np.zeros((1, 32))
    x[0, :12] = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.2500001, -5, -0.25, 4.9999]
    c, s = ref.quantise(x)
    assert s[0, 0] == 127
    assert list(ref.values(c, s)[0, :12]) == [6, 4, 4, 2, 2, 1, 1, 0, 0.5, -4, 0, 4]
    assert ref.quantise(x * 1.0001)[1][0, 0] == 128          # past 6: the next scale
    assert (ref.unpack(ref.pack(c)) == c).all()
