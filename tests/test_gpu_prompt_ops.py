"""4-bit rows and their products, rotary positions and attention over packed sequences against plain float64
forms, through the C ABI, at the sizes, strides and masks where they can go wrong."""
import numpy as np
import pytest

from paper_2608_09231_amd import binding
from tests import _operators as ref8
from tests import _prompt_ops as ref
from tests._gpu import dev, host_bf16, torch_cuda
from tests.test_gpu_kernels import bf16_bits, bits_to_f64
from tests.test_gpu_operators import strided

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8    # half a step, relative
FILL = 0x5A


def rng(*seed):
    return np.random.default_rng([78, *seed])


# ---------------------------------------------------------------- 4-bit rows

def check_quant(torch, x, *, ldx=None, ldq=None, lds=None):
    M, K = x.shape
    q = torch.full((M + 1, ldq or K // 2), FILL, dtype=torch.uint8, device="cuda")
    s = torch.full((M + 1, lds or binding.fp4_scale_ld(K)), FILL, dtype=torch.uint8, device="cuda")
    binding.quant_fp4(strided(torch, x, ldx or K), q, s, M=M, K=K)
    hq, hs = q.cpu().numpy(), s.cpu().numpy()
    assert (hq[:, K // 2:] == FILL).all() and (hs[:, K // 32:] == FILL).all()
    assert (hq[M] == FILL).all() and (hs[M] == FILL).all()
    x64 = bits_to_f64(x) if x.dtype == np.uint16 else x.astype(np.float64)
    rc, rs = ref.quantise(x64)
    np.testing.assert_array_equal(hs[:M, :K // 32], rs)
    want = ref.values(rc, rs)
    np.testing.assert_array_equal(ref.values(ref.unpack(hq[:M, :K // 2]), hs[:M, :K // 32]), want)
    # and back
    for bf16 in (True, False):
        ldy = K + 8
        y = torch.full((M + 1, ldy * (2 if bf16 else 4)), FILL, dtype=torch.uint8, device="cuda")
        y = y.view(torch.int16 if bf16 else torch.float32)
        binding.dequant_fp4(q, s, y, M=M, K=K)
        raw = y.cpu().numpy().view(np.uint8).reshape(M + 1, ldy, -1)
        assert (raw[M] == FILL).all() and (raw[:, K:] == FILL).all()
        got = host_bf16(y) if bf16 else y.cpu().numpy().astype(np.float64)
        # e2m1 times a power of two: exact in both, but for what rounding took to 2^128
        np.testing.assert_array_equal(got[:M, :K], np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,ldx,ldq,lds", [
    (1, 32, None, None, None), (3, 128, None, None, None), (5, 160, 176, 96, 12), (37, 2592, 2600, 1312, 84),
    (130, 1056, None, None, None), (1030, 992, 1008, 496, 36)])
def test_quant_rows(M, K, ldx, ldq, lds, dtype):
    torch = torch_cuda()
    r = rng(M, K)
    x = r.standard_normal((M, K)) * np.exp(3 * r.standard_normal((M, 1))) * np.exp(r.standard_normal(K))
    check_quant(torch, bf16_bits(x) if dtype == "bf16" else x.astype(np.float32), ldx=ldx, ldq=ldq, lds=lds)


def test_quant_borders_zeros_and_extremes():
    """Blocks whose largest value is a scale's last (6 * 2^e) or the next above it, ties between two e2m1 values,
    blocks of zeros, the type's smallest and largest values."""
    torch = torch_cuda()
    rows = []
    for e in (-151, -129, -128, -127, -126, -20, 0, 60, 125):
        top = np.float32(6 * 2.0 ** e) if e > -150 else np.float32(1e-45)
        for a in (top, np.nextafter(top, np.float32(np.inf)), np.nextafter(top, np.float32(0))):
            row = np.zeros(32, np.float32)
            row[17] = -a
            row[:8] = a * np.array([1, 5 / 6, 3.5 / 6, 2.5 / 6, 1.75 / 6, 1.25 / 6, 0.75 / 6, 0.25 / 6], np.float32)
            row[8:16] = -np.nextafter(row[:8], np.float32(0))
            rows.append(row)
    rows.append(np.zeros(32, np.float32))
    rows.append(np.full(32, np.finfo(np.float32).max))
    rows.append(np.full(32, -0.0, np.float32))
    check_quant(torch, np.stack(rows).astype(np.float32))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_quant_block_that_is_not_finite(bad):
    torch = torch_cuda()
    x = rng(5).standard_normal((6, 256)).astype(np.float32)
    x[2, 200] = bad
    check_quant(torch, x)
    check_quant(torch, bf16_bits(np.where(np.isfinite(x), x, 0)) | np.where(np.isnan(x), 0x7FC0, np.where(
        np.isinf(x), np.where(x > 0, 0x7F80, 0xFF80), 0)).astype(np.uint16))


def test_dequant_of_every_byte():
    """Every code with every scale byte: infinities past the type's range, rounding below its subnormals."""
    torch = torch_cuda()
    q = np.tile((np.arange(16) * 17).astype(np.uint8), (256, 1))          # 32 values: every code twice
    s = np.zeros((256, 4), np.uint8)
    s[:, 0] = np.arange(256)
    with np.errstate(over="ignore"):
        want = ref.values(ref.unpack(q), s[:, :1])
        for bf16 in (True, False):
            y = torch.empty(256, 32, dtype=torch.int16 if bf16 else torch.float32, device="cuda")
            binding.dequant_fp4(dev(torch, q), dev(torch, s), y, M=256, K=32)
            got = host_bf16(y) if bf16 else y.cpu().numpy().astype(np.float64)
            np.testing.assert_array_equal(got, np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want))


def test_rows_nothing_to_do():
    torch = torch_cuda()
    x = torch.zeros(4, 32, device="cuda")
    q = torch.full((4, 16), FILL, dtype=torch.uint8, device="cuda")
    s = torch.full((4, 4), FILL, dtype=torch.uint8, device="cuda")
    for M, K in ((0, 32), (4, 0)):
        binding.quant_fp4(x, q, s, M=M, K=K)
        binding.dequant_fp4(q, s, x, M=M, K=K)
    assert int((q != FILL).sum()) == 0 and int((s != FILL).sum()) == 0 and int((x != 0).sum()) == 0


# ---------------------------------------------------------------- products

def operand(r, M, K, spread=1.0):
    """4-bit rows with row and block scales of their own: (codes, scale bytes)."""
    x = r.standard_normal((M, K)) * np.exp(spread * r.standard_normal((M, 1))) / np.sqrt(K)
    return ref.quantise(bits_to_f64(bf16_bits(x * np.exp(0.5 * np.repeat(r.standard_normal((M, K // 32)), 32, 1)))))


def padded_scale(s, K, ld=None):
    out = np.full((s.shape[0], ld or binding.fp4_scale_ld(K)), 255, np.uint8)   # NaN scales past the last block
    out[:, :s.shape[1]] = s
    return out


def run_gemm(M, N, K, *, out="bf16", act="none", rms_cols=0, gelu_from=None, bias=True, gap_at=0, gap=0, pad=0,
             seed=0, operands=None):
    torch = torch_cuda()
    r = rng(M, N, K, seed)
    (aq, as_), (wq, ws) = operands or (operand(r, M, K), operand(r, N, K))
    b_bits = bf16_bits(0.1 * r.standard_normal(N))
    b = bits_to_f64(b_bits)
    a, w = ref.values(aq, as_), ref.values(wq, ws)
    y, d = ref8.product(a, w, b if bias else None, f32=True, act=act, rms_cols=rms_cols, gelu_from=gelu_from)
    flags = {"bf16": 0, "f32": binding.EPI_F32, "fp4": binding.EPI_FP4, "gated": binding.EPI_GATED_RES}[out]
    flags |= binding.EPI_SILU if act == "silu" else 0
    width = N // 2 + pad if out == "fp4" else N + gap + pad
    esize = {"bf16": 2, "gated": 2, "f32": 4, "fp4": 1}[out]
    old_bits = bf16_bits(r.standard_normal((M + 1, width)))
    C = dev(torch, old_bits) if out == "gated" else torch.full((M + 1, width * esize), FILL, dtype=torch.uint8,
                                                               device="cuda")
    if out != "gated":
        C = C.view({"bf16": torch.int16, "f32": torch.float32, "fp4": torch.uint8}[out])
    gate = r.standard_normal(N).astype(np.float32)
    cs = torch.full((M + 1, binding.fp4_scale_ld(N)), FILL, dtype=torch.uint8, device="cuda") if out == "fp4" else None
    sp = 4 if pad else 0
    binding.gemm_fp4(strided(torch, ref.pack(aq), K // 2 + (16 if pad else 0), 0x7F),
                     dev(torch, padded_scale(as_, K, binding.fp4_scale_ld(K) + sp)),
                     strided(torch, ref.pack(wq), K // 2 + (48 if pad else 0), 0x7F),
                     dev(torch, padded_scale(ws, K, binding.fp4_scale_ld(K) + 2 * sp)),
                     dev(torch, b_bits) if bias else None, C, M=M, N=N, K=K, flags=flags, c_scale=cs,
                     gate=dev(torch, gate) if out == "gated" else None, rms_cols=rms_cols, gelu_from=gelu_from,
                     gap_at=gap_at, gap=gap)
    torch.cuda.synchronize()
    host = C.cpu().numpy()
    if out == "fp4":
        scale, nb = cs.cpu().numpy(), N // 32
        assert (host[M] == FILL).all() and (host[:, N // 2:] == FILL).all()
        assert (scale[M] == FILL).all() and (scale[:, nb:] == FILL).all()
        scale = scale[:M, :nb]
        got = ref.values(ref.unpack(host[:M, :N // 2]), scale)
        # the scale is that of the largest value, up to what that may be off
        s = np.repeat(2.0 ** (scale.astype(np.float64) - 127), 32, 1)
        top = np.repeat(np.abs(y).reshape(M, nb, 32).max(2), 32, 1)
        off = np.repeat(d.reshape(M, nb, 32).max(2), 32, 1)
        fits = (top - off <= 6 * s) & ((top + off > 3 * s) | (scale.repeat(32, 1) == 0))
        assert (fits | np.isnan(top)).all()
        # half the distance to the next code: 1/4 up to 2, 1/2 up to 4, 1 above
        z = (np.abs(y) + d) / s
        return got, y, np.where(z <= 2, 0.25, np.where(z <= 4, 0.5, 1.0)) * s + d
    cols = np.arange(N) + np.where(np.arange(N) >= gap_at, gap, 0)
    rest = np.delete(np.arange(width), cols)
    if out == "gated":
        old = bits_to_f64(old_bits)
        got = host_bf16(C)
        assert (got[M] == old[M]).all() and (got[:, rest] == old[:, rest]).all()
        y, d = old[:M, cols] + gate * y, np.abs(gate) * d + 2.0 ** -22 * (np.abs(old[:M, cols]) + np.abs(gate * y))
        got = got[:M, cols]
    else:
        raw = host.view(np.uint8).reshape(M + 1, width, esize)
        assert (raw[M] == FILL).all() and (raw[:, rest] == FILL).all(), "bytes outside the output changed"
        got = (host_bf16(C) if out == "bf16" else host.astype(np.float64))[:M, cols]
    return got, y, d + (2.0 ** -24 if out == "f32" else BF16) * (np.abs(y) + d) + 1e-30


def check_gemm(*a, **kw):
    got, y, tol = run_gemm(*a, **kw)
    worst = np.max(np.abs(got - y) / tol)
    assert worst <= 1, f"{worst} of the tolerance at {np.unravel_index(np.argmax(np.abs(got - y) / tol), y.shape)}"


# few rows and columns, single blocks of K, blocks cut short in every way that a slice of 128 or 256 can be, ragged rows
# and columns, sizes of every tile
SIZES = [(1, 8, 32), (1, 1000, 2336), (1, 8, 64), (16, 72, 128), (17, 264, 416), (40, 136, 5120), (300, 2056, 288),
         (513, 1416, 1056), (70, 13824, 672), (1500, 5640, 160), (2100, 4104, 544), (1920, 4352, 416), (500, 10232, 1184),
         (5, 9000, 416), (16, 20008, 288), (100, 3000, 672), (300, 2056, 1952), (897, 1992, 1568), (33, 4096, 96)]
LARGE = [(4100, 4360, 32), (4100, 4360, 160), (4096, 4096, 1152), (4353, 3848, 928)]


@pytest.mark.parametrize("out", ["bf16", "f32", "gated"])
@pytest.mark.parametrize("M,N,K", SIZES + LARGE)
def test_gemm_sizes(M, N, K, out):
    check_gemm(M, N, K, out=out, pad=8 if (M + K) % 3 else 0, bias=(M % 4) > 0)


@pytest.mark.parametrize("act", ["none", "gelu", "silu", "rms"])
@pytest.mark.parametrize("M,N,K", [(1, 128, 544), (19, 256, 416), (257, 1152, 288), (700, 7040, 1056), (500, 10240, 416),
                                   (1913, 4352, 672), (4097, 4480, 288)])
def test_gemm_fp4_output(M, N, K, act):
    check_gemm(M, N, K, out="fp4", act=act, rms_cols=N if act == "rms" else 0, gelu_from=0 if act == "gelu" else None,
               pad=16 if M % 2 else 0)


@pytest.mark.parametrize("M,N,K", [(1, 32, 32), (3, 160, 96), (40, 1056, 416), (300, 2080, 288), (4100, 4192, 160)])
def test_gemm_fp4_output_of_part_of_a_tile(M, N, K):
    check_gemm(M, N, K, out="fp4", act="none", pad=0 if (N // 2) % 16 == 0 else 8)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(3, 512, 416), (30, 640, 288), (300, 2688, 416), (500, 10240, 416), (1913, 4352, 672),
                                   (70, 13824, 672), (2100, 4224, 288), (4100, 4352, 288)])
def test_gemm_norm_gelu_and_gap(M, N, K, out):
    """A fused projection: normed q and k columns, plain values, GELU past a gap; then per-column forms."""
    check_gemm(M, N, K, out=out, rms_cols=256, gelu_from=384, gap_at=384, gap=128, seed=1)
    check_gemm(M, N, K, out=out, rms_cols=128, gelu_from=204, gap_at=140, gap=12, pad=8 - (N + 12) % 8, seed=2)
    check_gemm(M, N, K, out=out, act="silu", seed=3)
    check_gemm(M, N, K, out=out, rms_cols=N, seed=4)


KERNELS = [(5, 64, 416), (40, 256, 416), (300, 2048, 416), (500, 10240, 544), (1920, 4352, 544), (4100, 4352, 416)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", KERNELS)
def test_gemm_scales_at_the_ends(M, N, K, out):
    """Blocks whose scale bytes are an end of the range in one operand and the opposite one in the other, so that
    every product is an ordinary number."""
    r = rng(M, N, K, 19)
    nb = K // 32
    ends = np.resize([0, 254, 1, 247, 2, 246, 9, 253, 120], nb)
    a = r.integers(0, 16, (M, K)).astype(np.uint8), np.tile(ends, (M, 1)).astype(np.uint8)
    w = r.integers(0, 16, (N, K)).astype(np.uint8), np.tile(254 - ends, (N, 1)).astype(np.uint8)
    check_gemm(M, N, K, out=out, operands=(a, w), bias=False)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", KERNELS)
def test_gemm_scale_of_255_is_nan(M, N, K, out):
    r = rng(M, N, K, 21)
    a, w = operand(r, M, K), operand(r, N, K)
    a[1][M // 2, K // 32 - 1] = 255
    a[0][M // 2, -32:] = 0                       # (zeros times NaN)
    w[1][N // 3, 3] = 255
    got, y, tol = run_gemm(M, N, K, out=out, operands=(a, w))
    gone = np.zeros(got.shape, bool)
    gone[M // 2], gone[:, N // 3] = True, True
    assert np.isnan(got[gone]).all() and (np.abs(got - y)[~gone] <= tol[~gone]).all()


# 256 x 256 tiles: one round of them, ragged and not
LARGE_TILES = [(900, 10240, 288), (1411, 6432, 416), (4096, 4096, 544)]


@pytest.mark.parametrize("M,N,K,act", [(*s, act) for s in LARGE_TILES for act in ("none", "gelu", "silu", "rms")
                                       if act != "rms" or s[1] % 128 == 0])
def test_gemm_fp4_output_of_large_tiles(M, N, K, act):
    check_gemm(M, N, K, out="fp4", act=act, rms_cols=N if act == "rms" else 0,
               gelu_from=0 if act == "gelu" else None, pad=16 if M % 2 else 0, bias=act != "silu")


@pytest.mark.parametrize("out", ["bf16", "f32", "gated", "fp4"])
@pytest.mark.parametrize("M,N,K", LARGE_TILES)
def test_gemm_scales_at_the_ends_of_large_tiles(M, N, K, out):
    r = rng(M, N, K, 43)
    nb = K // 32
    ends = np.resize([0, 254, 1, 247, 2, 246, 9, 253, 120], nb)
    a = r.integers(0, 16, (M, K)).astype(np.uint8), np.tile(ends, (M, 1)).astype(np.uint8)
    w = r.integers(0, 16, (N, K)).astype(np.uint8), np.tile(254 - ends, (N, 1)).astype(np.uint8)
    check_gemm(M, N, K, out=out, operands=(a, w), bias=False)


def test_gemm_fp4_output_of_nan_rows():
    r = rng(23)
    for M, N in ((4, 128), (300, 2048), (4100, 4352)):
        a, w = operand(r, M, 288), operand(r, N, 288)
        a[1][1, 2] = 255
        got, y, tol = run_gemm(M, N, 288, out="fp4", operands=(a, w))
        rest = np.arange(M) != 1
        assert np.isnan(got[1]).all() and (np.abs(got - y)[rest] <= tol[rest]).all()


@pytest.mark.parametrize("out", ["bf16", "f32", "gated", "fp4"])
@pytest.mark.parametrize("M,N", [(1050, 128), (1030, 1152), (4200, 4224)])
def test_gemm_rows_far_apart(M, N, out):
    """Rows 4 MiB apart, so that offsets pass 32 bits in every operand: the bits of dense rows."""
    torch = torch_cuda()
    K, far = 288, 1 << 22
    r = rng(M, N)
    esize = {"bf16": 2, "gated": 2, "f32": 4, "fp4": 1}[out]
    flags = {"bf16": 0, "f32": binding.EPI_F32, "fp4": binding.EPI_FP4, "gated": binding.EPI_GATED_RES}[out]
    x = dev(torch, r.standard_normal((M, K)).astype(np.float32))
    w = dev(torch, r.standard_normal((N, K)).astype(np.float32))
    gate = dev(torch, r.standard_normal(N).astype(np.float32))
    width = N // 2 if out == "fp4" else N * esize
    start = dev(torch, r.integers(0, 100, (M, width)).astype(np.uint8))
    res = []
    for apart in (False, True):
        bufs = []
        for t in (x, w):
            n = t.shape[0]
            q = torch.empty(n, far if apart else K // 2, dtype=torch.uint8, device="cuda")
            s = torch.empty(n, (1 << 20) if apart else binding.fp4_scale_ld(K), dtype=torch.uint8, device="cuda")
            src = torch.empty(n, far // 4 if apart else K, device="cuda")
            src[:, :K] = t
            binding.quant_fp4(src, q, s, M=n, K=K)
            back = torch.empty_like(src)
            binding.dequant_fp4(q, s, back, M=n, K=K)
            torch.cuda.synchronize()
            bufs += [q, s, back[:, :K].clone()]
            del src, back
        C = torch.empty(M, far if apart else width, dtype=torch.uint8, device="cuda")
        C[:, :width] = start
        cs = torch.zeros(M, binding.fp4_scale_ld(N), dtype=torch.uint8, device="cuda")
        binding.gemm_fp4(bufs[0], bufs[1], bufs[3], bufs[4], None,
                         C.view({1: torch.uint8, 2: torch.int16, 4: torch.float32}[esize]), M=M, N=N, K=K, flags=flags,
                         gate=gate if out == "gated" else None, c_scale=cs if out == "fp4" else None)
        res.append([t.clone() for t in (bufs[0][:, :K // 2], bufs[1][:, :9], bufs[2], bufs[3][:, :K // 2], C[:, :width], cs)])
        del C, bufs, q
    torch.cuda.empty_cache()
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_gemm_no_rows_or_columns():
    torch = torch_cuda()
    z = torch.full((64, 64), FILL, dtype=torch.uint8, device="cuda")
    for M, N in ((0, 64), (4, 0), (0, 0)):
        C = torch.full((4, 64), FILL, dtype=torch.int16, device="cuda")
        binding.gemm_fp4(z, z, z, z, None, C, M=M, N=N, K=64)
        assert int((C != FILL).sum()) == 0


# ---------------------------------------------------------------- rotary positions

def check_rotary(rows, heads, head_dim, rot, *, half, bf16, pairs=None, reach=5000, scale=1.0, pad=0, in_place=False,
                 seed=0, negative=False):
    torch = torch_cuda()
    r = rng(rows, heads, head_dim, rot, seed)
    n = rot // 2
    pairs = [n] if pairs is None else pairs
    x = r.standard_normal((rows, heads * head_dim))
    xb = bf16_bits(x) if bf16 else x.astype(np.float32)
    x64 = bits_to_f64(xb) if bf16 else xb.astype(np.float64)
    pos = r.integers(-reach if negative else 0, reach, (len(pairs), rows)).astype(np.int32)
    freq, one = binding.rotary_freqs(n)
    assert one == 1.0
    y64, d = ref.rotate(x64, pos, freq, heads=heads, head_dim=head_dim, pairs=pairs, half=half, scale=scale)
    ld = heads * head_dim + pad
    X = strided(torch, xb, ld)
    Y = X if in_place else torch.full((rows + 1, ld * (2 if bf16 else 4)), FILL, dtype=torch.uint8, device="cuda").view(
        torch.int16 if bf16 else torch.float32)
    before = X.cpu().numpy().view(np.uint8).reshape(rows, ld, -1)[:, heads * head_dim:]
    binding.rotary(X, Y, pos=dev(torch, pos), freq=dev(torch, freq), rows=rows, heads=heads, head_dim=head_dim,
                   pairs=pairs, layout=binding.ROTARY_HALF if half else binding.ROTARY_INTERLEAVED, scale=scale)
    raw = Y.cpu().numpy().view(np.uint8).reshape(Y.shape[0], ld, -1)
    assert (raw[:rows, heads * head_dim:] == (before if in_place else FILL)).all() and (raw[rows:] == FILL).all()
    got = (host_bf16(Y) if bf16 else Y.cpu().numpy().astype(np.float64))[:rows, :heads * head_dim]
    tol = d + (BF16 if bf16 else 2.0 ** -24) * (np.abs(y64) + d)
    worst = np.max(np.abs(got - y64) - tol) if got.size else 0
    assert worst <= 0, worst
    rest = np.ones((heads, head_dim), bool)
    rest[:, :rot] = False
    assert (got[:, rest.ravel()] == x64[:, rest.ravel()]).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("rows,heads,head_dim,rot,pairs", [
    (1, 1, 128, 128, None), (1, 40, 128, 128, None), (37, 7, 128, 64, None), (5, 3, 64, 64, None), (300, 5, 128, 128, [22, 21, 21]),
    (33, 2, 256, 96, [8, 20, 20]), (70, 3, 96, 20, None), (9, 2, 8, 2, None), (21, 3, 40, 26, [6, 0, 7]), (3, 2, 512, 512, [64, 64, 64, 64]), (6, 3, 128, 100, None),
    (7, 2, 24, 22, None), (4, 5, 16, 10, None), (5, 2, 72, 70, [30, 5]), (2, 3, 128, 126, None), (3, 2, 40, 16, None), (1000, 24, 128, 128, [8, 28, 28])])
def test_rotary(rows, heads, head_dim, rot, pairs, half, bf16, in_place):
    check_rotary(rows, heads, head_dim, rot, half=half, bf16=bf16, pairs=pairs, in_place=in_place,
                 pad=16 if rows % 2 else 0, scale=1.0 if rows % 3 else 1.277)


@pytest.mark.parametrize("half", [True, False])
def test_rotary_far_positions_both_ways(half):
    """Angles of up to 2^24 radians in f32, and of negative positions."""
    check_rotary(200, 2, 128, 128, half=half, bf16=False, reach=1 << 24, negative=True)


def test_rotary_extreme_positions():
    torch = torch_cuda()
    pos = np.array([2 ** 31 - 1, -2 ** 31, 0, 1], np.int32)
    x = np.zeros((4, 8), np.float32)
    x[:, 0] = 1
    freq = np.array([1.0, 0.37, 1e-3, 1e-9])
    x[:, :4] = 1
    y64, d = ref.rotate(x.astype(np.float64), pos[None], freq, heads=1, head_dim=8, pairs=[4], half=True)
    y = torch.empty(4, 8, device="cuda")
    binding.rotary(dev(torch, x), y, pos=dev(torch, pos), freq=dev(torch, freq), rows=4, heads=1, head_dim=8)
    assert (np.abs(y.cpu().numpy() - y64) <= d + 2.0 ** -24 * (np.abs(y64) + d)).all()


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("rot", [0, 36, 48])
def test_rotary_leaves_what_lies_past_it(rot, half):
    """Infinities and NaN (their bits, too) past the rotated width pass through and reach no pair."""
    torch = torch_cuda()
    r = rng(rot, 3)
    bits = bf16_bits(r.standard_normal((6, 2 * 64)))
    v = bits.reshape(6, 2, 64)
    v[..., rot:] = np.resize(np.array([0x7F80, 0xFF80, 0x7FC1, 0xFFC5, 0x0001, 0x8000], np.uint16), v[..., rot:].shape)
    freq = binding.rotary_freqs(rot // 2)[0]
    X = dev(torch, bits)
    Y = torch.zeros_like(X)
    binding.rotary(X, Y, pos=dev(torch, np.arange(6, dtype=np.int32)), freq=dev(torch, freq), rows=6, heads=2, head_dim=64,
                   layout=binding.ROTARY_HALF if half else binding.ROTARY_INTERLEAVED)
    got = Y.cpu().numpy().view(np.uint16).reshape(6, 2, 64)
    assert (got[..., rot:] == v[..., rot:]).all()
    assert np.isfinite(bits_to_f64(got[..., :rot])).all()


def test_rotary_of_columns_into_others_of_the_same_matrix():
    """The queries and keys of a fused projection, beside their values."""
    torch = torch_cuda()
    r = rng(8)
    bits = bf16_bits(r.standard_normal((50, 1024)))
    freq = binding.rotary_freqs(64)[0]
    m = dev(torch, bits)
    pos = np.arange(50, dtype=np.int32)
    binding.rotary(m[:, :384], m[:, 512:], pos=dev(torch, pos), freq=dev(torch, freq), rows=50, heads=3)
    got = host_bf16(m)
    x = bits_to_f64(bits)
    y, d = ref.rotate(x[:, :384], pos[None], freq, heads=3, head_dim=128, pairs=[64], half=True)
    assert (got[:, :512] == x[:, :512]).all() and (got[:, 896:] == x[:, 896:]).all()
    assert (np.abs(got[:, 512:896] - y) <= d + BF16 * (np.abs(y) + d)).all()


def test_rotary_back_and_forth():
    """Negative positions turn back; the rotation keeps a pair's length."""
    torch = torch_cuda()
    x = torch.randn(500, 3 * 128, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    pos = torch.arange(500, device="cuda", dtype=torch.int32) * 97
    freq = torch.from_numpy(binding.rotary_freqs(64)[0]).cuda()
    y, b = torch.empty_like(x), torch.empty_like(x)
    binding.rotary(x, y, pos=pos, freq=freq, rows=500, heads=3)
    binding.rotary(y, b, pos=-pos, freq=freq, rows=500, heads=3)
    # twice the error of one rotation and its rounding, of |a| + |b| <= sqrt(2) times the pair's length
    size = (x.view(500, 3, 2, 64).square().sum(2, keepdim=True).sqrt() * 2 ** 0.5).expand(-1, -1, 2, -1).reshape_as(x)
    assert bool(((b - x).abs() <= 2 * 9.5 * 2.0 ** -24 * size).all())


@pytest.mark.parametrize("rows,heads", [(0, 4), (4, 0)])
def test_rotary_nothing_to_do(rows, heads):
    torch = torch_cuda()
    x = torch.ones(4, 512, device="cuda")
    y = torch.zeros_like(x)
    freq = torch.ones(64, dtype=torch.float64, device="cuda")
    binding.rotary(x, y, pos=torch.ones(4, dtype=torch.int32, device="cuda"), freq=freq, rows=rows, heads=heads)
    assert int((y != 0).sum()) == 0


# ---------------------------------------------------------------- packed attention

def offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def packed(torch, ql, kl, heads, kv_heads=None, *, slots=None, causal=True, bounded=False, pad=0, seed=0, scale=1.0,
           change=None, exact_rows=True):
    """One call against the plain form.  slots: keys lie in a cache of so many rows a sequence.  Two more rows before and
    after the sequences' own hold what nothing may read or write."""
    G = kv_heads or heads
    r = rng(len(ql), sum(ql), sum(kl), heads, seed)
    qoff = offsets(ql) + 2
    koff = (np.arange(len(kl) + 1, dtype=np.int32) * slots if slots else offsets(kl)) + 2
    klen = np.array(kl, np.int32) if slots else None
    Tq, Tk = int(qoff[-1]) + 2, int(koff[-1]) + 2

    def tokens(rows, H, norm):
        x = r.standard_normal((rows, H, 128)) * scale
        if norm:
            x /= np.sqrt((x ** 2).mean(2, keepdims=True) + 1e-6)
        return bf16_bits(x.reshape(rows, H * 128))

    qb, kb, vb = tokens(Tq, heads, bounded), tokens(Tk, G, bounded), tokens(Tk, G, False)
    if slots:   # what lies past a slot's filled rows is never seen
        for z, n in enumerate(kl):
            kb[koff[z] + n:koff[z + 1]] = 0x7FC0
            vb[koff[z] + n:koff[z + 1]] = 0xFF80
    if change:
        change(qb, kb, vb, qoff, koff)
    q, k, v = (bits_to_f64(t) for t in (qb, kb, vb))
    ldo = heads * 128 + pad
    o = torch.full((Tq, ldo * 2), FILL, dtype=torch.uint8, device="cuda").view(torch.int16)
    binding.attention_packed_bf16(
        strided(torch, qb, heads * 128 + pad, 0xFF), strided(torch, kb, G * 128 + 2 * pad, 0xFF),
        strided(torch, vb, G * 128 + 3 * pad, 0xFF), o, qoff=dev(torch, qoff), koff=dev(torch, koff),
        klen=None if klen is None else dev(torch, klen), heads=heads, kv_heads=kv_heads,
        flags=(binding.ATTN_CAUSAL if causal else 0) | (binding.ATTN_BOUNDED_LOGITS if bounded else 0))
    torch.cuda.synchronize()
    raw = o.cpu().numpy().view(np.uint8).reshape(Tq, ldo, 2)
    assert (raw[:2] == FILL).all() and (raw[Tq - 2:] == FILL).all() and (raw[:, heads * 128:] == FILL).all()
    got = host_bf16(o)[2:Tq - 2, :heads * 128]
    with np.errstate(invalid="ignore"):
        y, d = ref.attend(q, k, v, qoff=qoff, koff=koff, heads=heads, kv_heads=kv_heads, klen=klen, causal=causal)
    y, d = y[2:Tq - 2], d[2:Tq - 2]
    if exact_rows:
        tol = d + BF16 * (np.abs(y) + d)
        worst = np.max(np.abs(got - y) - tol, initial=-1)
        assert worst <= 0, (worst, np.argwhere(np.abs(got - y) > tol)[:4])
    return got, y, d


LENGTHS = [
    ([1], [1], 1, 1), ([5], [5], 3, 1), ([128], [128], 2, 2), ([64, 1, 63, 129], [64, 1, 63, 129], 2, 1),
    ([300, 0, 17, 65], [300, 4, 17, 65], 7, 1), ([200, 33], [1000, 33], 6, 2), ([40, 70, 9], [10, 70, 0], 4, 2),
    ([1, 1, 1], [700, 64, 65], 8, 2), ([1, 1, 1, 1], [1, 0, 128, 1000], 5, 1), ([2, 31, 16], [900, 31, 500], 4, 4),
    ([1] * 70, list(range(70)), 4, 2), ([3] * 130, [3 + i % 7 for i in range(130)], 2, 1), ([511, 700], [511, 1300], 10, 2)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bounded", [False, True])
@pytest.mark.parametrize("ql,kl,heads,kv_heads", LENGTHS)
def test_packed_attention(ql, kl, heads, kv_heads, bounded, causal):
    torch = torch_cuda()
    packed(torch, ql, kl, heads, kv_heads, causal=causal, bounded=bounded, pad=8 if len(ql) % 2 else 0)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("ql,kl,heads,kv_heads", LENGTHS)
def test_packed_attention_against_a_cache(ql, kl, heads, kv_heads, causal):
    torch = torch_cuda()
    packed(torch, ql, kl, heads, kv_heads, causal=causal, slots=max(kl) + 3)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bounded", [False, True])
def test_packed_attention_of_long_sequences(bounded, causal):
    torch = torch_cuda()
    packed(torch, [2100, 3], [2900, 2000], 2, 1, causal=causal, bounded=bounded, seed=1)
    packed(torch, [1, 2, 1], [9000, 70, 5000], 4, 1, causal=causal, bounded=bounded, seed=2)
    packed(torch, [100], [8000], 3, 3, causal=causal, bounded=bounded, seed=3)


# long enough for the pipelined loop: whole tiles (odd and even counts of them, ragged ends, short sequences among long
# ones), and shares of few long ones
LONG = [([1100], [1100], 16, 16), ([1500, 40, 2000], [1500, 900, 2001], 12, 4), ([1300, 5], [1216, 1344], 16, 8)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bounded", [False, True])
@pytest.mark.parametrize("ql,kl,heads,kv_heads", LONG)
def test_packed_attention_pipelined(ql, kl, heads, kv_heads, bounded, causal):
    torch = torch_cuda()
    packed(torch, ql, kl, heads, kv_heads, causal=causal, bounded=bounded, pad=8 if len(ql) % 2 else 0)


@pytest.mark.parametrize("bounded,causal", [(False, True), (True, True), (False, False)])
def test_packed_attention_pipelined_shares(bounded, causal):
    torch = torch_cuda()
    packed(torch, [300], [60000], 12, 12, causal=causal, bounded=bounded)


@pytest.mark.parametrize("ql,kl,heads,top,causal", [
    *[([1100], [1100], 16, top, causal) for top in (1.0, 60.0, 90.0, 400.0) for causal in (True, False)],
    ([300], [60000], 12, 60.0, True), ([300], [60000], 12, 400.0, False)])
def test_logits_far_above_the_first_tile_s(ql, kl, heads, top, causal):
    """Logits that rise along the keys by `top`: the first tile's maximum is no shift for the last one's where
    e^top passes 2^100."""
    torch = torch_cuda()

    def rising(qb, kb, vb, qoff, koff):
        n = kb.shape[0]
        ramp = np.linspace(0, top / (2 * np.sqrt(128)), n)[:, None] * np.ones((1, 128))
        for h in range(0, kb.shape[1], 256):        # every other head; the others' logits are ordinary
            kb[:, h:h + 128] = bf16_bits(ramp)
            qb[:, h:h + 128] = bf16_bits(np.full((qb.shape[0], 128), 2.0))
    packed(torch, ql, kl, heads, heads, causal=causal, change=rising)


def test_values_near_the_largest_number():
    """Sums of values of 2^100 and more leave f32's range before they are divided, or pass it in parts."""
    torch = torch_cuda()

    def large(qb, kb, vb, qoff, koff):
        vb[:] = bf16_bits(bits_to_f64(vb) * 2.0 ** 118)
    for ql, kl, heads in (([1100], [1100], 16), ([300], [3000], 2), ([70], [70], 2), ([2], [5000], 2)):
        for causal in (True, False):
            packed(torch, ql, kl, heads, heads, causal=causal, change=large, bounded=True, scale=0.5)


@pytest.mark.parametrize("ql,kl,heads,kv_heads", [([300, 80], [300, 80], 4, 2), ([3, 2], [900, 700], 4, 2), ([20], [500], 4, 2),
                                                  ([2100], [2100], 4, 2), ([1100], [1100], 16, 16)])
def test_keys_that_a_query_does_not_see_do_not_reach_it(ql, kl, heads, kv_heads):
    """Infinities and NaN in later keys' values: causal queries before them keep their results, those from them on do not."""
    torch = torch_cuda()
    for bad in (0x7FC0, 0x7F80, 0xFF80):
        at = []

        def change(qb, kb, vb, qoff, koff):
            for z in range(len(ql)):
                j = kl[z] - max(1, ql[z] // 2)          # seen by the later half of the queries
                vb[koff[z] + j, 5], kb[koff[z] + j, 7] = bad, 0x7FC0 if bad == 0x7FC0 else kb[koff[z] + j, 7]
                at.append(j)
        got, y, d = packed(torch, ql, kl, heads, kv_heads, change=change, exact_rows=False)
        for z, j in enumerate(at):
            rows = np.arange(int(np.sum(ql[:z])), int(np.sum(ql[:z + 1])))
            before = rows[np.arange(ql[z]) + kl[z] - ql[z] < j]
            after = rows[np.arange(ql[z]) + kl[z] - ql[z] >= j]
            g, w, t = got[before], y[before], d[before]
            with np.errstate(invalid="ignore"):
                full, dd = packed(torch, ql, kl, heads, kv_heads, change=lambda qb, kb, vb, qo, ko: clear(vb, kb, ko, at), exact_rows=False)[1:]
            assert (np.abs(g - full[before]) <= dd[before] + BF16 * (np.abs(full[before]) + dd[before])).all()
            bad_col = got[after][:, 5]
            assert (~np.isfinite(bad_col)).all()


def clear(vb, kb, koff, at):
    for z, j in enumerate(at):
        vb[koff[z] + j] = 0
        kb[koff[z] + j] = 0


# few rows a sequence: tiles of one query's heads (16 and 32 of them), of queries without a key, of both kinds in shares
UNSEEN = [([2, 1] + [0] * 5, [40] * 7, 16, 1), ([2] + [0] * 5, [70, 5, 0, 9, 9, 9], 32, 1),
          ([3, 1] + [0] * 6, [9000, 200] + [0] * 6, 16, 1), ([2, 1, 1, 0, 0, 0, 0, 0], [5000, 33, 700, 0, 1, 2, 3, 4], 32, 2),
          ([20, 1, 1, 1], [4, 9, 9, 9], 1, 1), ([70, 1, 2], [30, 9, 3], 1, 1), ([40] + [1] * 30, [3000] + [1] * 30, 2, 2),
          ([5, 1, 0], [64, 32, 33], 8, 1)]


@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("ql,kl,heads,kv_heads", UNSEEN)
def test_values_that_no_row_of_a_tile_sees(ql, kl, heads, kv_heads, slots):
    """Infinities and NaN in the last key, which a sequence's last query alone sees: every other row, whatever tile it
    shares, is as if that key were zeros, and zeros where it sees no key."""
    torch = torch_cuda()
    assert (sum(ql) + 4) * (heads // kv_heads) <= 32 * len(ql)  # (the few-row kernels; `packed` adds four rows)
    kw = dict(slots=max(kl) + 3 if slots else None, exact_rows=False)
    last = np.cumsum(ql)[[n > 0 for n in ql]] - 1
    rest = np.setdiff1d(np.arange(sum(ql)), last)
    keyless = np.concatenate([np.arange(n) + m - n < 0 for n, m in zip(ql, kl)])

    def put(value, key):
        def change(qb, kb, vb, qoff, koff):
            for z, m in enumerate(kl):
                if m:
                    vb[koff[z] + m - 1, 5::128] = value
                    if key:
                        kb[koff[z] + m - 1] = value
        return change
    _, y, d = packed(torch, ql, kl, heads, kv_heads, change=put(0, True), **kw)
    for bad in (0x7FC0, 0x7F80, 0xFF80):
        got = packed(torch, ql, kl, heads, kv_heads, change=put(bad, bad == 0x7FC0), **kw)[0]
        assert (np.abs(got[rest] - y[rest]) <= d[rest] + BF16 * (np.abs(y[rest]) + d[rest])).all()
        assert (got[keyless] == 0).all()
        sees = last[~keyless[last]]
        assert (~np.isfinite(got[sees][:, 5::128])).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bounded", [False, True])
@pytest.mark.parametrize("ql,kl,heads,kv_heads", [
    ([1] * 5, [700, 1, 33, 64, 0], 4, 2), ([3] + [0] * 6, [9000] + [5] * 6, 8, 4), ([9, 2], [40, 300], 2, 2),   # few rows
    ([2, 1, 0, 0, 0], [3000, 40, 0, 0, 0], 32, 2), ([90], [100], 3, 1), ([300], [6000], 2, 2), ([1100], [1100], 16, 16)])
def test_infinite_values_that_a_query_sees(ql, kl, heads, kv_heads, bounded, causal):
    """An infinite value times a probability above zero: infinities of its sign, NaN where both signs meet or a NaN is
    seen, and every other column and row as ever."""
    torch = torch_cuda()
    kw = dict(causal=causal, bounded=bounded, exact_rows=False)
    cols = {3: (0x7F80, None), 40: (None, 0xFF80), 77: (0x7F80, 0xFF80), 100: (0xFF80, 0x7FC0), 127: (None, 0x7F80)}
    first = [m // 3 for m in kl]                    # a key that some see, and the last one
    at = {}

    def put(spoil):
        def change(qb, kb, vb, qoff, koff):
            for z, m in enumerate(kl):
                for c, bad in cols.items():
                    for key, b in zip((first[z], m - 1), bad):
                        if b is not None and m:
                            vb[koff[z] + key, c::128] = b if spoil else 0
            at["vb"], at["koff"] = vb.copy(), koff
        return change
    _, y, d = packed(torch, ql, kl, heads, kv_heads, change=put(False), **kw)
    got = packed(torch, ql, kl, heads, kv_heads, change=put(True), **kw)[0]
    v = bits_to_f64(at["vb"])
    want = np.zeros_like(y)                         # what is not finite adds up as it is
    for z, (n, m) in enumerate(zip(ql, kl)):
        for i in range(n):
            see = min(m, max(0, m - n + 1 + i)) if causal else m
            t = v[at["koff"][z]:at["koff"][z] + see]
            with np.errstate(invalid="ignore"):
                t = np.where(np.isfinite(t), 0, t).sum(0).reshape(kv_heads, 1, 128)
            want[sum(ql[:z]) + i] = np.broadcast_to(t, (kv_heads, heads // kv_heads, 128)).reshape(-1)
    fine = want == 0
    assert (np.abs(got - y) <= d + BF16 * (np.abs(y) + d))[fine].all()
    np.testing.assert_array_equal(got[~fine], want[~fine])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,batch,queries,keys,heads,kv_heads", [
    ("whole", 65, 100, 130, 2, 1), ("whole", 130, 70, 60, 4, 2), ("whole", 200, 45, 90, 1, 1), ("shared", 70, 50, 1300, 1, 1),
    ("shared", 130, 45, 1700, 1, 1)])
def test_many_sequences_of_many_rows(kind, batch, queries, keys, heads, kv_heads, causal):
    """More than 64 sequences in tiles of 128 rows, whole and shared out: lengths around the averages, every fifth
    sequence without queries and every seventh without keys, but for the 64th and the 65th."""
    torch = torch_cuda()
    r = rng(31, batch)
    ql, kl = (r.integers(n // 2, n + n // 2 + 1, batch) for n in (queries, keys))
    ql[::5], kl[::7] = 0, 0
    ql[63:65], kl[63:65] = queries, keys
    rows, Tk = (int(ql.sum()) + 4) * (heads // kv_heads), int(kl.sum()) + 4
    nbytes = binding.attention_packed_ws_bytes(batch=batch, Tq=int(ql.sum()) + 4, Tk=Tk, heads=heads, kv_heads=kv_heads)
    assert rows > 32 * batch and (nbytes > 0) == (kind == "shared")
    packed(torch, list(map(int, ql)), list(map(int, kl)), heads, kv_heads, causal=causal, bounded=batch == 130)


def test_packed_attention_rising_and_overflowing_logits():
    """Logits that rise along the keys, so that the running maximum moves in every tile; logits that overflow to
    infinities of either sign."""
    torch = torch_cuda()

    def rising(qb, kb, vb, qoff, koff):
        n = kb.shape[0]
        ramp = np.linspace(0, 6, n)[:, None] * np.ones((1, 128))
        kb[:, :128] = bf16_bits(ramp + 0.01 * bits_to_f64(kb[:, :128]))
        qb[:, :128] = bf16_bits(1 + 0.01 * bits_to_f64(qb[:, :128]))
    for ql, kl in (([300], [900]), ([2], [4000]), ([150], [150])):
        packed(torch, ql, kl, 1, 1, change=rising)

    def falling_out(qb, kb, vb, qoff, koff):
        qb[:, :128] = bf16_bits(np.full((qb.shape[0], 128), 1e30))
        kb[:, :128] = bf16_bits(np.where(np.arange(kb.shape[0])[:, None] % 3 == 0, 1.0, -1e30) * np.ones((1, 128)))
    for ql, kl in (([130], [400]), ([1], [400]), ([1100], [1100])):
        got, _, _ = packed(torch, ql, kl, 1, 1, causal=False, change=falling_out, exact_rows=False)
        assert np.isfinite(got).all()       # -inf logits count for nothing beside finite ones


def test_offsets_are_clamped():
    """Offsets past the matrices, falling ones and negative lengths stay inside them."""
    torch = torch_cuda()
    r = rng(12)
    q, k, v = (dev(torch, bf16_bits(r.standard_normal((64, 256)))) for _ in range(3))
    want = ref.attend(*(host_bf16(t) for t in (q, k, v)), qoff=[0, 30, 64], koff=[0, 64, 64], heads=2)
    for qoff, koff, klen in (([-5, 30, 1000], [-7, 2 ** 31 - 1, 5], None), ([0, 30, 64], [0, 64, 3], [99, -4]),
                             ([-2 ** 31, 30, 2 ** 31 - 1], [0, 64, 64], [2 ** 31 - 1, -2 ** 31])):
        o = torch.full((64, 256), FILL, dtype=torch.int16, device="cuda")
        binding.attention_packed_bf16(q, k, v, o, qoff=dev(torch, np.array(qoff, np.int32)),
                                      koff=dev(torch, np.array(koff, np.int32)),
                                      klen=None if klen is None else dev(torch, np.array(klen, np.int32)), heads=2)
        y, d = want
        got = host_bf16(o)
        assert (np.abs(got - y) <= d + BF16 * (np.abs(y) + d)).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,batch,Tq,Tk,heads,kv_heads", [
    ("few", 9, 60, 2000, 4, 2), ("few", 140, 200, 900, 2, 2), ("shared", 3, 500, 9000, 2, 1), ("shared", 70, 2300, 100000, 1, 1),
    ("whole", 20, 6000, 2500, 8, 2), ("whole", 100, 9000, 7000, 4, 2), ("whole", 1, 300, 300, 8, 8)])
def test_offsets_that_fall(kind, batch, Tq, Tk, heads, kv_heads, causal):
    """An offset below an earlier one counts as that one: sequences share no row, and each row's result is one
    sequence's, also where the earlier one lies more than 64 sequences before."""
    torch = torch_cuda()
    r = rng(13, batch, Tq)
    rows = Tq * (heads // kv_heads)
    assert (rows <= 32 * batch) == (kind == "few")
    nbytes = binding.attention_packed_ws_bytes(batch=batch, Tq=Tq, Tk=Tk, heads=heads, kv_heads=kv_heads)
    assert (nbytes > 0) == (kind != "whole")
    q, k, v = (dev(torch, bf16_bits(r.standard_normal((t, h * 128)))) for t, h in ((Tq, heads), (Tk, kv_heads), (Tk, kv_heads)))

    def falling(top):
        """Offsets that grow to `top`, every third one thrown anywhere or far outside."""
        at = np.sort(r.integers(0, top + 1, batch + 1))
        at[::3] = r.integers(-top, 2 * top, at[::3].size)
        if batch > 1:
            at[batch // 2] = -2 ** 31
        return at.astype(np.int32)
    for qoff, koff in ((falling(Tq), falling(Tk)), (np.resize([0, Tq], batch + 1), np.resize([0, Tk], batch + 1)),
                       (np.resize([0, Tq // 2, Tq // 4, Tq], batch + 1), np.resize([0, Tk // 3, Tk, 0, Tk // 2], batch + 1))):
        o = torch.full((Tq, heads * 128), FILL, dtype=torch.int16, device="cuda")
        binding.attention_packed_bf16(q, k, v, o, qoff=dev(torch, qoff.astype(np.int32)), koff=dev(torch, koff.astype(np.int32)),
                                      heads=heads, kv_heads=kv_heads, flags=binding.ATTN_CAUSAL if causal else 0)
        qm, km = (np.maximum.accumulate(np.clip(a.astype(np.int64), 0, t)) for a, t in ((qoff, Tq), (koff, Tk)))
        y, d = ref.attend(*(host_bf16(t) for t in (q, k, v)), qoff=qm, koff=km, heads=heads, kv_heads=kv_heads, causal=causal)
        raw, got = o.cpu().numpy(), host_bf16(o)
        own = np.arange(Tq)[(np.arange(Tq) >= qm[0]) & (np.arange(Tq) < qm[-1])]
        rest = np.setdiff1d(np.arange(Tq), own)
        assert (np.abs(got[own] - y[own]) <= d[own] + BF16 * (np.abs(y[own]) + d[own])).all()
        assert (raw[rest] == FILL).all()


def test_no_sequences_queries_or_keys():
    torch = torch_cuda()
    t = torch.ones(8, 256, dtype=torch.int16, device="cuda")
    for qoff, koff, Tq, Tk in (([0], [0], 8, 8), ([0, 0], [0, 8], 0, 8), ([0, 0, 0], [0, 8, 8], 8, 8)):
        o = torch.full((8, 256), FILL, dtype=torch.int16, device="cuda")
        binding.attention_packed_bf16(t, t, t, o, qoff=dev(torch, np.array(qoff, np.int32)),
                                      koff=dev(torch, np.array(koff, np.int32)), heads=2, Tq=Tq, Tk=Tk)
        assert int((o != FILL).sum()) == 0
    o = torch.full((8, 256), FILL, dtype=torch.int16, device="cuda")
    binding.attention_packed_bf16(t, t, t, o, qoff=dev(torch, np.array([0, 5], np.int32)),
                                  koff=dev(torch, np.array([0, 0], np.int32)), heads=2, Tk=0)
    assert int((o[:5] != 0).sum()) == 0 and int((o[5:] != FILL).sum()) == 0


@pytest.mark.parametrize("Lq", [1, 200])
def test_packed_rows_far_apart(Lq):
    """Rows of keys so far apart that offsets pass 32 bits: the bits of dense rows."""
    torch = torch_cuda()
    n, far = 1500, (1 << 22) - 8
    g = torch.Generator("cuda").manual_seed(3)
    k, v = (torch.randn(n, 128, device="cuda", generator=g).bfloat16() for _ in range(2))
    q = torch.randn(Lq, 256, device="cuda", generator=g).bfloat16()
    qoff, koff = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, Lq], [700, n]))
    res = []
    for apart in (False, True):
        kk, vv = (torch.empty(n, far if apart else 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        kk[:, :128], vv[:, :128] = k, v
        o = torch.empty_like(q)
        binding.attention_packed_bf16(q, kk, vv, o, qoff=qoff, koff=koff, heads=2, kv_heads=1, flags=binding.ATTN_CAUSAL)
        res.append(o.clone())
        del kk, vv
    torch.cuda.empty_cache()
    assert torch.equal(*res)


def test_packed_attention_is_the_dense_one():
    """A sequence of every query and key, not causal: the existing kernel's result up to both their roundings."""
    torch = torch_cuda()
    r = rng(40)
    qb, kb, vb = (bf16_bits(r.standard_normal((500, 3 * 128))) for _ in range(3))
    q, k, v = (dev(torch, t) for t in (qb, kb, vb))
    o, p = torch.empty_like(q), torch.empty_like(q)
    off = dev(torch, np.array([0, 500], np.int32))
    binding.attention_packed_bf16(q, k, v, p, qoff=off, koff=off, heads=3)
    binding.attention_bf16(q, k, v, o, Lq=500, Lk=500, heads=3, ldq=384, ldk=384, ldv=384, ldo=384,
                           vt_ws=torch.empty(3 * 128 * 512, dtype=torch.int16, device="cuda"))
    torch.cuda.synchronize()
    y, d = ref.attend(*(bits_to_f64(t) for t in (qb, kb, vb)), qoff=[0, 500], koff=[0, 500], heads=3)
    assert (np.abs(host_bf16(o) - host_bf16(p)) <= 2 * (d + BF16 * (np.abs(y) + d))).all()


# ---------------------------------------------------------------- together

class Layer:
    """One layer of a prompt encoder over packed prompts: 4-bit products, rotary positions, causal attention with
    grouped heads, an MLP whose middle stays in 4 bits; its buffers and workspaces."""

    def __init__(self, torch, seed, lengths=(70, 1, 200, 33), heads=4, kv_heads=2, F=512):
        r = rng(seed, 21)
        self.t, self.lengths, self.heads, self.G, self.F = torch, lengths, heads, kv_heads, F
        H = self.H = heads * 128
        L = self.L = sum(lengths)
        self.N = H + 2 * kv_heads * 128
        self.w = {name: self.rows(r.standard_normal((n, k)) / np.sqrt(k))
                  for name, n, k in (("qkv", self.N, H), ("o", H, H), ("up", F, H), ("down", H, F))}
        self.gate = dev(torch, r.standard_normal(H).astype(np.float32))
        self.x0 = dev(torch, bf16_bits(r.standard_normal((L, H))))
        self.off = dev(torch, offsets(lengths))
        self.pos = dev(torch, np.concatenate([np.arange(n) for n in lengths]).astype(np.int32))
        freq, self.scale = binding.rotary_freqs(64, method=binding.ROTARY_PARTS, factor=4.0, context=64.0)
        self.freq = dev(torch, freq)
        e = lambda *s, dt=torch.int16: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        self.x, self.qkv, self.raw, self.att = e(L, H), e(L, self.N), e(L, self.N), e(L, H)
        self.q4 = [e(L, n // 2, dt=torch.uint8) for n in (H, H, H, F)]
        self.s4 = [e(L, binding.fp4_scale_ld(n), dt=torch.uint8) for n in (H, H, H, F)]
        self.ws = e(max(16, binding.attention_packed_ws_bytes(batch=len(lengths), Tq=L, Tk=L, heads=heads, kv_heads=kv_heads)),
                    dt=torch.uint8)

    def rows(self, x):
        c, s = ref.quantise(x)
        return dev(self.t, ref.pack(c)), dev(self.t, padded_scale(s, x.shape[1])), ref.values(c, s)

    def linear(self, i, name, out, N, K, **kw):
        w = self.w[name]
        binding.gemm_fp4(self.q4[i], self.s4[i], w[0], w[1], None, out, M=self.L, N=N, K=K, stream=self.stream, **kw)

    def quant(self, i, x, K):
        binding.quant_fp4(x, self.q4[i], self.s4[i], M=self.L, K=K, stream=self.stream)

    def run(self, stream=None):
        self.stream, H, F, L, G = stream, self.H, self.F, self.L, self.G
        self.x.copy_(self.x0)
        self.quant(0, self.x, H)
        turned = (self.heads + G) * 128
        self.linear(0, "qkv", self.raw, self.N, H, rms_cols=turned)
        self.qkv.copy_(self.raw)
        both = self.qkv[:, :turned]
        binding.rotary(both, both, pos=self.pos, freq=self.freq, scale=self.scale, rows=L, heads=self.heads + G, stream=stream)
        q, k, v = self.qkv[:, :H], self.qkv[:, H:turned], self.qkv[:, turned:]
        binding.attention_packed_bf16(q, k, v, self.att, qoff=self.off, koff=self.off, heads=self.heads, kv_heads=G,
                                      flags=binding.ATTN_CAUSAL, ws=self.ws, stream=stream)
        self.quant(1, self.att, H)
        self.linear(1, "o", self.x, H, H, flags=binding.EPI_GATED_RES, gate=self.gate)
        self.quant(2, self.x, H)
        self.linear(2, "up", self.q4[3], F, H, flags=binding.EPI_FP4, c_scale=self.s4[3], gelu_from=0)
        self.linear(3, "down", self.x, H, F, flags=binding.EPI_GATED_RES, gate=self.gate)
        return self.x

    def host4(self, i):
        q, s = self.q4[i].cpu().numpy(), self.s4[i].cpu().numpy()
        return ref.values(ref.unpack(q), s[:, :q.shape[1] // 16])

    def step4(self, i, y, d):
        """Half the distance between the codes around y +- d."""
        q, s = self.q4[i], self.s4[i].cpu().numpy()
        s = np.repeat(2.0 ** (s[:, :q.shape[1] // 16].astype(np.float64) - 127), 32, 1)
        z = (np.abs(y) + d) / s
        return np.where(z <= 2, 0.25, np.where(z <= 4, 0.5, 1.0)) * s


def test_a_layer_of_a_prompt_encoder():
    """Each stage against float64 on the device's own input of that stage, so that every tolerance is one stage's."""
    torch = torch_cuda()
    b = Layer(torch, 1)
    H, L, G, turned = b.H, b.L, b.G, (b.heads + b.G) * 128
    out = host_bf16(b.run())
    x0 = host_bf16(b.x0)
    np.testing.assert_array_equal(b.host4(0), ref.values(*ref.quantise(x0)))
    y, d = ref8.product(b.host4(0), b.w["qkv"][2], None, f32=True, rms_cols=turned)
    raw = host_bf16(b.raw)
    assert (np.abs(raw - y) <= d + BF16 * (np.abs(y) + d) + 1e-30).all()
    qkv = host_bf16(b.qkv)
    y, d = ref.rotate(raw[:, :turned], b.pos.cpu().numpy()[None], b.freq.cpu().numpy(), heads=b.heads + G, head_dim=128,
                      pairs=[64], half=True, scale=b.scale)
    assert (np.abs(qkv[:, :turned] - y) <= d + BF16 * (np.abs(y) + d)).all()
    assert (qkv[:, turned:] == raw[:, turned:]).all()
    off = b.off.cpu().numpy()
    y, d = ref.attend(qkv[:, :H], qkv[:, H:turned], qkv[:, turned:], qoff=off, koff=off, heads=b.heads, kv_heads=G, causal=True)
    assert (np.abs(host_bf16(b.att) - y) <= d + BF16 * (np.abs(y) + d)).all()
    np.testing.assert_array_equal(b.host4(1), ref.values(*ref.quantise(host_bf16(b.att))))
    gate = b.gate.cpu().numpy().astype(np.float64)
    y, d = ref8.product(b.host4(1), b.w["o"][2], None, f32=True)
    mid, dm = x0 + gate * y, np.abs(gate) * d + 2.0 ** -22 * (np.abs(x0) + np.abs(gate * y))
    dm = dm + BF16 * (np.abs(mid) + dm)
    m4 = b.host4(2)
    assert (np.abs(m4 - mid) <= dm + b.step4(2, mid, dm)).all()
    y, d = ref8.product(m4, b.w["up"][2], None, f32=True, gelu_from=0)
    u4 = b.host4(3)
    assert (np.abs(u4 - y) <= d + b.step4(3, y, d)).all()
    y, d = ref8.product(u4, b.w["down"][2], None, f32=True)
    fin = mid + gate * y
    tol = dm + np.abs(gate) * d + 2.0 ** -22 * (np.abs(mid) + np.abs(gate * y))
    assert (np.abs(out - fin) <= tol + BF16 * (np.abs(fin) + tol)).all()


def test_tokens_one_by_one_are_the_prompt_at_once():
    """Keys and values appended to a cache, each token's query alone: the rows of the whole prompt, up to both calls'
    roundings."""
    torch = torch_cuda()
    r = rng(50)
    heads, G, n, slots = 6, 2, 150, 160
    qb, kb, vb = (bf16_bits(r.standard_normal((2 * n, h * 128))) for h in (heads, G, G))
    q, k, v = (dev(torch, t) for t in (qb, kb, vb))
    off = dev(torch, np.array([0, n, 2 * n], np.int32))
    whole = torch.empty_like(q)
    shape = dict(heads=heads, kv_heads=G, flags=binding.ATTN_CAUSAL)
    binding.attention_packed_bf16(q, k, v, whole, qoff=off, koff=off, **shape)
    ck, cv = (torch.full((2 * slots, G * 128), 0x7FC0, dtype=torch.int16, device="cuda") for _ in range(2))
    one = torch.empty_like(q)
    qoff, koff = (dev(torch, np.array(t, np.int32)) for t in ([0, 1, 2], [0, slots, 2 * slots]))
    for i in range(n):
        rows = [i, n + i]
        ck[[i, slots + i]], cv[[i, slots + i]] = k[rows], v[rows]
        o = torch.empty(2, heads * 128, dtype=torch.int16, device="cuda")
        binding.attention_packed_bf16(q[rows].contiguous(), ck, cv, o, qoff=qoff, koff=koff,
                                      klen=torch.full((2,), i + 1, dtype=torch.int32, device="cuda"), **shape)
        one[rows] = o
    y, d = ref.attend(*(bits_to_f64(t) for t in (qb, kb, vb)), qoff=[0, n, 2 * n], koff=[0, n, 2 * n], heads=heads,
                      kv_heads=G, causal=True)
    for got in (whole, one):
        assert (np.abs(host_bf16(got) - y) <= d + BF16 * (np.abs(y) + d)).all()


# lengths whose attention shares its keys out, has few rows a sequence, or goes whole tiles
LAYERS = [(70, 1, 200, 33), (1, 2, 1, 3, 1, 1), (2100,)]


def test_layers_captured_into_graphs():
    """Layers captured into graphs with their own workspaces, replayed in turn with eager work between: every
    replay gives the eager bits."""
    torch = torch_cuda()
    layers = [Layer(torch, s, lengths=n) for s, n in enumerate(LAYERS, 2)]
    want = [b.run().clone() for b in layers]
    other = Layer(torch, 9)
    stream = torch.cuda.Stream()
    graphs = []
    torch.cuda.synchronize()
    for b in layers:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            b.run(stream)
        graphs.append(g)
    for i in range(4):
        for b, g, w in zip(layers, graphs, want):
            b.x.zero_()
            b.ws.fill_(0xFF)
            g.replay()
            other.run()
            torch.cuda.synchronize()
            assert torch.equal(b.x, w), i


def test_layers_on_two_streams():
    torch = torch_cuda()
    layers = [Layer(torch, s, lengths=n) for s, n in ((5, (400, 900)), (6, (1, 1, 5)))]
    want = [b.run().clone() for b in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for b, s in zip(layers, streams):
        for _ in range(6):
            with torch.cuda.stream(s):
                b.run(s)
    torch.cuda.synchronize()
    for b, w in zip(layers, want):
        assert torch.equal(b.x, w)


@pytest.mark.parametrize("ql,kl,heads,kv_heads", [([1, 1, 3], [5000, 20, 900], 4, 1), ([300], [9000], 4, 2), ([20, 9], [700, 650], 8, 8),
                                                 ([1] * 200, [17] * 200, 4, 4)])
@pytest.mark.parametrize("bounded", [False, True])
def test_packed_attention_in_a_workspace_of_its_size(ql, kl, heads, kv_heads, bounded):
    """A workspace between guards: nothing before or behind it changes, and what it held does not matter."""
    torch = torch_cuda()
    r = rng(60, len(ql))
    q, k, v = (dev(torch, bf16_bits(r.standard_normal((n, h * 128)) / 4)) for n, h in ((sum(ql), heads), (sum(kl), kv_heads),
                                                                                     (sum(kl), kv_heads)))
    nbytes = binding.attention_packed_ws_bytes(batch=len(ql), Tq=sum(ql), Tk=sum(kl), heads=heads, kv_heads=kv_heads)
    assert nbytes > 0
    res = []
    for fill in (0x00, 0xFF, 0x7F):
        buf = torch.full((nbytes + 512,), fill, dtype=torch.uint8, device="cuda")
        o = torch.zeros_like(q)
        binding.attention_packed_bf16(q, k, v, o, qoff=dev(torch, offsets(ql)), koff=dev(torch, offsets(kl)), heads=heads,
                                      kv_heads=kv_heads, ws=buf[256:256 + nbytes],
                                      flags=binding.ATTN_CAUSAL | (binding.ATTN_BOUNDED_LOGITS if bounded else 0))
        assert bool((buf[:256] == fill).all()) and bool((buf[256 + nbytes:] == fill).all())
        res.append(o)
    assert torch.equal(res[0], res[1]) and torch.equal(res[0], res[2])


@pytest.mark.parametrize("n,heads,kv_heads,Tk", [(1, 4, 4, 500), (64, 2, 1, 5000), (300, 4, 2, 600)])
def test_sequences_that_overlap_stay_inside(n, heads, kv_heads, Tk):
    """Offsets that fall back name the same rows many times: nothing outside o's rows and the workspace is written."""
    torch = torch_cuda()
    g = torch.Generator("cuda").manual_seed(n)
    batch = 41
    q, k, v = (torch.randn(t, h * 128, device="cuda", generator=g).bfloat16() for t, h in ((n, heads), (Tk, kv_heads), (Tk, kv_heads)))
    qoff = torch.tensor([0, n] * (batch // 2) + [0, n], dtype=torch.int32, device="cuda")
    koff = torch.tensor([0, Tk] * (batch // 2) + [0, Tk], dtype=torch.int32, device="cuda")
    nbytes = binding.attention_packed_ws_bytes(batch=batch, Tq=n, Tk=Tk, heads=heads, kv_heads=kv_heads)
    buf = torch.full((nbytes + 512,), FILL, dtype=torch.uint8, device="cuda")
    o = torch.full((n + 2, heads * 128), 7.0, device="cuda", dtype=torch.bfloat16)
    binding.attention_packed_bf16(q, k, v, o[1:n + 1], qoff=qoff, koff=koff, heads=heads, kv_heads=kv_heads,
                                  ws=buf[256:256 + nbytes] if nbytes else None)
    assert bool((buf[:256] == FILL).all()) and bool((buf[256 + nbytes:] == FILL).all())
    assert bool((o[0] == 7).all()) and bool((o[n + 1] == 7).all())


def test_calls_lie_on_the_stream_they_are_given():
    """Calls behind others on a stream see their results."""
    torch = torch_cuda()
    s = torch.cuda.Stream()
    x = torch.zeros(4096, 4096, device="cuda")
    q = torch.empty(4096, 2048, dtype=torch.uint8, device="cuda")
    sc = torch.empty(4096, 128, dtype=torch.uint8, device="cuda")
    y = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            x.add_(1.0)
    binding.quant_fp4(x, q, sc, M=4096, K=4096, stream=s)
    binding.dequant_fp4(q, sc, y, M=4096, K=4096, stream=s)
    s.synchronize()
    assert bool((y == 16.0).all())          # 20 = 5 * 4: a tie, to the even code
