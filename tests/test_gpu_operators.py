"""8-bit rows and their products, block selection and sparse attention against
plain float64 forms, through the C ABI, at the sizes, strides and masks where
they can go wrong."""
import numpy as np
import pytest

from paper_2608_09231_amd import binding
from tests import _operators as ref
from tests._gpu import dev, host_bf16, torch_cuda
from tests.test_gpu_kernels import bf16_bits, bits_to_f64

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8    # half a step, relative
FILL = 0x5A


def rng(*seed):
    return np.random.default_rng([77, *seed])


def strided(torch, a, ld, fill=FILL):
    """A device buffer of rows `ld` elements apart whose gaps hold `fill` bytes."""
    M, K = a.shape
    buf = np.full((M, ld), 0, a.dtype)
    buf.view(np.uint8)[:] = fill
    buf[:, :K] = a
    return dev(torch, buf)


def run_quant(torch, x, *, ldx=None, ldq=None, lds=None):
    M, K = x.shape
    ld = ldx or K
    q = torch.full((M, ldq or K), FILL, dtype=torch.uint8, device="cuda")
    s = torch.full((M, lds or binding.fp8_scale_ld(K)), FILL, dtype=torch.uint8, device="cuda")
    binding.quant_fp8(strided(torch, x, ld), q, s, M=M, K=K)
    q, s = q.cpu().numpy(), s.cpu().numpy()
    nb = -(-K // 128)
    assert (q[:, K:] == FILL).all() and (s[:, nb:] == FILL).all()
    return q[:, :K], s[:, :nb]


def check_quant(torch, x, **kw):
    q, s = run_quant(torch, x, **kw)
    x64 = bits_to_f64(x) if x.dtype == np.uint16 else x.astype(np.float64)
    rq, rs = ref.quantise(x64)
    np.testing.assert_array_equal(s, rs)
    # -0 and +0 are one value; any NaN byte is a NaN
    np.testing.assert_array_equal(ref.TABLE[q], ref.TABLE[rq])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,ldx,ldq,lds", [
    (1, 16, None, None, None), (3, 128, None, None, None), (5, 144, 160, 176, 8), (37, 2608, 2616, 2624, 28),
    (130, 1040, None, None, None), (1030, 1008, 1024, 1008, 12)])
def test_quant_rows(M, K, ldx, ldq, lds, dtype):
    torch = torch_cuda()
    r = rng(M, K)
    x = r.standard_normal((M, K)) * np.exp(3 * r.standard_normal((M, 1))) * np.exp(r.standard_normal(K))
    check_quant(torch, bf16_bits(x) if dtype == "bf16" else x.astype(np.float32), ldx=ldx, ldq=ldq, lds=lds)


def test_quant_borders_zeros_and_extremes():
    """Blocks whose largest value is a scale's last (448 * 2^e) or the next above it, ties between two e4m3
    values, blocks of zeros, the type's smallest and largest values."""
    torch = torch_cuda()
    rows = []
    for e in (-150, -136, -135, -126, -20, 0, 60, 119):
        top = np.float32(448) * np.float32(2.0) ** e if e > -149 else np.float32(1e-45)
        for a in (top, np.nextafter(top, np.float32(np.inf)), np.nextafter(top, np.float32(0))):
            row = np.zeros(128, np.float32)
            row[17] = -a
            row[:8] = a * np.array([1, 15 / 16, 0.5, 0.53125, 0.59375, 1 / 448, 1 / 458752, 3 / 917504], np.float32)
            rows.append(row)
    rows.append(np.zeros(128, np.float32))
    rows.append(np.full(128, np.finfo(np.float32).max))
    rows.append(np.full(128, -0.0, np.float32))
    check_quant(torch, np.stack(rows).astype(np.float32))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_quant_block_that_is_not_finite(bad):
    torch = torch_cuda()
    x = rng(5).standard_normal((6, 512)).astype(np.float32)
    x[2, 200] = bad
    check_quant(torch, x)
    check_quant(torch, bf16_bits(np.where(np.isfinite(x), x, 0)) | np.where(np.isnan(x), 0x7FC0, np.where(
        np.isinf(x), np.where(x > 0, 0x7F80, 0xFF80), 0)).astype(np.uint16))


def test_quant_nothing_to_do():
    torch = torch_cuda()
    x = torch.zeros(4, 32, device="cuda")
    q = torch.full((4, 32), FILL, dtype=torch.uint8, device="cuda")
    s = torch.full((4, 4), FILL, dtype=torch.uint8, device="cuda")
    binding.quant_fp8(x, q, s, M=0, K=32)
    binding.quant_fp8(x, q, s, M=4, K=0)
    assert int((q != FILL).sum()) == 0 and int((s != FILL).sum()) == 0


# ---------------------------------------------------------------- products

def operand(r, M, K, spread=1.0):
    """8-bit rows with row and block scales of their own."""
    x = r.standard_normal((M, K)) * np.exp(spread * r.standard_normal((M, 1))) / np.sqrt(K)
    return ref.quantise(bits_to_f64(bf16_bits(x)))


def padded_scale(s, K, ld=None):
    out = np.full((s.shape[0], ld or binding.fp8_scale_ld(K)), 255, np.uint8)   # NaN scales past the last block
    out[:, :s.shape[1]] = s
    return out


def run_gemm(M, N, K, *, out="bf16", act="none", rms_cols=0, gelu_from=None, bias=True, gap_at=0, gap=0, pad=0,
             seed=0, operands=None, stream=None):
    torch = torch_cuda()
    r = rng(M, N, K, seed)
    (aq, as_), (wq, ws) = operands or (operand(r, M, K), operand(r, N, K))
    b_bits = bf16_bits(0.1 * r.standard_normal(N))
    b = bits_to_f64(b_bits)
    a, w = ref.values(aq, as_), ref.values(wq, ws)
    y, d = ref.product(a, w, b if bias else None, f32=out == "f32", act=act, rms_cols=rms_cols, gelu_from=gelu_from)
    flags = {"bf16": 0, "f32": binding.EPI_F32, "fp8": binding.EPI_FP8, "gated": binding.EPI_GATED_RES}[out]
    flags |= binding.EPI_SILU if act == "silu" else 0
    width = N + gap + pad
    esize = {"bf16": 2, "gated": 2, "f32": 4, "fp8": 1}[out]
    old_bits = bf16_bits(r.standard_normal((M + 1, width)))
    C = dev(torch, old_bits) if out == "gated" else torch.full((M + 1, width * esize), FILL, dtype=torch.uint8,
                                                               device="cuda")
    if out != "gated":
        C = C.view({"bf16": torch.int16, "f32": torch.float32, "fp8": torch.uint8}[out])
    gate = r.standard_normal(N).astype(np.float32)
    cs = torch.full((M + 1, binding.fp8_scale_ld(N)), FILL, dtype=torch.uint8, device="cuda") if out == "fp8" else None
    binding.gemm_fp8(strided(torch, aq, K + (16 if pad else 0), 0x7F), dev(torch, padded_scale(as_, K)),
                     strided(torch, wq, K + (48 if pad else 0), 0x7F), dev(torch, padded_scale(ws, K)),
                     dev(torch, b_bits) if bias else None, C, M=M, N=N, K=K, flags=flags, c_scale=cs,
                     gate=dev(torch, gate) if out == "gated" else None, rms_cols=rms_cols, gelu_from=gelu_from,
                     gap_at=gap_at, gap=gap)
    torch.cuda.synchronize()
    host = C.cpu().numpy()
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
        if out == "fp8":
            scale = cs.cpu().numpy()
            nb = N // 128
            assert (scale[M] == FILL).all() and (scale[:, nb:] == FILL).all()
            scale = scale[:M, :nb]
            got = ref.values(host[:M, :N], scale)
            # the scale is that of the largest value, up to what that may be off
            s = np.repeat(2.0 ** (scale.astype(np.float64) - 127), 128, 1)
            top = np.repeat((np.abs(y)).reshape(M, nb, 128).max(2), 128, 1)
            off = np.repeat(d.reshape(M, nb, 128).max(2), 128, 1)
            fits = (top - off <= 448 * s) & ((top + off > 224 * s) | (scale.repeat(128, 1) == 0))
            assert (fits | np.isnan(top)).all()     # (rows that are not finite have their own test)
            tol = np.maximum(2.0 ** -4 * (np.abs(y) + d), 2.0 ** -10 * s) + d
            return host[:M], scale, got, y, tol
        got = (host_bf16(C) if out == "bf16" else host.astype(np.float64))[:M, cols]
    tol = d + (2.0 ** -24 if out == "f32" else BF16) * (np.abs(y) + d) + 1e-30
    return host[:M], None, got, y, tol


def check_gemm(*a, **kw):
    _, _, got, y, tol = run_gemm(*a, **kw)
    worst = np.max(np.abs(got - y) / tol)
    assert worst <= 1, f"{worst} of the tolerance at {np.unravel_index(np.argmax(np.abs(got - y) / tol), y.shape)}"


# one size for each kernel and edge: few rows (one and two blocks of 16), tiles of 64 and 128 rows, 256 x 256 tiles;
# blocks of K cut short, fewer slices than stages
SIZES = [(1, 8, 16), (1, 1000, 2320), (16, 72, 128), (17, 264, 400), (40, 136, 5120), (300, 2056, 272), (513, 1416, 1040),
         (70, 13824, 656), (1500, 5640, 144), (2100, 4104, 528)]
RING = [(4100, 4360, 16), (4100, 4360, 144), (4096, 4096, 1152), (4353, 3848, 912)]


@pytest.mark.parametrize("out", ["bf16", "f32", "gated"])
@pytest.mark.parametrize("M,N,K", SIZES + RING)
def test_gemm_sizes(M, N, K, out):
    check_gemm(M, N, K, out=out, pad=8 if (M + K) % 3 else 0, bias=(M % 4) > 0)


# sizes whose tiles of 128 x 128 (510) and of 256 x 128 (160) fill the chip's CUs once
@pytest.mark.parametrize("out", ["bf16", "f32", "gated"])
@pytest.mark.parametrize("M,N,K", [(1920, 4352, 400), (1913, 4312, 1168), (512, 10240, 272), (500, 10232, 1168)])
def test_gemm_sizes_of_one_round(M, N, K, out):
    check_gemm(M, N, K, out=out, pad=8 if M % 8 else 0, bias=M % 8 == 0)


# narrow tiles of 64 and 128 columns; f32 outputs whose K is shared by two groups of waves, the second with one to
# as many slices as the first
@pytest.mark.parametrize("out", ["bf16", "f32", "gated"])
@pytest.mark.parametrize("M,N,K", [(5, 9000, 400), (16, 20008, 272), (100, 3000, 656), (300, 2056, 1936), (900, 2000, 1040),
                                   (897, 1992, 1552), (900, 2040, 2064), (850, 2048, 2048)])
def test_gemm_sizes_of_few_tiles(M, N, K, out):
    check_gemm(M, N, K, out=out, pad=8 if M % 8 else 0, bias=M % 8 == 0)


def test_gemm_f32_of_wide_tiles_norm_gelu_and_gap():
    """Tiles of 128 x 128: 512 and more of them."""
    for M, N, K in ((4096, 2048, 400), (4090, 2304, 656), (8192, 1408, 144)):
        check_gemm(M, N, K, out="f32", rms_cols=256, gelu_from=384, gap_at=384, gap=128, seed=1)
    check_gemm(4090, 2048, 656, out="f32", rms_cols=128, gelu_from=204, gap_at=140, gap=12, pad=4, seed=2)
    check_gemm(4090, 2040, 784, out="f32", act="silu", seed=3)
    a, w = operand(rng(1), 4096, 1168), operand(rng(2), 2048, 1168)
    a[1][700, 9] = 255
    _, _, got, y, tol = run_gemm(4096, 2048, 1168, out="f32", operands=(a, w))
    rest = np.arange(4096) != 700
    assert np.isnan(got[700]).all() and (np.abs(got - y)[rest] <= tol[rest]).all()


def test_gemm_f32_of_shared_k_norm_gelu_and_gap():
    check_gemm(900, 2048, 1168, out="f32", rms_cols=256, gelu_from=384, gap_at=384, gap=128, seed=1)
    check_gemm(900, 2048, 1296, out="f32", rms_cols=128, gelu_from=204, gap_at=140, gap=12, pad=4, seed=2)
    check_gemm(900, 2048, 1168, out="f32", act="silu", seed=3)
    a, w = operand(rng(1), 900, 1168), operand(rng(2), 2048, 1168)
    a[1][700, 9] = 255
    _, _, got, y, tol = run_gemm(900, 2048, 1168, out="f32", operands=(a, w))
    rest = np.arange(900) != 700
    assert np.isnan(got[700]).all() and (np.abs(got - y)[rest] <= tol[rest]).all()


@pytest.mark.parametrize("act", ["none", "gelu", "rms"])
@pytest.mark.parametrize("M,N,K", [(1913, 4352, 656), (500, 10240, 400)])
def test_gemm_fp8_output_of_one_round(M, N, K, act):
    check_gemm(M, N, K, out="fp8", act=act, rms_cols=N if act == "rms" else 0, gelu_from=0 if act == "gelu" else None)


@pytest.mark.parametrize("out", ["bf16", "f32", "gated", "fp8"])
@pytest.mark.parametrize("M,N", [(1050, 128), (1030, 1152), (4200, 4224)])
def test_gemm_rows_far_apart(M, N, out):
    """Rows 4 MiB apart, so that offsets pass 32 bits in every operand: the bits of dense rows."""
    torch = torch_cuda()
    K, far = 272, 1 << 22
    r = rng(M, N)
    esize = {"bf16": 2, "gated": 2, "f32": 4, "fp8": 1}[out]
    flags = {"bf16": 0, "f32": binding.EPI_F32, "fp8": binding.EPI_FP8, "gated": binding.EPI_GATED_RES}[out]
    x = dev(torch, r.standard_normal((M, K)).astype(np.float32))
    w = dev(torch, r.standard_normal((N, K)).astype(np.float32))
    gate = dev(torch, r.standard_normal(N).astype(np.float32))
    start = dev(torch, r.integers(0, 100, (M, N * esize)).astype(np.uint8))
    res = []
    for apart in (False, True):
        bufs = []
        for t in (x, w):
            n = t.shape[0]
            q = torch.empty(n, far if apart else K, dtype=torch.uint8, device="cuda")
            s = torch.empty(n, binding.fp8_scale_ld(K), dtype=torch.uint8, device="cuda")
            src = torch.empty(n, far // 4 if apart else K, device="cuda")
            src[:, :K] = t
            binding.quant_fp8(src, q, s, M=n, K=K)
            torch.cuda.synchronize()
            bufs += [q, s]
        del src
        C = torch.empty(M, far if apart else N * esize, dtype=torch.uint8, device="cuda")
        C[:, :N * esize] = start
        cs = torch.zeros(M, binding.fp8_scale_ld(N), dtype=torch.uint8, device="cuda")
        binding.gemm_fp8(bufs[0], bufs[1], bufs[2], bufs[3], None,
                         C.view({1: torch.uint8, 2: torch.int16, 4: torch.float32}[esize]), M=M, N=N, K=K, flags=flags,
                         gate=gate if out == "gated" else None, c_scale=cs if out == "fp8" else None)
        res.append([t.clone() for t in (bufs[0][:, :K], bufs[1][:, :3], bufs[2][:, :K], C[:, :N * esize], cs)])
        del C, bufs, q
    torch.cuda.empty_cache()
    for a, b in zip(*res):
        assert torch.equal(a, b)


@pytest.mark.parametrize("act", ["none", "gelu", "silu", "rms"])
@pytest.mark.parametrize("M,N,K", [(1, 128, 528), (19, 256, 400), (257, 1152, 272), (700, 7040, 1040), (4097, 4480, 272)])
def test_gemm_fp8_output(M, N, K, act):
    check_gemm(M, N, K, out="fp8", act=act, rms_cols=N if act == "rms" else 0, gelu_from=0 if act == "gelu" else None,
               pad=16 if M % 2 else 0)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(3, 512, 400), (30, 640, 272), (300, 2688, 400), (2100, 4224, 272), (4100, 4352, 272)])
def test_gemm_norm_gelu_and_gap(M, N, K, out):
    """A fused projection: normed q and k columns, plain values, GELU past a gap; then per-column forms."""
    check_gemm(M, N, K, out=out, rms_cols=256, gelu_from=384, gap_at=384, gap=128, seed=1)
    check_gemm(M, N, K, out=out, rms_cols=128, gelu_from=204, gap_at=140, gap=12, pad=8 - (N + 12) % 8, seed=2)
    check_gemm(M, N, K, out=out, act="silu", seed=3)


# tiles of 256 x 128 and 128 x 128, f32 tiles of 64 rows whose K is not shared
@pytest.mark.parametrize("M,N,K,out", [(500, 10240, 400, "bf16"), (1913, 4352, 656, "bf16"), (70, 13824, 656, "f32")])
def test_gemm_norm_gelu_and_gap_of_one_round(M, N, K, out):
    check_gemm(M, N, K, out=out, rms_cols=256, gelu_from=384, gap_at=384, gap=128, seed=1)
    check_gemm(M, N, K, out=out, rms_cols=128, gelu_from=204, gap_at=140, gap=12, pad=8 - (N + 12) % 8, seed=2)
    check_gemm(M, N, K, out=out, act="silu", seed=3)
    check_gemm(M, N, K, out=out, rms_cols=N, seed=4)


def test_gemm_scales_across_the_range():
    """Row scales over 2^-120 .. 2^120 whose products stay in range, and a smallest and a largest scale byte."""
    r = rng(9)
    for M, N, K in ((5, 64, 400), (300, 2048, 400), (4100, 4352, 400)):
        a, w = operand(r, M, K), operand(r, N, K)
        e = r.integers(-100, 100, K // 128 + 1)
        a[1][:] = np.clip(a[1].astype(int) + e, 0, 254)
        w[1][:] = np.clip(w[1].astype(int) - e, 0, 254)
        for out in ("bf16", "f32"):
            check_gemm(M, N, K, out=out, operands=(a, w), bias=False)


ENDS = [0, 254, 1, 247, 2, 246, 9, 10, 253, 120]     # least and largest scale bytes, and those beside bf16's range


# one size for each kernel; f32: narrow tiles of one and two blocks of rows, K shared by two groups, tiles of 64 and 128 rows
@pytest.mark.parametrize("out", ["bf16", "f32", "gated", "fp8"])
@pytest.mark.parametrize("M,N,K", [(5, 128, 1168), (5, 9088, 1168), (9, 20096, 528), (40, 256, 1168),
                                   (40, 4992, 528), (300, 2048, 1168), (900, 2048, 1296), (900, 2048, 1024),
                                   (500, 10240, 528), (1920, 4352, 528), (4096, 2048, 1168), (4100, 4352, 1168)])
def test_gemm_scales_at_the_ends(M, N, K, out):
    """Blocks whose scale bytes are an end of the range in one operand and the opposite one in the other, so that
    every product is an ordinary number though neither operand is one in bf16 or f32.  Every e4m3 value occurs, some
    rows hold subnormals only, and some hold zeros where others hold the largest values."""
    r = rng(M, N, K, 19)
    nb = -(-K // 128)
    ends = np.resize(ENDS, nb)

    def rows(n, scale):
        q = r.integers(0, 127, (n, K)) | 128 * r.integers(0, 2, (n, K))
        q[1::4] &= 0x87                                # subnormals and zeros
        s = np.broadcast_to(scale, (n, nb)).copy()
        for b in range(nb):
            q[3::8, 128 * b:128 * (b + 1)] &= 0x80 if b % 3 == 0 else 0xFF
            s[3::8, b] = r.integers(0, 255) if b % 3 == 0 else s[3::8, b]
        return q.astype(np.uint8), s.astype(np.uint8)

    check_gemm(M, N, K, out=out, operands=(rows(M, ends), rows(N, 254 - ends)), bias=False)


@pytest.mark.parametrize("M,N,K", [(5, 128, 400), (40, 256, 400), (900, 2048, 1296), (900, 2048, 400), (4096, 2048, 400)])
def test_gemm_f32_sums_near_the_largest_number(M, N, K):
    """Sums of up to 2^125, of blocks whose scale bytes lie on both sides of 236."""
    r = rng(M, N, 20)
    a, w = operand(r, M, K, spread=0), operand(r, N, K, spread=0)
    nb = -(-K // 128)
    a[1][:] = 127 + 100 + r.integers(0, 12, (M, 1)) + np.array([0, 0, 0, 1])[np.arange(nb) % 4]
    w[1][:] = 127 + r.integers(-27, -23, (N, 1)) + 16 * (np.arange(N) % 3 == 0)[:, None]
    check_gemm(M, N, K, out="f32", operands=(a, w), bias=False)


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("M,N", [(4, 128), (300, 2048), (4100, 4352)])
def test_gemm_nan_rows_stay_in_their_rows(M, N, out):
    K = 272
    r = rng(M, N, 3)
    x = r.standard_normal((M, K))
    x[3, 200] = np.inf
    a = ref.quantise(x)
    w = operand(r, N, K)
    host, scale, got, y, tol = run_gemm(M, N, K, out=out, operands=(a, w))
    assert np.isnan(got[3]).all()
    rest = np.arange(M) != 3
    assert (np.abs(got - y)[rest] <= tol[rest]).all()
    if out == "fp8":
        assert (scale[3] == 255).all()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(4, 128), (300, 2048), (1920, 4352), (4100, 4352)])
def test_gemm_scale_of_255_is_nan(M, N, out):
    """Also above finite values, in rows of either operand."""
    K = 400
    r = rng(M, N, 4)
    a, w = operand(r, M, K), operand(r, N, K)
    a[1][2, 1] = w[1][5, 3] = 255
    _, _, got, y, tol = run_gemm(M, N, K, out=out, operands=(a, w), bias=False)
    assert np.isnan(got[2]).all() and np.isnan(got[:, 5]).all()
    rest = np.ones(y.shape, bool)
    rest[2], rest[:, 5] = False, False
    assert (np.abs(got - y)[rest] <= tol[rest]).all()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(4, 128, 400), (40, 256, 400), (900, 2048, 1296), (900, 2048, 400), (4096, 2048, 400)])
def test_gemm_scale_of_255_is_nan_on_zeros(M, N, K, out):
    r = rng(M, N, 6)
    a, w = operand(r, M, K), operand(r, N, K)
    a[0][2, 128:256], w[0][5, 384:] = 0, 0
    a[1][2, 1] = w[1][5, 3] = 255
    a[0][3], a[1][3] = 0, 0                             # a row of zeros
    _, _, got, y, tol = run_gemm(M, N, K, out=out, operands=(a, w), bias=False)
    assert np.isnan(got[2]).all() and np.isnan(got[:, 5]).all()
    rest = np.ones(y.shape, bool)
    rest[2], rest[:, 5] = False, False
    assert (np.abs(got - y)[rest] <= tol[rest]).all()


def test_gemm_no_rows_or_columns():
    torch = torch_cuda()
    z = torch.zeros(64, 64, dtype=torch.uint8, device="cuda")
    C = torch.full((8, 8), 7.0, device="cuda")
    for M, N in ((0, 8), (8, 0)):
        binding.gemm_fp8(z, z, z, z, None, C, M=M, N=N, K=64, flags=binding.EPI_F32)
    assert int((C != 7).sum()) == 0


# ---------------------------------------------------------------- selection and attention

def tokens(r, rows, heads, pad=0, scale=1.0):
    """bf16 bits [rows, heads 128 + pad] (gaps NaN) and their float64 values."""
    x = r.standard_normal((rows, heads, 128)) + r.standard_normal((rows // 40 + 1, heads, 128)).repeat(40, 0)[:rows]
    x *= scale / np.sqrt((x ** 2).mean(2, keepdims=True))
    bits = np.full((rows, heads * 128 + pad), 0x7FC0, np.uint16)
    bits[:, :heads * 128] = bf16_bits(x.reshape(rows, -1))
    return bits, bits_to_f64(bits[:, :heads * 128])


def shape_of(Lq, Lk, heads, topk, kv_heads=None, batch=1, klen=None):
    return dict(Lq=Lq, Lk=Lk, heads=heads, topk=topk, kv_heads=kv_heads, batch=batch, klen=klen)


def on_device(torch, shape):
    k = shape["klen"]
    return dict(shape, klen=None if k is None else torch.tensor(k, dtype=torch.int32, device="cuda"))


def run_select(torch, qb, kb, shape, first):
    nqb = -(-shape["Lq"] // 128)
    idx = torch.full((shape["batch"], shape["heads"], nqb, shape["topk"]), -77, dtype=torch.int32, device="cuda")
    binding.select_blocks_bf16(dev(torch, qb), dev(torch, kb), idx, first=first, **on_device(torch, shape))
    return idx.cpu().numpy()


SELECT = [
    (shape_of(1, 1, 1, 1), 0), (shape_of(1, 63, 2, 3), 0), (shape_of(127, 64, 1, 1), 1), (shape_of(129, 65, 3, 2), 0),
    (shape_of(300, 5000, 4, 9, kv_heads=2), 2), (shape_of(1, 5000, 6, 17, kv_heads=3, batch=3, klen=[5000, 0, 4033]), 1),
    (shape_of(2049, 1025, 2, 5, batch=2, klen=[1, 1025]), 0), (shape_of(700, 20000, 1, 33), 0),
    (shape_of(130, 40000, 1, 600), 3), (shape_of(130, 70000, 1, 64, klen=[69999]), 1), (shape_of(64, 300000, 1, 7), 0)]


@pytest.mark.parametrize("shape,first", SELECT)
@pytest.mark.parametrize("pad", [0, 24])
def test_select_blocks(shape, first, pad):
    torch = torch_cuda()
    r = rng(shape["Lq"], shape["Lk"])
    qb, q = tokens(r, shape["batch"] * shape["Lq"], shape["heads"], pad)
    kb, k = tokens(r, shape["batch"] * shape["Lk"], shape["kv_heads"] or shape["heads"], pad)
    if shape["klen"]:   # rows past a sequence's keys may hold anything
        for z, n in enumerate(shape["klen"]):
            kb[z * shape["Lk"] + n:(z + 1) * shape["Lk"], :] = 0x7FC0
    np.testing.assert_array_equal(run_select(torch, qb, kb, shape, first), ref.select(q, k, first=first, **shape))


@pytest.mark.parametrize("Lk,topk", [(700, 3), (9000, 20), (21000, 40), (40000, 64)])
@pytest.mark.parametrize("first", [0, 2])
def test_select_blocks_of_many_heads(Lk, topk, first):
    """More lists than the chip has CUs."""
    torch = torch_cuda()
    r = rng(Lk, 2)
    shape = shape_of(131, Lk, 136, topk, kv_heads=1, batch=2, klen=[Lk, Lk - 333])
    qb, q = tokens(r, 2 * 131, 136)
    kb, k = tokens(r, 2 * Lk, 1)
    kb[2 * Lk - 333:] = 0x7FC0
    np.testing.assert_array_equal(run_select(torch, qb, kb, shape, first), ref.select(q, k, first=first, **shape))


@pytest.mark.parametrize("Lk", [640, 5000, 40000, 70000])
def test_select_ties_go_to_the_lowest_block(Lk):
    """Small whole numbers, equal blocks: sums, means and products are exact, so ties are ties."""
    torch = torch_cuda()
    r = rng(Lk)
    nkb = -(-Lk // 64)
    kinds = r.integers(-2, 3, (4, 128)).astype(float)
    k = kinds[r.integers(0, 4, nkb)].repeat(64, 0)[:Lk]
    q = r.integers(-2, 3, (256, 128)).astype(float)
    q[128:] = 0                                     # every product is zero
    shape = shape_of(256, Lk, 1, min(nkb, 7))
    got = run_select(torch, bf16_bits(q), bf16_bits(k), shape, 0)
    np.testing.assert_array_equal(got, ref.select(q, k, **shape))
    np.testing.assert_array_equal(got[0, 0, 1], np.arange(min(nkb, 7)))


def test_select_infinities_and_nan():
    torch = torch_cuda()
    r = rng(4)
    shape = shape_of(128, 64 * 6, 1, 3)
    qb, q = tokens(r, 128, 1)
    kb, k = tokens(r, 64 * 6, 1)
    for block, bits in ((1, 0x7FC0), (2, 0x7F80), (4, 0xFF80)):
        kb[64 * block + 5, 9] = bits
    k = bits_to_f64(kb)
    np.testing.assert_array_equal(run_select(torch, qb, kb, shape, 0), ref.select(q, k, **shape))
    np.testing.assert_array_equal(run_select(torch, qb, kb, shape, 2), ref.select(q, k, first=2, **shape))


def run_attention(torch, qb, kb, vb, idx, shape, bounded=False, pad=0):
    H = shape["heads"] * 128
    o = torch.full((shape["batch"] * shape["Lq"] + 3, H + pad), 0x2A2A, dtype=torch.int16, device="cuda")
    binding.attention_sparse_bf16(dev(torch, qb), dev(torch, kb), dev(torch, vb), o, dev(torch, idx),
                                  flags=binding.ATTN_BOUNDED_LOGITS if bounded else 0, **on_device(torch, shape))
    raw = o.cpu().numpy()
    rows = shape["batch"] * shape["Lq"]
    assert (raw[rows:] == 0x2A2A).all() and (raw[:, H:] == 0x2A2A).all(), "rows or columns past the output changed"
    return host_bf16(o)[:rows, :H]


def check_attention(got, q, k, v, idx, shape):
    y, tol = ref.attend(q, k, v, idx, **shape)
    tol = tol + BF16 * (np.abs(y) + tol) + 1e-30
    worst = np.max(np.abs(got - y) / tol, initial=0)
    assert worst <= 1, f"{worst} of the tolerance"
    return y


ATTEND = [
    shape_of(1, 1, 1, 1), shape_of(1, 4097, 3, 40), shape_of(1, 9000, 2, 140, batch=2, klen=[9000, 130]),
    shape_of(5, 63, 2, 1), shape_of(33, 64, 1, 2), shape_of(128, 65, 2, 2), shape_of(129, 1000, 2, 7),
    shape_of(300, 3000, 6, 11, kv_heads=2), shape_of(257, 517, 4, 9, kv_heads=1, batch=3, klen=[517, 0, 1]),
    shape_of(1000, 2000, 8, 5, batch=2), shape_of(9000, 1500, 8, 6)]


@pytest.mark.parametrize("bounded", [False, True])
@pytest.mark.parametrize("shape", ATTEND)
def test_sparse_attention(shape, bounded):
    """Random lists with holes (-1 and blocks that do not exist), unordered, one block twice; keys past a
    sequence's end hold NaN."""
    torch = torch_cuda()
    r = rng(shape["Lq"], shape["Lk"], shape["heads"])
    G = shape["kv_heads"] or shape["heads"]
    pad = 8 * (shape["Lq"] % 3)
    qb, q = tokens(r, shape["batch"] * shape["Lq"], shape["heads"], pad)
    kb, k = tokens(r, shape["batch"] * shape["Lk"], G, pad)
    vb, v = tokens(r, shape["batch"] * shape["Lk"], G, pad, scale=2.0)
    if shape["klen"]:
        for z, n in enumerate(shape["klen"]):
            kb[z * shape["Lk"] + n:(z + 1) * shape["Lk"], :] = 0x7FC0
            vb[z * shape["Lk"] + n:(z + 1) * shape["Lk"], :] = 0x7F80
    nqb, nkb = -(-shape["Lq"] // 128), -(-shape["Lk"] // 64)
    idx = r.integers(0, nkb, (shape["batch"], shape["heads"], nqb, shape["topk"])).astype(np.int32)
    idx[r.random(idx.shape) < 0.1] = -1
    idx[r.random(idx.shape) < 0.05] = nkb + 3
    idx[r.random(idx.shape) < 0.02] = -2 ** 31
    if shape["topk"] > 1:
        idx[..., -1] = idx[..., 0]
        idx[0, 0, 0] = -1                           # a block of queries without keys
    got = run_attention(torch, qb, kb, vb, idx, shape, bounded, pad)
    y = check_attention(got, q, k, v, idx, shape)
    if shape["topk"] > 1:
        assert (got[:min(128, shape["Lq"]), :128] == 0).all() and (y[:min(128, shape["Lq"]), :128] == 0).all()


@pytest.mark.parametrize("bounded", [False, True])
@pytest.mark.parametrize("shape", [
    shape_of(40, 1500, 90, 20, kv_heads=2, batch=3, klen=[1500, 0, 1025]), shape_of(130, 1100, 132, 17, kv_heads=4),
    shape_of(97, 4000, 260, 16, kv_heads=1), shape_of(33, 900, 300, 70, kv_heads=3)])
def test_sparse_attention_of_many_lists(shape, bounded):
    """More lists than the chip has CUs, of 16 and more entries; every count of tiles from none on, blocks of
    queries that leave waves without rows."""
    torch = torch_cuda()
    r = rng(shape["Lq"], shape["Lk"], shape["heads"])
    G = shape["kv_heads"]
    qb, q = tokens(r, shape["batch"] * shape["Lq"], shape["heads"])
    kb, k = tokens(r, shape["batch"] * shape["Lk"], G)
    vb, v = tokens(r, shape["batch"] * shape["Lk"], G, scale=2.0)
    for z, n in enumerate(shape["klen"] or []):
        kb[z * shape["Lk"] + n:(z + 1) * shape["Lk"], :] = 0x7FC0
        vb[z * shape["Lk"] + n:(z + 1) * shape["Lk"], :] = 0x7F80
    nqb, nkb = -(-shape["Lq"] // 128), -(-shape["Lk"] // 64)
    idx = r.integers(0, nkb, (shape["batch"], shape["heads"], nqb, shape["topk"])).astype(np.int32)
    kept = np.arange(shape["heads"]) % (shape["topk"] + 1)     # entries of a head's lists
    idx[r.permuted(np.broadcast_to(np.arange(shape["topk"]), idx.shape), axis=3) >= kept[:, None, None]] = -1
    got = run_attention(torch, qb, kb, vb, idx, shape, bounded)
    check_attention(got, q, k, v, idx, shape)
    assert (got[:, :128] == 0).all()


@pytest.mark.parametrize("Lq", [16, 17, 20, 32])
def test_sparse_attention_of_few_queries(Lq):
    torch = torch_cuda()
    r = rng(Lq, 41)
    for heads, Lk, topk in ((2, 3000, 37), (200, 700, 5)):
        shape = shape_of(Lq, Lk, heads, topk, kv_heads=2, batch=2, klen=[Lk, Lk - 90])
        qb, q = tokens(r, 2 * Lq, heads)
        kb, k = tokens(r, 2 * Lk, 2)
        vb, v = tokens(r, 2 * Lk, 2)
        kb[2 * Lk - 90:], vb[2 * Lk - 90:] = 0x7FC0, 0x7F80
        idx = r.integers(-1, -(-Lk // 64), (2, heads, 1, topk)).astype(np.int32)
        for bounded in (False, True):
            check_attention(run_attention(torch, qb, kb, vb, idx, shape, bounded), q, k, v, idx, shape)


@pytest.mark.parametrize("Lq,heads,topk", [(1, 2, 6), (40, 2, 6), (300, 100, 16)])
def test_rows_far_apart(Lq, heads, topk):
    """Rows of up to 8 MiB, so that offsets pass 32 bits in every operand: the bits of dense rows."""
    torch = torch_cuda()
    Lk, far = 650, (1 << 22) - 8
    r = rng(Lq, 55)
    rows = [dev(torch, tokens(r, n, g)[0]) for n, g in ((Lq, heads), (Lk, 2), (Lk, 2))]
    shape = dict(Lq=Lq, Lk=Lk, heads=heads, topk=topk, kv_heads=2)
    res = []
    for apart in (False, True):
        q, k, v = (torch.empty(t.shape[0], far if apart else t.shape[1], dtype=torch.int16, device="cuda") for t in rows)
        for t, x in zip((q, k, v), rows):
            t[:, :x.shape[1]] = x
        idx = torch.empty(1, heads, -(-Lq // 128), topk, dtype=torch.int32, device="cuda")
        o = torch.empty(Lq, far if apart else heads * 128, dtype=torch.int16, device="cuda")
        binding.select_blocks_bf16(q, k, idx, **shape)
        binding.attention_sparse_bf16(q, k, v, o, idx, flags=binding.ATTN_BOUNDED_LOGITS, **shape)
        res.append((idx, o[:, :heads * 128].clone()))
        del q, k, v, o, t
    torch.cuda.empty_cache()
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])


def guarded(torch, nbytes):
    """A workspace of NaNs and the bytes behind it, which no call may change."""
    buf = torch.full((nbytes + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    return buf[:nbytes], buf[nbytes:]


@pytest.mark.parametrize("Lq,Lk,topk,klen", [(1, 63, 2, None), (300, 5000, 9, [5000, 4030]), (2049, 9000, 30, [1, 9000]),
                                             (130, 40000, 600, None), (130, 70000, 64, [69999, 0])])
def test_selection_in_a_workspace_of_its_size(Lq, Lk, topk, klen):
    """Block counts that leave groups of 16 unfilled: what was never written is NaN."""
    torch = torch_cuda()
    r = rng(Lq, Lk, 61)
    shape = shape_of(Lq, Lk, 4, topk, kv_heads=2, batch=len(klen or [0]), klen=klen)
    qb, q = tokens(r, shape["batch"] * Lq, 4)
    kb, k = tokens(r, shape["batch"] * Lk, 2)
    on = on_device(torch, shape)
    ws, rest = guarded(torch, binding.select_blocks_ws_bytes(**on))
    idx = torch.empty(shape["batch"], 4, -(-Lq // 128), topk, dtype=torch.int32, device="cuda")
    binding.select_blocks_bf16(dev(torch, qb), dev(torch, kb), idx, first=1, ws=ws, **on)
    assert (rest == 0xFF).all()
    np.testing.assert_array_equal(idx.cpu().numpy(), ref.select(q, k, first=1, **shape))


@pytest.mark.parametrize("bounded", [False, True])
@pytest.mark.parametrize("Lq,heads,topk", [(1, 2, 200), (1, 30, 40), (17, 3, 60), (33, 4, 30), (128, 9, 12), (300, 5, 100)])
def test_attention_in_a_workspace_of_its_size(Lq, heads, topk, bounded):
    torch = torch_cuda()
    r = rng(Lq, heads, 62)
    shape = shape_of(Lq, 4097, heads, topk, kv_heads=1)
    qb, q = tokens(r, Lq, heads)
    kb, k = tokens(r, 4097, 1)
    vb, v = tokens(r, 4097, 1)
    nqb = -(-Lq // 128)
    idx = r.integers(-1, 65, (1, heads, nqb, topk)).astype(np.int32)
    idx[0, 0, 0, topk // 4:] = -1                      # pieces of a list that hold no entry
    n = binding.attention_sparse_ws_bytes(**shape)
    assert n > 0
    ws, rest = guarded(torch, n)
    o = torch.empty(Lq, heads * 128, dtype=torch.int16, device="cuda")
    binding.attention_sparse_bf16(dev(torch, qb), dev(torch, kb), dev(torch, vb), o, dev(torch, idx), ws=ws,
                                  flags=binding.ATTN_BOUNDED_LOGITS if bounded else 0, **shape)
    assert (rest == 0xFF).all()
    check_attention(host_bf16(o), q, k, v, idx, shape)


def test_lengths_of_zero():
    """No keys: lists of -1 and rows of zeros.  No queries, no sequences: nothing is written."""
    torch = torch_cuda()
    x = torch.full((200, 256), 0x7FC0, dtype=torch.int16, device="cuda")
    for Lq, Lk, batch, klen in ((200, 0, 1, None), (100, 70, 2, [0, -3]), (0, 64, 1, None), (200, 64, 0, None)):
        kl = None if klen is None else torch.tensor(klen, dtype=torch.int32, device="cuda")
        shape = dict(Lq=Lq, Lk=Lk, heads=2, topk=3, batch=batch, klen=kl)
        idx = torch.full((2, 2, 2, 3), 1, dtype=torch.int32, device="cuda")
        o = torch.full((200, 256), 0x2A2A, dtype=torch.int16, device="cuda")
        ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        n = batch * 2 * -(-Lq // 128) * 3
        binding.select_blocks_bf16(x, x, idx, ws=ws, **shape)
        assert (idx.view(-1)[:n] == -1).all() and (idx.view(-1)[n:] == 1).all()
        idx.fill_(0)
        binding.attention_sparse_bf16(x, x, x, o, idx, ws=ws, **shape)
        assert (o[:batch * Lq] == 0).all() and (o[batch * Lq:] == 0x2A2A).all()
    # empty tensors, whose pointers are null
    for Lq, Lk in ((200, 0), (0, 64), (40, 0), (20, 0)):
        shape = dict(Lq=Lq, Lk=Lk, heads=2, topk=20)
        q, k = (torch.empty(n, 256, dtype=torch.int16, device="cuda") for n in (Lq, Lk))
        idx = torch.full((1, 2, -(-Lq // 128), 20), 1, dtype=torch.int32, device="cuda")
        o = torch.full((Lq, 256), 1, dtype=torch.int16, device="cuda")
        binding.attention_sparse_bf16(q, k, k, o, idx, **shape)
        binding.select_blocks_bf16(q, k, idx, **shape)
        assert (o == 0).all() and (idx == -1).all()
    e = torch.empty(0, 256, dtype=torch.uint8, device="cuda")
    w, c = torch.zeros(64, 256, dtype=torch.uint8, device="cuda"), torch.empty(0, 64, dtype=torch.int16, device="cuda")
    binding.quant_fp8(torch.empty(0, 256, device="cuda"), e, e, M=0, K=256)
    binding.gemm_fp8(e, e, w, w, None, c, M=0, N=64, K=256)


@pytest.mark.parametrize("Lq", [1, 200])
def test_sparse_attention_rising_logits(Lq):
    """Logits that grow along the list by more than f32's exponent range in all: the running maximum moves at
    every tile and old parts vanish; and logits far below zero, whose plain exponentials would."""
    torch = torch_cuda()
    r = rng(Lq, 8)
    shape = shape_of(Lq, 64 * 12, 1, 12)
    for sign in (1, -1):
        k = np.repeat(np.arange(12), 64)[:, None] * np.ones(128) * 2 + r.standard_normal((64 * 12, 128)) * 0.1
        q = sign * (1 + 0.1 * r.standard_normal((Lq, 128)))
        v = r.standard_normal((64 * 12, 128))
        (qb, kb, vb) = (bf16_bits(t) for t in (q, k, v))
        idx = np.broadcast_to(np.arange(12, dtype=np.int32), (1, 1, -(-Lq // 128), 12)).copy()
        got = run_attention(torch, qb, kb, vb, idx, shape)
        check_attention(got, *(bits_to_f64(t) for t in (qb, kb, vb)), idx, shape)


def test_sparse_attention_overflowing_logits():
    """A key whose logit overflows to -inf weighs nothing; one listed alone leaves zeros."""
    torch = torch_cuda()
    shape = shape_of(64, 128, 1, 2)
    q = np.full((64, 128), 2.0 ** 100)
    k = np.zeros((128, 128))
    k[:64] = -2.0 ** 100
    v = rng(6).standard_normal((128, 128))
    qb, kb, vb = (bf16_bits(t) for t in (q, k, v))
    idx = np.array([[[[0, 1]]]], np.int32)
    got = run_attention(torch, qb, kb, vb, idx, shape)
    want = bits_to_f64(vb)[64:].mean(0)
    assert np.abs(got - want).max() <= 2.0 ** -7 * np.abs(bits_to_f64(vb)).max()
    idx[...] = 0
    assert (run_attention(torch, qb, kb, vb, idx, shape) == 0).all()


def test_sparse_attention_over_every_block_is_the_dense_one():
    torch = torch_cuda()
    Lq, Lk, heads = 700, 1500, 3
    shape = shape_of(Lq, Lk, heads, 24)
    r = rng(12)
    qb, q = tokens(r, Lq, heads)
    kb, k = tokens(r, Lk, heads)
    vb, v = tokens(r, Lk, heads)
    idx = run_select(torch, qb, kb, shape, 0)
    assert (idx == np.arange(24)).all()
    got = run_attention(torch, qb, kb, vb, idx, shape)
    check_attention(got, q, k, v, idx, shape)
    o = torch.empty((Lq, heads * 128), dtype=torch.int16, device="cuda")
    ws = torch.empty(heads * 128 * 1536, dtype=torch.int16, device="cuda")
    binding.attention_bf16(dev(torch, qb), dev(torch, kb), dev(torch, vb), o, Lq=Lq, Lk=Lk, heads=heads,
                           ldq=heads * 128, ldk=heads * 128, ldv=heads * 128, ldo=heads * 128, vt_ws=ws)
    # the two round their probabilities to bf16 around different maxima: twice one side's bound
    y, tol = ref.attend(q, k, v, idx, **shape)
    assert (np.abs(got - host_bf16(o)) <= 2 * (tol + BF16 * (np.abs(y) + tol))).all()


# ---------------------------------------------------------------- together

class Block:
    """Attention half and MLP of one block on 8-bit products and chosen key blocks, its buffers and workspaces."""

    def __init__(self, torch, seed, L=700, heads=2, F=512, topk=4):
        r = rng(seed, 21)
        H = self.H = heads * 128
        self.t, self.L, self.heads, self.F, self.topk = torch, L, heads, F, topk
        self.w = {}
        for name, n, k in (("qkv", 3 * H, H), ("o", H, H), ("up", F, H), ("down", H, F)):
            self.w[name] = self.rows(r.standard_normal((n, k)) / np.sqrt(k))
        self.gate = dev(torch, r.standard_normal(H).astype(np.float32))
        self.x0 = dev(torch, bf16_bits(r.standard_normal((L, H))))
        e = lambda *s, dt=torch.int16: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        self.x, self.qkv, self.att = e(L, H), e(L, 3 * H), e(L, H)
        self.q8 = [e(L, n, dt=torch.uint8) for n in (H, H, H, F)]
        self.s8 = [e(L, binding.fp8_scale_ld(n), dt=torch.uint8) for n in (H, H, H, F)]
        self.idx = e(1, heads, -(-L // 128), topk, dt=torch.int32)
        self.shape = dict(Lq=L, Lk=L, heads=heads, topk=topk)
        self.ws = [e(max(16, f(**self.shape)), dt=torch.uint8)
                   for f in (binding.select_blocks_ws_bytes, binding.attention_sparse_ws_bytes)]

    def rows(self, x):
        q, s = ref.quantise(x)
        return dev(self.t, q), dev(self.t, padded_scale(s, x.shape[1])), ref.values(q, s)

    def linear(self, i, name, out, N, K, **kw):
        w = self.w[name]
        binding.gemm_fp8(self.q8[i], self.s8[i], w[0], w[1], None, out, M=self.L, N=N, K=K, stream=self.stream, **kw)

    def quant(self, i, x, K):
        binding.quant_fp8(x, self.q8[i], self.s8[i], M=self.L, K=K, stream=self.stream)

    def run(self, stream=None):
        self.stream, H, F, L = stream, self.H, self.F, self.L
        self.x.copy_(self.x0)
        self.quant(0, self.x, H)
        self.linear(0, "qkv", self.qkv, 3 * H, H, rms_cols=2 * H)
        q, k, v = (self.qkv[:, i * H:(i + 1) * H] for i in range(3))
        binding.select_blocks_bf16(q, k, self.idx, first=1, ws=self.ws[0], stream=stream, **self.shape)
        binding.attention_sparse_bf16(q, k, v, self.att, self.idx, ws=self.ws[1], stream=stream,
                                      flags=binding.ATTN_BOUNDED_LOGITS, **self.shape)
        self.quant(1, self.att, H)
        self.linear(1, "o", self.x, H, H, flags=binding.EPI_GATED_RES, gate=self.gate)
        self.quant(2, self.x, H)
        self.linear(2, "up", self.q8[3], F, H, flags=binding.EPI_FP8, c_scale=self.s8[3], gelu_from=0)
        self.linear(3, "down", self.x, H, F, flags=binding.EPI_GATED_RES, gate=self.gate)
        return self.x

    def host8(self, i):
        q, s = self.q8[i].cpu().numpy(), self.s8[i].cpu().numpy()
        return ref.values(q, s[:, :-(-q.shape[1] // 128)])


def test_a_block_on_all_four_operators():
    """Each stage against float64 on the device's own input of that stage, so that every tolerance is one stage's."""
    torch = torch_cuda()
    b = Block(torch, 1)
    H, L = b.H, b.L
    out = host_bf16(b.run())
    x0 = host_bf16(b.x0)
    rq, rs = ref.quantise(x0)
    np.testing.assert_array_equal(b.host8(0), ref.values(rq, rs))
    y, d = ref.product(b.host8(0), b.w["qkv"][2], None, f32=False, rms_cols=2 * H)
    qkv = host_bf16(b.qkv)
    assert (np.abs(qkv - y) <= d + BF16 * (np.abs(y) + d) + 1e-30).all()
    q, k, v = (qkv[:, i * H:(i + 1) * H] for i in range(3))
    idx = b.idx.cpu().numpy()
    np.testing.assert_array_equal(idx, ref.select(q, k, first=1, **b.shape))
    check_attention(host_bf16(b.att), q, k, v, idx, b.shape)
    rq, rs = ref.quantise(host_bf16(b.att))
    np.testing.assert_array_equal(b.host8(1), ref.values(rq, rs))
    gate = b.gate.cpu().numpy().astype(np.float64)
    y, d = ref.product(b.host8(1), b.w["o"][2], None, f32=False)
    mid, dm = x0 + gate * y, np.abs(gate) * d + 2.0 ** -22 * (np.abs(x0) + np.abs(gate * y))
    dm = dm + BF16 * (np.abs(mid) + dm)
    # the 8-bit rows of the middle residual lie within its error and their own half step
    m8 = b.host8(2)
    s = np.repeat(2.0 ** (b.s8[2].cpu().numpy()[:, :H // 128].astype(np.float64) - 127), 128, 1)
    assert (np.abs(m8 - mid) <= dm + np.maximum(2.0 ** -4 * (np.abs(mid) + dm), 2.0 ** -10 * s)).all()
    y, d = ref.product(m8, b.w["up"][2], None, f32=False, gelu_from=0)
    u8 = b.host8(3)
    s = np.repeat(2.0 ** (b.s8[3].cpu().numpy()[:, :b.F // 128].astype(np.float64) - 127), 128, 1)
    assert (np.abs(u8 - y) <= d + np.maximum(2.0 ** -4 * (np.abs(y) + d), 2.0 ** -10 * s)).all()
    y, d = ref.product(u8, b.w["down"][2], None, f32=False)
    fin = mid + gate * y
    tol = dm + np.abs(gate) * d + 2.0 ** -22 * (np.abs(mid) + np.abs(gate * y))
    assert (np.abs(out - fin) <= tol + BF16 * (np.abs(fin) + tol)).all()


def test_blocks_captured_into_two_graphs():
    """Two blocks captured into graphs with their own workspaces, replayed in turn with eager work between: every
    replay gives the eager bits."""
    torch = torch_cuda()
    blocks = [Block(torch, s) for s in (2, 3)]
    want = [b.run().clone() for b in blocks]
    other = Block(torch, 4)
    stream = torch.cuda.Stream()
    graphs = []
    torch.cuda.synchronize()
    for b in blocks:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            b.run(stream)
        graphs.append(g)
    for i in range(4):
        for b, g, w in zip(blocks, graphs, want):
            b.x.zero_()
            b.idx.fill_(-1)
            g.replay()
            other.run()
            torch.cuda.synchronize()
            assert torch.equal(b.x, w), i


def test_blocks_on_two_streams():
    torch = torch_cuda()
    blocks = [Block(torch, s, L=1500) for s in (5, 6)]
    want = [b.run().clone() for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for b, s in zip(blocks, streams):
        for _ in range(6):
            with torch.cuda.stream(s):
                b.run(s)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert torch.equal(b.x, w)


def test_workspaces_of_the_caching_allocator():
    """Without a workspace argument the binding takes one on the call's stream; results are those of a kept one."""
    torch = torch_cuda()
    r = rng(31)
    shape = shape_of(1, 5000, 3, 30)
    qb, _ = tokens(r, 1, 3)
    kb, _ = tokens(r, 5000, 3)
    q, k = dev(torch, qb), dev(torch, kb)
    torch.cuda.synchronize()
    outs = []
    for stream in (None, torch.cuda.Stream()):
        for _ in range(3):
            idx = torch.empty(1, 3, 1, 30, dtype=torch.int32, device="cuda")
            o = torch.empty(1, 384, dtype=torch.int16, device="cuda")
            torch.cuda.synchronize()
            binding.select_blocks_bf16(q, k, idx, stream=stream, **shape)
            binding.attention_sparse_bf16(q, k, k, o, idx, stream=stream, **shape)
            torch.cuda.synchronize()
            outs.append((idx, o))
    for idx, o in outs:
        assert torch.equal(idx, outs[0][0]) and torch.equal(o, outs[0][1])


def test_workspaces_of_a_captured_call():
    """Workspaces that the binding takes during a capture stay the graph's own: other allocations between the
    replays do not touch them."""
    torch = torch_cuda()
    r = rng(33)
    shape = shape_of(1, 5000, 3, 64)
    q, k = dev(torch, tokens(r, 1, 3)[0]), dev(torch, tokens(r, 5000, 3)[0])
    idx = torch.empty(1, 3, 1, 64, dtype=torch.int32, device="cuda")
    o = torch.empty(1, 384, dtype=torch.int16, device="cuda")

    def run():
        binding.select_blocks_bf16(q, k, idx, **shape)
        binding.attention_sparse_bf16(q, k, k, o, idx, **shape)

    run()
    want = idx.clone(), o.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(4):
        junk = [torch.full((n,), -1, dtype=torch.int32, device="cuda") for n in (300, 5000, 70000, 10 ** 6)]
        idx.fill_(7)
        o.zero_()
        g.replay()
        junk += [torch.full((n,), -1, dtype=torch.int32, device="cuda") for n in (300, 5000, 70000)]
        torch.cuda.synchronize()
        assert torch.equal(idx, want[0]) and torch.equal(o, want[1]), i
        del junk
