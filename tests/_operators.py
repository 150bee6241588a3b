"""Plain float64 forms of the 8-bit and sparse operators, on the host (numpy),
written from their definitions, with the error bounds that the tests use."""
import numpy as np

E4M3_MAX = 448.0


def e4m3_table():
    """Values of the 256 e4m3 bytes (NaN for 0x7f and 0xff)."""
    v = np.zeros(256)
    for b in range(128):
        e, m = b >> 3, b & 7
        v[b] = np.nan if b == 127 else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[b + 128] = -v[b]
    return v


TABLE = e4m3_table()


def quantise(x):
    """float64 [M, K] -> (e4m3 bytes, scale bytes [M, ceil(K / 128)]) by the definition: per block the least
    e >= -127 with max |x| <= 448 2^e, the nearest e4m3 of x / 2^e, ties to the even byte; a block that is not
    finite gets 255 and NaNs."""
    x = np.asarray(x, np.float64)
    M, K = x.shape
    nb = -(-K // 128)
    q = np.zeros((M, K), np.uint8)
    scale = np.zeros((M, nb), np.uint8)
    pos = TABLE[:127]                      # ascending
    for b in range(nb):
        blk = x[:, 128 * b:128 * (b + 1)]
        a = np.abs(blk).max(1)
        fin = np.isfinite(a)
        e = np.full(M, -127)
        for i in np.flatnonzero(fin & (a > 0)):
            k = int(np.floor(np.log2(a[i]))) - 10
            while a[i] > E4M3_MAX * 2.0 ** k:
                k += 1
            e[i] = max(k, -127)
        y = np.abs(np.where(fin[:, None], blk, 0)) / 2.0 ** e[:, None]
        hi = np.clip(np.searchsorted(pos, y), 0, 126)
        lo = np.clip(hi - 1, 0, 126)
        dl, dh = y - pos[lo], pos[hi] - y
        byte = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
        byte = np.where(np.signbit(blk), byte | 128, byte)
        q[:, 128 * b:128 * (b + 1)] = np.where(fin[:, None], byte, 0x7F)
        scale[:, b] = np.where(fin, e + 127, 255)
    return q, scale


def values(q, scale):
    K = q.shape[1]
    s = 2.0 ** (scale.astype(np.float64) - 127)
    s[scale == 255] = np.nan
    return TABLE[q] * np.repeat(s, 128, 1)[:, :K]


def gelu(y):
    return 0.5 * y * (1 + np.tanh(np.sqrt(2 / np.pi) * (y + 0.044715 * y ** 3)))


def silu(y):
    return y / (1 + np.exp(-y))


def product(a, w, bias, *, f32, act="none", rms_cols=0, gelu_from=None):
    """The layer in float64 and a bound on what the device may be off before the output's rounding.

    Sum: with S = sum |a w|, the 8-bit matrix cores lose at most 2^-13 S (a few neighbouring products are cut
    2^-14 below their largest, each at most once), bf16 ones and every f32 chain at most (K + 16) 2^-24 S.
    GELU and SiLU have slopes below 1.13 and are evaluated with two hardware functions of 1 ulp, 2^-21 with the
    argument's roundings.  The norm divides by the row's size: its relative error is at most the
    2-norm error over the 2-norm."""
    y = a @ w.T
    S = np.abs(a) @ np.abs(w).T
    K = a.shape[1]
    d = S * (K + 16) * 2.0 ** -24 + (0 if f32 else S * 2.0 ** -13)
    if bias is not None:
        y = y + bias
        d = d + np.abs(y) * 2.0 ** -24
    if rms_cols:
        for h in range(0, rms_cols, 128):
            v, dv = y[:, h:h + 128], d[:, h:h + 128]
            n = np.sqrt((v ** 2).mean(1, keepdims=True) + 1e-6)
            off = np.sqrt((dv ** 2).mean(1, keepdims=True)) / n
            y[:, h:h + 128] = v / n
            d[:, h:h + 128] = dv / n + np.abs(v / n) * (off + 2.0 ** -20)
    if gelu_from is not None:
        v = y[:, gelu_from:]
        d[:, gelu_from:] = 1.13 * d[:, gelu_from:] + np.abs(v) * 2.0 ** -21 * (1 + np.abs(v))
        y[:, gelu_from:] = gelu(v)
    if act == "silu":
        d = 1.13 * d + np.abs(y) * 2.0 ** -21 * (1 + np.abs(y))
        y = silu(y)
    return y, d


def mean_blocks(x, L, H, blk, n):
    """[blocks, H, 128] means of the rows below n."""
    nb = -(-L // blk)
    out = np.zeros((nb, H, 128))
    for b in range(nb):
        rows = x[b * blk:min((b + 1) * blk, n)]
        if len(rows):
            out[b] = rows.reshape(len(rows), H, 128).sum(0) / len(rows)
    return out


def select(q, k, *, Lq, Lk, heads, topk, kv_heads=None, batch=1, klen=None, first=0):
    G = kv_heads or heads
    nqb, nkb = -(-Lq // 128), -(-Lk // 64)
    idx = np.full((batch, heads, nqb, topk), -1, np.int32)
    for z in range(batch):
        n = Lk if klen is None else int(np.clip(klen[z], 0, Lk))
        qm = mean_blocks(q[z * Lq:(z + 1) * Lq], Lq, heads, 128, Lq)
        km = mean_blocks(k[z * Lk:(z + 1) * Lk], Lk, G, 64, n)
        valid = -(-n // 64)
        for h in range(heads):
            with np.errstate(invalid="ignore"):
                s = qm[:, h] @ km[:, h // (heads // G)].T
            s[np.isnan(s)] = -np.inf
            s[:, :first] = np.inf
            order = np.argsort(-s[:, :valid], axis=1, kind="stable")[:, :topk]
            order.sort(1)
            idx[z, h, :, :order.shape[1]] = order
    return idx


def attend(q, k, v, idx, *, Lq, Lk, heads, topk, kv_heads=None, batch=1, klen=None):
    """float64 outputs [batch Lq, heads 128] and the bound of what the device may be off before its rounding.

    With weights w_j: every probability carries a relative error of at most e = 2^-8 (its rounding to bf16) plus
    that of its logit: f32 sums of 128 products (128 2^-24 |q||k|), two roundings and exp2's.  Numerator and
    sum take the same rounded values, so the output moves by at most e sum w_j |v_j - o| / (1 - e); the f32 sums
    over n keys add n 2^-24 sum w_j |v_j|."""
    G = kv_heads or heads
    out = np.zeros((batch * Lq, heads * 128))
    tol = np.zeros_like(out)
    for z in range(batch):
        n = Lk if klen is None else int(np.clip(klen[z], 0, Lk))
        nkb = -(-n // 64)
        for h in range(heads):
            g = h // (heads // G)
            for b in range(-(-Lq // 128)):
                rows = slice(z * Lq + 128 * b, z * Lq + min(128 * (b + 1), Lq))
                at = [j for j in idx[z, h, b] if 0 <= j < nkb]
                keys = np.concatenate([np.arange(64 * j, min(64 * (j + 1), n)) for j in at]).astype(int) if at else []
                if not len(keys):
                    continue
                qq = q[rows, h * 128:(h + 1) * 128]
                kk, vv = (t[z * Lk + keys, g * 128:(g + 1) * 128] for t in (k, v))
                s = qq @ kk.T / np.sqrt(128)
                w = np.exp(s - s.max(1, keepdims=True))
                w /= w.sum(1, keepdims=True)
                o = w @ vv
                size = np.linalg.norm(qq, axis=1, keepdims=True) * np.linalg.norm(kk, axis=1).max() / np.sqrt(128)
                e = 2.0 ** -8 + (130 * 2.0 ** -24) * size + 2.0 ** -21 * (1 + np.abs(s).max(1, keepdims=True))
                spread = np.stack([(w * np.abs(vv[:, c][None, :] - o[:, c][:, None])).sum(1) for c in range(128)], 1)
                out[rows, h * 128:(h + 1) * 128] = o
                tol[rows, h * 128:(h + 1) * 128] = e * spread * 1.01 + (len(keys) + 16) * 2.0 ** -24 * (w @ np.abs(vv))
    return out, tol
