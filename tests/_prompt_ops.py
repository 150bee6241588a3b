"""Plain float64 forms of a prompt encoder's operators (4-bit rows, rotary positions, packed attention), on the host
(numpy), written from their definitions, with the error bounds that the tests use."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
TABLE = np.concatenate([E2M1, -E2M1])


def quantise(x):
    """float64 [M, K] -> (codes, scale bytes [M, K / 32]) by the definition: per block the least e >= -127 with
    max |x| <= 6 2^e, the nearest e2m1 of x / 2^e, ties to the even code; a block that is not finite gets 255."""
    x = np.asarray(x, np.float64)
    M, K = x.shape
    blk = x.reshape(M, K // 32, 32)
    a = np.abs(blk).max(2)
    fin = np.isfinite(a)
    # a = m 2^k with m in [1/2, 1), and 6 = 3/4 * 2^3
    m, k = np.frexp(np.where(fin, a, 0))
    e = np.maximum(np.where(m > 0, k - 3 + (m > 0.75), -127), -127)
    top = np.where(fin, a, 0)
    assert (top <= 6 * 2.0 ** e).all() and ((top > 6 * 2.0 ** (e - 1.0)) | (e == -127)).all()
    y = np.abs(np.where(fin[..., None], blk, 0)) / (2.0 ** e)[..., None]
    middle = (E2M1[:-1] + E2M1[1:]) / 2
    below, above = np.searchsorted(middle, y, "left"), np.searchsorted(middle, y, "right")   # one code, or two at a tie
    code = np.where(below % 2 == 0, below, above)
    code = np.where(np.signbit(blk), code | 8, code)
    return np.where(fin[..., None], code, 0).reshape(M, K).astype(np.uint8), np.where(fin, e + 127, 255).astype(np.uint8)


def pack(codes):
    return (codes[:, ::2] | codes[:, 1::2] << 4).astype(np.uint8)


def unpack(q):
    return np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)


def values(codes, scale):
    s = 2.0 ** (scale.astype(np.float64) - 127)
    s[scale == 255] = np.nan
    return TABLE[codes] * np.repeat(s, 32, 1)


def rotate(x, pos, freq, *, heads, head_dim, pairs, half, scale=1.0):
    """float64 rotation of [rows, heads head_dim] and the bound on what the device may be off before its rounding.

    Cosine and sine: the reduced angle's rounding to f32, its product with pi / 2, a rounded pi / 2 and the
    polynomials' own roundings and rests stay below 4 of 2^-24, the factor, two products and a sum add a rounding each:
    8 2^-24 |scale| (|a| + |b|).  The angle itself is formed in double: 2^-50 of it."""
    n = len(freq)
    rows = x.shape[0]
    axis = np.repeat(np.arange(len(pairs)), pairs)
    t = pos[axis].T.astype(np.float64) * freq
    c, s = (f(t)[:, None] * scale for f in (np.cos, np.sin))
    x = x.reshape(rows, heads, head_dim)
    y, tol = x.copy(), np.zeros_like(x)
    i, j = (slice(0, n), slice(n, 2 * n)) if half else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    tol[..., i] = tol[..., j] = abs(scale) * (np.abs(a) + np.abs(b)) * (8 * 2.0 ** -24 + 2.0 ** -50 * np.abs(t)[:, None])
    return y.reshape(rows, -1), tol.reshape(rows, -1)


def attend(q, k, v, *, qoff, koff, heads, kv_heads=None, klen=None, causal=False):
    """float64 outputs of the rows that belong to a sequence (NaN elsewhere) and the bound of what the device may be off
    before its rounding.

    With weights w_j: every probability carries a relative error of at most e = 2^-8 (its rounding to bf16) plus
    that of its logit: f32 sums of 128 products (128 2^-24 |q||k|), two roundings and exp2's.  Numerator and
    sum take the same rounded values, so the output moves by at most e sum w_j |v_j - o| / (1 - e); the f32 sums
    over n keys add n 2^-24 sum w_j |v_j|.  Of many keys sum w_j |v_j - o| is bounded by the square root of
    sum w_j (v_j - o)^2 = sum w_j v_j^2 - o^2, as means are by root mean squares."""
    G = kv_heads or heads
    Tq, Tk = q.shape[0], k.shape[0]
    out = np.full((Tq, heads * 128), np.nan)
    tol = np.zeros_like(out)
    for z in range(len(qoff) - 1):
        q0 = int(np.clip(qoff[z], 0, Tq))
        q1 = int(np.clip(qoff[z + 1], q0, Tq))
        k0 = int(np.clip(koff[z], 0, Tk))
        n = int(np.clip(koff[z + 1], k0, Tk)) - k0
        if klen is not None:
            n = int(np.clip(klen[z], 0, n))
        for h in range(heads):
            c, g = slice(h * 128, h * 128 + 128), slice(h // (heads // G) * 128, h // (heads // G) * 128 + 128)
            for r0 in range(q0, q1, 512):
                r1 = min(q1, r0 + 512)
                limit = np.arange(r0 - q0, r1 - q0) + n - (q1 - q0) + 1 if causal else np.full(r1 - r0, n)
                m = int(np.clip(limit[-1], 0, n))
                qq, kk, vv = q[r0:r1, c], k[k0:k0 + m, g], v[k0:k0 + m, g]
                see = np.arange(m) < limit[:, None]
                out[r0:r1, c] = 0
                if not see.any():
                    continue
                kk, vv = np.where(see.any(0)[:, None], kk, 0), np.where(see.any(0)[:, None], vv, 0)
                s = np.where(see, qq @ kk.T / np.sqrt(128), -np.inf)
                top = s.max(1, keepdims=True)
                w = np.exp(s - np.where(np.isinf(top), 0, top))
                den = w.sum(1, keepdims=True)
                w /= np.where(den == 0, 1, den)
                o = w @ vv
                size = np.linalg.norm(qq, axis=1, keepdims=True) * np.linalg.norm(kk, axis=1).max() / np.sqrt(128)
                e = 2.0 ** -8 + (130 * 2.0 ** -24) * size + 2.0 ** -21 * (1 + np.abs(np.where(see, s, 0)).max(1, keepdims=True))
                spread = np.sqrt(np.maximum(w @ vv ** 2 - o ** 2, 0)) if m > 600 else np.stack([(w * np.abs(vv[:, i][None] - o[:, i][:, None])).sum(1) for i in range(128)], 1)
                out[r0:r1, c] = o
                tol[r0:r1, c] = e * spread * 1.01 + (m + 16) * 2.0 ** -24 * (w @ np.abs(vv))
    return out, tol
