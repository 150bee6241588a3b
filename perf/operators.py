"""Cases of the low-precision and sparse operators of a full step, with their plain forms.

Four operators: rows quantised to 8-bit floating point with one scale per 128
values (``quant``), the product of two such matrices with a layer's epilogue
(``gemm``), the choice of key blocks per query block by a cheap score
(``select``) and attention over the chosen blocks (``sparse``).

``run`` computes an operator from elementary torch operations where ``own``
is false, and calls the library where it is true.  ``exact`` computes the same
in float64 from the definition.
"""
import math

import torch

own = False

QB, KB, D = 128, 64, 128   # queries and keys of a block, width of a head
FP8 = torch.float8_e4m3fn
E8 = torch.float8_e8m0fnu
MAX_PAIRS = 40 * 32760 * 52 * KB            # listed (query, key, head) triples of the largest sparse case
MAX_PRODUCT = 32760 * 13824 * 5120          # M N K of the largest product


def listed():
    return [
        # one row of conditioning entering a quantised layer
        dict(name="quant_row", op="quant", M=1, K=5120, dtype="bf16"),
        # odd f32 rows whose last block is cut short
        dict(name="quant_ragged_f32", op="quant", M=1357, K=2608, dtype="f32"),
        # activations of a video block (32760 tokens) entering its linear layers
        dict(name="quant_video", op="quant", M=32760, K=5120, dtype="bf16"),
        # one row against a layer's weights: SiLU of a conditioning vector
        dict(name="gemm_row", op="gemm", M=1, N=13824, K=5120, out="bf16", act="silu"),
        # the text tokens' key and value projection of a video block, keys normed per head
        dict(name="gemm_text", op="gemm", M=512, N=10240, K=5120, out="bf16", act="rms"),
        # odd sizes: ragged in all three, f32 output
        dict(name="gemm_ragged_f32", op="gemm", M=1333, N=1000, K=2320, out="f32", act="none"),
        # the video block's MLP: up-projection with GELU, its output quantised for the down-projection
        dict(name="gemm_video_mlp", op="gemm", M=32760, N=13824, K=5120, out="fp8", act="gelu"),
        # an image's joint sequence: 512 text tokens (8 key blocks, always kept) and 4096 image tokens
        dict(name="select_image", op="select", B=1, Lq=4608, Lk=4608, heads=24, kv_heads=24, topk=24, first=8, pad=False),
        # the video block's self-attention, a tenth of the key blocks
        dict(name="select_video", op="select", B=1, Lq=32760, Lk=32760, heads=40, kv_heads=40, topk=52, first=1, pad=False),
        # a single token per head over a long context
        dict(name="sparse_token", op="sparse", B=1, Lq=1, Lk=32760, heads=40, kv_heads=40, topk=64, first=1, pad=False,
             bounded=False),
        # a padded batch with shared key heads and odd lengths
        dict(name="sparse_ragged", op="sparse", B=2, Lq=1000, Lk=5003, heads=12, kv_heads=4, topk=9, first=1, pad=True,
             bounded=False),
        # the video block's self-attention over a tenth of its key blocks, normed queries and keys
        dict(name="sparse_video", op="sparse", B=1, Lq=32760, Lk=32760, heads=40, kv_heads=40, topk=52, first=1, pad=False,
             bounded=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quant", "gemm", "gemm", "select", "sparse", "sparse"])
    if op == "quant":
        return dict(op=op, M=_log(rng, 1, 32760), K=16 * _log(rng, 1, 320), dtype=rng.choice(["bf16", "f32"]))
    if op == "gemm":
        while True:
            M, K = _log(rng, 1, 32760), 16 * _log(rng, 4, 864)
            out = rng.choice(["bf16", "f32", "fp8"])
            act = rng.choice(["none", "silu", "gelu"] if out == "f32" else ["none", "silu", "gelu", "rms"])
            N = 128 * _log(rng, 1, 108) if out == "fp8" or act == "rms" else 8 * _log(rng, 8, 1728)
            if M * N * K <= MAX_PRODUCT:
                return dict(op=op, M=M, N=N, K=K, out=out, act=act)
    while True:
        kv = rng.choice([1, 2, 3, 4, 8, 24, 40])
        heads = kv * rng.choice([1, 1, 1, 2, 3])
        B = rng.choice([1, 1, 1, 2, 3])
        Lk = _log(rng, 1, 32760) if op == "sparse" else _log(rng, 1024, 32760)   # select: with something to choose
        Lq = rng.choice([1, _log(rng, 1, 32760), Lk])
        nkb = -(-Lk // KB)
        topk = _log(rng, 1, min(64, nkb)) if op == "sparse" else _log(rng, 2, min(64, nkb // 2))
        pairs = B * heads * Lq * topk * KB
        if heads <= 40 and pairs <= MAX_PAIRS and B * Lk * kv <= 40 * 32760 and B * Lq * heads <= 40 * 32760:
            c = dict(op=op, B=B, Lq=Lq, Lk=Lk, heads=heads, kv_heads=kv, topk=topk, first=rng.choice([0, 1]),
                     pad=rng.random() < 0.4)
            return dict(c, bounded=rng.random() < 0.5) if op == "sparse" else c


def _scale_ld(K):
    return 4 * -(-K // 512)


# ---------------------------------------------------------------- inputs

def _rows(gen, M, K, dtype):
    """Activations as they leave a norm: unit rows with some wide channels, and a few tokens far larger than the rest."""
    x = torch.randn(M, K, generator=gen, device="cuda")
    x *= torch.exp(0.7 * torch.randn(K, generator=gen, device="cuda"))
    x *= torch.where(torch.rand(M, 1, generator=gen, device="cuda") < 0.02, 30.0, 1.0)
    return x.to(dtype)


def _tokens(gen, B, L, H):
    """Queries or keys after the per-head norm: a slow course along the sequence and noise."""
    n = L // 192 + 2
    base = torch.randn(B, n, H * D, generator=gen, device="cuda")
    at = torch.arange(L, device="cuda", dtype=torch.float32) / 192
    i = at.long()
    f = (at - i)[:, None]
    x = base[:, i] * (1 - f) + base[:, i + 1] * f
    x = (x + torch.randn(B, L, H * D, generator=gen, device="cuda")).view(B, L, H, D)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    return x.to(torch.bfloat16).view(B * L, H * D)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=c)
    if c["op"] == "quant":
        M, K = c["M"], c["K"]
        s["x"] = _rows(gen, M, K, torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
        s["q"] = torch.empty(M, K, dtype=FP8, device="cuda")
        s["scale"] = torch.empty(M, _scale_ld(K), dtype=torch.uint8, device="cuda").view(E8)
    elif c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        for name, x in (("A", _rows(gen, M, K, torch.bfloat16)),
                        ("W", (torch.randn(N, K, generator=gen, device="cuda") / math.sqrt(K)).to(torch.bfloat16))):
            q, e = _quantise(x.float())
            sc = torch.full((x.shape[0], _scale_ld(K)), 127, dtype=torch.uint8, device="cuda")
            sc[:, :e.shape[1]] = e
            s[name], s[name + "s"] = q, sc.view(E8)
        s["bias"] = (0.1 * torch.randn(N, generator=gen, device="cuda")).to(torch.bfloat16)
        dt = dict(bf16=torch.bfloat16, f32=torch.float32, fp8=FP8)[c["out"]]
        s["C"] = torch.empty(M, N, dtype=dt, device="cuda")
        if c["out"] == "fp8":
            s["Cs"] = torch.empty(M, _scale_ld(N), dtype=torch.uint8, device="cuda").view(E8)
    else:
        B, Lq, Lk, H, G = c["B"], c["Lq"], c["Lk"], c["heads"], c["kv_heads"]
        s["q"], s["k"] = _tokens(gen, B, Lq, H), _tokens(gen, B, Lk, G)
        s["klen"] = None
        if c["pad"]:  # filled to different lengths
            s["klen"] = torch.randint((Lk + 1) // 2, Lk + 1, (B,), generator=gen, device="cuda").int()
        nqb = -(-Lq // QB)
        if c["op"] == "select":
            s["idx"] = torch.empty(B, H, nqb, c["topk"], dtype=torch.int32, device="cuda")
        else:
            s["v"] = torch.randn(B * Lk, G * D, generator=gen, device="cuda").to(torch.bfloat16)
            s["idx"] = _select(c, s["q"], s["k"], s["klen"])
            s["o"] = torch.empty(B * Lq, H * D, dtype=torch.bfloat16, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms

def _quantise(x):
    """f32 rows -> (e4m3 values of x / 2^e, e + 127): e the least with max |x| <= 448 * 2^e over 128 values."""
    M, K = x.shape
    nb = -(-K // 128)
    xb = torch.nn.functional.pad(x, (0, nb * 128 - K)).view(M, nb, 128)
    m, e = torch.frexp(xb.abs().amax(-1))          # m 2^e, 1/2 <= m < 1;  448 = 7/8 * 2^9
    byte = (e - 9 + (m > 0.875).int() + 127).clamp(min=0)
    byte = torch.where(m == 0, 0, byte)
    q = torch.ldexp(xb, (127 - byte)[..., None]).to(FP8)
    return q.view(M, nb * 128)[:, :K].contiguous(), byte.to(torch.uint8)


def _values(q, scale):
    """The f32 values that 8-bit rows and their scales stand for."""
    M, K = q.shape
    s = scale[:, :-(-K // 128)].float().repeat_interleave(128, 1)[:, :K]
    return q.float() * s


def _epilogue(c, y):
    if c["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    elif c["act"] == "gelu":
        u = math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)
        y = y / (1 + torch.exp(-2 * u))
    elif c["act"] == "rms":
        h = y.view(y.shape[0], -1, 128)
        y = (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6)).view_as(y)
    return y


def _pooled(x, B, L, H, block, klen):
    """Mean of each block's valid rows, float64 [B, H, blocks, D]."""
    n = -(-L // block)
    x = x.double().view(B, L, H, D)
    rows = torch.arange(n * block, device=x.device).view(1, n, block)
    limit = torch.full((B, 1, 1), L, device=x.device) if klen is None else klen.long().view(B, 1, 1)
    ok = rows < limit
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, n * block - L)).view(B, n, block, H, D)
    x = torch.where(ok[..., None, None], x, 0.0).sum(2) / ok.sum(-1).clamp(min=1)[..., None, None]
    return x.permute(0, 2, 1, 3), ok[:, :, 0]


def _select(c, q, k, klen):
    B, H, G, topk = c["B"], c["heads"], c["kv_heads"], c["topk"]
    qm, _ = _pooled(q, B, c["Lq"], H, QB, None)
    km, ok = _pooled(k, B, c["Lk"], G, KB, klen)
    nkb = km.shape[2]
    s = qm @ km.repeat_interleave(H // G, 1).transpose(2, 3).contiguous()
    s = torch.where(torch.isnan(s), -math.inf, s)
    s[..., :c["first"]] = math.inf
    s = torch.where(ok[:, None, None], s, -math.inf)   # these lie behind all others: equal values go by index
    idx = torch.sort(s, dim=-1, descending=True, stable=True).indices[..., :topk]
    idx = torch.where(idx < ok.sum(-1).view(B, 1, 1, 1), idx, nkb)
    idx = torch.sort(idx, dim=-1).values
    idx = torch.nn.functional.pad(idx, (0, topk - idx.shape[-1]), value=nkb)
    return torch.where(idx == nkb, -1, idx).int()


def _attend(q, k, v, idx, klen, Lk):
    """Attention of one query block per row of idx: q [..., QB, D], k and v the listed blocks [..., topk, KB, D]."""
    at = idx[..., None] * KB + torch.arange(KB, device=idx.device)
    ok = ((idx[..., None] >= 0) & (at < klen)).flatten(-2)
    k, v = k.flatten(-3, -2), torch.where(ok[..., None], v.flatten(-3, -2), 0.0)
    s = q @ k.transpose(-1, -2).contiguous() / math.sqrt(D)
    s = torch.where(ok[..., None, :], s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(m), 0.0, m))
    den = p.sum(-1, keepdim=True)
    return (p @ v) / torch.where(den == 0, 1.0, den)


def _blocks(x, B, L, H, block, dtype):
    n = -(-L // block)
    x = torch.nn.functional.pad(x.view(B, L, H, D), (0, 0, 0, 0, 0, n * block - L))
    return x.view(B, n, block, H, D).permute(0, 3, 1, 2, 4).to(dtype)


def _plain(s):
    c = s["case"]
    if c["op"] == "quant":
        q, e = _quantise(s["x"].float())
        return dict(q=q, scale=e.view(E8))
    if c["op"] == "gemm":
        y = _values(s["A"], s["As"]) @ _values(s["W"], s["Ws"]).t() + s["bias"].float()
        y = _epilogue(c, y)
        if c["out"] == "fp8":
            q, e = _quantise(y)
            return dict(q=q, scale=e.view(E8))
        return y.to(s["C"].dtype)
    if c["op"] == "select":
        return _select(c, s["q"], s["k"], s["klen"])
    B, Lq, Lk, H, G = c["B"], c["Lq"], c["Lk"], c["heads"], c["kv_heads"]
    q = _blocks(s["q"], B, Lq, H, QB, torch.float32)
    k, v = (_blocks(s[n], B, Lk, G, KB, torch.float32) for n in "kv")
    idx = s["idx"].long()
    b = torch.arange(B, device=idx.device).view(B, 1, 1, 1)
    h = (torch.arange(H, device=idx.device) // (H // G)).view(1, H, 1, 1)
    at = idx.clamp(min=0)
    klen = Lk if s["klen"] is None else s["klen"].view(B, 1, 1, 1, 1)
    o = _attend(q, k[b, h, at], v[b, h, at], idx, klen, Lk)
    return o.permute(0, 2, 3, 1, 4).reshape(B, -1, H * D)[:, :Lq].reshape(B * Lq, H * D).to(torch.bfloat16)


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2608_09231_amd import binding as lib
    c = s["case"]
    if c["op"] == "quant":
        lib.quant_fp8(s["x"], s["q"], s["scale"], M=c["M"], K=c["K"])
        return dict(q=s["q"], scale=s["scale"][:, :-(-c["K"] // 128)])
    if c["op"] == "gemm":
        flags = dict(bf16=lib.EPI_STORE, f32=lib.EPI_F32, fp8=lib.EPI_FP8)[c["out"]]
        lib.gemm_fp8(s["A"], s["As"], s["W"], s["Ws"], s["bias"], s["C"], M=c["M"], N=c["N"], K=c["K"],
                     flags=flags | (lib.EPI_SILU if c["act"] == "silu" else 0), c_scale=s.get("Cs"),
                     gelu_from=0 if c["act"] == "gelu" else None, rms_cols=c["N"] if c["act"] == "rms" else 0)
        if c["out"] == "fp8":
            return dict(q=s["C"], scale=s["Cs"][:, :c["N"] // 128])
        return s["C"]
    shape = dict(Lq=c["Lq"], Lk=c["Lk"], heads=c["heads"], kv_heads=c["kv_heads"], batch=c["B"], topk=c["topk"],
                 klen=s["klen"])
    if c["op"] == "select":
        lib.select_blocks_bf16(s["q"], s["k"], s["idx"], first=c["first"], **shape)
        return s["idx"]
    lib.attention_sparse_bf16(s["q"], s["k"], s["v"], s["o"], s["idx"],
                              flags=lib.ATTN_BOUNDED_LOGITS if c["bounded"] else 0, **shape)
    return s["o"]


# ---------------------------------------------------------------- measure and reference

def work(case):
    c = case
    if c["op"] == "quant":
        M, K = c["M"], c["K"]
        return dict(bytes=M * K * ((2 if c["dtype"] == "bf16" else 4) + 1) + M * -(-K // 128), flops=2 * M * K)
    if c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        out = dict(bf16=2, f32=4, fp8=1 + 1 / 128)[c["out"]]
        return dict(bytes=(M + N) * (K + -(-K // 128)) + 2 * N + M * N * out, flops=2 * M * N * K)
    B, Lq, Lk, H, G, topk = (c[n] for n in ("B", "Lq", "Lk", "heads", "kv_heads", "topk"))
    nqb, nkb = -(-Lq // QB), -(-Lk // KB)
    index = 4 * B * H * nqb * topk
    if c["op"] == "select":
        return dict(bytes=2 * D * B * (Lq * H + Lk * G) + index,
                    flops=D * B * (Lq * H + Lk * G) + 2 * D * B * H * nqb * nkb)
    listed_keys = min(topk * KB, Lk)
    keys = min(Lk * G, H * nqb * listed_keys)   # rows of K and V that are read at all, at most
    return dict(bytes=2 * D * B * (2 * Lq * H + 2 * keys) + index, flops=4 * D * B * H * Lq * listed_keys)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "quant":
        x = s["x"].double()
        M, K = x.shape
        nb = -(-K // 128)
        xb = torch.cat([x, x.new_zeros(M, nb * 128 - K)], 1).view(M, nb, 128)
        a = xb.abs().amax(-1)
        e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 448)).clamp(min=-127)
        e += (a > 448 * torch.exp2(e)).double()       # the logarithm may be a step off at the borders
        e -= ((e > -127) & (a <= 448 * torch.exp2(e - 1))).double()
        y = xb / torch.exp2(e)[..., None]
        grid = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)   # e4m3's spacing at y
        return dict(q=(torch.round(y / grid) * grid).view(M, -1)[:, :K], scale=torch.exp2(e))
    if c["op"] == "gemm":
        if c["out"] == "fp8":
            return None   # rounded to 8 bits with a scale of its own: there is no such value in 64 bits
        M, K = s["A"].shape

        def full(q, sc):
            v = q.double()
            for b in range(-(-K // 128)):
                v[:, 128 * b:128 * b + 128] *= sc[:, b:b + 1].double()
            return v
        y = torch.addmm(s["bias"].double(), full(s["A"], s["As"]), full(s["W"], s["Ws"]).t())
        if c["act"] == "silu":
            y = y * torch.sigmoid(y)
        elif c["act"] == "gelu":
            y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        elif c["act"] == "rms":
            for h in range(0, y.shape[1], 128):
                y[:, h:h + 128] /= (y[:, h:h + 128].pow(2).mean(1, keepdim=True) + 1e-6).sqrt()
        return y
    if c["op"] == "select":
        return None
    B, Lq, Lk, H, G = c["B"], c["Lq"], c["Lk"], c["heads"], c["kv_heads"]
    out = torch.zeros(B * Lq, H * D, dtype=torch.float64, device="cuda")
    nqb, nkb = -(-Lq // QB), -(-Lk // KB)
    for b in range(B):
        n = Lk if s["klen"] is None else int(s["klen"][b])
        for h in range(H):
            kv = slice(h // (H // G) * D, h // (H // G) * D + D)
            q = torch.zeros(nqb * QB, D, dtype=torch.float64, device="cuda")
            q[:Lq] = s["q"][b * Lq:(b + 1) * Lq, h * D:(h + 1) * D].double()
            k, v = (torch.zeros(nkb * KB, D, dtype=torch.float64, device="cuda") for _ in range(2))
            k[:n] = s["k"][b * Lk:b * Lk + n, kv].double()
            v[:n] = s["v"][b * Lk:b * Lk + n, kv].double()
            idx = s["idx"][b, h].long()
            rows = (idx[..., None] * KB + torch.arange(KB, device="cuda")).view(nqb, -1)
            gone = (rows < 0) | (rows >= n)
            rows = rows.clamp(min=0)
            t = torch.bmm(q.view(nqb, QB, D), k[rows].transpose(1, 2).contiguous()) / math.sqrt(D)
            t = t.masked_fill(gone[:, None], -math.inf)
            w = torch.nan_to_num(torch.softmax(t, -1), nan=0.0)
            out[b * Lq:(b + 1) * Lq, h * D:(h + 1) * D] = torch.bmm(w, v[rows]).view(-1, D)[:Lq]
    return out
