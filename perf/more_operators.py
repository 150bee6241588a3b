"""Cases of a prompt encoder's operators, with their plain forms.

The text tokens that the sampler is given come from a decoder-only encoder, and its blocks' own attention wants
positions: rotary positions of one to three axes (``rotary``), attention over packed sequences of different lengths
with grouped heads, causal or not, down to single tokens against a cache (``attend``), rows quantised to 4-bit
floating point with one scale per 32 values and back (``quant``), the product of two such matrices with a layer's
epilogue (``gemm``), and an MLP of them, whose middle stays in 4 bits (``mlp``).

``run`` computes an operator from elementary torch operations where ``own`` is false, and calls the library where
it is true.  ``exact`` computes the same in float64 from the definition.
"""
import math
import random

import torch

own = False

D = 128                                       # width of an attention head
E8 = torch.float8_e8m0fnu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
MAX_ROTARY = 32760 * 40 * 128                 # values of the largest rotation
MAX_PAIRS = 16 * 16384 * 16384                # (query, key, head) triples of the largest attention, masked ones included
MAX_CACHE = 64 * 8192 * 8                     # key rows times key heads
MAX_PRODUCT = 32760 * 13824 * 5120            # M N K of the largest product


def listed():
    return [
        # a few tokens far into a long text, f32, half of each head's width rotated, frequencies scaled for the length
        dict(name="rotary_far_f32", op="rotary", rows=37, heads=7, head_dim=128, rot=64, layout="half", axes=1,
             dtype="f32", reach=1 << 20, scaled=True),
        # queries of a video block: frame, row and column of 32760 tokens
        dict(name="rotary_video", op="rotary", rows=32760, heads=40, head_dim=128, rot=128, layout="interleaved", axes=3,
             dtype="bf16", reach=64, scaled=False),
        # one more token of 16 texts, each with its own length, keys and values in a cache of 8192 slots
        dict(name="attend_tokens", op="attend", mode="token", B=16, Lq=1, Lk=8192, heads=32, kv_heads=8, bounded=False),
        # a batch of prompts of up to 512 tokens, packed
        dict(name="attend_prompts", op="attend", mode="prompt", B=8, Lq=512, Lk=512, heads=28, kv_heads=4, bounded=False),
        # the next piece of texts whose beginnings are cached: odd lengths, one of them empty
        dict(name="attend_chunks", op="attend", mode="chunk", B=5, Lq=701, Lk=5003, heads=12, kv_heads=4, bounded=True),
        # one long text
        dict(name="attend_long", op="attend", mode="prompt", B=1, Lq=16384, Lk=16384, heads=16, kv_heads=4, bounded=False),
        # odd f32 rows
        dict(name="quant_ragged_f32", op="quant", M=1357, K=2592, dtype="f32"),
        # activations of a video block entering its linear layers
        dict(name="quant_video", op="quant", M=32760, K=5120, dtype="bf16"),
        # one row against a layer's weights: SiLU of a conditioning vector
        dict(name="gemm_row", op="gemm", M=1, N=13824, K=5120, out="bf16", act="silu"),
        # odd sizes: ragged in all three, f32 output
        dict(name="gemm_ragged_f32", op="gemm", M=1333, N=1000, K=2336, out="f32", act="none"),
        # the text tokens' key and value projection of a video block, keys normed per head
        dict(name="gemm_text", op="gemm", M=512, N=10240, K=5120, out="bf16", act="rms"),
        # the video block's MLP: its input quantised, up with GELU and 4-bit rows out, down
        dict(name="mlp_video", op="mlp", M=32760, N=13824, K=5120),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "attend", "attend", "quant", "gemm", "gemm", "mlp"])
    while op == "rotary":
        head_dim = rng.choice([64, 96, 128, 256])
        rot = head_dim if rng.random() < 0.6 else 2 * rng.randint(4, head_dim // 2)
        c = dict(op=op, rows=_log(rng, 1, 32760), heads=_log(rng, 1, 64), head_dim=head_dim, rot=rot,
                 layout=rng.choice(["half", "interleaved"]), axes=rng.choice([1, 1, 2, 3]),
                 dtype=rng.choice(["bf16", "bf16", "f32"]), reach=_log(rng, 64, 1 << 20), scaled=rng.random() < 0.3)
        if c["rows"] * c["heads"] * head_dim * (2 if c["dtype"] == "f32" else 1) <= MAX_ROTARY:
            return c
    if op == "quant":
        return dict(op=op, M=_log(rng, 1, 32760), K=32 * _log(rng, 1, 160), dtype=rng.choice(["bf16", "f32"]))
    while op == "gemm":
        M, K = _log(rng, 1, 32760), 32 * _log(rng, 2, 432)
        out = rng.choice(["bf16", "bf16", "f32"])
        act = rng.choice(["none", "silu", "gelu"] if out == "f32" else ["none", "silu", "gelu", "rms"])
        N = 128 * _log(rng, 1, 108) if act == "rms" else 8 * _log(rng, 8, 1728)
        if M * N * K <= MAX_PRODUCT:
            return dict(op=op, M=M, N=N, K=K, out=out, act=act)
    while op == "mlp":
        M, N, K = _log(rng, 1, 32760), 128 * _log(rng, 2, 108), 32 * _log(rng, 4, 160)
        if M * N * K <= MAX_PRODUCT:
            return dict(op=op, M=M, N=N, K=K)
    while True:
        mode = rng.choice(["token", "prompt", "chunk", "cross"])
        kv = rng.choice([1, 2, 3, 4, 8, 16])
        heads = kv * rng.choice([1, 1, 2, 4, 5, 7])
        B = _log(rng, 1, 64)
        Lk = _log(rng, 1, 16384)
        Lq = 1 if mode == "token" else Lk if mode == "prompt" else _log(rng, 1, 4096)
        if mode == "chunk":
            Lq = min(Lq, Lk)
        if heads <= 40 and B * heads * Lq * Lk <= MAX_PAIRS and B * Lk * kv <= MAX_CACHE and B * Lq * heads <= MAX_CACHE:
            return dict(op="attend", mode=mode, B=B, Lq=Lq, Lk=Lk, heads=heads, kv_heads=kv, bounded=rng.random() < 0.4)


def _scale_ld(K):
    return 4 * -(-K // 128)


def _lengths(c):
    """Queries and keys of each sequence; the first is the longest, the second, of three or more chunks, empty."""
    rng = random.Random("%(mode)s %(B)d %(Lq)d %(Lk)d" % c)
    kl = [c["Lk"]] + [rng.randint(min(c["Lk"], 1 + c["Lk"] // 16), c["Lk"]) for _ in range(c["B"] - 1)]
    if c["mode"] == "token":
        return [1] * c["B"], kl
    if c["mode"] == "prompt":
        return kl, kl
    ql = [c["Lq"]] + [rng.randint(1, c["Lq"]) for _ in range(c["B"] - 1)]
    if c["mode"] == "chunk":
        ql = [min(q, k) for q, k in zip(ql, kl)]
        if c["B"] > 2:
            ql[1] = 0
    return ql, kl


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _pairs_of_axes(c):
    n, a = c["rot"] // 2, c["axes"]
    return [n - (a - 1) * (n // a)] + [n // a] * (a - 1)


# ---------------------------------------------------------------- inputs

def _rows(gen, M, K, dtype):
    """Activations as they leave a norm: unit rows with some wide channels, and a few tokens far larger than the rest."""
    x = torch.randn(M, K, generator=gen, device="cuda")
    x *= torch.exp(0.7 * torch.randn(K, generator=gen, device="cuda"))
    x *= torch.where(torch.rand(M, 1, generator=gen, device="cuda") < 0.02, 30.0, 1.0)
    return x.to(dtype)


def _frequencies(c):
    """Radians per position of every pair, and the factor on cosine and sine: 10000^(-i / pairs) along each axis; where
    scaled, 16 times the trained 4096 positions: slow pairs (under a turn in those) divided by 16, fast ones (over 32
    turns) as they are, a ramp between."""
    axes = []
    for n in _pairs_of_axes(c):
        f = torch.exp(-math.log(1e4) / max(n, 1) * torch.arange(n, dtype=F64))
        if c["scaled"]:
            keep = ((4096 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
            f = f * keep + f / 16 * (1 - keep)
        axes.append(f)
    return torch.cat(axes), 0.1 * math.log(16) + 1 if c["scaled"] else 1.0


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def four_bits(rows, K, x):
        codes, e = _quantise(x.float())
        sc = torch.full((rows, _scale_ld(K)), 127, dtype=torch.uint8, device="cuda")
        sc[:, :e.shape[1]] = e
        return _pack(codes), sc.view(E8)

    s = dict(case=c)
    if c["op"] == "rotary":
        rows, width = c["rows"], c["heads"] * c["head_dim"]
        s["x"] = randn(rows, width).to(BF16 if c["dtype"] == "bf16" else F32)
        s["y"] = torch.empty_like(s["x"])
        s["pos"] = torch.randint(0, c["reach"], (c["axes"], rows), generator=gen, device="cuda").int()
        freq, s["scale"] = _frequencies(c)
        s["freq"], s["pairs"] = freq.cuda(), _pairs_of_axes(c)
    elif c["op"] == "attend":
        H, G = c["heads"], c["kv_heads"]
        ql, kl = _lengths(c)
        s["qoff"] = torch.tensor(_starts(ql), dtype=torch.int32).cuda()
        if c["mode"] in ("token", "chunk"):   # a cache: slots of Lk rows, filled to klen
            s["koff"] = torch.tensor([c["Lk"] * i for i in range(c["B"] + 1)], dtype=torch.int32).cuda()
            s["klen"] = torch.tensor(kl, dtype=torch.int32).cuda()
            rows_k = c["B"] * c["Lk"]
        else:
            s["koff"], s["klen"], rows_k = torch.tensor(_starts(kl), dtype=torch.int32).cuda(), None, sum(kl)
        q, k = randn(sum(ql), H, D), randn(rows_k, G, D)
        if c["bounded"]:
            q, k = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) for x in (q, k))
        s["q"], s["k"] = q.to(BF16).view(-1, H * D), k.to(BF16).view(-1, G * D)
        s["v"] = randn(rows_k, G * D).to(BF16)
        s["o"] = torch.empty(sum(ql), H * D, dtype=BF16, device="cuda")
    elif c["op"] == "quant":
        M, K = c["M"], c["K"]
        s["x"] = _rows(gen, M, K, BF16 if c["dtype"] == "bf16" else F32)
        s["q"] = torch.empty(M, K // 2, dtype=torch.uint8, device="cuda")
        s["qs"] = torch.empty(M, _scale_ld(K), dtype=torch.uint8, device="cuda").view(E8)
        s["y"] = torch.empty(M, K, dtype=BF16, device="cuda")
    else:
        M, N, K = c["M"], c["N"], c["K"]
        x = _rows(gen, M, K, BF16)
        s["W"], s["Ws"] = four_bits(N, K, (randn(N, K) / math.sqrt(K)).to(BF16))
        s["bias"] = (0.1 * randn(N)).to(BF16)
        if c["op"] == "gemm":
            s["A"], s["As"] = four_bits(M, K, x)
            s["C"] = torch.empty(M, N, dtype=BF16 if c["out"] == "bf16" else F32, device="cuda")
        else:
            s["x"] = x
            s["A"] = torch.empty(M, K // 2, dtype=torch.uint8, device="cuda")
            s["As"] = torch.empty(M, _scale_ld(K), dtype=torch.uint8, device="cuda").view(E8)
            s["h"] = torch.empty(M, N // 2, dtype=torch.uint8, device="cuda")
            s["hs"] = torch.empty(M, _scale_ld(N), dtype=torch.uint8, device="cuda").view(E8)
            s["W2"], s["W2s"] = four_bits(K, N, (randn(K, N) / math.sqrt(N)).to(BF16))
            s["bias2"] = (0.1 * randn(K)).to(BF16)
            s["C"] = torch.empty(M, K, dtype=BF16, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms

def _quantise(x):
    """f32 rows -> (e2m1 codes of x / 2^e, e + 127): e the least with max |x| <= 6 * 2^e over 32 values."""
    M, K = x.shape
    xb = x.view(M, K // 32, 32)
    m, e = torch.frexp(xb.abs().amax(-1))          # m 2^e, 1/2 <= m < 1;  6 = 3/4 * 2^3
    byte = (e - 3 + (m > 0.75).int() + 127).clamp(min=0)
    byte = torch.where(m == 0, 0, byte)
    y = torch.ldexp(xb, (127 - byte)[..., None])
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))   # between neighbours: 0 .5 1 1.5 2, 3 4, 6
    r = torch.round(a / step)                      # halves to even
    code = torch.where(a < 2, r, torch.where(a < 4, r + 2, r + 4)).to(torch.uint8)
    return (code + 8 * torch.signbit(y)).view(M, K), byte.to(torch.uint8)


def _pack(codes):
    """Two codes a byte, the first in the low half."""
    return codes[:, ::2] + 16 * codes[:, 1::2]


def _unpack(q):
    return torch.stack((q & 15, q >> 4), -1).view(q.shape[0], -1)


def _values(codes, byte):
    """The f32 values that 4-bit codes and their scales (E8M0) stand for."""
    e2m1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    v = e2m1[(codes & 7).int()] * (1 - 2 * (codes >> 3).float())
    return (v.view(codes.shape[0], -1, 32) * byte.float()[..., None]).view_as(v)


def _product(s, name, A, As, K):
    """A . W^T + bias in f32: A as codes, W as `name` of the state."""
    n = K // 32
    return _values(A, As[:, :n]) @ _values(_unpack(s[name]), s[name + "s"][:, :n]).t()


def _epilogue(act, y):
    if act == "silu":
        y = y / (1 + torch.exp(-y))
    elif act == "gelu":
        u = math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)
        y = y / (1 + torch.exp(-2 * u))
    elif act == "rms":
        h = y.view(y.shape[0], -1, 128)
        y = (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6)).view_as(y)
    return y


def _rotate(s):
    c = s["case"]
    n, rot = c["rot"] // 2, c["rot"]
    axis = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(s["pairs"])).cuda()
    angle = s["pos"].double()[axis].t() * s["freq"]             # [rows, pairs]
    cos, sin = ((f(angle) * s["scale"]).float()[:, None] for f in (torch.cos, torch.sin))
    x = s["x"].float().view(c["rows"], c["heads"], c["head_dim"])
    y = x.clone()
    first, second = (slice(0, n), slice(n, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = x[..., first], x[..., second]
    y[..., first] = a * cos - b * sin
    y[..., second] = b * cos + a * sin
    return y.view(c["rows"], -1).to(s["x"].dtype)


def _attend(s):
    c = s["case"]
    B, H, G, mq, mk = c["B"], c["heads"], c["kv_heads"], c["Lq"], c["Lk"]
    dev = s["q"].device
    q0, k0 = s["qoff"][:-1].long(), s["koff"][:-1].long()
    ql = s["qoff"][1:].long() - q0
    kl = s["klen"].long() if s["klen"] is not None else s["koff"][1:].long() - k0
    i, j = torch.arange(mq, device=dev), torch.arange(mk, device=dev)
    Tq, Tk = s["q"].shape[0], s["k"].shape[0]
    qi = (q0[:, None] + i).clamp(max=Tq - 1)
    ki = (k0[:, None] + j).clamp(max=Tk - 1)
    q = s["q"].float().view(Tq, H, D)[qi].view(B, mq, G, H // G, D).permute(0, 2, 3, 1, 4)
    k, v = (s[n].float().view(Tk, G, D)[ki].permute(0, 2, 1, 3) for n in "kv")
    t = q.reshape(B, G, -1, D) @ k.transpose(2, 3).contiguous()
    t = t.view(B, G, H // G, mq, mk).div_(math.sqrt(D))
    seen = (j < kl[:, None])[:, None]                             # [B, queries, keys]
    if c["mode"] != "cross":                                     # a sequence's last query sees its last key
        seen = seen & (j <= i[:, None] + (kl - ql)[:, None, None])
    t.masked_fill_(~seen[:, None, None], -math.inf)
    m = t.amax(-1, keepdim=True)
    t = t.sub_(torch.where(torch.isinf(m), 0.0, m)).exp_()
    den = t.sum(-1, keepdim=True)
    o = (t.view(B, G, -1, mk) @ v.contiguous()).view(B, G, H // G, mq, D) / torch.where(den == 0, 1.0, den)
    rows = torch.where(i < ql[:, None], qi, Tq).view(-1)          # (past the last query: a row that is dropped)
    out = torch.empty(Tq + 1, H * D, dtype=BF16, device=dev)
    out[rows] = o.permute(0, 3, 1, 2, 4).reshape(B * mq, H * D).to(BF16)
    return out[:Tq]


def _plain(s):
    c = s["case"]
    if c["op"] == "rotary":
        return _rotate(s)
    if c["op"] == "attend":
        return _attend(s)
    if c["op"] == "quant":
        codes, e = _quantise(s["x"].float())
        return dict(values=_values(codes, e.view(E8)).to(BF16), scale=e.view(E8))
    K, N = c["K"], c["N"]
    if c["op"] == "gemm":
        y = _product(s, "W", _unpack(s["A"]), s["As"], K) + s["bias"].float()
        return _epilogue(c["act"], y).to(s["C"].dtype)
    codes, e = _quantise(s["x"].float())
    y = _epilogue("gelu", _product(s, "W", codes, e.view(E8), K) + s["bias"].float())
    codes, e = _quantise(y)
    return (_product(s, "W2", codes, e.view(E8), N) + s["bias2"].float()).to(BF16)


def run(state):
    s = state
    if not own:
        return _plain(s)
    else:  # (the rows that prepare packs are whole numbers of 64 bits; the calls take bytes)
        s = {**s, **{n: s[n].to(torch.uint8) for n in ("A", "W", "W2") if n in s}}
    from paper_2608_09231_amd import binding as lib
    c = s["case"]
    if c["op"] == "rotary":
        lib.rotary(s["x"], s["y"], pos=s["pos"], freq=s["freq"], rows=c["rows"], heads=c["heads"],
                   head_dim=c["head_dim"], pairs=s["pairs"], scale=s["scale"],
                   layout=lib.ROTARY_HALF if c["layout"] == "half" else lib.ROTARY_INTERLEAVED)
        return s["y"]
    if c["op"] == "attend":
        lib.attention_packed_bf16(s["q"], s["k"], s["v"], s["o"], qoff=s["qoff"], koff=s["koff"], klen=s["klen"],
                                  heads=c["heads"], kv_heads=c["kv_heads"],
                                  flags=(lib.ATTN_BOUNDED_LOGITS if c["bounded"] else 0)
                                  | (lib.ATTN_CAUSAL if c["mode"] != "cross" else 0))
        return s["o"]
    M, K = c["M"], c["K"]
    if c["op"] == "quant":
        lib.quant_fp4(s["x"], s["q"], s["qs"], M=M, K=K)
        lib.dequant_fp4(s["q"], s["qs"], s["y"], M=M, K=K)
        return dict(values=s["y"], scale=s["qs"][:, :K // 32])
    N = c["N"]
    if c["op"] == "gemm":
        flags = (lib.EPI_F32 if c["out"] == "f32" else lib.EPI_STORE) | (lib.EPI_SILU if c["act"] == "silu" else 0)
        lib.gemm_fp4(s["A"], s["As"], s["W"], s["Ws"], s["bias"], s["C"], M=M, N=N, K=K, flags=flags,
                     gelu_from=0 if c["act"] == "gelu" else None, rms_cols=N if c["act"] == "rms" else 0)
        return s["C"]
    lib.quant_fp4(s["x"], s["A"], s["As"], M=M, K=K)
    lib.gemm_fp4(s["A"], s["As"], s["W"], s["Ws"], s["bias"], s["h"], M=M, N=N, K=K, flags=lib.EPI_FP4, gelu_from=0,
                 c_scale=s["hs"])
    lib.gemm_fp4(s["h"], s["hs"], s["W2"], s["W2s"], s["bias2"], s["C"], M=M, N=K, K=N)
    return s["C"]


# ---------------------------------------------------------------- measure and reference

def work(case):
    c = case
    if c["op"] == "rotary":
        n = c["rows"] * c["heads"] * c["head_dim"]
        return dict(bytes=2 * n * (2 if c["dtype"] == "bf16" else 4) + 4 * c["axes"] * c["rows"] + 4 * c["rot"],
                    flops=3 * c["rows"] * c["heads"] * c["rot"])
    if c["op"] == "attend":
        H, G = c["heads"], c["kv_heads"]
        ql, kl = _lengths(c)
        # pairs that the mask leaves: query i of n sees the first m - n + 1 + i of m keys
        pairs = sum(q * k - (q * (q - 1) // 2 if c["mode"] != "cross" else 0) for q, k in zip(ql, kl))
        keys = sum(k for q, k in zip(ql, kl) if q)
        return dict(bytes=2 * D * (2 * H * sum(ql) + 2 * G * keys) + 12 * c["B"], flops=4 * D * H * pairs)
    M, K = c["M"], c["K"]

    def four(rows, width):
        return rows * width // 2 + rows * width // 32

    if c["op"] == "quant":
        return dict(bytes=M * K * ((2 if c["dtype"] == "bf16" else 4) + 2) + 2 * four(M, K), flops=3 * M * K)
    N = c["N"]
    if c["op"] == "gemm":
        return dict(bytes=four(M, K) + four(N, K) + 2 * N + M * N * (2 if c["out"] == "bf16" else 4), flops=2 * M * N * K)
    return dict(bytes=2 * M * K + 2 * four(N, K) + 2 * N + 2 * K + 2 * M * K, flops=4 * M * N * K)


def _grid(x):
    """float64 rows -> (the nearest values of their 4-bit form, scales)."""
    M, K = x.shape
    xb = x.reshape(M, K // 32, 32)
    a = xb.abs().amax(-1)
    e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 6)).clamp(min=-127)
    e += (a > 6 * torch.exp2(e)).double()         # the logarithm may be a step off at the borders
    e -= ((e > -127) & (a <= 6 * torch.exp2(e - 1))).double()
    sc = torch.exp2(e)[..., None]
    y = xb / sc
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1))) - 1)
    return (torch.round(y / step) * step * sc).view(M, K), sc[..., 0]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "rotary":
        n, rot = c["rot"] // 2, c["rot"]
        turn = torch.cat([s["pos"][a].double()[:, None] * f for a, f in enumerate(torch.split(s["freq"], s["pairs"]))], 1)
        w = torch.polar(torch.full_like(turn, s["scale"]), turn)[:, None]
        y = s["x"].double().view(c["rows"], c["heads"], c["head_dim"])
        if c["layout"] == "half":
            z = torch.complex(y[..., :n], y[..., n:rot]) * w
            z = torch.cat([z.real, z.imag], -1)
        else:
            z = torch.view_as_real(torch.view_as_complex(y[..., :rot].reshape(*y.shape[:2], n, 2)) * w).flatten(-2)
        return torch.cat([z, y[..., rot:]], -1).view(c["rows"], -1)
    if c["op"] == "attend":
        H, G = c["heads"], c["kv_heads"]
        out = torch.zeros(s["q"].shape[0], H * D, dtype=F64, device="cuda")
        qoff, koff = s["qoff"].tolist(), s["koff"].tolist()
        for b, n in enumerate(_lengths(c)[1]):
            lq = qoff[b + 1] - qoff[b]
            if not lq or not n:
                continue
            for h in range(H):
                kv = slice(h // (H // G) * D, h // (H // G) * D + D)
                k, v = (s[x][koff[b]:koff[b] + n, kv].double() for x in "kv")
                for r in range(0, lq, 4096):
                    at = torch.arange(r, min(lq, r + 4096), device="cuda")
                    t = s["q"][qoff[b] + at, h * D:h * D + D].double() @ k.t() / math.sqrt(D)
                    if c["mode"] != "cross":
                        t = t.masked_fill(torch.arange(n, device="cuda") > at[:, None] + (n - lq), -math.inf)
                    out[qoff[b] + at, h * D:h * D + D] = torch.nan_to_num(torch.softmax(t, -1), nan=0.0) @ v
        return out
    if c["op"] == "quant":
        y, sc = _grid(s["x"].double())
        return dict(values=y, scale=sc)

    def full(q, sc):
        table = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
        table = torch.tensor(table + [-x for x in table], dtype=F64, device="cuda")
        v = torch.empty(q.shape[0], 2 * q.shape[1], dtype=F64, device="cuda")
        v[:, ::2], v[:, 1::2] = table[(q % 16).long()], table[(q // 16).long()]
        n = q.shape[1] // 16
        return v * torch.repeat_interleave(sc[:, :n].double(), 32, 1)

    def gelu(y):
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))

    W = full(s["W"], s["Ws"])
    if c["op"] == "mlp":
        y = gelu(torch.addmm(s["bias"].double(), _grid(s["x"].double())[0], W.t()))
        return torch.addmm(s["bias2"].double(), _grid(y)[0], full(s["W2"], s["W2s"]).t())
    y = torch.addmm(s["bias"].double(), full(s["A"], s["As"]), W.t())
    if c["act"] == "silu":
        y = y * torch.sigmoid(y)
    elif c["act"] == "gelu":
        y = gelu(y)
    elif c["act"] == "rms":
        y = y.view(y.shape[0], -1, 128)
        y = (y / (y.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()).flatten(1)
    return y
