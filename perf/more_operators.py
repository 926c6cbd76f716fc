"""The model's end in front of the vocabulary projection, and that projection in 4
bits: the last residual addition with its root-mean-square norm and an output in
8-bit integers (norm8) or in microscaled 4-bit floating point (norm4), matrices
into the 4-bit format and back (mx4), and the logits from 4-bit weights under the
grammar's masks, with the norm in front (head4).

Every case runs either the operators' plain forms (elementary torch operations in
32 bits) or, where `own` is true, the calls of the library's binding.

norm     h = x + residual, rounded to their type;  r = 1 / sqrt(mean(h^2) + eps);
         v = h * gain in 32 bits
norm8    s = max|v| / 127, q = rint(v / s), scale = s r
mx4      blocks of 32 columns share 2^e, e = floor(log2 max|v|) - 2; a value is the
         nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^e with its sign (ties to the even
         code, 6 at most)
norm4    v in mx4, scale = r
head4    y[t][n] = (sum_k x_t[k] w_n[k]) scale_t c_n over values of mx4, -inf where the
         mask forbids n
Codes are packed two a byte, the even column in the low half.  Blocks' exponents are
bytes e + 127 in tiles of 128 rows by 4 blocks (512 bytes; tiles of the same rows
follow each other): row r, block b of a tile at 16 (r % 32) + 4 (r / 32) + b.
"""
import math

import torch

own = False

NEG = -math.inf
EPS = 1e-5
INV127 = 1.0 / 127.0


def _psc():
    from paper_2608_03065_gb300 import psc
    return psc


# ------------------------------------------------------------------- the cases
def listed():
    return [
        # one stream's token: latency
        {"name": "norm8 t1 k2048", "op": "norm8", "T": 1, "K": 2048, "dtype": "bf16", "residual": True},
        # an odd batch in f32, a width that no vector divides
        {"name": "norm8 t201 k5001 f32", "op": "norm8", "T": 201, "K": 5001, "dtype": "f32", "residual": True},
        # all tokens of a prompt, as teacher forcing scores them
        {"name": "norm8 t16384 k4096", "op": "norm8", "T": 16384, "K": 4096, "dtype": "bf16", "residual": True},
        # hidden states that come without a residual, ragged rows
        {"name": "mx4 t37 k2047", "op": "mx4", "T": 37, "K": 2047, "dtype": "bf16"},
        # the projection's weights, laid out once from f32 and read back to measure what 4 bits lose
        {"name": "mx4 t151936 k1024 f32", "op": "mx4", "T": 151936, "K": 1024, "dtype": "f32"},
        # one stream's token
        {"name": "norm4 t1 k4096", "op": "norm4", "T": 1, "K": 4096, "dtype": "bf16", "residual": True},
        # a verification batch of many drafts, no residual
        {"name": "norm4 t8192 k2048", "op": "norm4", "T": 8192, "K": 2048, "dtype": "bf16", "residual": False},
        # one stream: the weights are read for one token
        {"name": "head4 t1 v128256 k2048", "op": "head4", "T": 1, "V": 128256, "K": 2048, "dtype": "bf16",
         "mask": "none", "w_scale": False},
        # few rows inside punctuation and keywords: the grammar leaves a few dozen tokens each
        {"name": "head4 t16 v151936 k1024 tight", "op": "head4", "T": 16, "V": 151936, "K": 1024, "dtype": "f32",
         "mask": "tight", "w_scale": True},
        # an odd batch over a small vocabulary of odd size and a ragged width
        {"name": "head4 t45 v32001 k1500", "op": "head4", "T": 45, "V": 32001, "K": 1500, "dtype": "f32",
         "mask": "mixed", "w_scale": True},
        # a serving batch
        {"name": "head4 t256 v128256 k4096", "op": "head4", "T": 256, "V": 128256, "K": 4096, "dtype": "bf16",
         "mask": "none", "w_scale": False},
        # the benchmark's batch and vocabulary
        {"name": "head4 t1024 v262144 k2048", "op": "head4", "T": 1024, "V": 262144, "K": 2048, "dtype": "bf16",
         "mask": "mixed", "w_scale": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["norm8", "mx4", "norm4", "head4", "head4"])
    c = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "head4":
        T, V, K = _log_int(rng, 1, 1024), _log_int(rng, 500, 262144), _log_int(rng, 64, 4096)
        if rng.random() < 0.7:
            K = -(-K // 32) * 32
        while T * V * K > 1024 * 262144 * 2048:
            T = max(1, T // 2)
        if c["dtype"] == "f32" and T * V > 512 * 262144:
            c["dtype"] = "bf16"
        c.update(T=T, V=V, K=K, mask=rng.choice(["none", "tight", "mixed"]), w_scale=rng.random() < 0.5)
    else:
        T, K = _log_int(rng, 1, 65536 if op == "mx4" else 16384), _log_int(rng, 64, 16384)
        if rng.random() < 0.6:
            K = -(-K // 8) * 8
        while T * K > 16384 * 4096:
            T = max(1, T // 2)
        if c["dtype"] == "f32" and T * K > 8192 * 4096:
            c["dtype"] = "bf16"
        c.update(T=T, K=K)
        if op != "mx4":
            c["residual"] = rng.random() < 0.7
    return c


# ------------------------------------------------------------------- the inputs
#: Shares of a vocabulary that grammars leave open: nothing (a failed row), one token
#: (a literal's rest), a few dozen (keywords, punctuation), and rows inside names,
#: strings or comments.  Negative: a number of tokens.
_SHARES = {"mixed": ([0.0, -1.0, -48.0, 0.02, 0.45, 0.95], [0.03, 0.05, 0.22, 0.20, 0.30, 0.20]),
           "tight": ([0.0, -1.0, -8.0, -48.0], [0.04, 0.16, 0.4, 0.4])}
_TOKENS = {"tight": 0.16 + 0.4 * 8 + 0.4 * 48}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _pack_bits(bits):
    """[B, V] truth values -> int32 [B, ceil(V / 32)], bit v & 31 of word v >> 5."""
    B, V = bits.shape
    bits = torch.nn.functional.pad(bits, (0, -V % 32)).view(B, -1, 32)
    words = (bits.to(torch.int32) << torch.arange(32, device=bits.device, dtype=torch.int32)).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def _bitmask(kind, B, V, g):
    if kind == "none":
        return None
    shares, odds = _SHARES[kind]
    pick = torch.multinomial(torch.tensor(odds, device="cuda"), B, replacement=True, generator=g)
    share = torch.tensor([s if s >= 0 else -s / V for s in shares], device="cuda")[pick]
    out = torch.empty(B, (V + 31) // 32, dtype=torch.int32, device="cuda")
    for lo in range(0, B, 128):
        hi = min(B, lo + 128)
        out[lo:hi] = _pack_bits(torch.rand(hi - lo, V, device="cuda", generator=g) < share[lo:hi, None])
    return out


def _hidden(T, K, g, dtype):
    """Hidden states: rows of different sizes, a few loud channels."""
    out = torch.empty(T, K, dtype=dtype, device="cuda")
    loud = 1 + 9 * (torch.rand(1, K, device="cuda", generator=g) < 0.01)
    for lo in range(0, T, 4096):
        n = min(T, lo + 4096) - lo
        x = torch.randn(n, K, device="cuda", generator=g)
        out[lo:lo + n] = x * loud * (0.5 + torch.rand(n, 1, device="cuda", generator=g))
    return out


def _row_bytes(K):
    return (K + 31) // 32 * 16


def _tile_bytes(rows, K):
    return (rows + 127) // 128 * ((K + 127) // 128) * 512


def _weights(V, K, g):
    """The projection's weights in mx4: packed codes [V, row bytes] and tiles of exponents."""
    RT, KT = (V + 127) // 128, (K + 127) // 128
    w = torch.zeros(V, _row_bytes(K), dtype=torch.uint8, device="cuda")
    tiles = torch.zeros(RT, KT, 32, 4, 4, dtype=torch.uint8, device="cuda")
    for lo in range(0, V, 16384):
        n = min(V, lo + 16384) - lo
        f = torch.zeros(n, KT * 128, device="cuda")
        # rows of different sizes, as those of frequent and rare tokens
        f[:, :K] = torch.randn(n, K, device="cuda", generator=g) * (K ** -0.5)
        f *= 0.5 + torch.rand(n, 1, device="cuda", generator=g)
        f = f.view(n, -1, 32)
        e = torch.frexp(f.abs().amax(-1)).exponent - 3
        u = torch.ldexp(f, -e[..., None])
        a = u.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        a = ((a / step).round() * step).clamp(max=6)
        code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)) + 8 * (u < 0)
        code = code.to(torch.uint8).view(n, -1)
        w[lo:lo + n] = (code[:, 0::2] | (code[:, 1::2] << 4))[:, :w.shape[1]]
        full = torch.zeros(-(-n // 128) * 128, KT * 4, dtype=torch.uint8, device="cuda")
        full[:n] = (e + 127).to(torch.uint8)
        tiles[lo // 128:lo // 128 + full.shape[0] // 128] = full.view(-1, 4, 32, KT, 4).permute(0, 3, 2, 1, 4)
    return w, tiles.view(-1)


def prepare(case, seed):
    c, g = case, _gen(seed)
    T, K, dt = c["T"], c["K"], _dtype(c)
    s = {"op": c["op"], "K": K, "dtype": dt, "x": _hidden(T, K, g, torch.bfloat16 if c["op"] == "head4" else dt)}
    if c["op"] != "mx4":
        s["gain"] = 1 + 0.2 * torch.randn(K, device="cuda", generator=g)
        s["residual"] = 3 * _hidden(T, K, g, s["x"].dtype) if c.get("residual", True) else None
        s["sum"] = torch.empty_like(s["x"]) if c.get("residual", True) else None
        s["scale"] = torch.empty(T, device="cuda")
    if c["op"] == "norm8":
        s["q"] = torch.empty(T, K, dtype=torch.int8, device="cuda")
    else:
        s["q"] = torch.zeros(T, _row_bytes(K), dtype=torch.uint8, device="cuda")
        s["blocks"] = torch.zeros(_tile_bytes(T, K), dtype=torch.uint8, device="cuda")
        if c["op"] != "head4":
            s["y"] = torch.empty(T, K, dtype=dt, device="cuda")
    if c["op"] == "head4":
        V = c["V"]
        s["w"], s["w_blocks"] = _weights(V, K, g)
        s["w_scale"] = 0.5 + torch.rand(V, device="cuda", generator=g) if c["w_scale"] else None
        s["bitmask"] = _bitmask(c["mask"], T, V, g)
        s["logits"] = torch.empty(T, V, dtype=dt, device="cuda")
    return s


# --------------------------------------------------------------- the plain forms
def _plain_norm(s):
    """h in its type (None without a residual), v and r in 32 bits."""
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(h.dtype)
    f = h.float()
    r = 1.0 / torch.sqrt((f * f).mean(1) + EPS)
    return (h if s["residual"] is not None else None), f * s["gain"][None], r


def _plain_mx4(v):
    """The values that 4 bits keep of v."""
    T, K = v.shape
    b = torch.nn.functional.pad(v, (0, -K % 32)).view(T, -1, 32)
    top = torch.ldexp(torch.ones((), device=v.device), torch.frexp(b.abs().amax(-1, keepdim=True)).exponent - 3)
    u = b / top
    a = u.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = ((a / step).round() * step).clamp(max=6)
    return (torch.where(u < 0, -a, a) * top).view(T, -1)[:, :K]


def _plain_weights(w, blocks, V, K):
    """Packed codes and tiles of exponents -> values [V, K]."""
    values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=w.device)
    f = torch.stack((values[(w & 15).int()], values[(w >> 4).int()]), -1).view(V, -1, 32)
    e = blocks.view((V + 127) // 128, -1, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, (K + 127) // 128 * 4)
    top = torch.ldexp(torch.ones((), device=w.device), e[:V, :f.shape[1]].int() - 127)
    return (f * top[..., None]).view(V, -1)[:, :K]


def _allowed(words, V):
    """[B, W] packed words -> [B, V] truth values."""
    bits = (words[:, :, None] >> torch.arange(32, device=words.device, dtype=torch.int32)) & 1
    return bits.view(words.shape[0], -1)[:, :V].bool()


def _plain_norm8(s):
    h, v, r = _plain_norm(s)
    m = v.abs().amax(1) * INV127
    q = (v / m[:, None]).round().clamp(-127, 127).to(torch.int8)
    return {"sum": h, "q": q, "scale": m * r}


def _plain_norm4(s):
    h, v, r = _plain_norm(s)
    return {"sum": h, "y": (_plain_mx4(v) * r[:, None]).to(s["dtype"]), "scale": r}


def _plain_head4(s):
    h, v, r = _plain_norm(s)
    V, K = s["w"].shape[0], s["K"]
    y = (_plain_mx4(v) @ _plain_weights(s["w"], s["w_blocks"], V, K).t()) * r[:, None]
    if s["w_scale"] is not None:
        y = y * s["w_scale"][None]
    if s["bitmask"] is not None:
        y = torch.where(_allowed(s["bitmask"], V), y, NEG)
    return {"sum": h, "logits": y.to(s["dtype"]), "scale": r}


# ------------------------------------------------------------------- one pass
def run(state):
    s = state
    if not own:
        if s["op"] == "mx4":
            return _plain_mx4(s["x"].float()).to(s["dtype"])
        return {"norm8": _plain_norm8, "norm4": _plain_norm4, "head4": _plain_head4}[s["op"]](s)
    psc = _psc()
    if s["op"] == "mx4":
        psc.psc_quantize_mx4(s["x"], s["q"], s["blocks"])
        psc.psc_dequantize_mx4(s["q"], s["blocks"], s["y"])
        return s["y"]
    if s["op"] == "norm8":
        psc.psc_norm_quantize_rows(s["x"], s["q"], s["scale"], gain=s["gain"], eps=EPS, residual=s["residual"],
                                   sum_out=s["sum"])
        return {"sum": s["sum"], "q": s["q"], "scale": s["scale"]}
    psc.psc_norm_quantize_mx4(s["x"], s["q"], s["blocks"], s["scale"], gain=s["gain"], eps=EPS, residual=s["residual"],
                              sum_out=s["sum"])
    if s["op"] == "norm4":
        psc.psc_dequantize_mx4(s["q"], s["blocks"], s["y"], scale=s["scale"])
        return {"sum": s["sum"], "y": s["y"], "scale": s["scale"]}
    psc.psc_head_logits_mx4(s["q"], s["blocks"], s["w"], s["w_blocks"], s["logits"], s["K"], scale=s["scale"],
                            w_scale=s["w_scale"], bitmask=s["bitmask"])
    return {"sum": s["sum"], "logits": s["logits"], "scale": s["scale"]}


# ------------------------------------------------------------------- its bounds
def work(case):
    c = case
    T, K, e = c["T"], c["K"], 2 if c["dtype"] == "bf16" else 4
    codes = T * K / 2 + T * K / 32
    if c["op"] == "mx4":                        # in, codes out, codes in, values out
        return {"bytes": 2 * T * K * e + 2 * codes, "flops": 6 * T * K}
    if c["op"] == "head4":
        e_x, V = 2, c["V"]
        mask = 0 if c["mask"] == "none" else T * ((V + 31) // 32) * 4
        # of a tight mask, the rows of the weights that some token allows
        dots = T * V if c["mask"] != "tight" else T * min(V, _TOKENS["tight"])
        read = V if c["mask"] != "tight" else min(V, dots)
        per = K / 2 + K / 32 + (4 if c["w_scale"] else 0)
        return {"bytes": read * per + 3 * T * K * e_x + 4 * K + 2 * codes + 4 * T + T * V * e + mask,
                "flops": 2 * dots * K + 12 * T * K}
    x = T * K * e * (3 if c["residual"] else 1) + 4 * K + 4 * T
    if c["op"] == "norm8":
        return {"bytes": x + T * K, "flops": 8 * T * K}
    return {"bytes": x + 2 * codes + T * K * e, "flops": 10 * T * K}


# ------------------------------------------------------ the definitions in 64 bits
def _exact_norm(s):
    h = s["x"].double()
    if s["residual"] is not None:               # rounded as the stream holds it
        h = (h + s["residual"].double()).float().to(s["x"].dtype).double()
    r = (h.square().sum(1) / h.shape[1] + EPS) ** -0.5
    v = (h * s["gain"].double()).float().double()           # codes are those of products in 32 bits
    return (h if s["residual"] is not None else None), v, r


def _exact_mx4(v):
    """By the distance to each of the eight magnitudes; of two at the same distance the even code's."""
    T, K = v.shape
    out = torch.empty_like(v)
    grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    for k in range(0, K, 32):
        b = v[:, k:k + 32]
        m = b.abs().amax(1, keepdim=True).clamp(min=2.0 ** -120)
        e = torch.floor(torch.log2(m))
        e = e + (torch.exp2(e + 1) <= m).double() - (torch.exp2(e) > m).double()   # a logarithm may be a step off
        top = torch.exp2(e - 2)
        u = (b / top).abs()
        best, at = (u - grid[0]).abs(), torch.zeros_like(u)
        for code in range(1, 8):
            d = (u - grid[code]).abs()
            nearer = (d < best) | ((d == best) & (code % 2 == 0))
            best, at = torch.where(nearer, d, best), torch.where(nearer, grid[code], at)
        out[:, k:k + 32] = torch.sign(b) * at * top
    return out


def _exact_rows(w, blocks, lo, hi, K):
    """Rows lo to hi of the weights, by the formula of a code and of an exponent's place."""
    k = torch.arange(K, device=w.device)
    r = torch.arange(lo, hi, device=w.device)[:, None]
    code = (w[lo:hi].long()[:, k // 2] >> (4 * (k % 2))) & 15
    e, m = (code >> 1) & 3, code & 1
    a = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e - 1).double())
    b = k // 32
    at = ((r // 128) * ((K + 127) // 128) + b // 4) * 512 + 16 * (r % 32) + 4 * (r % 128 // 32) + b % 4
    return torch.where(code >= 8, -a, a) * 2.0 ** (blocks[at].double() - 127)


def _bits64(words, V):
    """Bit by bit from the words as unsigned 64-bit numbers."""
    v = torch.arange(V, device=words.device)
    w = words.long() & 0xFFFFFFFF
    return (w[v // 32] >> (v % 32)) % 2 == 1


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "mx4":
        return _exact_mx4(s["x"].double())
    h, v, r = _exact_norm(s)
    if s["op"] == "norm8":
        return {"sum": h, "q": None, "scale": v.abs().amax(1) / 127 * r}
    if s["op"] == "norm4":
        return {"sum": h, "y": _exact_mx4(v) * r[:, None], "scale": r}
    K, V = s["K"], s["w"].shape[0]
    x = _exact_mx4(v)
    y = torch.empty(x.shape[0], V, dtype=torch.float64, device=x.device)
    for lo in range(0, V, 8192):
        hi = min(V, lo + 8192)
        y[:, lo:hi] = x @ _exact_rows(s["w"], s["w_blocks"], lo, hi, K).t()
    y *= r[:, None]
    if s["w_scale"] is not None:
        y *= s["w_scale"].double()[None]
    if s["bitmask"] is not None:
        for t in range(x.shape[0]):
            y[t, ~_bits64(s["bitmask"][t], V)] = NEG
    return {"sum": h, "logits": y, "scale": r}
