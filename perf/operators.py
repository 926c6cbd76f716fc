"""The operators between a model's last hidden states and the token that the
parser consumes: the vocabulary projection in 8-bit integers under the grammar's
masks (head), penalties, biases and masks on logits (process), and the draw of a
token among the allowed ones (sample).

Every case runs either the operators' plain forms (elementary torch operations in
32 bits) or, where `own` is true, the calls of the library's binding.

head     s_t = max|x_t| / 127, q_t = rint(x_t / s_t);
         y[t][v] = (sum_k q_t[k] w[v][k]) * s_t * c_v, -inf where the mask forbids v
process  y = x; repetition r over prompt and output: y > 0 ? y / r : y * r; for tokens
         of the output, n times there: y - f n - p; plus the row's biases; then the mask
sample   z = (x - max) / T, weights rint(2^40 e^z) (whole numbers, so that sums have no
         order); a token stays if fewer than k tokens are larger, if the larger ones
         hold less than p of the weight that top-k leaves, and if e^z >= min_p; the
         draw is the first token, by index, whose running weight passes u * (sum)
"""
import math

import torch

own = False

FLT_MAX = 3.4028234663852886e38
NEG = -math.inf


def _psc():
    from paper_2608_03065_gb300 import psc
    return psc


# ------------------------------------------------------------------- the cases
def listed():
    return [
        # one stream, the Llama 3 size of vocabulary, a chat turn behind it
        {"name": "process b1 v128256 h600", "op": "process", "B": 1, "V": 128256, "H": 600, "bias": 0, "dtype": "bf16",
         "mask": "open"},
        # a small vocabulary in f32, biases as an API's callers send them, no grammar
        {"name": "process b64 v32000 h2047 f32", "op": "process", "B": 64, "V": 32000, "H": 2047, "bias": 300,
         "dtype": "f32", "mask": "none"},
        # an odd batch with long documents behind it
        {"name": "process b201 v151936 h20000", "op": "process", "B": 201, "V": 151936, "H": 20000, "bias": 8,
         "dtype": "bf16", "mask": "mixed"},
        # the benchmark's batch and vocabulary
        {"name": "process b1024 v262144 h1024", "op": "process", "B": 1024, "V": 262144, "H": 1024, "bias": 16,
         "dtype": "bf16", "mask": "mixed"},
        # one stream: the weights are read for one token
        {"name": "head t1 v128256 k2048", "op": "head", "T": 1, "V": 128256, "K": 2048, "dtype": "bf16",
         "mask": "none"},
        # few rows inside punctuation and keywords: the grammar leaves a few dozen tokens each
        {"name": "head t16 v151936 k1024 tight", "op": "head", "T": 16, "V": 151936, "K": 1024, "dtype": "f32",
         "mask": "tight"},
        # a serving batch
        {"name": "head t256 v128256 k4096", "op": "head", "T": 256, "V": 128256, "K": 4096, "dtype": "bf16",
         "mask": "none"},
        # the benchmark's batch and vocabulary
        {"name": "head t1024 v262144 k2048", "op": "head", "T": 1024, "V": 262144, "K": 2048, "dtype": "bf16",
         "mask": "mixed"},
        # one stream with the usual settings
        {"name": "sample b1 v262144 k+p", "op": "sample", "B": 1, "V": 262144, "dtype": "bf16", "mask": "open",
         "filters": "kp"},
        # nucleus sampling without a grammar, f32 logits
        {"name": "sample b64 v32000 p f32", "op": "sample", "B": 64, "V": 32000, "dtype": "f32", "mask": "none",
         "filters": "p"},
        # a serving batch, every row with its own settings
        {"name": "sample b256 v128256 mixed", "op": "sample", "B": 256, "V": 128256, "dtype": "bf16", "mask": "mixed",
         "filters": "mixed"},
        # the benchmark's batch and vocabulary, temperature alone for some rows, filters for others
        {"name": "sample b1024 v262144 mixed", "op": "sample", "B": 1024, "V": 262144, "dtype": "bf16",
         "mask": "mixed", "filters": "mixed"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["process", "head", "sample"])
    V = _log_int(rng, 500, 262144)
    if rng.random() < 0.5:
        V = -(-V // 64) * 64
    rows = _log_int(rng, 1, 1024)
    c = {"op": op, "V": min(V, 262144), "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "process":
        H = _log_int(rng, 1, 32768)
        while rows * H > 8_000_000:
            rows = max(1, rows // 2)
        c.update(B=rows, H=H, bias=rng.choice([0, 1, 16, 300]), mask=rng.choice(["none", "open", "mixed"]))
    elif op == "head":
        K = _log_int(rng, 64, 4096)
        if rng.random() < 0.75:
            K = -(-K // 16) * 16
        while rows * c["V"] * K > 1024 * 262144 * 2048:
            rows = max(1, rows // 2)
        c.update(T=rows, K=K, mask=rng.choice(["none", "tight", "mixed"]))
    else:
        c.update(B=rows, mask=rng.choice(["none", "open", "mixed"]), filters=rng.choice(["none", "k", "p", "kp", "mixed"]))
    if c["dtype"] == "f32" and rows * c["V"] > 512 * 262144:
        c["dtype"] = "bf16"
    return c


# ------------------------------------------------------------------- the inputs
#: Shares of a vocabulary that grammars leave open: nothing (a failed row), one token
#: (a literal's rest), a few dozen (keywords, punctuation), and rows inside names,
#: strings or comments.
_SHARES = {"mixed": ([0.0, -1.0, -48.0, 0.02, 0.45, 0.95], [0.03, 0.05, 0.22, 0.20, 0.30, 0.20]),
           "open": ([0.45, 0.95], [0.5, 0.5]),
           "tight": ([0.0, -1.0, -8.0, -48.0], [0.04, 0.16, 0.4, 0.4])}
_OPEN_ROWS = {"mixed": 0.97, "open": 1.0, "tight": 0.96, "none": 1.0}
_TOKENS = {"tight": 0.16 + 0.4 * 8 + 0.4 * 48}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _pack(bits):
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
        out[lo:hi] = _pack(torch.rand(hi - lo, V, device="cuda", generator=g) < share[lo:hi, None])
    return out


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _zipf_logits(B, V, g, dtype):
    """Logits whose probabilities fall like a power of the rank, as a language model's do."""
    out = torch.empty(B, V, dtype=dtype, device="cuda")
    for lo in range(0, B, 128):
        hi = min(B, lo + 128)
        a = torch.rand(hi - lo, 1, device="cuda", generator=g) + 1.0
        x = torch.empty(hi - lo, V, device="cuda").exponential_(generator=g)
        out[lo:hi] = x * a + 0.25 * torch.randn(hi - lo, V, device="cuda", generator=g) - 4.0
    return out


def _choose(values, B, g, dtype):
    at = torch.randint(len(values), (B,), device="cuda", generator=g)
    return torch.tensor(values, device="cuda", dtype=dtype)[at]


def _prepare_process(c, g):
    B, V, H = c["B"], c["V"], c["H"]
    s = {"logits": _zipf_logits(B, V, g, _dtype(c)), "bitmask": _bitmask(c["mask"], B, V, g)}
    s["out"] = torch.empty_like(s["logits"])
    # text repeats itself: ids by a power law; a row's history is between half of H and H long
    ids = (V * torch.rand(B, H, device="cuda", generator=g) ** 3).to(torch.int32).clamp(max=V - 1)
    s["history_len"] = torch.randint((H + 1) // 2, H + 1, (B,), device="cuda", generator=g).to(torch.int32)
    s["prompt_len"] = (s["history_len"] * torch.rand(B, device="cuda", generator=g)).to(torch.int32)
    s["history"] = torch.where(torch.arange(H, device="cuda")[None] < s["history_len"][:, None], ids, -1)
    s["repetition"] = _choose([1.0, 1.05, 1.2, 1.5], B, g, torch.float32)
    s["frequency"] = _choose([0.0, 0.25, 0.5, -0.1], B, g, torch.float32)
    s["presence"] = _choose([0.0, 0.4, 1.0], B, g, torch.float32)
    if c["bias"]:
        n = min(c["bias"], V)
        step = V // n      # ids of a row are distinct: one of every n-th part of the vocabulary
        at = torch.randint(step, (B, n), device="cuda", generator=g)
        s["bias_ids"] = (at + step * torch.arange(n, device="cuda")[None]).to(torch.int32)
        bias = 4.0 * torch.randn(B, n, device="cuda", generator=g)
        s["bias"] = torch.where(torch.rand(B, n, device="cuda", generator=g) < 0.05, NEG, bias)
    else:
        s["bias_ids"] = s["bias"] = None
    return s


def _prepare_head(c, g):
    T, V, K = c["T"], c["V"], c["K"]
    x = torch.randn(T, K, device="cuda", generator=g) * (0.5 + torch.rand(T, 1, device="cuda", generator=g))
    x = x * (1 + 9 * (torch.rand(1, K, device="cuda", generator=g) < 0.01))    # a few loud channels
    w = torch.empty(V, K, dtype=torch.int8, device="cuda")
    scale = torch.empty(V, device="cuda")
    for lo in range(0, V, 32768):
        hi = min(V, lo + 32768)
        f = torch.randn(hi - lo, K, device="cuda", generator=g) * (K ** -0.5)
        scale[lo:hi] = f.abs().amax(1) / 127.0
        w[lo:hi] = (f / scale[lo:hi, None]).round().to(torch.int8)
    s = {"x": x.to(torch.bfloat16), "w": w, "w_scale": scale, "bitmask": _bitmask(c["mask"], T, V, g)}
    s["q"] = torch.empty(T, K, dtype=torch.int8, device="cuda")
    s["scale"] = torch.empty(T, device="cuda")
    s["logits"] = torch.empty(T, V, dtype=_dtype(c), device="cuda")
    return s


def _prepare_sample(c, g):
    B, V = c["B"], c["V"]
    s = {"logits": _zipf_logits(B, V, g, _dtype(c)), "bitmask": _bitmask(c["mask"], B, V, g)}
    s["uniform"] = torch.rand(B, device="cuda", generator=g)
    s["temperature"] = _choose([0.0, 0.6, 0.8, 1.0, 1.0, 1.3] if c["filters"] == "mixed" else [0.6, 0.8, 1.0], B, g,
                               torch.float32)
    ks, ps, ms = {"none": (None, None, None), "k": ([1, 20, 50, 200], None, None), "p": (None, [0.8, 0.9, 0.95], None),
                  "kp": ([20, 50, 100], [0.8, 0.9, 0.95], None),
                  "mixed": ([0, 0, 1, 40, 50, 1000], [1.0, 1.0, 0.9, 0.95], [0.0, 0.0, 0.0, 0.05, 0.1])}[c["filters"]]
    s["top_k"] = _choose(ks, B, g, torch.int32) if ks else None
    s["top_p"] = _choose(ps, B, g, torch.float32) if ps else None
    s["min_p"] = _choose(ms, B, g, torch.float32) if ms else None
    s["tokens"] = torch.empty(B, dtype=torch.int32, device="cuda")
    s["logprobs"] = torch.empty(B, device="cuda")
    return s


def prepare(case, seed):
    g = _gen(seed)
    s = {"process": _prepare_process, "head": _prepare_head, "sample": _prepare_sample}[case["op"]](case, g)
    s["op"], s["V"] = case["op"], case["V"]
    return s


# --------------------------------------------------------------- the plain forms
def _allowed(words, V):
    """[B, W] packed words -> [B, V] truth values."""
    bits = (words[:, :, None] >> torch.arange(32, device=words.device, dtype=torch.int32)) & 1
    return bits.view(words.shape[0], -1)[:, :V].bool()


def _plain_process(s):
    V = s["V"]
    y = s["logits"].float()
    B = y.shape[0]
    ids = torch.where(s["history"] < 0, V, s["history"]).long()
    at = torch.arange(ids.shape[1], device=ids.device)[None]
    there = at < s["history_len"][:, None]
    out = (there & (at >= s["prompt_len"][:, None])).float()
    zeros = torch.zeros(B, V + 1, device=y.device)
    seen = zeros.scatter_add(1, ids, there.float())[:, :V] > 0
    n = zeros.scatter_add(1, ids, out)[:, :V]
    r = s["repetition"][:, None]
    y = torch.where(seen, torch.where(y > 0, y / r, y * r), y)
    y = torch.where(n > 0, y - s["frequency"][:, None] * n - s["presence"][:, None], y)
    if s["bias"] is not None:
        y = y + zeros.scatter(1, s["bias_ids"].long(), s["bias"])[:, :V]
    if s["bitmask"] is not None:
        y = torch.where(_allowed(s["bitmask"], V), y, NEG)
    return y.to(s["logits"].dtype)


def _plain_head(s):
    x = s["x"].float()
    scale = x.abs().amax(1) / 127.0
    q = (x / scale[:, None]).round().clamp(-127, 127)
    y = (q @ s["w"].float().t()) * scale[:, None] * s["w_scale"][None]
    if s["bitmask"] is not None:
        y = torch.where(_allowed(s["bitmask"], s["V"]), y, NEG)
    return {"logits": y.to(s["logits"].dtype), "scale": scale}


def _plain_sample(s):
    V = s["V"]
    x = s["logits"].float()
    valid = x > NEG
    if s["bitmask"] is not None:
        valid = valid & _allowed(s["bitmask"], V)
    x = torch.where(valid, x.clamp(max=FLT_MAX), NEG)
    m = x.amax(1, keepdim=True)
    some = m[:, 0] > NEG
    greedy = s["temperature"] < 1e-6
    inv = (1.0 / torch.where(greedy, 1.0, s["temperature"]))[:, None]
    z = (x - torch.where(some[:, None], m, 0.0)) * inv
    e = torch.exp(z)
    w = (e * 2.0 ** 40).round().long()
    keep = valid
    if s["top_k"] is not None or s["top_p"] is not None:
        d, at = torch.sort(x, dim=1, descending=True)
        dw = w.gather(1, at)
        if s["top_k"] is not None:
            k = torch.where(s["top_k"] <= 0, V, s["top_k"]).clamp(max=V).long()
            low = d.gather(1, k[:, None] - 1)
            keep = keep & (x >= low)
            dw = torch.where(d >= low, dw, 0)
        if s["top_p"] is not None:
            c = dw.cumsum(1)
            total = c[:, -1:]
            p = (s["top_p"].clamp(0, 1) * 2.0 ** 24).round().long()[:, None]
            limit = (p * (total >> 24) + ((p * (total & (2 ** 24 - 1))) >> 24)).clamp(min=1)
            last = (c - dw < limit).sum(1, keepdim=True).clamp(min=1) - 1
            keep = keep & ((x >= d.gather(1, last)) | (s["top_p"] >= 1)[:, None])
    if s["min_p"] is not None:
        keep = keep & (e >= s["min_p"].clamp(max=1)[:, None])
    c = torch.where(keep, w, 0).cumsum(1)
    total = c[:, -1:]
    u = (s["uniform"] * 2.0 ** 24).long()[:, None]
    t = u * (total >> 24) + ((u * (total & (2 ** 24 - 1))) >> 24)
    tok = (c <= t).sum(1).clamp(max=V - 1)
    lp = z.gather(1, tok[:, None])[:, 0] - torch.log(total[:, 0].float() * 2.0 ** -40)
    tok = torch.where(greedy, (x == m).long().argmax(1), tok)
    lp = torch.where(greedy, 0.0, lp)
    return {"tokens": torch.where(some, tok, -1).to(torch.int32), "logprobs": torch.where(some, lp, NEG)}


# ------------------------------------------------------------------- one pass
def run(state):
    s = state
    if not own:
        return {"process": _plain_process, "head": _plain_head, "sample": _plain_sample}[s["op"]](s)
    psc = _psc()
    if s["op"] == "process":
        psc.psc_process_logits(s["logits"], out=s["out"], history=s["history"], history_len=s["history_len"],
                               prompt_len=s["prompt_len"], repetition=s["repetition"], frequency=s["frequency"],
                               presence=s["presence"], bias_ids=s["bias_ids"], bias=s["bias"], bitmask=s["bitmask"])
        return s["out"]
    if s["op"] == "head":
        psc.psc_quantize_rows(s["x"], s["q"], s["scale"])
        psc.psc_head_logits(s["q"], s["scale"], s["w"], s["w_scale"], s["logits"], bitmask=s["bitmask"])
        return {"logits": s["logits"], "scale": s["scale"]}
    psc.psc_sample(s["logits"], s["uniform"], s["tokens"], logprobs=s["logprobs"], bitmask=s["bitmask"],
                   temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return {"tokens": s["tokens"], "logprobs": s["logprobs"]}


# ------------------------------------------------------------------- its bounds
def work(case):
    c = case
    V, e = c["V"], 2 if c["dtype"] == "bf16" else 4
    rows = c.get("B", c.get("T"))
    mask = 0 if c["mask"] == "none" else rows * ((V + 31) // 32) * 4
    if c["op"] == "process":
        hist = int(0.75 * rows * c["H"])
        return {"bytes": 2 * rows * V * e + mask + 4 * hist + 8 * rows * c["bias"] + 20 * rows, "flops": 4 * hist}
    if c["op"] == "head":
        K = c["K"]
        # of a tight mask, the rows of the weights that some token allows
        dots = rows * V if c["mask"] != "tight" else rows * min(V, _TOKENS["tight"])
        read = V if c["mask"] != "tight" else min(V, dots)
        return {"bytes": int(read * (K + 4) + rows * K * 2 + rows * V * e + mask + 4 * rows),
                "flops": int(2 * dots * K + 2 * rows * K)}
    return {"bytes": rows * V * e + mask + 28 * rows, "flops": 4 * rows * V}


# ------------------------------------------------------ the definitions in 64 bits
def _bits64(words, V):
    """Bit by bit from the words as unsigned 64-bit numbers."""
    v = torch.arange(V, device=words.device)
    w = words.long() & 0xFFFFFFFF
    return (w[v // 32] >> (v % 32)) % 2 == 1


def _exact_process(s):
    x, V = s["logits"], s["V"]
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    lens, prompts = s["history_len"].tolist(), s["prompt_len"].tolist()
    for b in range(x.shape[0]):
        y = x[b].double()
        ids = s["history"][b, :lens[b]].long()
        both = torch.bincount(ids, minlength=V)
        n = torch.bincount(ids[prompts[b]:], minlength=V).double()
        r, f, p = (s[k][b].double() for k in ("repetition", "frequency", "presence"))
        again = both > 0
        y = torch.where(again & (y > 0), y / r, torch.where(again, y * r, y))
        y = y - f * n - p * (n > 0)
        if s["bias"] is not None:
            y[s["bias_ids"][b].long()] += s["bias"][b].double()
        if s["bitmask"] is not None:
            y[~_bits64(s["bitmask"][b], V)] = NEG
        out[b] = y
    return out


def _exact_head(s):
    x = s["x"].double()
    scale = x.abs().max(1).values / 127
    # a quotient is rounded to 32 bits before it is rounded to a whole number
    q = torch.round((x / scale.float().double()[:, None]).float()).double()
    y = torch.empty(x.shape[0], s["V"], dtype=torch.float64, device=x.device)
    for lo in range(0, s["V"], 16384):
        y[:, lo:lo + 16384] = q @ s["w"][lo:lo + 16384].double().t()
    y *= scale[:, None]
    y *= s["w_scale"].double()[None]
    if s["bitmask"] is not None:
        for t in range(x.shape[0]):
            y[t, ~_bits64(s["bitmask"][t], s["V"])] = NEG
    return {"logits": y, "scale": scale}


def _exact_sample(s):
    x, V = s["logits"], s["V"]
    B = x.shape[0]
    lp = torch.full((B,), NEG, dtype=torch.float64, device=x.device)
    at = lambda k, b, d: d if s[k] is None else s[k][b].item()  # noqa: E731
    for b in range(B):
        y = x[b].double()
        ok = y > NEG if s["bitmask"] is None else (y > NEG) & _bits64(s["bitmask"][b], V)
        y = y[ok]
        if y.numel() == 0:
            continue
        T = s["temperature"][b].item()
        if T < 1e-6:
            lp[b] = 0.0
            continue
        z = (y - y.max()) / T
        levels, back, n = torch.unique(-z, return_inverse=True, return_counts=True)   # the largest first
        mass = n * torch.exp(-levels)
        keep = torch.ones_like(levels, dtype=torch.bool)
        k, p, m = at("top_k", b, 0), at("top_p", b, 1.0), at("min_p", b, 0.0)
        if k > 0:
            keep &= n.cumsum(0) - n < k
        if p < 1:
            left = torch.where(keep, mass, 0.0)
            keep &= (left.cumsum(0) - left < p * left.sum()) | (levels == levels[0])
        keep &= torch.exp(-levels) >= min(m, 1.0)
        weight = torch.exp(z) * keep[back]
        c = weight.cumsum(0)
        u = math.floor(s["uniform"][b].item() * 2 ** 24) / 2 ** 24
        i = int((c <= u * c[-1]).sum().clamp(max=len(c) - 1))
        lp[b] = z[i] - torch.log(c[-1])
    return {"tokens": None, "logprobs": lp}


def exact(case, seed):
    s = prepare(case, seed)
    return {"process": _exact_process, "head": _exact_head, "sample": _exact_sample}[case["op"]](s)
