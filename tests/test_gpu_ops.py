"""The operators around the mask on the GPU, against plain implementations in 64
bits (numpy), at the sizes, masks and values where they can go wrong.

Tolerances follow from the arithmetic.  u = 2^-24 is the unit roundoff of f32 (24
bits), 2^-8 that of bf16 (8 bits).  head: one rounding of the integer sum and two
products, 3u, then the rounding to bf16; where partial sums can pass 2^24, a tensor core may round or
cut each of its K / 16 additions, 2u each of the sum of magnitudes.  process:
at most five roundings of numbers no larger than the sum of the magnitudes
involved.  sample: z is rounded twice and exp is good to 2 ulp, so a weight is off
by (2|z| + 4)u of itself, |z| <= 29 wherever a weight is not 0: 62u, so that every
partial sum lies within 62u of its total, 4e-6; DELTA = 1e-5 leaves a factor of two
over it for the two sums that a comparison involves.
"""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, UB, DELTA = 2.0 ** -24, 2.0 ** -8, 1e-5
NEG = -np.inf
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def psc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_03065_gb300 import build, psc as mod
    build.build()
    mod.load()
    return mod


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def _pack(allowed):
    B, V = allowed.shape
    bits = np.zeros((B, (V + 31) // 32 * 32), dtype=np.uint8)
    bits[:, :V] = allowed
    return _dev(np.packbits(bits, axis=1, bitorder="little").view(np.int32))


def _mask(rng, kind, B, V):
    """Truth values: rows of every density, the first empty, the last of one token."""
    if kind == "none":
        return None
    share = rng.choice([0.002, 0.05, 0.5, 0.97], size=(B, 1)) if kind == "mixed" else np.full((B, 1), 0.003)
    a = rng.random((B, V)) < share
    a[0] = False
    if B > 1:
        a[-1] = False
        a[-1, rng.integers(V)] = True
    return a


def _strided(x, dtype, pad, shift):
    """x as a device tensor whose rows are `pad` apart and start `shift` elements in."""
    B, V = x.shape
    big = torch.full((B, V + pad + shift), 7.0, dtype=dtype, device="cuda")
    view = big[:, shift:shift + V]
    view.copy_(_dev(x.astype(np.float32)))
    return big, view


def _f64(t):
    return t.double().cpu().numpy()


# --------------------------------------------------------------------- quantise
@pytest.mark.parametrize("T,K,pad", [(1, 1, 0), (3, 7, 5), (17, 64, 0), (5, 1000, 3), (2, 8192, 0), (300, 33, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_rows(psc, T, K, pad, dtype):
    rng = np.random.default_rng([T, K])
    x = rng.standard_normal((T, K)) * rng.uniform(0.1, 30, (T, 1))
    x[0, K // 2] = 0
    if T > 2:
        x[1] = 0
    _, xd = _strided(x, DT[dtype], pad, 0)
    q = torch.full((T, K + pad), 99, dtype=torch.int8, device="cuda")
    scale = torch.empty(T, device="cuda")
    psc.psc_quantize_rows(xd, q[:, :K], scale)
    ref = _f64(xd)
    s = np.abs(ref).max(1).astype(np.float32) * (np.float32(1) / np.float32(127))
    np.testing.assert_array_equal(scale.cpu().numpy(), s)       # correctly rounded products and quotients on both sides
    safe = np.where(s > 0, s, 1).astype(np.float32)
    want = np.rint(ref.astype(np.float32) / safe[:, None])      # ties to even
    np.testing.assert_array_equal(q[:, :K].cpu().numpy(), want)
    assert (q[:, K:] == 99).all()


def test_quantize_rows_shows_what_is_not_finite(psc):
    x = torch.randn(5, 300, device="cuda")
    x[1, 7] = float("inf")
    x[2, 0] = float("nan")
    x[3] = 1e-45                       # the scale underflows
    x[4] = 3e38
    q, s = torch.empty(5, 300, dtype=torch.int8, device="cuda"), torch.empty(5, device="cuda")
    psc.psc_quantize_rows(x, q, s)
    s, q = s.cpu(), q.cpu()
    assert torch.isnan(s[1]) and torch.isnan(s[2]) and s[3] == 0 and s[4] > 0
    assert (q[1:4] == 0).all() and (q[4] == 127).all()


# ------------------------------------------------------------------------- head
def _head_case(psc, T, V, K, dtype, mask, pad=0, shift=0, fill=None, out_pad=0, stream=None):
    rng = np.random.default_rng([T, V, K])
    q = rng.integers(-127, 128, (T, K)) if fill is None else np.full((T, K), fill)
    w = np.clip(np.rint(rng.standard_normal((V, K)) * 40), -127, 127) if fill is None else np.full((V, K), 127)
    sx, sw = rng.uniform(0.01, 0.1, T).astype(np.float32), rng.uniform(1e-4, 1e-3, V).astype(np.float32)
    allowed = _mask(rng, mask, T, V)

    def place(a):      # rows K + pad apart, the first `shift` bytes in; what lies between is not zero
        flat = torch.full((a.shape[0] * (K + pad) + shift,), 55, dtype=torch.int8, device="cuda")
        v = flat[shift:].view(a.shape[0], K + pad)[:, :K]
        v.copy_(_dev(a, torch.int8))
        return v

    big = torch.full((T, V + out_pad), 7.0, dtype=DT[dtype], device="cuda")
    psc.psc_head_logits(place(q), _dev(sx), place(w), _dev(sw), big[:, :V],
                        bitmask=None if allowed is None else _pack(allowed), stream=stream)
    got = _f64(big)
    assert (got[:, V:] == 7).all()
    got = got[:, :V]
    # sums of whole numbers: f64 products are exact
    exact = q.astype(np.float64) @ w.astype(np.float64).T * sx.astype(np.float64)[:, None] * sw.astype(np.float64)
    tol = (3 * U + (UB if dtype == "bf16" else 0)) * np.abs(exact)
    if K > 1040:
        size = np.abs(q).astype(np.float64) @ np.abs(w).astype(np.float64).T
        big_sums = size >= 2.0 ** 24      # only there can a partial sum leave the whole numbers of f32
        tol = tol + np.where(big_sums, 2 * U * (K / 16) * size * sx[:, None] * sw, 0)
    if allowed is not None:
        assert (got[~allowed] == NEG).all()
        exact, tol, got = exact[allowed], tol[allowed], got[allowed]
    assert (np.abs(got - exact) <= tol * 1.0000001).all(), np.max(np.abs(got - exact) / np.maximum(tol, 1e-300))


@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (1, 130, 16), (1, 1000, 48), (2, 257, 64), (3, 129, 100), (7, 512, 257),
                                   (8, 1000, 1024), (9, 640, 320), (16, 333, 512), (17, 300, 80), (33, 1024, 1040),
                                   (64, 129, 128), (100, 1500, 192), (130, 260, 2048), (256, 384, 64), (257, 500, 336),
                                   (300, 127, 96), (513, 1300, 160), (4, 300, 4096), (8, 700, 2048), (12, 3000, 2048),
                                   (16, 2500, 4080), (16, 200, 4200)])
@pytest.mark.parametrize("dtype,mask", [("bf16", "none"), ("f32", "mixed"), ("bf16", "tight")])
def test_head_logits(psc, T, V, K, dtype, mask):
    _head_case(psc, T, V, K, dtype, mask, pad=-K % 16)


@pytest.mark.parametrize("T,V,K", [(16, 40000, 1024), (128, 20500, 2048), (256, 21000, 4096), (500, 9000, 1500)])
def test_head_logits_of_many_tiles_a_block(psc, T, V, K):
    """Several tiles per SM and long sums: every ring of the pipeline goes round many times."""
    _head_case(psc, T, V, K, "bf16", "none", pad=-K % 16)
    _head_case(psc, T, V, K, "f32", "mixed", pad=-K % 16)


@pytest.mark.parametrize("T", [1, 5, 40, 200])
@pytest.mark.parametrize("K,pad,shift", [(65, 0, 0), (64, 4, 0), (64, 0, 4), (64, 0, 1), (31, 17, 0), (100, 28, 16)])
def test_head_logits_at_any_alignment(psc, T, K, pad, shift):
    _head_case(psc, T, 321, K, "f32", "mixed", pad=pad, shift=shift, out_pad=3)
    _head_case(psc, T, 321, K, "bf16", "none", pad=pad, shift=shift, out_pad=1)


@pytest.mark.parametrize("T,V,K,pad,shift", [(1, 50000, 1001, 0, 0), (3, 20000, 4095, 0, 0), (12, 30001, 2047, 0, 3),
                                             (40, 25000, 2050, 0, 2), (257, 21000, 2047, 0, 0)])
def test_head_logits_of_several_slabs(psc, T, V, K, pad, shift):
    """Unaligned rows over more than one slab of the workspace."""
    _head_case(psc, T, V, K, "bf16", "mixed", pad=pad, shift=shift)
    _head_case(psc, T, V, K, "f32", "none", pad=pad, shift=shift, out_pad=2)


@pytest.mark.parametrize("T", [1, 12, 257])
def test_head_logits_of_large_unaligned_weights_are_those_of_aligned_ones(psc, T):
    """The same sums and the same epilogue, so the same bits, where the packed rows pass a slab of 256 MB."""
    V, K = 140001, 2047
    g = torch.Generator(device="cuda").manual_seed(T)
    q = torch.randint(-127, 128, (T, K), generator=g, dtype=torch.int8, device="cuda")
    w = torch.randint(-127, 128, (V, K), generator=g, dtype=torch.int8, device="cuda")
    sx, sw = torch.rand(T, generator=g, device="cuda"), torch.rand(V, generator=g, device="cuda")
    bits = torch.randint(-2 ** 31, 2 ** 31 - 1, (T, (V + 31) // 32), generator=g, dtype=torch.int32, device="cuda")
    aligned = torch.zeros(V, 2048, dtype=torch.int8, device="cuda")
    aligned[:, :K] = w
    for mask in (None, bits):
        here, there = (torch.empty(T, V, device="cuda") for _ in range(2))
        psc.psc_head_logits(q, sx, w, sw, here, bitmask=mask)
        psc.psc_head_logits(q, sx, aligned[:, :K], sw, there, bitmask=mask)
        assert torch.equal(here, there)


@pytest.mark.parametrize("T", [1, 4, 20, 150])
@pytest.mark.parametrize("fill", [127, -128])
def test_head_logits_largest_sums(psc, T, fill):
    _head_case(psc, T, 200, 8192, "f32", "none", fill=fill)


def test_head_logits_passes_on_what_is_not_finite(psc):
    q = torch.zeros(3, 64, dtype=torch.int8, device="cuda")
    w = torch.ones(100, 64, dtype=torch.int8, device="cuda")
    sx = torch.tensor([1.0, float("nan"), 1.0], device="cuda")
    out = torch.zeros(3, 100, device="cuda")
    psc.psc_head_logits(q, sx, w, torch.ones(100, device="cuda"), out)
    assert torch.isnan(out[1]).all() and (out[0] == 0).all() and (out[2] == 0).all()


# ---------------------------------------------------------------------- process
def _process_ref(x, lens, plens, hist, rep, freq, pres, ids, bias, allowed):
    """64-bit result and the sum of the magnitudes that each value went through."""
    y, size, touched = x.copy(), np.abs(x), np.zeros(x.shape, dtype=bool)
    B, V = x.shape
    for b in range(B):
        L = max(0, min(int(lens[b]), hist.shape[1]))
        seen, out = set(), {}
        for i in range(L):
            v = int(hist[b, i])
            if 0 <= v < V:
                seen.add(v)
                if i >= plens[b]:
                    out[v] = out.get(v, 0) + 1
        for v in seen:
            y[b, v] = y[b, v] / rep[b] if y[b, v] > 0 else y[b, v] * rep[b]
            size[b, v] = max(abs(y[b, v]), size[b, v])
            touched[b, v] = True
            if v in out:
                y[b, v] -= freq[b] * out[v] + pres[b]
                size[b, v] += abs(freq[b] * out[v]) + abs(pres[b])
        last = {int(v): float(z) for v, z in zip(ids[b], bias[b]) if 0 <= v < V}
        for v, z in last.items():
            y[b, v] += z
            size[b, v] += abs(z)
            touched[b, v] = True
    if allowed is not None:
        y[~allowed] = NEG
        touched &= allowed
    return y, size, touched


@pytest.mark.parametrize("B,V,H,n", [(1, 1, 1, 0), (1, 33, 0, 3), (3, 1000, 1, 1), (2, 1025, 257, 40), (5, 4099, 700, 0),
                                     (4, 32000, 8000, 300), (3, 50001, 9000, 17), (2, 70000, 40000, 0), (1, 1, 32767, 2), (2, 270001, 9001, 9),
                                     (2, 300, 20000, 5), (7, 2048, 100, 2048), (2, 5000, 2047, 300)])
@pytest.mark.parametrize("dtype,mask,where", [("bf16", "mixed", "out"), ("f32", "none", "in"), ("f32", "mixed", "in"),
                                              ("bf16", "none", "out"), ("bf16", "mixed", "ragged")])
def test_process_logits(psc, B, V, H, n, dtype, mask, where):
    rng = np.random.default_rng([B, V, H, n])
    pad, shift = (5, 1) if where == "ragged" else (0, 0)
    big, xd = _strided(rng.standard_normal((B, V)) * 4, DT[dtype], pad, shift)
    hist = (rng.random((B, H)) ** 3 * V).astype(np.int32)
    hist[rng.random((B, H)) < 0.02] = -1
    hist[rng.random((B, H)) < 0.02] = V + 3
    lens = rng.integers(0, H + 1, B).astype(np.int32)
    lens[0] = H + 9                                   # more than there is: H
    if B > 2:
        lens[1] = -4                                  # fewer than none: 0
    plens = (rng.integers(-2, H + 5, B)).astype(np.int32)
    rep, freq, pres = (rng.choice(c, B).astype(np.float32) for c in
                       ([0.7, 1.0, 1.3], [0.0, 0.125, -0.3], [0.0, 0.6]))
    ids = rng.integers(-1, V + 1, (B, n)).astype(np.int32)      # repeated ids too: the last counts
    bias = (rng.standard_normal((B, n)) * 3).astype(np.float32)
    allowed = _mask(rng, mask, B, V)
    x = _f64(xd)
    ref, size, touched = _process_ref(x, lens, plens, hist, rep.astype(np.float64), freq.astype(np.float64),
                                      pres.astype(np.float64), ids, bias.astype(np.float64), allowed)
    out = None if where == "in" else torch.full_like(big, 9.0)[:, shift:shift + V]
    psc.psc_process_logits(xd, out=out, history=_dev(hist) if H else None, history_len=_dev(lens),
                           prompt_len=_dev(plens), repetition=_dev(rep), frequency=_dev(freq), presence=_dev(pres),
                           bias_ids=_dev(ids) if n else None, bias=_dev(bias) if n else None,
                           bitmask=None if allowed is None else _pack(allowed))
    got = _f64(xd if out is None else out)
    if out is not None:
        np.testing.assert_array_equal(_f64(xd), x)              # the input is as it was
    if pad:
        assert (out._base[:, :shift] == 9).all() and (out._base[:, shift + V:] == 9).all()
    if allowed is not None:
        assert (got[~allowed] == NEG).all()
    same = ~touched if allowed is None else allowed & ~touched
    np.testing.assert_array_equal(got[same], x[same])
    tol = 5 * U * size + (UB * np.abs(ref) if dtype == "bf16" else 0)
    # a bf16 rounding is of the f32 value, itself off by a little
    assert (np.abs(got[touched] - ref[touched]) <= tol[touched] * 1.01).all()


def test_process_logits_infinities_and_nan(psc):
    x = torch.zeros(1, 64, device="cuda")
    x[0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 2.0])
    hist = torch.tensor([[0, 1, 2, 3, 5]], dtype=torch.int32, device="cuda")
    ids = torch.tensor([[3, 6, 7]], dtype=torch.int32, device="cuda")
    bias = torch.tensor([[float("-inf"), float("inf"), 1.5]], device="cuda")
    allowed = np.ones((1, 64), dtype=bool)
    allowed[0, [2, 6]] = False
    psc.psc_process_logits(x, history=hist, repetition=torch.full((1,), 2.0, device="cuda"),
                           presence=torch.ones(1, device="cuda"), bias_ids=ids, bias=bias, bitmask=_pack(allowed))
    got = x[0].cpu().numpy()
    assert got[0] == np.inf and got[1] == NEG and got[2] == NEG and got[3] == NEG and got[6] == NEG
    assert got[5] == -1 and got[7] == 1.5 and (got[8:] == 0).all()


def test_process_logits_rows_that_alternate_in_one_buffer(psc):
    big = torch.randn(4, 200, device="cuda")
    a, b = big[:, :100], big[:, 100:]
    want = a.clone()
    psc.psc_process_logits(a, out=b)
    assert torch.equal(a, want) and torch.equal(b, want)


# ----------------------------------------------------------------------- sample
def _draw_ref(x, allowed, u, T, k, p, m):
    """The draw in 64 bits: (token, ln probability)."""
    ok = (x > NEG) & (allowed if allowed is not None else True)
    if not ok.any():
        return -1, NEG
    x = np.where(ok, np.minimum(x, np.finfo(np.float32).max), NEG)
    top = x.max()
    if not T >= 1e-6:
        return int(np.argmax(x == top)), 0.0
    z = (x - top) / T
    w = np.where(ok, np.exp(z), 0.0)
    keep = ok.copy()
    if 0 < k < len(x):
        keep &= x >= np.sort(x)[-k]
    if p < 1:
        order = np.argsort(-x, kind="stable")
        mass = np.where(keep, w, 0.0)[order]
        before = mass.cumsum() - mass
        low = x[order][np.flatnonzero(before < max(p, 0) * mass.sum())[-1]] if p > 0 else top
        keep &= x >= low
    keep &= w >= min(m, 1.0)
    w = np.where(keep, w, 0.0)
    c = w.cumsum()
    i = min(int((c <= u * c[-1]).sum()), np.flatnonzero(keep)[-1])
    return i, z[i] - np.log(w.sum())


def _check_draws(tokens, logprobs, x, allowed, u, T, k, p, m):
    for b in range(len(u)):
        a = None if allowed is None else allowed[b]
        ub = np.floor(u[b] * 2.0 ** 24) / 2.0 ** 24
        # a boundary of top_p, min_p or the draw itself may fall within DELTA of its limit
        near = {_draw_ref(x[b], a, min(max(ub + du, 0), 1 - 1e-9), T[b], k[b], p[b] + dp if p[b] < 1 else 1.0,
                          m[b] * (1 + dm))
                for du in (-DELTA, 0, DELTA) for dp in (-DELTA, 0, DELTA) for dm in (-DELTA, 0, DELTA)}
        assert any(tokens[b] == t and (lp == logprobs[b] or abs(lp - logprobs[b]) <= 62 * U + 4 * U * abs(lp) + DELTA)
                   for t, lp in near), (b, tokens[b], logprobs[b], near)


def _settings(rng, B, kind):
    T = rng.choice([0.0, 0.5, 0.9, 1.0, 1.7], B) if kind == "mixed" else np.full(B, 0.8)
    k = rng.choice([-1, 0, 1, 2, 40, 1000, 10 ** 6], B) if kind in ("mixed", "k") else np.zeros(B)
    p = rng.choice([0.0, 0.3, 0.9, 0.999, 1.0, 1.5], B) if kind in ("mixed", "p") else np.ones(B)
    m = rng.choice([-1.0, 0.0, 0.02, 1.0, 2.0], B) if kind in ("mixed", "m") else np.zeros(B)
    return T.astype(np.float32), k.astype(np.int32), p.astype(np.float32), m.astype(np.float32)


@pytest.mark.parametrize("B,V", [(1, 1), (3, 7), (40, 33), (25, 257), (30, 1000), (12, 4099), (10, 32000), (6, 140001),
                                 (2, 600000)])
@pytest.mark.parametrize("dtype,mask,kind", [("bf16", "mixed", "mixed"), ("f32", "none", "mixed"), ("f32", "mixed", "p"),
                                             ("bf16", "none", "k"), ("bf16", "none", "none"), ("f32", "tight", "m")])
@pytest.mark.parametrize("shape", ["zipf", "flat", "ties"])
def test_sample(psc, B, V, dtype, mask, kind, shape):
    rng = np.random.default_rng([B, V, len(shape)])
    x = {"zipf": rng.exponential(1.5, (B, V)), "flat": rng.standard_normal((B, V)) * 1.4,
         "ties": rng.integers(0, 4, (B, V)) * 1.0}[shape]
    pad, shift = ((3, 1), (0, 0), (8, 0))[B % 3]
    _, xd = _strided(x, DT[dtype], pad, shift)
    T, k, p, m = _settings(rng, B, kind)
    u = rng.random(B).astype(np.float32)
    u[0] = 0.0
    u[-1] = np.float32(1 - 2.0 ** -24)
    allowed = _mask(rng, mask, B, V)
    before = _f64(xd)
    tok, lp = torch.full((B,), -7, dtype=torch.int32, device="cuda"), torch.full((B,), 7.0, device="cuda")
    off = kind == "none"
    psc.psc_sample(xd, _dev(u), tok, logprobs=lp, bitmask=None if allowed is None else _pack(allowed),
                   temperature=_dev(T), top_k=None if off else _dev(k), top_p=None if off else _dev(p),
                   min_p=None if off else _dev(m))
    _check_draws(tok.cpu().numpy(), _f64(lp), before, allowed, u, T.astype(np.float64), k, p.astype(np.float64),
                 m.astype(np.float64))
    np.testing.assert_array_equal(_f64(xd), before)
    again, lp2 = torch.empty_like(tok), torch.empty_like(lp)
    psc.psc_sample(xd, _dev(u), again, logprobs=lp2, bitmask=None if allowed is None else _pack(allowed),
                   temperature=_dev(T), top_k=None if off else _dev(k), top_p=None if off else _dev(p),
                   min_p=None if off else _dev(m))
    assert torch.equal(tok, again) and torch.equal(lp, lp2)


@pytest.mark.parametrize("V", [9000, 100001, 262144])
@pytest.mark.parametrize("dtype,mask", [("f32", "none"), ("bf16", "mixed")])
@pytest.mark.parametrize("shape", ["narrow", "lumpy", "long"])
def test_sample_a_nucleus_that_is_hard_to_find(psc, V, dtype, mask, shape):
    """Rows that no list holds and that a sample misjudges: values hardly apart, values that
    depend on a block of 1024 tokens, and a heavy start with a long even tail."""
    B = 5
    rng = np.random.default_rng([V, len(shape)])
    x = rng.standard_normal((B, V))
    lump = (np.arange(V) // 1024) % 8 == 0
    x = {"narrow": x * 1e-3, "lumpy": x + np.where(lump, -3.0, 2.0) * (1 - 2 * (np.arange(B)[:, None] % 2)),
         "long": np.where(np.arange(V) < 3000, x + 5, x * 0.05)}[shape]
    _, xd = _strided(x, DT[dtype], 8, 0)
    u = rng.random(B).astype(np.float32)
    p = np.array([0.2, 0.55, 0.8, 0.95, 0.999], dtype=np.float32)
    allowed = _mask(rng, mask, B, V)
    tok, lp = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda")
    psc.psc_sample(xd, _dev(u), tok, logprobs=lp, bitmask=None if allowed is None else _pack(allowed), top_p=_dev(p))
    _check_draws(tok.cpu().numpy(), _f64(lp), _f64(xd), allowed, u, np.ones(B), np.zeros(B, dtype=int),
                 p.astype(np.float64), np.zeros(B))


@pytest.mark.parametrize("B,V", [(160, 150001), (400, 50000)])
@pytest.mark.parametrize("shape", ["flat", "lumpy"])
def test_sample_a_batch_in_which_every_row_is_heavy(psc, B, V, shape):
    """With top_k given but off: many rows, few blocks each, and the first rows checked."""
    rng = np.random.default_rng([B, V])
    g = torch.Generator(device="cuda").manual_seed(B)
    xd = torch.randn(B, V, generator=g, device="cuda")
    if shape == "lumpy":
        xd += torch.where(torch.arange(V, device="cuda") // 1024 % 8 == 0, -3.0, 2.0)
    xd = xd.bfloat16()
    u = rng.random(B).astype(np.float32)
    p = np.tile(np.array([0.5, 0.9, 0.97, 0.999], dtype=np.float32), B // 4)
    tok, lp = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda")
    psc.psc_sample(xd, _dev(u), tok, logprobs=lp, top_k=torch.zeros(B, dtype=torch.int32, device="cuda"), top_p=_dev(p))
    rows = [0, 1, 2, 3, B // 2, B // 2 + 1, B - 2, B - 1]
    n = len(rows)
    _check_draws(tok.cpu().numpy()[rows], _f64(lp)[rows], _f64(xd[rows]), None, u[rows], np.ones(n),
                 np.zeros(n, dtype=int), p[rows].astype(np.float64), np.zeros(n))


@pytest.mark.parametrize("V", [100, 5000, 70000])
def test_sample_infinities_nan_and_masked_values(psc, V):
    rng = np.random.default_rng(V)
    x = rng.standard_normal((8, V))
    allowed = np.ones((8, V), dtype=bool)
    x[0, 5] = np.nan                                        # skipped
    x[1, :] = NEG                                           # nothing
    x[2, 3] = x[2, 9] = np.inf                              # one of the two
    x[3, 2], allowed[3, 2] = np.inf, False                  # masked: not looked at
    x[4, 2], allowed[4, 2] = np.nan, False
    x[5, :] = np.nan
    x[6, :] = np.finfo(np.float32).min                      # the lowest value is a value
    x[7, :] = NEG
    x[7, V - 1] = -3e38
    u = np.linspace(0.01, 0.9, 8).astype(np.float32)
    one, k, p = np.ones(8), np.full(8, 50), np.full(8, 0.9)
    for filters in (False, True):
        tok, lp = torch.empty(8, dtype=torch.int32, device="cuda"), torch.empty(8, device="cuda")
        psc.psc_sample(_dev(x, torch.float32), _dev(u), tok, logprobs=lp, bitmask=_pack(allowed),
                       top_k=_dev(k, torch.int32) if filters else None, top_p=_dev(p, torch.float32) if filters else None)
        _check_draws(tok.cpu().numpy(), _f64(lp), x.astype(np.float32).astype(np.float64), allowed, u, one,
                     k if filters else one * 0, np.full(8, np.float32(0.9), dtype=np.float64) if filters else one,
                     one * 0)
        t = tok.cpu().numpy()
        assert t[1] == -1 and t[5] == -1 and t[2] in (3, 9) and t[3] != 2 and t[4] != 2 and t[7] == V - 1


def test_sample_draws_with_the_right_probabilities(psc):
    """Every u = (i + 1/2) / n once: token v comes out n * p(v) times, give or take
    the two ends of its interval."""
    rng = np.random.default_rng(0)
    V, n = 777, 1 << 14
    x = (rng.exponential(1.5, V)).astype(np.float32)
    xd = _dev(x)[None].expand(n, V).contiguous()
    u = _dev(((np.arange(n) + 0.5) / n).astype(np.float32))
    tok = torch.empty(n, dtype=torch.int32, device="cuda")
    psc.psc_sample(xd, u, tok)
    got = np.bincount(tok.cpu().numpy(), minlength=V)
    p = np.exp(x.astype(np.float64) - x.max())
    p /= p.sum()
    assert (np.abs(got - n * p) <= 1 + n * DELTA).all()


# ------------------------------------------------------- streams, graphs, the chain
def _chain(psc, s, stream):
    psc.psc_quantize_rows(s["x"], s["q"], s["sx"], stream=stream)
    psc.psc_head_logits(s["q"], s["sx"], s["w"], s["sw"], s["logits"], bitmask=s["mask"], work=s["work"], stream=stream)
    psc.psc_process_logits(s["logits"], history=s["hist"], repetition=s["rep"], stream=stream)
    psc.psc_sample(s["logits"], s["u"], s["tok"], logprobs=s["lp"], bitmask=s["mask"], top_k=s["k"], stream=stream)


@pytest.mark.parametrize("T,V,K", [(1, 5000, 128), (24, 9001, 256), (200, 3000, 64)])
def test_chain_on_a_stream_and_from_a_graph(psc, T, V, K):
    rng = np.random.default_rng([T, V])
    g = torch.Generator(device="cuda").manual_seed(V)
    s = {"x": torch.randn(T, K, device="cuda", generator=g).bfloat16(),
         "q": torch.empty(T, K, dtype=torch.int8, device="cuda"), "sx": torch.empty(T, device="cuda"),
         "w": torch.randint(-127, 128, (V, K), dtype=torch.int8, device="cuda", generator=g),
         "sw": torch.rand(V, device="cuda", generator=g) * 0.01, "logits": torch.empty(T, V, device="cuda"),
         "mask": _pack(_mask(rng, "mixed", T, V)), "hist": torch.randint(0, V, (T, 50), device="cuda", generator=g).int(),
         "rep": torch.full((T,), 1.2, device="cuda"), "u": torch.rand(T, device="cuda", generator=g),
         "tok": torch.empty(T, dtype=torch.int32, device="cuda"), "lp": torch.empty(T, device="cuda"),
         "k": torch.full((T,), 30, dtype=torch.int32, device="cuda"),
         "work": torch.empty(psc.psc_head_work_bytes(T, V, K), dtype=torch.uint8, device="cuda")}
    _chain(psc, s, None)
    want = [s[k].clone() for k in ("logits", "tok", "lp")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):                 # back to back on a stream of its own: buffers are reused at once
        s["x"].copy_(s["x"])
        _chain(psc, s, side)
    side.synchronize()
    for k, t in zip(("logits", "tok", "lp"), want):
        assert torch.equal(s[k], t), k
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _chain(psc, s, None)
    for k in ("logits", "tok", "lp"):
        s[k].zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for k, t in zip(("logits", "tok", "lp"), want):
        assert torch.equal(s[k], t), k


def test_results_do_not_depend_on_the_batch_around_a_row(psc):
    """A row alone gives the bits that it gives in a batch (other variants run there)."""
    g = torch.Generator(device="cuda").manual_seed(5)
    B, V, K = 70, 20000, 256
    q = torch.randint(-127, 128, (B, K), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-127, 128, (V, K), dtype=torch.int8, device="cuda", generator=g)
    sx, sw = torch.rand(B, device="cuda", generator=g), torch.rand(V, device="cuda", generator=g) * 1e-4
    logits = torch.empty(B, V, device="cuda")
    psc.psc_head_logits(q, sx, w, sw, logits)
    u = torch.rand(B, device="cuda", generator=g)
    p = torch.full((B,), 0.9, device="cuda")
    tok, lp = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda")
    psc.psc_sample(logits, u, tok, logprobs=lp, top_p=p)
    for b in (0, 33, 69):
        one = torch.empty(1, V, device="cuda")
        psc.psc_head_logits(q[b:b + 1], sx[b:b + 1], w, sw, one)
        assert torch.equal(one[0], logits[b])
        t1, l1 = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, device="cuda")
        psc.psc_sample(one, u[b:b + 1], t1, logprobs=l1, top_p=p[b:b + 1])
        assert t1[0] == tok[b] and l1[0] == lp[b]


def test_buffers_that_change_between_calls_without_a_wait(psc):
    """Kernels overlap the ends of those before them: twenty steps on the same buffers, each
    input written on the stream right before the call, give what each gives alone."""
    g = torch.Generator(device="cuda").manual_seed(11)
    B, V, K, H = 60, 40000, 128, 9000
    x = torch.empty(B, K, device="cuda", dtype=torch.bfloat16)
    wf = torch.empty(V, K, device="cuda")
    q, sx = torch.empty(B, K, dtype=torch.int8, device="cuda"), torch.empty(B, device="cuda")
    w, sw = torch.empty(V, K, dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    logits, out = torch.empty(B, V, device="cuda"), torch.empty(B, V, device="cuda")
    hist = torch.empty(B, H, dtype=torch.int32, device="cuda")
    mask = torch.empty(B, (V + 31) // 32, dtype=torch.int32, device="cuda")
    k, p = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda")
    u, tok = torch.empty(B, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    pres = torch.full((B,), 0.5, device="cuda")
    steps = [{"x": torch.randn(B, K, device="cuda", generator=g).bfloat16(),
              "wf": torch.randn(V, K, device="cuda", generator=g),
              "hist": torch.randint(0, V, (B, H), device="cuda", generator=g).int(),
              "mask": torch.randint(-2 ** 31, 2 ** 31, mask.shape, device="cuda", generator=g).int(),
              "k": torch.randint(0, 2, (B,), device="cuda", generator=g).int() * 30,
              "p": torch.rand(B, device="cuda", generator=g) + 0.3, "u": torch.rand(B, device="cuda", generator=g)}
             for _ in range(20)]

    def step(s):
        for name, buf in (("x", x), ("wf", wf), ("hist", hist), ("mask", mask), ("k", k), ("p", p), ("u", u)):
            buf.copy_(s[name])
        psc.psc_quantize_rows(x, q, sx)
        psc.psc_quantize_rows(wf, w, sw)              # the weights straight before their use
        psc.psc_head_logits(q, sx, w, sw, logits, bitmask=mask)
        psc.psc_process_logits(logits, out=out, history=hist, presence=pres, bitmask=mask)
        psc.psc_sample(out, u, tok, bitmask=mask, top_k=k, top_p=p)
        return tok.clone(), out.clone()

    chained = [step(s) for s in steps]
    torch.cuda.synchronize()
    for s, (t, y) in zip(steps, chained):
        t2, y2 = step(s)
        torch.cuda.synchronize()
        assert torch.equal(t, t2) and torch.equal(y, y2)
