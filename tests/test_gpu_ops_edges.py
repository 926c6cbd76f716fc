"""The operators around the mask on the GPU where their variants meet: values and masks
that send a row from one way of drawing to another, sizes at which rings and slabs go
round.  Reference forms and tolerances are those of test_gpu_ops."""
from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_ops import DT, NEG, U, UB, _check_draws, _dev, _f64, _head_case, _pack, psc  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------- sample
def _draw(psc, x, dtype, u, allowed=None, T=None, k=None, p=None, m=None, rows=None):  # noqa: F811
    """One call, checked against the 64-bit draw on `rows` (all if None); None leaves a filter out."""
    B, V = x.shape
    xd = _dev(x.astype(np.float32)).to(DT[dtype])
    tok, lp = torch.full((B,), -7, dtype=torch.int32, device="cuda"), torch.full((B,), 7.0, device="cuda")
    f32 = [None if a is None else np.asarray(a, dtype=np.float32) for a in (T, p, m)]
    psc.psc_sample(xd, _dev(u), tok, logprobs=lp, bitmask=None if allowed is None else _pack(allowed),
                   temperature=None if T is None else _dev(f32[0]), top_p=None if p is None else _dev(f32[1]),
                   min_p=None if m is None else _dev(f32[2]),
                   top_k=None if k is None else _dev(np.asarray(k, dtype=np.int32)))
    rows = np.arange(B) if rows is None else np.asarray(rows)
    T, p, m = (np.full(B, d) if a is None else a.astype(np.float64) for a, d in zip(f32, (1.0, 1.0, 0.0)))
    k = np.zeros(B, dtype=int) if k is None else np.asarray(k)
    _check_draws(tok.cpu().numpy()[rows], _f64(lp)[rows], _f64(xd[rows]), None if allowed is None else allowed[rows],
                 u[rows], T[rows], k[rows], p[rows], m[rows])
    return tok.cpu().numpy(), _f64(lp)


@pytest.mark.parametrize("V,first,n", [(262144, 1024, 400), (262144, 1000, 1000), (200001, 1564, 380),
                                       (151936, 600, 280), (140001, 100, 2000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 60])
def test_sample_among_neighbouring_tokens(psc, V, first, n, dtype, B):  # noqa: F811
    """What stays lies close together (the digits of a number, the names of one prefix), and the
    filters leave all that is listed: min-p alone, top-k of no fewer than the candidates."""
    rng = np.random.default_rng([V, n, B])
    x = np.full((B, V), -20.0)
    x[:, first:first + n] = rng.standard_normal((B, n)) * 0.25
    allowed = np.zeros((B, V), dtype=bool)
    allowed[:, first:first + n] = True
    u = rng.random(B).astype(np.float32)
    rows = np.unique([0, B // 2, B - 1])
    for mask in (None, allowed):
        _draw(psc, x, dtype, u, mask, m=np.full(B, 0.01), rows=rows)
        _draw(psc, x, dtype, u, mask, m=np.full(B, 1e-4), T=np.full(B, 0.8), rows=rows)
    _draw(psc, x, dtype, u, allowed, k=np.full(B, n), rows=rows)
    _draw(psc, x, dtype, u, allowed, k=np.full(B, 5000), rows=rows)
    _draw(psc, x, dtype, u, allowed, k=np.full(B, 5000), m=np.full(B, 0.3), rows=rows)
    _draw(psc, x, dtype, u, allowed, k=np.full(B, 5000), p=np.full(B, 0.9), rows=rows)


def test_sample_top_k_of_as_many_tokens_as_reach_the_bound(psc):  # noqa: F811
    """Every one of the k largest lies in a group of its own, so that the list holds them and no
    other; the tokens below it would take nearly all of the weight."""
    V, n = 1 << 22, 400
    x = np.full((1, V), -3.0)
    x[0, np.arange(n) * 8] = np.arange(n) * 1e-3
    for u in (0.25, 0.75):
        _draw(psc, x, "f32", np.array([u], dtype=np.float32), k=[n])


@pytest.mark.parametrize("B,V", [(7, 1000), (60, 9000), (5, 150001)])
@pytest.mark.parametrize("dtype,filters", [("bf16", ""), ("f32", "k"), ("bf16", "p"), ("f32", "m"), ("bf16", "kpm")])
@pytest.mark.filterwarnings("ignore:invalid value")          # -inf / inf of the reference's masked tokens
def test_sample_at_an_infinite_temperature_is_uniform(psc, B, V, dtype, filters):  # noqa: F811
    """z = (x - m) * (1 / T) is 0 for every candidate: what the filters keep is drawn evenly.  Rows
    at the largest finite temperature, at 0 and NaN (greedy) and at 1 beside them."""
    rng = np.random.default_rng([V, B])
    x = rng.integers(-12, 12, (B, V)) * 0.25
    allowed = rng.random((B, V)) < 0.5
    T = np.resize([np.inf, np.finfo(np.float32).max, 0.0, np.inf, 1.0, np.nan, np.inf], B)
    u = ((np.arange(B) + 0.5) / B).astype(np.float32)
    rows = np.arange(min(B, 7))
    tok, lp = _draw(psc, x, dtype, u, allowed, T=T, rows=rows, k=np.full(B, 50) if "k" in filters else None,
                    p=np.full(B, 0.3) if "p" in filters else None, m=np.full(B, 0.5) if "m" in filters else None)
    if not filters:                                          # the u-th of the allowed, in order
        for b in np.flatnonzero(np.isinf(T)):
            at = np.flatnonzero(allowed[b])
            assert tok[b] == at[int(np.floor(u[b] * 2.0 ** 24)) * len(at) >> 24]
            assert abs(lp[b] + np.log(len(at))) <= 1e-6 * np.log(len(at))


# ------------------------------------------------------------------------- head
@pytest.mark.parametrize("T,V,K", [(20, 300001, 64), (24, 280000, 16), (48, 290000, 48), (100, 280001, 64),
                                   (128, 280000, 64), (200, 270001, 64), (300, 150000, 33), (1000, 70000, 64),
                                   (20, 120001, 129), (160000, 100, 192), (160000, 128, 320), (128000, 77, 448),
                                   (110000, 60, 64)])
def test_head_logits_of_short_rows_and_many_tiles(psc, T, V, K):  # noqa: F811
    """A tile is one or few stages of the pipeline, and a block has a dozen tiles and more: the
    rings go round across tiles, and a byte slot is used by one group after another."""
    _head_case(psc, T, V, K, "bf16", "none", pad=-K % 16)
    _head_case(psc, T, V, K, "f32", "mixed" if T < 2000 else "none", pad=-K % 16)


@pytest.mark.parametrize("T,V,K,shift,mask", [(1, 5000, 256, 0, 0), (4, 5000, 256, 0, 1), (8, 5000, 256, 0, 1),
                                              (12, 30000, 512, 0, 1), (12, 30000, 512, 0, 2), (12, 30000, 512, 0, 0),
                                              (60, 30000, 512, 0, 1), (200, 60000, 512, 0, 1), (200, 60000, 512, 0, 0),
                                              (3, 9000, 2047, 1, 0), (40, 140000, 2047, 1, 1), (300, 140000, 2047, 1, 0)])
def test_head_faults_is_what_the_last_call_says(psc, T, V, K, shift, mask):  # noqa: F811
    """Rows, single blocks, pairs, one slab and several: a call leaves the number of blocks that gave
    up, whatever the workspace held before.  (No wait is made to give up on the GPU: a number is written in.)"""
    g = torch.Generator(device="cuda").manual_seed(T)
    q = torch.randint(-127, 128, (T, K), generator=g, dtype=torch.int8, device="cuda")
    w = torch.randint(-127, 128, (V, K + shift), generator=g, dtype=torch.int8, device="cuda")[:, shift:]
    sx, sw, out = torch.rand(T, device="cuda"), torch.rand(V, device="cuda"), torch.empty(T, V, device="cuda")
    bits = torch.randint(-2 ** 31, 2 ** 31 - 1, (T, (V + 31) // 32), generator=g, dtype=torch.int32, device="cuda")
    bits = None if mask == 0 else bits if mask == 1 else bits * (torch.arange((V + 31) // 32, device="cuda") % 50 == 0)
    bits = bits if bits is None else bits.int()
    work = psc.psc_head_logits(q, sx, w, sw, out, bitmask=bits)          # one of its own
    assert psc.psc_head_faults(work) == 0
    work.fill_(1)
    assert psc.psc_head_faults(work) == 0x01010101
    assert psc.psc_head_logits(q, sx, w, sw, out, bitmask=bits, work=work) is work
    assert psc.psc_head_faults(work) == 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    work[:4].view(torch.int32).fill_(3)
    side.wait_stream(torch.cuda.current_stream())
    for s in (side, side.cuda_stream):
        psc.psc_head_logits(q, sx, w, sw, out, bitmask=bits, work=work, stream=s)
        assert psc.psc_head_faults(work, stream=s) == 0
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("K", [1024, 1000])
@pytest.mark.parametrize("T", [1, 4, 16, 24, 150])
def test_head_sums_of_any_bytes_are_exact_up_to_1024_columns(psc, T, K):  # noqa: F811
    """-128 on both sides: every sum is a whole number within 2^24, and with scales of 1 the
    logits are those numbers, whichever variant forms them."""
    rng = np.random.default_rng([T, K])
    V = 700
    q, w = rng.integers(-128, 128, (T, K)), rng.integers(-128, 128, (V, K))
    q[0] = w[0] = w[V - 1] = -128
    w[1] = 127
    w[2] = np.where(np.arange(K) % 2, 127, -128)
    out = torch.empty(T, V, device="cuda")
    pitch = (K + 15) // 16 * 16
    wd = torch.empty(V, pitch, dtype=torch.int8, device="cuda")[:, :K]
    wd.copy_(_dev(w, torch.int8))
    psc.psc_head_logits(_dev(q, torch.int8), torch.ones(T, device="cuda"), wd, torch.ones(V, device="cuda"), out)
    np.testing.assert_array_equal(_f64(out), (q @ w.T).astype(np.float64))


@pytest.mark.parametrize("T,V,K,pad,shift", [(3, 70001, 4095, 0, 0), (12, 70001, 4095, 0, 1), (40, 70001, 4095, 0, 0),
                                             (140, 280003, 1001, 0, 2), (2, 1100000, 250, 1, 0)])
@pytest.mark.parametrize("dtype,mask", [("f32", "none"), ("bf16", "mixed"), ("f32", "tight")])
def test_head_logits_of_packed_rows_over_two_slabs(psc, T, V, K, pad, shift, dtype, mask):  # noqa: F811
    """Packed rows of more than 256 MB: the second slab's rows, scales and mask words against 64
    bits, on the rows around the slabs' edge, the first and the last."""
    pitch = (K + 15) // 16 * 16
    edge = (256 << 20) // pitch // 128 * 128
    assert edge < V < 2 * edge
    rng = np.random.default_rng([T, V, K])
    q = rng.integers(-127, 128, (T, K), dtype=np.int8)
    flat = torch.randint(-127, 128, (V * (K + pad) + shift,), dtype=torch.int8, device="cuda",
                         generator=torch.Generator(device="cuda").manual_seed(K))
    w = flat[shift:].view(V, K + pad)[:, :K]
    sx, sw = rng.uniform(0.01, 0.1, T).astype(np.float32), rng.uniform(1e-4, 1e-3, V).astype(np.float32)
    allowed = None if mask == "none" else rng.random((T, V)) < (0.5 if mask == "mixed" else 0.001)
    if allowed is not None:
        allowed[0] = False
        allowed[-1, edge - 3:edge + 3] = allowed[-1, V - 1] = True
    big = torch.full((T, V + 3), 7.0, dtype=DT[dtype], device="cuda")
    psc.psc_head_logits(_dev(q), _dev(sx), w, _dev(sw), big[:, :V], bitmask=None if allowed is None else _pack(allowed))
    assert (big[:, V:] == 7).all()
    rows = np.unique(np.r_[0:300, edge - 300:edge + 300, V - 300:V, rng.integers(0, V, 300)])
    at = torch.from_numpy(rows).cuda()
    got, wr = _f64(big[:, at]), w[at].cpu().numpy().astype(np.float64)
    exact = q.astype(np.float64) @ wr.T * sx.astype(np.float64)[:, None] * sw[rows].astype(np.float64)
    tol = (3 * U + (UB if dtype == "bf16" else 0)) * np.abs(exact)
    if K > 1040:                          # as in _head_case
        size = np.abs(q).astype(np.float64) @ np.abs(wr).T
        tol = tol + np.where(size >= 2.0 ** 24, 2 * U * (K / 16) * size * sx[:, None] * sw[rows], 0)
    if allowed is not None:
        assert (got[~allowed[:, rows]] == NEG).all()
        assert int(big[:, :V].isneginf().sum()) == int((~allowed).sum())
        exact, tol, got = (a[allowed[:, rows]] for a in (exact, tol, got))
    assert (np.abs(got - exact) <= tol * 1.0000001).all()
