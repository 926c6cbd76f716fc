"""The norms with a quantised output on the GPU, against numpy.

Codes and the sum h are compared exactly: they are made of correctly rounded f32 products,
sums and quotients on both sides.  A scale holds r = 1 / sqrt(mean h^2 + eps): the squares are
all positive, so a sum of K of them in f32, no addend passing through more additions than a
thread has columns (32, or K / 1024 rounded up to a chunk of 8 in wider rows) and 12 across
threads, is off by that many u = 2^-24 of itself at most; the quotient by K, the addition of
eps, the root and the reciprocal are a rounding each, and the root halves what is in front of it.
"""
from __future__ import annotations

import numpy as np
import pytest

from tests import _mx4_ref as ref
from tests.test_gpu_ops import DT, U, _dev, _f64, _strided, psc  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _adds(K):
    return max(32, 8 * -(-K // 8192)) + 12


def _tolerance(K):
    return (_adds(K) + 2) / 2 * U + 3 * U


def _data(rng, T, K, dtype, loud=True):
    x = rng.standard_normal((T, K)) * rng.uniform(0.1, 10, (T, 1))
    if loud:
        x *= 1 + 20 * (rng.random((1, K)) < 0.02)
    x = x.astype(np.float32)
    return ref.round_bf16(x) if dtype == "bf16" else x


def _int8(v, r):
    """Codes and scale of v with the factor r."""
    unit = np.abs(v).max(1) * (np.float32(1) / np.float32(127))
    safe = np.where(unit > 0, unit, 1).astype(np.float32)
    q = np.clip(np.rint((v / safe[:, None]).astype(np.float32)), -127, 127)
    return np.where(unit[:, None] > 0, q, 0), unit.astype(np.float64) * r


SIZES = [(1, 1, 0), (1, 7, 1), (3, 8, 0), (5, 31, 3), (2, 32, 0), (130, 33, 0), (17, 128, 0), (4, 129, 7), (9, 256, 0),
         (6, 500, 0), (300, 1000, 0), (2, 2048, 8), (3, 2047, 0), (2, 5001, 0), (2, 8192, 0), (2, 8200, 0),
         (3, 16384, 0), (2, 16391, 1), (1, 40000, 0), (2, 70001, 0)]


@pytest.mark.parametrize("T,K,pad", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual,gain,out", [(True, True, "new"), (False, True, None), (True, False, "residual"),
                                               (True, True, "x"), (True, True, None), (False, False, "new")])
def test_norm_quantize(psc, T, K, pad, dtype, residual, gain, out):  # noqa: F811
    rng = np.random.default_rng([T, K, pad, residual, gain])
    x, res = _data(rng, T, K, dtype), _data(rng, T, K, dtype) if residual else None
    g = (rng.uniform(0.5, 1.5, K) * rng.choice([-1, 1], K)).astype(np.float32) if gain else None
    if T > 2:
        x[1] = 0
        if residual:
            res[1] = 0
    h, v, r = ref.norm(x, res, g, 1e-5, dtype == "bf16")
    tol = _tolerance(K)

    def place():
        xb, xd = _strided(x, DT[dtype], pad, 0)
        rb, rd = (None, None) if res is None else _strided(res, DT[dtype], pad, 0)
        sb, sd = {"new": _strided(np.zeros((T, K)), DT[dtype], pad + 1, 1), "x": (xb, xd), "residual": (rb, rd),
                  None: (None, None)}[out]
        return xd, rd, sb, sd, [b for b in (xb, rb) if b is not None]

    def check_sum(sb, sd, others):
        if sd is not None:
            np.testing.assert_array_equal(_f64(sd), h)
            lead = 1 if out == "new" else 0
            assert (sb[:, lead + K:] == 7).all() and (sb[:, :lead] == 7).all()
        for b in others:
            assert (b[:, K:] == 7).all()

    scale = torch.full((T + 1,), 7.0, device="cuda")
    xd, rd, sb, sd, others = place()
    big = torch.full((T, K + 5), 99, dtype=torch.int8, device="cuda")
    psc.psc_norm_quantize_rows(xd, big[:, :K], scale[:T], gain=None if g is None else _dev(g), eps=1e-5, residual=rd,
                               sum_out=sd)
    q, s = _int8(v, r)
    np.testing.assert_array_equal(big[:, :K].cpu().numpy(), q)
    assert (big[:, K:] == 99).all() and scale[T] == 7
    np.testing.assert_allclose(_f64(scale[:T]), s, rtol=tol + U, atol=0)
    check_sum(sb, sd, others)

    xd, rd, sb, sd, others = place()
    n = psc.psc_mx4_row_bytes(K)
    big = torch.full((T, n + 16), 99, dtype=torch.uint8, device="cuda")
    blocks = torch.full((psc.psc_mx4_block_bytes(T, K),), 77, dtype=torch.uint8, device="cuda")
    psc.psc_norm_quantize_mx4(xd, big[:, :n], blocks, scale[:T], gain=None if g is None else _dev(g), eps=1e-5,
                              residual=rd, sum_out=sd)
    codes, e = ref.quantize(v)
    np.testing.assert_array_equal(big[:, :n].cpu().numpy(), ref.pack(codes))
    assert (big[:, n:] == 99).all() and scale[T] == 7
    np.testing.assert_array_equal(blocks.cpu().numpy(), ref.tiles(e, K, 77))
    np.testing.assert_allclose(_f64(scale[:T]), r, rtol=tol, atol=0)
    check_sum(sb, sd, others)


@pytest.mark.parametrize("K", [40, 2048, 20000])
def test_rows_that_are_not_finite_or_zero(psc, K):  # noqa: F811
    T = 7
    x = np.random.default_rng(K).standard_normal((T, K)).astype(np.float32)
    g = np.ones(K, dtype=np.float32)
    x[1, K // 2], x[2, 0], x[3, K - 1] = np.inf, np.nan, -np.inf
    x[4] = 0
    x[5, 3] = 1e30
    g[3] = 1e30                                  # h * gain leaves f32 in row 5
    q, s = torch.full((T, K), 9, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    psc.psc_norm_quantize_rows(_dev(x), q, s, gain=_dev(g), eps=0.0)
    q, s = q.cpu().numpy(), s.cpu().numpy()
    bad = [1, 2, 3, 5]
    assert np.isnan(s[bad]).all() and (q[bad] == 0).all()
    assert s[4] == 0 and (q[4] == 0).all() and np.isfinite(s[[0, 6]]).all()
    c = torch.empty(T, psc.psc_mx4_row_bytes(K), dtype=torch.uint8, device="cuda")
    b = torch.empty(psc.psc_mx4_block_bytes(T, K), dtype=torch.uint8, device="cuda")
    psc.psc_norm_quantize_mx4(_dev(x), c, b, t := torch.empty(T, device="cuda"),
                              gain=_dev(g), eps=0.0)
    with np.errstate(over="ignore", invalid="ignore"):
        codes, e = ref.quantize(x * g[None])
    assert (e == 255).sum() == 4
    np.testing.assert_array_equal(c.cpu().numpy(), ref.pack(codes))
    full = ref.tiles(e, K, 0)
    rows = ref.tiles(np.ones_like(e), K, 0) == 1         # what rows of the matrix write
    np.testing.assert_array_equal(b.cpu().numpy()[rows], full[rows])
    t = t.cpu().numpy()
    assert np.isnan(t[bad]).all() and t[4] == 0 and np.isfinite(t[[0, 6]]).all()
    # with eps, a row of zeros has a finite factor and zero codes
    psc.psc_norm_quantize_mx4(_dev(x), c, b, s2 := torch.empty(T, device="cuda"), gain=_dev(g), eps=1e-4)
    assert abs(s2[4].item() - 100) < 1e-3


@pytest.mark.parametrize("K", [48, 4096, 9000, 33000])
@pytest.mark.parametrize("size", [1e-42, 1e-30, 1e-14, 1e14, 1e25, 3e37])
def test_sizes_whose_squares_leave_f32(psc, K, size):  # noqa: F811
    rng = np.random.default_rng(K)
    x = (rng.uniform(-1, 1, (3, K)) * size).astype(np.float32)
    x[:, 0] = size
    for eps in (0.0, 1e-6):
        h, v, r = ref.norm(x, None, None, eps, False)
        q, s = torch.empty(3, K, dtype=torch.int8, device="cuda"), torch.empty(3, device="cuda")
        for out in (None, torch.empty(3, K, device="cuda")):
            psc.psc_norm_quantize_rows(_dev(x), q, s, eps=eps, sum_out=out)
            want, scale = _int8(v, r)
            np.testing.assert_array_equal(q.cpu().numpy(), want)
            # the product's own rounding is a whole step where the scale is below the normal numbers
            np.testing.assert_allclose(_f64(s), scale, rtol=_tolerance(K) + U, atol=2.0 ** -149)
        n = psc.psc_mx4_row_bytes(K)
        c = torch.empty(3, n, dtype=torch.uint8, device="cuda")
        b = torch.full((psc.psc_mx4_block_bytes(3, K),), 5, dtype=torch.uint8, device="cuda")
        psc.psc_norm_quantize_mx4(_dev(x), c, b, s, eps=eps)
        codes, e = ref.quantize(v)
        np.testing.assert_array_equal(c.cpu().numpy(), ref.pack(codes))
        np.testing.assert_array_equal(b.cpu().numpy(), ref.tiles(e, K, 5))
        if r.max() < 3e38:
            np.testing.assert_allclose(_f64(s), r, rtol=_tolerance(K), atol=0)
        else:
            assert (s[torch.from_numpy(r > 3.5e38)] == float("inf")).all()


def test_a_row_does_not_depend_on_its_batch(psc):  # noqa: F811
    rng = np.random.default_rng(3)
    for K in (1000, 4096, 9000):
        x, g = _dev(_data(rng, 500, K, "bf16")).bfloat16(), _dev(rng.uniform(0.5, 1.5, K).astype(np.float32))
        q, s = torch.empty(500, K, dtype=torch.int8, device="cuda"), torch.empty(500, device="cuda")
        psc.psc_norm_quantize_rows(x, q, s, gain=g)
        for t in (0, 77, 499):
            q1, s1 = torch.empty(1, K, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
            psc.psc_norm_quantize_rows(x[t:t + 1], q1, s1, gain=g)
            assert torch.equal(q1[0], q[t]) and torch.equal(s1[0], s[t])


@pytest.mark.parametrize("T,K,dtype,residual", [(20000, 72, "bf16", True), (16000, 40, "f32", False), (4001, 4096, "bf16", True),
                                                (7000, 2048, "bf16", False), (4000, 2056, "f32", True),
                                                (3000, 8192, "bf16", True), (9000, 1000, "bf16", True),
                                                (4001, 4095, "bf16", True), (9000, 1003, "f32", True), (20000, 61, "bf16", False),
                                                (700, 16384, "bf16", True), (700, 13001, "bf16", True)])
def test_many_rows_are_what_a_few_are(psc, T, K, dtype, residual):  # noqa: F811
    """A batch that is worked on in turns, rows that need a second pass among it, against the same
    rows a few at a time; the sum in place of the residual."""
    rng = np.random.default_rng([T, K])
    x = _dev(_data(rng, T, K, dtype)).to(DT[dtype])
    x[5], x[6, 3], x[T - 1] = 0, float("inf"), 0
    x[7], x[T // 2], x[T // 2 + 1] = x[7] * 1e28, x[T // 2] * 1e-28, float("nan")
    res = _dev(_data(rng, T, K, dtype)).to(DT[dtype]) if residual else None
    if residual:
        res[5:8], res[T // 2:T // 2 + 2], res[T - 1] = 0, 0, 0
    g, n = _dev(rng.uniform(0.5, 1.5, K).astype(np.float32)), psc.psc_mx4_row_bytes(K)

    def run(lo, hi):
        rows = hi - lo
        r8 = None if res is None else res[lo:hi].clone()
        r4 = None if res is None else res[lo:hi].clone()
        q8, s8 = torch.zeros(rows, K, dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
        q4, s4 = torch.zeros(rows, n, dtype=torch.uint8, device="cuda"), torch.zeros(rows, device="cuda")
        b = torch.zeros(psc.psc_mx4_block_bytes(rows, K), dtype=torch.uint8, device="cuda")
        psc.psc_norm_quantize_rows(x[lo:hi], q8, s8, gain=g, residual=r8, sum_out=r8, eps=0.0)
        psc.psc_norm_quantize_mx4(x[lo:hi], q4, b, s4, gain=g, residual=r4, sum_out=r4, eps=0.0)
        return [t for t in (q8, s8.view(torch.int32), q4, s4.view(torch.int32), r8, r4) if t is not None], b

    whole, blocks = run(0, T)
    tiles = blocks.view((T + 127) // 128, -1)
    for lo in (0, 256, T // 2 // 128 * 128, (T - 1) // 128 * 128):
        few, b = run(lo, min(T, lo + 128))
        for u, v in zip(whole, few):
            assert torch.equal(u[lo:lo + 128].view(torch.uint8), v.view(torch.uint8))
        assert torch.equal(tiles[lo // 128], b)


def test_feeds_the_projections(psc):  # noqa: F811
    """The norm and both projections after it, against the normalised rows in 64 bits: a value of 8 bits
    is off by half a step of its row's largest / 127, one of 4 bits by a quarter of its block's largest."""
    rng = np.random.default_rng(11)
    T, V, K = 33, 700, 512
    x, res, g = _data(rng, T, K, "bf16"), _data(rng, T, K, "bf16"), rng.uniform(0.5, 1.5, K).astype(np.float32)
    h, v, r = ref.norm(x, res, g, 1e-6, True)
    y = v.astype(np.float64) * r[:, None]
    w = rng.standard_normal((V, K)).astype(np.float32)
    xd, rd, gd, wd = _dev(x).bfloat16(), _dev(res).bfloat16(), _dev(g), _dev(w)
    q, s, out = (torch.empty(T, K, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"),
                 torch.empty(T, V, device="cuda"))
    wq, ws = torch.empty(V, K, dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    psc.psc_quantize_rows(wd, wq, ws)
    psc.psc_norm_quantize_rows(xd, q, s, gain=gd, residual=rd)
    psc.psc_head_logits(q, s, wq, ws, out)
    w8 = wq.double().cpu().numpy() * _f64(ws)[:, None]
    bound = np.abs(y).max(1)[:, None] / 254 * np.abs(w8).sum(1)[None] * 1.001
    assert (np.abs(_f64(out) - y @ w8.T) <= bound).all()
    n = psc.psc_mx4_row_bytes(K)
    q, b = torch.empty(T, n, dtype=torch.uint8, device="cuda"), torch.empty(psc.psc_mx4_block_bytes(T, K),
                                                                            dtype=torch.uint8, device="cuda")
    wq, wb = torch.empty(V, n, dtype=torch.uint8, device="cuda"), torch.empty(psc.psc_mx4_block_bytes(V, K),
                                                                              dtype=torch.uint8, device="cuda")
    psc.psc_quantize_mx4(wd, wq, wb)
    psc.psc_norm_quantize_mx4(xd, q, b, s, gain=gd, residual=rd)
    psc.psc_head_logits_mx4(q, b, wq, wb, out, K, scale=s)
    w4 = ref.decode(*ref.quantize(w))
    # up to 6 of 8 in the largest's binade is cut: a quarter of it; elsewhere half a step of 2
    top = np.repeat(np.abs(y).reshape(T, -1, 32).max(-1), 32, axis=1)
    bound = (top / 4 * 1.001) @ np.abs(w4).T
    assert (np.abs(_f64(out) - y @ w4.T) <= bound + 1e-4).all()


def test_other_streams_and_graphs(psc):  # noqa: F811
    rng = np.random.default_rng(5)
    T, K = 65, 1500
    x, res, g = (_dev(_data(rng, T, K, "f32")) for _ in range(3))
    g = g[0].contiguous()
    n = psc.psc_mx4_row_bytes(K)

    def buffers():
        return (torch.zeros(T, K, dtype=torch.int8, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, K, device="cuda"),
                torch.zeros(T, n, dtype=torch.uint8, device="cuda"),
                torch.zeros(psc.psc_mx4_block_bytes(T, K), dtype=torch.uint8, device="cuda"), torch.zeros(T, device="cuda"))

    def call(o, stream=None):
        psc.psc_norm_quantize_rows(x, o[0], o[1], gain=g, residual=res, sum_out=o[2], stream=stream)
        psc.psc_norm_quantize_mx4(o[2], o[3], o[4], o[5], gain=g, stream=stream)

    a, b, c = buffers(), buffers(), buffers()
    call(a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(b, side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c)
    x.mul_(2)
    graph.replay()
    call(a)
    torch.cuda.synchronize()
    for u, w in zip(a, c):
        assert torch.equal(u, w)
    x.mul_(0.5)
    call(a)
    torch.cuda.synchronize()
    for u, w in zip(a, b):
        assert torch.equal(u, w)


@pytest.mark.parametrize("T", [3, 8000])
def test_sums_of_any_two_bf16(psc, T):  # noqa: F811
    """x + residual over all bit patterns, subnormal ones among them: the f32 sum, rounded once more."""
    K, rng = 64, np.random.default_rng(T)
    bits = rng.integers(-32768, 32768, (2, T, K)).astype(np.int16)
    bits[1, ::2] = (bits[0, ::2] ^ -32768) + rng.integers(-4, 5, bits[0, ::2].shape)      # nearly -x
    bits[1, 1::4] = bits[0, 1::4] - rng.integers(0, 1 << 11, bits[0, 1::4].shape)        # a smaller exponent, often
    x, res = (torch.from_numpy(b).view(torch.bfloat16) for b in bits)
    out = torch.empty(T, K, dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty(T, K, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    psc.psc_norm_quantize_rows(x.cuda(), q, s, residual=res.cuda(), sum_out=out)
    want, got = (x.float() + res.float()).bfloat16(), out.cpu()
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan) and (want.float().abs()[~nan] < 2.0 ** -126).any()
    assert torch.equal(got[~nan].view(torch.int16), want[~nan].view(torch.int16))


@pytest.mark.parametrize("K,dtype", [(1001, "bf16"), (4095, "bf16"), (130, "f32")])
def test_a_row_at_any_address_has_the_same_codes(psc, K, dtype):  # noqa: F811
    """Rows that start anywhere: the codes are those of the row alone, the scale up to the order of its sum."""
    rng = np.random.default_rng(K)
    x = _dev(_data(rng, 9, K, dtype)).to(DT[dtype])
    q, s = torch.empty(9, K, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    psc.psc_norm_quantize_rows(x, q, s)
    for t in range(9):
        q1, s1 = torch.empty(1, K, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
        psc.psc_norm_quantize_rows(x[t:t + 1].clone(), q1, s1)
        assert torch.equal(q1[0], q[t])
        np.testing.assert_allclose(_f64(s1), _f64(s[t:t + 1]), rtol=2 * _tolerance(K), atol=0)
