"""Microscaled 4-bit floating point on the GPU, against numpy in 64 bits.

Codes, exponents and values read back are compared exactly.  The projection's products are
exact (whole quarters times powers of two); its sums over K are in f32: up to K / 64 partial
sums of 64 products, in each of which a tensor core may cut the addends below its 24 bits, the
running sum among them, and round or cut the result: 4u of the sum of magnitudes, u = 2^-24;
by rows a sum passes through K / 1024 + 6 roundings, which is less where K >= 512 and 8u below.
Two products by scales and the rounding to the logits' type (2^-8 for bf16) come on top.
"""
from __future__ import annotations

import numpy as np
import pytest

from tests import _mx4_ref as ref
from tests.test_gpu_ops import DT, NEG, U, UB, _dev, _f64, _mask, _pack, _strided, psc  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _blocks_of(psc, rows, K, fill=0):  # noqa: F811
    return torch.full((psc.psc_mx4_block_bytes(rows, K),), fill, dtype=torch.uint8, device="cuda")


def _values(rng, T, K, dtype):
    """Values of all sizes, ties and borders of the format among them."""
    x = rng.standard_normal((T, K)) * np.exp2(rng.integers(-30, 30, (T, 1)))
    ties = rng.random((T, K)) < 0.3
    x = np.where(ties, rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.99, 0, -0.0, 4], (T, K)) * rng.choice([-1, 1], (T, K)), x)
    x = x.astype(np.float32)
    return ref.round_bf16(x) if dtype == "bf16" else x


@pytest.mark.parametrize("T,K,pad", [(1, 1, 0), (1, 8, 0), (3, 31, 0), (2, 32, 0), (5, 33, 2), (129, 64, 0), (33, 100, 0),
                                     (128, 128, 0), (260, 129, 0), (3, 1000, 8), (7, 2047, 0), (2, 2048, 0), (1, 9000, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_and_back(psc, T, K, pad, dtype):  # noqa: F811
    rng = np.random.default_rng([T, K])
    x = _values(rng, T, K, dtype)
    if T > 2:
        x[1] = 0
    _, xd = _strided(x, DT[dtype], pad, 0)
    n = psc.psc_mx4_row_bytes(K)
    big, blocks = torch.full((T, n + 16), 99, dtype=torch.uint8, device="cuda"), _blocks_of(psc, T, K, 77)
    psc.psc_quantize_mx4(xd, big[:, :n], blocks)
    codes, e = ref.quantize(x)
    np.testing.assert_array_equal(big[:, :n].cpu().numpy(), ref.pack(codes))
    assert (big[:, n:] == 99).all()
    np.testing.assert_array_equal(blocks.cpu().numpy(), ref.tiles(e, K, 77))
    values = ref.decode(codes, e)
    for out in ("bf16", "f32"):
        for shift in (0, 1):
            full, y = _strided(np.zeros((T, K)), DT[out], pad, shift)
            psc.psc_dequantize_mx4(big[:, :n], blocks, y)
            np.testing.assert_array_equal(_f64(y), values)
            assert (full[:, :shift] == 7).all() and (full[:, shift + K:] == 7).all()
    scale = rng.uniform(0.1, 3, T).astype(np.float32)
    y = torch.empty(T, K, device="cuda")
    psc.psc_dequantize_mx4(big[:, :n], blocks, y, scale=_dev(scale))
    np.testing.assert_array_equal(_f64(y), (values.astype(np.float32) * scale[:, None]).astype(np.float64))


def test_quantize_at_the_ends_of_f32(psc):  # noqa: F811
    tops = [1e-45, 1e-40, 2.0 ** -127, 2.0 ** -126, 2.0 ** -125, 2.0 ** -124, 3e38, np.float32(3.4028235e38), 2.0 ** 127, float(np.finfo(np.float32).max)]
    x = np.zeros((len(tops) + 3, 64), dtype=np.float32)
    for i, t in enumerate(tops):                # the largest as an f32 passes it on the way, and is not finite then
        x[i, :32] = np.linspace(-t, t, 32, dtype=np.float64).astype(np.float32)
        x[i, 33] = t
    x[-3, 5], x[-2, 40], x[-1, 0] = np.inf, np.nan, -np.inf
    n = psc.psc_mx4_row_bytes(64)
    q, b = torch.empty(len(x), n, dtype=torch.uint8, device="cuda"), _blocks_of(psc, len(x), 64, 3)
    psc.psc_quantize_mx4(_dev(x), q, b)
    codes, e = ref.quantize(x)
    np.testing.assert_array_equal(b.cpu().numpy(), ref.tiles(e, 64, 3))
    np.testing.assert_array_equal(q.cpu().numpy(), ref.pack(codes))
    with np.errstate(invalid="ignore"):
        assert ((e == 255) == ~np.isfinite(x).reshape(len(x), 2, 32).all(-1)).all()
    y = torch.empty(len(x), 64, device="cuda")
    psc.psc_dequantize_mx4(q, b, y)
    np.testing.assert_array_equal(_f64(y), ref.decode(codes, e))


# --------------------------------------------------------------------- the projection
def _matrix(psc, codes, e, K, pad=0, rows_fill=0xA5):  # noqa: F811
    """Codes and exponents on the device, rows `pad` bytes further apart; what is not the matrix's is not zero."""
    p = ref.pack(codes)
    big = torch.full((p.shape[0], p.shape[1] + pad), 0x7B, dtype=torch.uint8, device="cuda")
    big[:, :p.shape[1]] = _dev(p)
    return big[:, :p.shape[1]], _dev(ref.tiles(e, K, rows_fill))


def _head_case(psc, T, V, K, dtype, mask, scales=True, pad=0, out_pad=0, spread=3, stream=None, seed=0):  # noqa: F811
    rng = np.random.default_rng([T, V, K, seed])
    qc, wc = rng.integers(0, 16, (T, K), dtype=np.uint8), rng.integers(0, 16, (V, K), dtype=np.uint8)
    nb = (K + 31) // 32
    qe = rng.integers(127 - spread, 128 + spread, (T, nb)).astype(np.uint8)
    we = rng.integers(120 - spread, 121 + spread, (V, nb)).astype(np.uint8)
    sx, sw = rng.uniform(0.01, 0.1, T).astype(np.float32), rng.uniform(0.1, 10, V).astype(np.float32)
    allowed = _mask(rng, mask, T, V)
    big = torch.full((T, V + out_pad), 7.0, dtype=DT[dtype], device="cuda")
    psc.psc_head_logits_mx4(*_matrix(psc, qc, qe, K, pad), *_matrix(psc, wc, we, K, pad), big[:, :V], K,
                            scale=_dev(sx) if scales else None, w_scale=_dev(sw) if scales else None,
                            bitmask=None if allowed is None else _pack(allowed), stream=stream)
    assert psc.psc_mx4_faults(stream=stream) == 0
    got = _f64(big)
    assert (got[:, V:] == 7).all()
    got = got[:, :V]
    x, w = ref.decode(qc, qe), ref.decode(wc, we)
    f = sx.astype(np.float64)[:, None] * sw.astype(np.float64) if scales else np.ones((1, 1))
    exact, size = x @ w.T * f, np.abs(x) @ np.abs(w).T * f
    tol = 4 * U * (K / 64 + 2) * size + (2 * U + (UB if dtype == "bf16" else 0)) * np.abs(exact)
    if allowed is not None:
        assert (got[~allowed] == NEG).all()
        exact, tol, got = exact[allowed], tol[allowed], got[allowed]
    assert (np.abs(got - exact) <= tol * 1.0000001).all(), np.max(np.abs(got - exact) / np.maximum(tol, 1e-300))


SIZES = [(1, 1, 1), (1, 130, 16), (1, 1000, 48), (2, 257, 64), (3, 129, 100), (7, 512, 257), (8, 1000, 1024),
         (9, 640, 320), (16, 333, 512), (17, 300, 80), (33, 1024, 1040), (64, 129, 128), (100, 1500, 192),
         (128, 500, 600), (130, 260, 2048), (190, 700, 384), (200, 300, 1000), (256, 384, 64), (257, 500, 336),
         (300, 127, 96), (385, 1000, 640), (513, 1300, 160), (4, 300, 4096), (8, 700, 2048), (16, 2500, 4080),
         (16, 200, 4200), (5, 200, 33000), (140, 300, 8192)]


@pytest.mark.parametrize("T,V,K", SIZES)
@pytest.mark.parametrize("dtype,mask,scales", [("bf16", "none", True), ("f32", "mixed", False), ("bf16", "tight", True),
                                               ("f32", "none", True)])
def test_head_logits(psc, T, V, K, dtype, mask, scales):  # noqa: F811
    _head_case(psc, T, V, K, dtype, mask, scales, pad=16 * (K % 3), out_pad=K % 5)


@pytest.mark.parametrize("T,V,K", [(1, 30000, 512), (5, 40001, 256), (40, 60000, 256), (300, 50000, 256),
                                   (600, 45000, 512), (129, 33333, 1300)])
def test_head_of_many_tiles(psc, T, V, K):  # noqa: F811
    """More tiles than blocks that run at once: rings and accumulators go round."""
    _head_case(psc, T, V, K, "f32", "none")
    _head_case(psc, T, V, K, "bf16", "mixed")
    _head_case(psc, T, V, K, "f32", "tight")


@pytest.mark.parametrize("T", [3, 40, 300])
def test_head_of_values_far_apart(psc, T):  # noqa: F811
    """Blocks whose sizes differ by powers up to 2^40 within a row."""
    _head_case(psc, T, 400, 700, "f32", "none", spread=20)


@pytest.mark.parametrize("T", [1, 20, 200])
def test_head_masks(psc, T):  # noqa: F811
    """Nothing allowed anywhere, one token in the whole batch, all of one tile, the last token."""
    rng = np.random.default_rng(T)
    V, K = 1333, 320
    x, w = rng.standard_normal((T, K)).astype(np.float32), rng.standard_normal((V, K)).astype(np.float32)
    qc, qe = ref.quantize(x)
    wc, we = ref.quantize(w)
    q, w4 = _matrix(psc, qc, qe, K), _matrix(psc, wc, we, K)
    exact = ref.decode(qc, qe) @ ref.decode(wc, we).T
    size = np.abs(ref.decode(qc, qe)) @ np.abs(ref.decode(wc, we)).T
    for kind in ("none", "one", "tile", "last", "all"):
        a = np.zeros((T, V), dtype=bool)
        if kind == "one":
            a[T // 2, 777] = True
        elif kind == "tile":
            a[:, 256:384] = True
        elif kind == "last":
            a[T - 1, V - 1] = True
        elif kind == "all":
            a[:] = True
        out = torch.full((T, V), 7.0, device="cuda")
        psc.psc_head_logits_mx4(*q, *w4, out, K, bitmask=_pack(a))
        got = _f64(out)
        assert (got[~a] == NEG).all()
        assert (np.abs(got - exact)[a] <= 4 * U * (K / 64 + 2) * size[a]).all()


@pytest.mark.parametrize("T", [2, 70, 260])
@pytest.mark.parametrize("masked", [False, True])
def test_what_is_not_a_number_stays_in_its_rows(psc, T, masked):  # noqa: F811
    rng = np.random.default_rng(T)
    V, K = 700, 400
    qc, wc = rng.integers(0, 16, (T, K), dtype=np.uint8), rng.integers(0, 16, (V, K), dtype=np.uint8)
    qe, we = np.full((T, 13), 127, dtype=np.uint8), np.full((V, 13), 127, dtype=np.uint8)
    qe[1, 12], we[5, 0], we[699, 3] = 255, 255, 255
    a = np.zeros((T, V), dtype=bool)
    a[:, ::7] = True
    a[:, 5], a[:, 699] = True, True
    sw = np.ones(V, dtype=np.float32)
    sw[14] = np.inf
    out = torch.empty(T, V, device="cuda")
    psc.psc_head_logits_mx4(*_matrix(psc, qc, qe, K, rows_fill=255), *_matrix(psc, wc, we, K, rows_fill=255), out, K,
                            w_scale=_dev(sw), bitmask=_pack(a) if masked else None)
    got = out.cpu().numpy()
    nan = np.zeros((T, V), dtype=bool)
    nan[1], nan[:, 5], nan[:, 699] = True, True, True
    see = a if masked else np.ones_like(a)
    x, w = ref.decode(qc, np.where(qe == 255, 0, qe)), ref.decode(wc, np.where(we == 255, 0, we))
    inf = np.zeros((T, V), dtype=bool)
    inf[:, 14] = (x @ w.T)[:, 14] != 0
    assert np.isnan(got[see & nan]).all()
    assert np.isfinite(got[see & ~nan & (sw == 1)[None]]).all()
    assert np.isinf(got[see & ~nan & inf]).all()
    if masked:
        assert (got[~a] == NEG).all()


def test_streams_and_graphs(psc):  # noqa: F811
    rng = np.random.default_rng(9)
    for T, V, K, mask in [(1, 3000, 512, None), (12, 3000, 512, "tight"), (90, 3000, 512, "mixed"), (400, 3000, 512, None)]:
        x, w = rng.standard_normal((T, K)).astype(np.float32), rng.standard_normal((V, K)).astype(np.float32)
        n = psc.psc_mx4_row_bytes(K)
        xd, wd = _dev(x), _dev(w)
        bm = None if mask is None else _pack(_mask(rng, mask, T, V))

        def buffers():
            return (torch.zeros(T, n, dtype=torch.uint8, device="cuda"), _blocks_of(psc, T, K),
                    torch.zeros(V, n, dtype=torch.uint8, device="cuda"), _blocks_of(psc, V, K),
                    torch.zeros(T, V, device="cuda"))

        def call(o, stream=None):
            # the weights are made by the kernel in front, so that nothing may be read before it is done
            psc.psc_quantize_mx4(xd, o[0], o[1], stream=stream)
            psc.psc_quantize_mx4(wd, o[2], o[3], stream=stream)
            psc.psc_head_logits_mx4(o[0], o[1], o[2], o[3], o[4], K, bitmask=bm, stream=stream)

        a, b, c = buffers(), buffers(), buffers()
        call(a)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        call(b, side)
        assert psc.psc_mx4_faults(stream=side) == 0
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(c)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a[4], b[4]) and torch.equal(a[4], c[4])
        xd.neg_()
        wd.mul_(4)
        graph.replay()
        call(a)
        torch.cuda.synchronize()
        assert torch.equal(a[4], c[4])
        for _ in range(20):                              # one after the other, no wait between
            call(b, side)
        side.synchronize()
        assert torch.equal(a[4], b[4])


def test_binding_without_its_module(psc, monkeypatch):  # noqa: F811
    """The same calls from Python alone, for tensors that are plainly in order and for others."""
    rng = np.random.default_rng(2)
    for T, V, K, pad in [(1, 300, 256, 0), (1, 300, 250, 8), (9, 300, 256, 8), (140, 200, 100, 0)]:
        x = _strided(rng.standard_normal((T, K)), torch.bfloat16, pad, 0)[1]
        w = _dev(rng.standard_normal((V, K)).astype(np.float32))
        n = psc.psc_mx4_row_bytes(K)
        bm = _pack(rng.random((T, V)) < 0.5)

        def run():
            q, b, s = torch.zeros(T, n + 16, dtype=torch.uint8, device="cuda"), _blocks_of(psc, T, K), torch.zeros(T, device="cuda")
            wq, wb = torch.zeros(V, n, dtype=torch.uint8, device="cuda"), _blocks_of(psc, V, K)
            h, y, out = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, K, device="cuda"), torch.zeros(T, V, device="cuda")
            q8, s8 = torch.zeros(T, K, dtype=torch.int8, device="cuda"), torch.zeros(T, device="cuda")
            psc.psc_quantize_mx4(w, wq, wb)
            psc.psc_norm_quantize_mx4(x, q, b, s, residual=x, sum_out=h)
            psc.psc_norm_quantize_rows(x, q8, s8, residual=x, sum_out=h)
            psc.psc_dequantize_mx4(q, b, y, scale=s)
            psc.psc_head_logits_mx4(q, b, wq, wb, out, K, scale=s, bitmask=bm)
            torch.cuda.synchronize()
            return wq, wb, q, b, s, h, y, out, q8, s8

        with monkeypatch.context() as m:
            m.setattr(psc, "_marshal", None)
            a = run()
        assert psc._marshal is not None
        for u, v in zip(a, run()):
            assert torch.equal(u, v)


@pytest.mark.parametrize("module", [True, False])
def test_tensors_of_another_device_are_refused(psc, monkeypatch, module):  # noqa: F811
    if not module:
        monkeypatch.setattr(psc, "_marshal", None)
    else:
        psc._load_marshal(psc.load(), lambda: 3)
    monkeypatch.setattr(psc, "_device", lambda: 3)
    x, q, s = torch.zeros(2, 64, device="cuda"), torch.zeros(2, 32, dtype=torch.uint8, device="cuda"), torch.zeros(2, device="cuda")
    b, q8, y = _blocks_of(psc, 2, 64), torch.zeros(2, 64, dtype=torch.int8, device="cuda"), torch.zeros(2, 2, device="cuda")
    try:
        for call in (lambda: psc.psc_norm_quantize_rows(x, q8, s), lambda: psc.psc_norm_quantize_mx4(x, q, b, s),
                     lambda: psc.psc_quantize_mx4(x, q, b), lambda: psc.psc_dequantize_mx4(q, b, x),
                     lambda: psc.psc_head_logits_mx4(q, b, q, b, y, 64)):
            with pytest.raises(ValueError, match="current device"):
                call()
    finally:
        psc._load_marshal(psc.load())


def test_values_back_where_the_factor_leaves_the_normal_numbers(psc):  # noqa: F811
    """code * 2^e * scale with 2^e * scale above the largest or below the smallest normal number: the power of two
    first, then one rounding of the product with the scale (and that to the type)."""
    rng = np.random.default_rng(4)
    for K in (64, 61):
        e = np.array([[0, 0], [1, 3], [252, 254], [254, 250], [10, 20], [127, 127], [255, 127], [130, 0]], dtype=np.uint8)
        scale = np.array([1.3, 1e-3, 2.0, 3e38, 1e-36, 0, 1, np.inf], dtype=np.float32)
        codes = rng.integers(0, 16, (8, K), dtype=np.uint8)
        q, blocks = _matrix(psc, codes, e, K)
        with np.errstate(over="ignore", invalid="ignore", under="ignore"):
            want = ref.decode(codes, e).astype(np.float32) * scale[:, None]
        for pad in (0, 3):
            _, y = _strided(np.zeros((8, K)), torch.float32, pad, 0)
            psc.psc_dequantize_mx4(q, blocks, y, scale=_dev(scale))
            np.testing.assert_array_equal(y.cpu().numpy(), want)
