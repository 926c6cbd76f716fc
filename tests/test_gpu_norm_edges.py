"""The norms where rows are read a second time, against numpy in 64 bits.  Reference forms and tolerances are those
of test_gpu_norm."""
from __future__ import annotations

import numpy as np
import pytest

from tests import _mx4_ref as ref
from tests.test_gpu_norm import _data, _int8, _tolerance
from tests.test_gpu_ops import DT, U, _dev, _f64, psc  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [1001, 1003, 250])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("out", ["new", "x", "residual"])
def test_sums_read_again_by_blocks_of_one_warp(psc, K, dtype, out):  # noqa: F811
    """Many rows of up to 1024 columns that start anywhere: a warp a row, whose lanes store the ends of each other's sums
    and read them again in rows whose squares leave f32, and in rows of zeros."""
    T = 1300
    rng = np.random.default_rng([K, T])
    x, res = _data(rng, T, K, dtype), _data(rng, T, K, dtype)
    x[::5], res[::5] = 0, 0
    for start, size in ((1, 1e28), (2, 1e-28)):
        for a in (x, res):
            scaled = (a[start::5] * np.float32(size)).astype(np.float32)
            a[start::5] = ref.round_bf16(scaled) if dtype == "bf16" else scaled
    g = (rng.uniform(0.5, 1.5, K) * rng.choice([-1, 1], K)).astype(np.float32)
    with np.errstate(divide="ignore"):
        h, v, r = ref.norm(x, res, g, 0.0, dtype == "bf16")
    r = np.where((h == 0).all(1), 0, r)                     # a row of zeros has the factor 0
    codes, e = ref.quantize(v)
    n = psc.psc_mx4_row_bytes(K)

    def inputs():
        xd, rd = _dev(x).to(DT[dtype]), _dev(res).to(DT[dtype])
        return xd, rd, {"new": torch.full((T, K), 7.0, dtype=DT[dtype], device="cuda"), "x": xd, "residual": rd}[out]

    xd, rd, sd = inputs()
    q, s = torch.zeros(T, n, dtype=torch.uint8, device="cuda"), torch.full((T,), 7.0, device="cuda")
    b = torch.full((psc.psc_mx4_block_bytes(T, K),), 5, dtype=torch.uint8, device="cuda")
    psc.psc_norm_quantize_mx4(xd, q, b, s, gain=_dev(g), eps=0.0, residual=rd, sum_out=sd)
    np.testing.assert_array_equal(_f64(sd), h)
    np.testing.assert_array_equal(q.cpu().numpy(), ref.pack(codes))
    np.testing.assert_array_equal(b.cpu().numpy(), ref.tiles(e, K, 5))
    np.testing.assert_allclose(_f64(s), r, rtol=_tolerance(K), atol=0)

    xd, rd, sd = inputs()
    q = torch.zeros(T, K, dtype=torch.int8, device="cuda")
    psc.psc_norm_quantize_rows(xd, q, s, gain=_dev(g), eps=0.0, residual=rd, sum_out=sd)
    want, scale = _int8(v, r)
    np.testing.assert_array_equal(_f64(sd), h)
    np.testing.assert_array_equal(q.cpu().numpy(), want)
    np.testing.assert_allclose(_f64(s), scale, rtol=_tolerance(K) + U, atol=0)


@pytest.mark.parametrize("K", [1, 64, 1001, 4096])
@pytest.mark.parametrize("T", [2, 3000])
def test_eps_up_to_the_largest_number(psc, K, T):  # noqa: F811
    """mean h^2 + eps beyond f32, for squares that are not: the root of it is a number, and so is its inverse."""
    x = np.full((T, K), 9e18 / np.sqrt(K), dtype=np.float32)          # squares of 8.1e37 in all, below 2^126
    x[1::2] *= np.float32(1e-3)
    xd, n = _dev(x), psc.psc_mx4_row_bytes(K)
    q, s = torch.empty(T, K, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    c, b = torch.empty(T, n, dtype=torch.uint8, device="cuda"), torch.empty(psc.psc_mx4_block_bytes(T, K), dtype=torch.uint8,
                                                                            device="cuda")
    for eps in (1e30, 2.0 ** 125, 2.0 ** 126, 2.0 ** 127, float(np.finfo(np.float32).max)):
        h, v, r = ref.norm(x, None, None, eps, False)
        psc.psc_norm_quantize_rows(xd, q, s, eps=eps)
        want, scale = _int8(v, r)
        np.testing.assert_array_equal(q.cpu().numpy(), want)
        np.testing.assert_allclose(_f64(s), scale, rtol=_tolerance(K) + U, atol=0)
        psc.psc_norm_quantize_mx4(xd, c, b, s, eps=eps)
        np.testing.assert_allclose(_f64(s), r, rtol=_tolerance(K), atol=0)


@pytest.mark.parametrize("T,K", [(5, 1024), (3000, 1024), (7, 2048), (1500, 2048), (400, 8192)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_do_not_depend_on_how_the_other_tensors_lie(psc, T, K, dtype):  # noqa: F811
    """Rows of x at aligned addresses: gain, codes, residual and sum may lie anywhere, and every result has the same bits."""
    rng = np.random.default_rng([T, K])
    x, res = _dev(_data(rng, T, K, dtype)).to(DT[dtype]), _dev(_data(rng, T, K, dtype)).to(DT[dtype])
    g = _dev(rng.uniform(0.5, 1.5, K).astype(np.float32))

    def moved(t, by):
        """The same values, `by` elements off in rows of 8 + by elements more."""
        if t.dim() == 1:
            out = torch.empty(K + by, dtype=t.dtype, device="cuda")[by:]
        else:
            out = torch.empty(T, K + 8 + by, dtype=t.dtype, device="cuda")[:, by:by + K]
        out.copy_(t)
        return out

    def run(gain=g, residual=res, pad=0, sum_by=0):
        big = torch.zeros(T, K + pad, dtype=torch.int8, device="cuda")
        h = moved(res, sum_by) if sum_by else torch.empty_like(res)
        s = torch.empty(T, device="cuda")
        psc.psc_norm_quantize_rows(x, big[:, :K], s, gain=gain, residual=residual, sum_out=h)
        q4 = torch.zeros(T, psc.psc_mx4_row_bytes(K), dtype=torch.uint8, device="cuda")
        b, s4 = torch.zeros(psc.psc_mx4_block_bytes(T, K), dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")
        psc.psc_norm_quantize_mx4(x, q4, b, s4, gain=gain, residual=residual)
        return big[:, :K], s, h, q4, b, s4

    want = run()
    for other in (run(gain=moved(g, 1)), run(pad=4), run(residual=moved(res, 3)), run(sum_by=1), run(pad=5, sum_by=2)):
        for u, v in zip(want, other):
            assert torch.equal(u, v)


@pytest.mark.parametrize("T", [3, 140])
@pytest.mark.parametrize("power", [-106, -60, 0, 60, 112])
def test_norm_and_projection_in_4_bits_over_the_range_of_rows(psc, T, power):  # noqa: F811
    """The codes hold h * gain as it is, so that its size goes through the projection's sums: those of magnitudes lie
    between 2^-100 and 2^127 here, as the header asks for.  Tolerances as in test_gpu_mx4, and the factor's."""
    rng = np.random.default_rng([T, power + 200])
    V, K = 500, 512
    x = np.ldexp(rng.uniform(0.5, 1, (T, K)) * rng.choice([-1, 1], (T, K)), power).astype(np.float32)
    w = (rng.uniform(0.5, 4, (V, K)) * rng.choice([-1, 1], (V, K))).astype(np.float32)
    h, v, r = ref.norm(x, None, None, 0.0, False)
    n = psc.psc_mx4_row_bytes(K)
    q, b = torch.empty(T, n, dtype=torch.uint8, device="cuda"), torch.empty(psc.psc_mx4_block_bytes(T, K), dtype=torch.uint8,
                                                                            device="cuda")
    wq, wb = torch.empty(V, n, dtype=torch.uint8, device="cuda"), torch.empty(psc.psc_mx4_block_bytes(V, K), dtype=torch.uint8,
                                                                              device="cuda")
    s, out = torch.empty(T, device="cuda"), torch.empty(T, V, device="cuda")
    psc.psc_quantize_mx4(_dev(w), wq, wb)
    psc.psc_norm_quantize_mx4(_dev(x), q, b, s, eps=0.0)
    psc.psc_head_logits_mx4(q, b, wq, wb, out, K, scale=s)
    y, m = ref.decode(*ref.quantize(v)), ref.decode(*ref.quantize(w))
    sums = np.abs(y) @ np.abs(m).T
    assert 2.0 ** -100 < sums.min() and sums.max() < 2.0 ** 127
    exact = y @ m.T * r[:, None]
    tol = 4 * U * (K / 64 + 2) * sums * r[:, None] + (_tolerance(K) + 2 * U) * np.abs(exact)
    assert (np.abs(_f64(out) - exact) <= tol * 1.0000001).all()


def test_the_factor_of_tiny_rows(psc):  # noqa: F811
    """Beyond f32 only with eps 0 and a root mean square of 2^-128 or less; any eps that is a number of f32 keeps it finite."""
    x = np.zeros((4, 64), dtype=np.float32)
    x[0], x[1], x[2] = 1e-42, 2.0 ** -127, 2.0 ** -129
    n = psc.psc_mx4_row_bytes(64)
    q, b = torch.empty(4, n, dtype=torch.uint8, device="cuda"), torch.empty(512, dtype=torch.uint8, device="cuda")
    for eps in (0.0, 2.0 ** -149, 1e-12):
        psc.psc_norm_quantize_mx4(_dev(x), q, b, s := torch.empty(4, device="cuda"), eps=eps)
        with np.errstate(divide="ignore"):
            r = ref.norm(x, None, None, eps, False)[2]
        r[r > 3.5e38] = np.inf
        if eps == 0:
            r[3] = 0
            assert np.isinf(r).tolist() == [True, False, True, False]
        np.testing.assert_allclose(_f64(s), r, rtol=_tolerance(64), atol=0)
