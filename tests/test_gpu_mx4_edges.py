"""The norms and the 4-bit operators where a batch, a vocabulary or a capture is unusual: offsets beyond 32 bits,
logits that start between aligned addresses, captures without a call before, calls at the same time.
Reference forms and tolerances are those of test_gpu_mx4 and test_gpu_norm."""
from __future__ import annotations

import os
import subprocess
import sys

import numpy as np
import pytest

from tests import _mx4_ref as ref
from tests.test_gpu_mx4 import _blocks_of, _matrix
from tests.test_gpu_ops import DT, NEG, U, UB, _dev, _f64, _mask, _pack, psc  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("T,V", [(1, 170_000_001), (12, 200_000_000), (130, 17_000_000)])
@pytest.mark.parametrize("masked", [False, True])
def test_head_beyond_32_bits(psc, T, V, masked):  # noqa: F811
    """More than 2^32 bytes of logits, or more tiles than a block looks at masks of beforehand."""
    K = 32
    rng = np.random.default_rng([T, V])
    g = torch.Generator(device="cuda").manual_seed(V)
    w = torch.randint(0, 256, (V, 16), dtype=torch.uint8, device="cuda", generator=g)
    wb = torch.randint(120, 130, (psc.psc_mx4_block_bytes(V, K),), dtype=torch.uint8, device="cuda", generator=g)
    wb.view(-1, 32, 4, 4)[:, :, :, 1:] = 0                 # past K
    qc, qe = rng.integers(0, 16, (T, K), dtype=np.uint8), np.full((T, 1), 127, dtype=np.uint8)
    out = torch.full((T, V), 7.0, dtype=torch.bfloat16, device="cuda")
    bm = torch.randint(-2 ** 31, 2 ** 31, (T, (V + 31) // 32), dtype=torch.int32, device="cuda", generator=g) if masked else None
    psc.psc_head_logits_mx4(*_matrix(psc, qc, qe, K), w, wb, out, K, bitmask=bm)
    assert psc.psc_mx4_faults() == 0
    x = ref.decode(qc, qe)
    for lo in (0, V // 2 // 128 * 128, V - 4000):
        v = np.arange(lo, min(V, lo + 4000))
        packed = w[lo:lo + 4000].cpu().numpy()
        codes = np.stack((packed & 15, packed >> 4), -1).reshape(len(v), K)
        at = torch.from_numpy(512 * (v // 128) + 16 * (v % 32) + 4 * (v % 128 // 32)).cuda()
        e = wb[at].cpu().numpy()[:, None]
        exact = x @ ref.decode(codes, e).T
        size = np.abs(x) @ np.abs(ref.decode(codes, e)).T
        got = _f64(out[:, lo:lo + 4000])
        tol = 4 * U * 3 * size + UB * np.abs(exact)
        allowed = np.ones_like(got, dtype=bool)
        if masked:
            words = bm[:, torch.from_numpy(v // 32).cuda()].cpu().numpy().view(np.uint32)
            allowed = (words >> (v % 32).astype(np.uint32)[None]) & 1 == 1
            assert (got[~allowed] == NEG).all()
        assert (np.abs(got - exact) <= tol)[allowed].all()


def test_norm_and_format_beyond_32_bits(psc):  # noqa: F811
    T, K = 70_000, 65_544                                  # 9.2 GB of bf16
    x = torch.empty(T, K, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, T, 10_000):
        x[lo:lo + 10_000].normal_()
    q, s = torch.empty(T, K, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    psc.psc_norm_quantize_rows(x, q, s)
    q4, b4 = torch.empty(T, psc.psc_mx4_row_bytes(K), dtype=torch.uint8, device="cuda"), _blocks_of(psc, T, K)
    psc.psc_quantize_mx4(x, q4, b4)
    rows = [0, 1, 40_000, T - 1]
    h, v, r = ref.norm(x[rows].float().cpu().numpy(), None, None, 1e-6, True)
    unit = np.abs(v).max(1) * (np.float32(1) / np.float32(127))
    np.testing.assert_array_equal(q[rows].cpu().numpy(), np.rint((v / unit[:, None]).astype(np.float32)))
    np.testing.assert_allclose(_f64(s[rows]), unit.astype(np.float64) * r, rtol=((8 * 9 + 12 + 2) / 2 + 4) * U)
    codes, e = ref.quantize(v)
    np.testing.assert_array_equal(q4[rows].cpu().numpy(), ref.pack(codes))
    x.zero_()
    psc.psc_dequantize_mx4(q4, b4, x)
    np.testing.assert_array_equal(_f64(x[rows]), ref.decode(codes, e))


@pytest.mark.parametrize("T,V,K", [(3, 700, 64), (40, 515, 200), (140, 700, 96), (300, 1000, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift,pad", [(1, 0), (2, 2), (4, 4), (8, 8), (3, 5)])
def test_logits_between_aligned_addresses(psc, T, V, K, dtype, shift, pad):  # noqa: F811
    rng = np.random.default_rng([T, V, shift])
    qc, wc = rng.integers(0, 16, (T, K), dtype=np.uint8), rng.integers(0, 16, (V, K), dtype=np.uint8)
    nb = (K + 31) // 32
    qe, we = np.full((T, nb), 126, dtype=np.uint8), rng.integers(124, 128, (V, nb)).astype(np.uint8)
    allowed = _mask(rng, "mixed", T, V)
    exact = ref.decode(qc, qe) @ ref.decode(wc, we).T
    size = np.abs(ref.decode(qc, qe)) @ np.abs(ref.decode(wc, we)).T
    tol = 4 * U * (K / 64 + 2) * size + (UB if dtype == "bf16" else 0) * np.abs(exact)
    for mask in (None, allowed):
        big = torch.full((T, V + shift + pad), 7.0, dtype=DT[dtype], device="cuda")
        psc.psc_head_logits_mx4(*_matrix(psc, qc, qe, K), *_matrix(psc, wc, we, K), big[:, shift:shift + V], K,
                                bitmask=None if mask is None else _pack(mask))
        assert (big[:, :shift] == 7).all() and (big[:, shift + V:] == 7).all()
        got = _f64(big[:, shift:shift + V])
        a = np.ones_like(allowed) if mask is None else mask
        assert (got[~a] == NEG).all()
        assert (np.abs(got - exact) <= tol)[a].all()


CAPTURE = """
import sys, torch
sys.path.insert(0, {root!r})
from paper_2608_03065_gb300 import psc
psc.load()
K, V = 512, 2000
for T, masked in ((2, True), (2, False), (300, True), (20000, False)):
    n = psc.psc_mx4_row_bytes(K)
    x, w = torch.randn(T, K, device="cuda").bfloat16(), torch.randn(V, K, device="cuda")
    q, b, s = torch.zeros(T, n, dtype=torch.uint8, device="cuda"), torch.zeros(psc.psc_mx4_block_bytes(T, K), dtype=torch.uint8, device="cuda"), torch.zeros(T, device="cuda")
    wq, wb = torch.zeros(V, n, dtype=torch.uint8, device="cuda"), torch.zeros(psc.psc_mx4_block_bytes(V, K), dtype=torch.uint8, device="cuda")
    y, h, q8, s8 = torch.zeros(T, K, device="cuda"), torch.zeros_like(x), torch.zeros(T, K, dtype=torch.int8, device="cuda"), torch.zeros(T, device="cuda")
    out = torch.zeros(min(T, 300), V, device="cuda")
    bm = torch.randint(-2 ** 31, 2 ** 31, (min(T, 300), (V + 31) // 32), dtype=torch.int32, device="cuda") if masked else None

    def step():
        psc.psc_quantize_mx4(w, wq, wb)
        psc.psc_norm_quantize_mx4(x, q, b, s, residual=x, sum_out=h)
        psc.psc_norm_quantize_rows(x, q8, s8, residual=x, sum_out=h)
        psc.psc_dequantize_mx4(q, b, y, scale=s)
        psc.psc_head_logits_mx4(q[:300], b, wq, wb, out, K, scale=s, bitmask=bm)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    g.replay()
    torch.cuda.synchronize()
    first = [t.clone() for t in (wq, wb, q, b, s, y, h, q8, s8, out)]
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(first, (wq, wb, q, b, s, y, h, q8, s8, out)))
    assert out.abs().sum() > 0 and psc.psc_mx4_faults() == 0
print("same")
"""


def test_captures_without_a_call_before(psc):  # noqa: F811
    """In a process of its own, where no kernel has run: the first calls are captured."""
    r = subprocess.run([sys.executable, "-c", CAPTURE.format(root=ROOT)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("T", [5, 100, 400])
def test_calls_at_the_same_time(psc, T):  # noqa: F811
    """Two streams, each with its own buffers, and threads that call at once: the results of one call after the other."""
    import threading
    rng = np.random.default_rng(T)
    V, K = 6000, 384
    n = psc.psc_mx4_row_bytes(K)
    xs = [_dev(rng.standard_normal((T, K)).astype(np.float32)) for _ in range(4)]
    wc, we = ref.quantize(rng.standard_normal((V, K)).astype(np.float32))
    w = _matrix(psc, wc, we, K)
    bm = _pack(_mask(rng, "mixed", T, V))
    bufs = [(torch.zeros(T, n, dtype=torch.uint8, device="cuda"), _blocks_of(psc, T, K), torch.zeros(T, device="cuda"),
             torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")) for _ in range(4)]
    streams = [torch.cuda.Stream() for _ in range(4)]

    def call(i, stream=None):
        q, b, s, out = bufs[i]
        psc.psc_norm_quantize_mx4(xs[i], q, b, s, stream=stream)
        psc.psc_head_logits_mx4(q, b, *w, out, K, scale=s, bitmask=bm, stream=stream)

    want = []
    for i in range(4):
        call(i)
        torch.cuda.synchronize()
        want.append(bufs[i][3].clone())
        bufs[i][3].zero_()
    torch.cuda.synchronize()
    threads = [threading.Thread(target=lambda i=i: [call(i, streams[i]) for _ in range(25)]) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(4):
        assert torch.equal(bufs[i][3], want[i])
    assert psc.psc_mx4_faults() == 0


def test_the_same_tensor_in_several_places(psc):  # noqa: F811
    """x as its own residual, the sum in its place; tokens and weights one matrix."""
    rng = np.random.default_rng(8)
    for T, K in [(7, 96), (200, 1000), (5000, 1024)]:
        x = ref.round_bf16(rng.standard_normal((T, K)).astype(np.float32))
        xd = _dev(x).bfloat16()
        q, s = torch.empty(T, K, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        psc.psc_norm_quantize_rows(xd, q, s, residual=xd, sum_out=xd)
        h, v, r = ref.norm(x, x, None, 1e-6, True)
        np.testing.assert_array_equal(_f64(xd), h)
        unit = np.abs(v).max(1) * (np.float32(1) / np.float32(127))
        np.testing.assert_array_equal(q.cpu().numpy(), np.rint((v / unit[:, None]).astype(np.float32)))
    for T in (50, 300):
        c, e = ref.quantize(rng.standard_normal((T, 256)).astype(np.float32))
        m, out = _matrix(psc, c, e, 256), torch.empty(T, T, device="cuda")
        psc.psc_head_logits_mx4(*m, *m, out, 256)
        y = ref.decode(c, e)
        assert (np.abs(_f64(out) - y @ y.T) <= 4 * U * 6 * (np.abs(y) @ np.abs(y).T)).all()
