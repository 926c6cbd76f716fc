"""The 4-bit operators and the norm on the CPU: the binding matches include/psc_mx4.h and
psc_norm.h, and wrong arguments are refused before anything is launched (the library's own
checks are reached with addresses that it must not use)."""
from __future__ import annotations

import os
import re

import pytest

from tests.test_library_cpu import ROOT, _c_type, psc  # noqa: F401
from tests.test_ops_binding import ARG, LIMIT, P

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("header,names", [("psc_mx4.h", "EXPORTED_MX4"), ("psc_norm.h", "EXPORTED_NORM")])
def test_binding_matches_the_header(psc, header, names):  # noqa: F811
    lib = psc.load()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    protos = re.findall(r"([A-Za-z_][\w ]*?\**)\s*\b(psc_\w+)\s*\(([^)]*)\)\s*;", text)
    assert sorted(p[1] for p in protos) == sorted(getattr(psc, names))
    import ctypes
    for ret, name, params in protos:
        f = getattr(lib, name)
        args = [p.strip() for p in params.split(",")]
        assert len(f.argtypes) == len(args), name
        for decl, t in zip(args, f.argtypes):
            if decl.startswith("float ") and "*" not in decl:
                assert t is ctypes.c_float, (name, decl)
                continue
            want = _c_type(decl.rsplit(" ", 1)[0] if "*" not in decl.split()[-1] else decl)
            assert t in want, (name, decl, t)
        assert f.restype in _c_type(ret), (name, ret, f.restype)


def _norm(op="rows", x=P, dtype=1, stride=64, res=None, res_stride=0, sum_=None, sum_stride=0, gain=None, eps=1e-6,
          T=4, K=64, q=P, q_stride=64, blocks=P, scale=P):
    head = (x, dtype, stride, res, res_stride, sum_, sum_stride, gain, eps, T, K, q, q_stride)
    if op == "rows":
        return "psc_norm_quantize_rows", head + (scale, None)
    return "psc_norm_quantize_mx4", head + (blocks, scale, None)


def _quantize(x=P, dtype=1, stride=64, T=4, K=64, q=P, q_stride=32, blocks=P):
    return "psc_quantize_mx4", (x, dtype, stride, T, K, q, q_stride, blocks, None)


def _dequantize(q=P, q_stride=32, blocks=P, scale=None, T=4, K=64, y=P, dtype=1, stride=64):
    return "psc_dequantize_mx4", (q, q_stride, blocks, scale, T, K, y, dtype, stride, None)


def _head(q=P, q_stride=32, qb=P, T=4, w=P, w_stride=32, wb=P, V=100, K=64, out=P, dtype=1, stride=100):
    return "psc_head_logits_mx4", (q, q_stride, qb, None, T, w, w_stride, wb, None, V, K, None, out, dtype, stride,
                                   None)


M = 2 ** 31 - 1


@pytest.mark.parametrize("call,code", [
    (_norm(op, **kw), code) for op in ("rows", "mx4") for kw, code in [
        (dict(x=None), ARG), (dict(q=None), ARG), (dict(scale=None), ARG), (dict(dtype=2), ARG), (dict(stride=63), ARG),
        (dict(q_stride=16), ARG), (dict(T=-1), ARG), (dict(K=0), ARG), (dict(res=P, res_stride=63), ARG),
        (dict(sum_=2 * P, sum_stride=63), ARG), (dict(sum_=P, sum_stride=80), ARG),
        (dict(res=2 * P, res_stride=64, sum_=2 * P, sum_stride=72), ARG), (dict(eps=-1e-9), ARG),
        (dict(x=P + 1), ARG), (dict(res=P + 1, res_stride=64), ARG), (dict(sum_=P + 3, sum_stride=64), ARG),
        (dict(gain=P + 2), ARG), (dict(scale=P + 1), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG),
        (dict(K=2 ** 30 + 1, stride=M, q_stride=M // 16 * 16), LIMIT)]
] + [
    (_norm("mx4", blocks=None), ARG), (_norm("mx4", q=P + 8), ARG), (_norm("mx4", q_stride=40), ARG),
    (_norm("mx4", blocks=P + 4), ARG),
    (_quantize(x=None), ARG), (_quantize(q=None), ARG), (_quantize(blocks=None), ARG), (_quantize(dtype=-1), ARG),
    (_quantize(stride=63), ARG), (_quantize(q_stride=16), ARG), (_quantize(q_stride=40), ARG), (_quantize(q=P + 4), ARG),
    (_quantize(blocks=P + 8), ARG), (_quantize(x=P + 1), ARG), (_quantize(x=P + 2, dtype=0), ARG),
    (_dequantize(y=P + 1), ARG), (_dequantize(scale=P + 2), ARG), (_head(out=P + 1), ARG), (_head(out=P + 2, dtype=0), ARG), (_quantize(T=-1), ARG), (_quantize(K=0), ARG), (_quantize(K=65, stride=65), ARG),
    (_quantize(K=M, stride=M, q_stride=2 ** 31), LIMIT),
    (_dequantize(q=None), ARG), (_dequantize(y=None), ARG), (_dequantize(blocks=None), ARG), (_dequantize(dtype=5), ARG),
    (_dequantize(stride=63), ARG), (_dequantize(q_stride=16), ARG), (_dequantize(q=P + 1), ARG),
    (_dequantize(T=-1), ARG), (_dequantize(K=-3), ARG), (_dequantize(K=M, stride=M, q_stride=2 ** 31), LIMIT),
    (_head(q=None), ARG), (_head(qb=None), ARG), (_head(w=None), ARG), (_head(wb=None), ARG), (_head(out=None), ARG),
    (_head(dtype=2), ARG), (_head(stride=99), ARG), (_head(T=-1), ARG), (_head(V=0), ARG), (_head(K=0), ARG),
    (_head(q=P + 8), ARG), (_head(q_stride=24), ARG), (_head(w=P + 8), ARG), (_head(w_stride=40), ARG),
    (_head(qb=P + 8), ARG), (_head(wb=P + 2), ARG),
    (("psc_mx4_faults", (None, 0, None)), ARG), (_head(K=131073, q_stride=65552, w_stride=65552), LIMIT), (_head(T=2 ** 24 + 1), LIMIT),
    (_head(V=2 ** 30 + 1, stride=M), LIMIT),
])
def test_wrong_arguments_are_refused(psc, call, code):  # noqa: F811
    name, args = call
    assert getattr(psc.load(), name)(*args) == code
    assert name in psc.load().psc_last_error().decode()


@pytest.mark.parametrize("call", [_norm("rows", x=None, q=None, scale=None, T=0), _norm("mx4", x=None, scale=None, T=0),
                                  _quantize(x=None, T=0), _dequantize(y=None, T=0),
                                  _head(q=None, qb=None, out=None, T=0)])
def test_empty_batches_are_nothing_to_do(psc, call):  # noqa: F811
    name, args = call
    assert getattr(psc.load(), name)(*args) == 0


def test_sizes(psc):  # noqa: F811
    for rows, K, n in [(1, 1, 512), (128, 128, 512), (129, 128, 1024), (128, 129, 1024), (300, 1000, 3 * 8 * 512),
                       (M, 2 ** 30, 2 ** 24 * 2 ** 23 * 512), (0, 5, 0), (5, 0, 0), (-1, 5, 0), (5, 2 ** 30 + 1, 0)]:
        assert psc.psc_mx4_block_bytes(rows, K) == n
    assert [psc.psc_mx4_row_bytes(k) for k in (1, 32, 33, 2048)] == [16, 16, 32, 1024]


def test_binding_refuses_tensors_of_the_wrong_kind(psc):  # noqa: F811
    x, s = torch.zeros(4, 100), torch.zeros(4)
    q, b = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        psc.psc_quantize_mx4(x, q, b)
    with pytest.raises(ValueError, match="2-D"):
        psc.psc_quantize_mx4(s, q, b)
    with pytest.raises(ValueError, match="bf16 or f32"):
        psc.psc_quantize_mx4(x.half(), q, b)
    with pytest.raises(ValueError, match="unit column stride"):
        psc.psc_dequantize_mx4(q, b, x.t())
    with pytest.raises(ValueError, match="bf16 or f32"):
        psc.psc_dequantize_mx4(q, b, x.double())
    with pytest.raises(ValueError, match="2-D"):
        psc.psc_norm_quantize_rows(s, q, s)
    with pytest.raises(ValueError, match="CUDA"):
        psc.psc_norm_quantize_mx4(x, q, b, s)
    with pytest.raises(ValueError, match="2-D"):
        psc.psc_head_logits_mx4(s, b, q, b, x, 100)


def test_the_formats_values_by_hand():
    """The reference of the GPU tests against the format's own table."""
    from tests._mx4_ref import decode, quantize
    import numpy as np
    x = np.zeros((1, 33), dtype=np.float32)
    x[0, :12] = [6, -0.5, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.2, 4.99, -7.9]      # the largest in [4, 8): e = 0
    x[0, 32] = -1e-3
    codes, e = quantize(x)
    assert e.tolist() == [[127, 127 - 12]]      # 1e-3 lies in 2^-10 (1, 2)
    assert codes[0, :12].tolist() == [7, 9, 0, 2, 2, 4, 4, 6, 6, 8, 6, 15]
    assert codes[0, 32] == 8 + 6                # 1e-3 * 2^12 = 4.096
    assert decode(codes, e)[0, :12].tolist() == [6, -0.5, 0, 1, 1, 2, 2, 4, 4, 0, 4, -6]


class _Tensor:
    """As much of a CUDA tensor as the binding asks for; of an empty batch, so that nothing is launched."""

    def __init__(self, *shape, dtype, device=0):
        self.shape, self.dtype, self.device, self.is_cuda = shape, dtype, device, True

    def stride(self):
        return self.shape[1:] + (1,)

    def dim(self):
        return len(self.shape)

    def data_ptr(self):
        return P

    def numel(self):
        return self.shape[0] * (self.shape[1] if len(self.shape) > 1 else 1)

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device


def _calls(psc):  # noqa: F811
    """Each entry with the tensors it takes, over no rows."""
    f32, u8 = torch.float32, torch.uint8
    x = lambda: _Tensor(0, 64, dtype=f32)  # noqa: E731
    v = lambda n: _Tensor(n, dtype=f32)  # noqa: E731
    q, b = (lambda n: _Tensor(n, 32, dtype=u8)), (lambda n: _Tensor(n, dtype=u8))
    return [(psc.psc_norm_quantize_rows, dict(x=x(), q=_Tensor(0, 64, dtype=torch.int8), scale=v(0), gain=v(64),
                                              residual=x(), sum_out=x())),
            (psc.psc_norm_quantize_mx4, dict(x=x(), q=q(0), blocks=b(0), scale=v(0), gain=v(64), residual=x(), sum_out=x())),
            (psc.psc_quantize_mx4, dict(x=x(), q=q(0), blocks=b(0))),
            (psc.psc_dequantize_mx4, dict(q=q(0), blocks=b(0), y=x(), scale=v(0))),
            (psc.psc_head_logits_mx4, dict(q=q(0), q_blocks=b(0), w=q(100), w_blocks=b(512), logits=_Tensor(0, 100, dtype=f32),
                                           K=64, scale=v(0), w_scale=v(100), bitmask=_Tensor(0, 4, dtype=torch.int32)))]


@pytest.mark.parametrize("marshal", [True, False])
def test_tensors_of_another_device_are_refused(psc, monkeypatch, marshal):  # noqa: F811
    """Every tensor of a call has to be on the current device (here the binding's idea of it), with the calls taken
    apart in C and in Python."""
    lib = psc.load()
    monkeypatch.setattr(psc, "_device", lambda: 1)
    if marshal:
        psc._load_marshal(lib, lambda: 1)
        if psc._marshal is None:
            pytest.skip("the module is not built here")
    else:
        monkeypatch.setattr(psc, "_marshal", None)
    try:
        for entry, tensors in _calls(psc):
            for t in tensors.values():
                if isinstance(t, _Tensor):
                    t.device = 1
            entry(**tensors, stream=0)
            for name, t in tensors.items():
                if not isinstance(t, _Tensor):
                    continue
                t.device = 0
                with pytest.raises(ValueError, match=f"{name} is on cuda:0"):
                    entry(**tensors, stream=0)
                t.device = 1
    finally:
        if marshal:
            psc._load_marshal(lib)


@pytest.mark.parametrize("limit,kw,code", [(-1, {}, ARG), (2 ** 22 + 1, {}, ARG), (5, dict(w=None), ARG), (5, dict(q=P + 8), ARG),
                                           (5, dict(dtype=1), ARG), (5, dict(dtype=2), ARG), (5, dict(T=2 ** 24 + 1), LIMIT),
                                           (0, dict(q=None, qb=None, out=None, T=0), 0)])
def test_the_self_test_of_waits_has_the_projections_checks(psc, limit, kw, code):  # noqa: F811
    args = _head(**{"dtype": 0, **kw})[1]
    assert psc.load().psc_mx4_check_wait(*args[:-1], limit, None) == code
    if code:
        assert "psc_mx4_check_wait" in psc.load().psc_last_error().decode()
