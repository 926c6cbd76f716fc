"""The operators around the mask on the CPU: the binding matches include/psc_ops.h,
and wrong arguments are refused before anything is launched (the library's own
checks are reached with addresses that it must not use)."""
from __future__ import annotations

import os
import re

import pytest

from tests.test_library_cpu import ROOT, _c_type, psc  # noqa: F401

torch = pytest.importorskip("torch")


def test_binding_matches_the_operators_header(psc):  # noqa: F811
    lib = psc.load()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "psc_ops.h")).read(), flags=re.S)
    protos = re.findall(r"([A-Za-z_][\w ]*?\**)\s*\b(psc_[a-z_]+)\s*\(([^)]*)\)\s*;", text)
    assert sorted(p[1] for p in protos) == sorted(psc.EXPORTED_OPS)
    for ret, name, params in protos:
        f = getattr(lib, name)
        args = [p.strip() for p in params.split(",")]
        assert len(f.argtypes) == len(args), name
        for decl, t in zip(args, f.argtypes):
            want = _c_type(decl.rsplit(" ", 1)[0] if "*" not in decl.split()[-1] else decl)
            assert t in want, (name, decl, t)
        assert f.restype in _c_type(ret), (name, ret, f.restype)


P = 1 << 20      # an address that no refused call reads


def _quantize(x=P, dtype=1, stride=64, T=4, K=64, q=P, q_stride=64, scale=P):
    return "psc_quantize_rows", (x, dtype, stride, T, K, q, q_stride, scale, None)


def _head(q=P, q_stride=64, scale=P, T=4, w=P, w_stride=64, w_scale=P, V=100, K=64, mask=None, out=P, dtype=1,
          stride=100, work=P, n=1 << 30):
    return "psc_head_logits", (q, q_stride, scale, T, w, w_stride, w_scale, V, K, mask, out, dtype, stride, work, n,
                               None)


def _process(logits=P, dtype=1, stride=100, out=P, out_stride=100, B=4, V=100, hist=None, hist_stride=0, H=0,
             ids=None, bias=None, n=0):
    return "psc_process_logits", (logits, dtype, stride, out, out_stride, B, V, hist, hist_stride, H, None, None,
                                  None, None, None, ids, bias, n, None, None)


def _sample(logits=P, dtype=1, stride=100, B=4, V=100, u=P, tokens=P, work=P, n=16):
    return "psc_sample", (logits, dtype, stride, B, V, None, u, None, None, None, None, tokens, None, work, n, None)


ARG, LIMIT = 1, 5


@pytest.mark.parametrize("call,code", [
    (_quantize(x=None), ARG), (_quantize(q=None), ARG), (_quantize(scale=None), ARG), (_quantize(dtype=2), ARG),
    (_quantize(stride=63), ARG), (_quantize(q_stride=63), ARG), (_quantize(T=-1), ARG), (_quantize(K=0), ARG),
    (_head(q=None), ARG), (_head(scale=None), ARG), (_head(w=None), ARG), (_head(w_scale=None), ARG),
    (_head(out=None), ARG), (_head(q_stride=63), ARG), (_head(w_stride=63), ARG), (_head(stride=99), ARG),
    (_head(dtype=-1), ARG), (_head(T=-1), ARG), (_head(V=0), ARG), (_head(K=0), ARG), (_head(work=None), ARG),
    (_head(work=P + 16), ARG), (_head(n=0), ARG),
    (_head(K=131073, q_stride=131088, w_stride=131088), LIMIT),
    (_process(logits=None), ARG), (_process(out=None), ARG), (_process(dtype=7), ARG), (_process(stride=99), ARG),
    (_process(out_stride=99, out=P * 2), ARG), (_process(out_stride=101), ARG), (_process(B=-1), ARG),
    (_process(V=0), ARG), (_process(H=-1), ARG), (_process(H=3), ARG), (_process(hist=P, H=3, hist_stride=2), ARG),
    (_process(n=2), ARG), (_process(n=2, ids=P), ARG), (_process(n=-1), ARG),
    (_process(out=P + 50), ARG), (_process(out=P + 198, stride=198, out_stride=198), ARG),
    (_process(hist=P, H=1 << 24, hist_stride=1 << 24), LIMIT), (_process(n=4097, ids=P, bias=P), LIMIT),
    (_sample(logits=None), ARG), (_sample(u=None), ARG), (_sample(tokens=None), ARG), (_sample(dtype=3), ARG),
    (_sample(stride=99), ARG), (_sample(B=48, work=None), ARG), (_sample(B=49, n=63), ARG), (_sample(B=-1), ARG), (_sample(V=0), ARG), (_sample(V=(1 << 22) + 1, stride=1 << 23), LIMIT),
])
def test_wrong_arguments_are_refused(psc, call, code):  # noqa: F811
    name, args = call
    assert getattr(psc.load(), name)(*args) == code
    assert name in psc.load().psc_last_error().decode()


@pytest.mark.parametrize("call", [_quantize(x=None, q=None, scale=None, T=0), _head(q=None, scale=None, out=None, T=0),
                                  _process(logits=None, out=None, B=0), _sample(logits=None, u=None, tokens=None, B=0)])
def test_empty_batches_are_nothing_to_do(psc, call):  # noqa: F811
    name, args = call
    assert getattr(psc.load(), name)(*args) == 0


def test_binding_refuses_tensors_of_the_wrong_kind(psc):  # noqa: F811
    x, u, t = torch.zeros(4, 100), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        psc.psc_sample(x, u, t)
    with pytest.raises(ValueError, match="bf16 or f32"):
        psc.psc_sample(x.half(), u, t)
    with pytest.raises(ValueError, match="unit column stride"):
        psc.psc_sample(x.t(), u, t)
    with pytest.raises(ValueError, match=">=101"):
        psc.psc_process_logits(x, V=101)
    with pytest.raises(ValueError, match="2-D"):
        psc.psc_process_logits(x[0])
    with pytest.raises(ValueError):
        psc.psc_process_logits(x, bias_ids=t[:, None])
    q = torch.zeros(4, 64, dtype=torch.int8)
    with pytest.raises(ValueError, match=r"\[T, K\]"):
        psc.psc_head_logits(q, u, q[:, :63], u, x)
    with pytest.raises(ValueError, match="2-D"):
        psc.psc_quantize_rows(u, q, u)
