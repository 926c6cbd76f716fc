"""The operators' binding and C entries on the CPU at the ends of their ranges."""
from __future__ import annotations

import pytest

from tests.test_library_cpu import psc  # noqa: F401

from tests.test_ops_binding import LIMIT, _head, _quantize

torch = pytest.importorskip("torch")


def test_head_faults_refuses_what_is_no_workspace(psc):  # noqa: F811
    with pytest.raises(ValueError, match="work"):
        psc.psc_head_faults(torch.zeros(3, dtype=torch.uint8))
    with pytest.raises(ValueError, match="CUDA"):
        psc.psc_head_faults(torch.zeros(256, dtype=torch.uint8))


M = 2 ** 31 - 1


@pytest.mark.parametrize("call", [_head(V=M, stride=M), _head(V=M - 31, stride=M), _head(V=M - 127, stride=M, T=1),
                                  _head(V=2 ** 30 + 1, stride=M), _head(T=M), _head(T=2 ** 24 + 1),
                                  _head(T=2 ** 24, V=2 ** 30, stride=M), _quantize(K=M, stride=M, q_stride=M),
                                  _quantize(K=2 ** 30 + 1, stride=M, q_stride=M)])
def test_sizes_that_indexes_cannot_hold_are_refused(psc, call):  # noqa: F811
    name, args = call
    assert getattr(psc.load(), name)(*args) == LIMIT
    assert name in psc.load().psc_last_error().decode()


def test_workspaces_of_sizes_at_the_limits(psc):  # noqa: F811
    for T, V, K in [(M, 100, 64), (4, M, 64), (4, 100, M), (2 ** 24 + 1, 1, 1), (1, 2 ** 30 + 1, 1), (1, 1, 131073)]:
        for aligned in (True, False):
            assert psc.psc_head_work_bytes(T, V, K, aligned) == 256
    for T, V, K in [(2 ** 24, 1, 131072), (1, 2 ** 30, 131072), (1, 1, 131072)]:
        tokens = T * K * 2
        assert tokens <= psc.psc_head_work_bytes(T, V, K) < psc.psc_head_work_bytes(T, V, K, False)
