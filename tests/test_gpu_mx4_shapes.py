"""The 4-bit projection in the shapes that go round most: more than four tiles of tokens at a time, tokens that come along
with the weights over several tiles of rows, the widest rows.  Tolerances are those of test_gpu_mx4."""
from __future__ import annotations

import pytest

from tests.test_gpu_mx4 import _head_case
from tests.test_gpu_ops import psc  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V,K", [(1300, 11000, 512), (1100, 9000, 2048), (1300, 11000, 2304), (2500, 4000, 96)])
def test_more_tokens_than_are_worked_on_at_a_time(psc, T, V, K):  # noqa: F811
    """Tokens' slots, accumulators and parities are carried from one group of tiles of tokens to the next."""
    _head_case(psc, T, V, K, "f32", "none")
    _head_case(psc, T, V, K, "bf16", "mixed")


@pytest.mark.parametrize("T,V,K", [(200, 40000, 2304), (300, 30000, 2100), (513, 20001, 4096), (700, 9001, 8192)])
def test_tokens_that_come_along_over_several_tiles(psc, T, V, K):  # noqa: F811
    _head_case(psc, T, V, K, "bf16", "tight")
    _head_case(psc, T, V, K, "f32", "none")


@pytest.mark.parametrize("T,V,K", [(1, 150, 131072), (3, 40, 131072), (100, 300, 65600), (140, 200, 131072), (260, 30, 100000),
                                   (16, 20000, 33001)])
def test_the_widest_rows(psc, T, V, K):  # noqa: F811
    _head_case(psc, T, V, K, "f32", "none")
    _head_case(psc, T, V, K, "bf16", "mixed")
