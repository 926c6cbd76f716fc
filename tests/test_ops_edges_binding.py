"""The operators' binding and C entries on the CPU at the ends of their ranges."""
from __future__ import annotations

import pytest

from tests.test_library_cpu import psc  # noqa: F401

torch = pytest.importorskip("torch")


def test_head_faults_refuses_what_is_no_workspace(psc):  # noqa: F811
    with pytest.raises(ValueError, match="work"):
        psc.psc_head_faults(torch.zeros(3, dtype=torch.uint8))
    with pytest.raises(ValueError, match="CUDA"):
        psc.psc_head_faults(torch.zeros(256, dtype=torch.uint8))
