"""The operators together, as the example runs them: every token that it draws is one
that the oracle's mask allows, and the steps replayed from a CUDA graph are the steps."""
from __future__ import annotations

import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_03065_gb300 import build, psc
    build.build()
    psc.load()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import sampled_decode
    return sampled_decode


def test_sampled_documents_stay_in_the_language(example):
    from oracle import Oracle, Vocab
    rows, steps = 12, 24
    w, tokens, logprobs, status = example.run(rows, steps, seed=3)
    o = Oracle(w.grammar_text)
    voc = Vocab.from_list(w.vocab, w.eos_id)
    configs = [o.initial() for _ in range(rows)]
    for i in range(steps):
        mask = o.masks(configs, voc)
        allowed = np.unpackbits(mask.view(np.uint8), axis=-1, bitorder="little")[:, :len(w.vocab)]
        for b, c in enumerate(configs):
            t = int(tokens[b, i])
            assert allowed[b, t], (b, i, t)
            o.advance_tokens(c, voc, [t])
    assert set(status.tolist()) <= {0, 1}
    assert torch.isfinite(logprobs).all() and (logprobs <= 0).all()
    assert len({tuple(r) for r in tokens.tolist()}) > 1


def test_graph_replay_gives_the_same_documents(example):
    a = example.run(6, 12, use_graph=True, seed=5)
    b = example.run(6, 12, use_graph=False, seed=5)
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
