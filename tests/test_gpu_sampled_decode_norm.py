"""The decoding loop with the norm in front of the projection, in 8 and in 4 bits: every token that it draws is one
that the oracle's mask allows, the steps replayed from a CUDA graph are the steps, and its logits are those of
the steps' definitions in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest

from tests import _mx4_ref as ref
from tests.test_gpu_sampled_decode import example  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("projection", ["norm8", "mx4"])
@pytest.mark.parametrize("rows", [3, 20])
def test_sampled_documents_stay_in_the_language(example, projection, rows):  # noqa: F811
    from oracle import Oracle, Vocab
    steps = 16
    w, tokens, logprobs, status = example.run(rows, steps, seed=3, projection=projection)
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


@pytest.mark.parametrize("projection", ["norm8", "mx4"])
def test_graph_replay_gives_the_same_documents(example, projection):  # noqa: F811
    a = example.run(6, 12, use_graph=True, seed=5, projection=projection)
    b = example.run(6, 12, use_graph=False, seed=5, projection=projection)
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_logits_of_a_step(example):  # noqa: F811
    """Two steps' residual sums and masked logits (before penalties) against numpy; sums over K = 256 in f32 as in the
    projection's own tests, the norm's factor off by 24 u of itself."""
    from workloads import configs
    rows, u = 5, 2.0 ** -24
    d = example.Decoder(configs.load(2, batch=1), rows, 4, projection="mx4", repetition=1.0)
    h = np.zeros((rows, 256), dtype=np.float32)
    K, V = 256, d.h.V
    w = torch.empty(V, K, device="cuda")
    d.psc.psc_dequantize_mx4(d.w4, d.w4_blocks, w)
    w = w.double().cpu().numpy()
    for _ in range(2):
        d.new_inputs()
        x = d.x.float().cpu().numpy()
        h, v, r = ref.norm(x, h, d.gain.cpu().numpy(), 1e-6, True)
        d.step()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(d.residual.float().cpu().numpy(), h)
        y = ref.decode(*ref.quantize(v))
        exact, size = y @ w.T * r[:, None], np.abs(y) @ np.abs(w).T * r[:, None]
        allowed = np.unpackbits(d.mask.cpu().numpy().view(np.uint8), axis=-1, bitorder="little")[:, :V].astype(bool)
        got = d.logits.double().cpu().numpy()
        assert (got[~allowed] == -np.inf).all()
        tol = 4 * u * (K / 64 + 2) * size + 27 * u * np.abs(exact)
        assert (np.abs(got - exact) <= tol)[allowed].all()
