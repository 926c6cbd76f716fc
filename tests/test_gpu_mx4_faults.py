"""The 4-bit projection where its waits give up, without any fault: psc_mx4_check_wait runs it with waits that are
too short, and what matters is that it ends, counts the blocks, writes no logit that is not right, and leaves the device
as it was."""
from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_mx4 import _matrix
from tests.test_gpu_ops import _mask, _pack, psc  # noqa: F401
from tests.test_gpu_sampled_decode import example  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# few tokens, with one part of a stage small and with all alike; pairs of blocks whose tokens stay, and whose come along
SIZES = [(1, 30001, 2048), (16, 25000, 512), (128, 20001, 1024), (300, 30001, 512), (200, 15000, 2304), (600, 9000, 300)]


def _call(psc, T, V, K, masked):  # noqa: F811
    rng = np.random.default_rng([T, V, K])
    qc, wc = rng.integers(0, 16, (T, K), dtype=np.uint8), rng.integers(0, 16, (V, K), dtype=np.uint8)
    nb = (K + 31) // 32
    qe, we = rng.integers(124, 130, (T, nb)).astype(np.uint8), rng.integers(118, 124, (V, nb)).astype(np.uint8)
    matrices = (*_matrix(psc, qc, qe, K), *_matrix(psc, wc, we, K))
    bm = _pack(_mask(rng, "mixed", T, V)) if masked else None

    def call(limit=None):
        big = torch.full((T, V + 3), 7.0, device="cuda")
        if limit is None:
            psc.psc_head_logits_mx4(*matrices, big[:, :V], K, bitmask=bm)
        else:
            psc.psc_mx4_check_wait(*matrices, big[:, :V], K, limit, bitmask=bm)
        assert (big[:, V:] == 7).all()
        return big[:, :V]

    return call


@pytest.mark.parametrize("T,V,K", SIZES)
def test_waits_that_give_up_at_once(psc, T, V, K):  # noqa: F811
    """Every block gives up, with nothing under way."""
    call = _call(psc, T, V, K, False)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    tokens, rows = (1, 128) if T <= 128 else (-(-T // 256), 192)
    tiles = -(-V // rows)
    blocks = min(tiles, sms) if T <= 128 else 2 * tokens * min(sms // 2 // tokens, tiles)
    want = call()
    before = psc.psc_mx4_faults()
    assert (call(0) == 7).all()
    assert psc.psc_mx4_faults() - before == blocks
    assert torch.equal(call(), want)
    assert psc.psc_mx4_faults() - before == blocks


@pytest.mark.parametrize("T,V,K", SIZES)
@pytest.mark.parametrize("masked", [False, True])
def test_waits_that_give_up_midway(psc, T, V, K, masked):  # noqa: F811
    """Blocks give up with copies and products under way: what is written is right, and the calls after it are.  A look at
    once does not find copies that have just been asked for; 4,000 take about a hundred microseconds."""
    call = _call(psc, T, V, K, masked)
    want = call()
    for limit in (1, 2, 4, 6, 7, 8, 9, 10, 11, 12, 14, 16, 18, 20, 22, 25, 28, 32, 36, 40, 50, 80, 300, 4000):
        before = psc.psc_mx4_faults()
        got = call(limit)
        gave_up = psc.psc_mx4_faults() - before
        assert ((got == 7) | (got == want)).all(), limit
        assert gave_up > 0 or torch.equal(got, want)
        # (where the masks allow nothing at all, as the one of a single row, there is nothing to wait for)
        assert gave_up > 0 or limit > 1 or not torch.isfinite(want).any()
        assert torch.equal(call(), want)
    before = psc.psc_mx4_faults()
    assert torch.equal(call(1 << 22), want)                 # as many as the projection itself waits for
    assert psc.psc_mx4_faults() == before


def test_counts_are_kept_until_they_are_reset(psc):  # noqa: F811
    call = _call(psc, 3, 5000, 256, False)
    psc.psc_mx4_faults(reset=True)
    assert psc.psc_mx4_faults() == 0
    call(0), call(0)
    assert psc.psc_mx4_faults() == 2 * 40
    assert psc.psc_mx4_faults(reset=True) == 2 * 40
    assert psc.psc_mx4_faults() == 0


def test_resets_lose_no_fault_of_another_stream(psc):  # noqa: F811
    """Two threads count and reset while others' projections give up on streams of their own: every fault is reported
    once."""
    import threading
    call = _call(psc, 3, 5000, 256, False)
    psc.psc_mx4_faults(reset=True)
    streams, reports, errors = [torch.cuda.Stream() for _ in range(4)], [0, 0], []
    rounds, done = 150, threading.Event()

    def work(stream):
        try:
            with torch.cuda.stream(stream):
                for _ in range(rounds):
                    call(0)
                stream.synchronize()
        except Exception as e:              # noqa: BLE001
            errors.append(e)

    def count(i):
        try:
            while not done.is_set():
                reports[i] += psc.psc_mx4_faults(reset=True, stream=streams[2 + i])
        except Exception as e:              # noqa: BLE001
            errors.append(e)

    workers = [threading.Thread(target=work, args=(s,)) for s in streams[:2]]
    counters = [threading.Thread(target=count, args=(i,)) for i in range(2)]
    for t in workers + counters:
        t.start()
    for t in workers:
        t.join()
    done.set()
    for t in counters:
        t.join()
    assert not errors
    assert sum(reports) + psc.psc_mx4_faults(reset=True) == 2 * rounds * 40
    assert psc.psc_mx4_faults() == 0


@pytest.mark.parametrize("projection", ["int8", "norm8", "mx4"])
def test_the_example_counts_its_own_faults(psc, example, projection):  # noqa: F811
    """What gave up before a run is not the run's; what gives up during a run in 4 bits is."""
    call = _call(psc, 3, 5000, 256, False)
    call(0)
    before = psc.psc_mx4_faults()
    assert before > 0
    example.run(3, 4, projection=projection)
    assert psc.psc_mx4_faults() == before
    if projection == "mx4":
        step = example.Decoder.step

        def step_beside_a_fault(self):
            step(self)
            call(0)

        with pytest.MonkeyPatch.context() as m:
            m.setattr(example.Decoder, "step", step_beside_a_fault)
            with pytest.raises(RuntimeError, match="gave up"):
                example.run(3, 2, use_graph=False, projection=projection)
    psc.psc_mx4_faults(reset=True)
