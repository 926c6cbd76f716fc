"""Sampled decoding under a grammar, every step on the device.

A batch of JSON documents is drawn token by token: the grammar's masks
(psc_fill_mask), the vocabulary projection in 8-bit integers under them
(psc_quantize_rows, psc_head_logits), penalties for what has been said
(psc_process_logits), the draw (psc_sample) and the parser (psc_advance).  The
steps are captured once in a CUDA graph and replayed.  There is no model: a
step's hidden states are random, so the documents are grammatical and nothing
more.

    python examples/sampled_decode.py [--rows 8] [--steps 40]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


class Decoder:
    """The buffers of a decoding loop, and one step of it."""

    def __init__(self, workload, rows: int, max_steps: int, hidden: int = 256, seed: int = 0, temperature: float = 0.8,
                 top_k: int = 40, top_p: float = 0.95, repetition: float = 1.1):
        import torch
        from paper_2608_03065_gb300 import psc
        self.psc = psc
        self.h = psc.psc_compile(workload.grammar_text, workload.vocab, workload.eos_id)
        self.states = psc.psc_state_init(self.h, rows, 256)
        V, dev = self.h.V, "cuda"
        self.gen = torch.Generator(device=dev).manual_seed(seed)
        # the projection's weights, quantised once: a scale per vocabulary row
        weights = torch.randn(V, hidden, device=dev, generator=self.gen).bfloat16()
        self.w = torch.empty(V, hidden, dtype=torch.int8, device=dev)
        self.w_scale = torch.empty(V, device=dev)
        psc.psc_quantize_rows(weights, self.w, self.w_scale)
        self.w_scale *= hidden ** -0.5 * 2.0
        # a step's inputs: hidden states, one uniform number a row
        self.x = torch.empty(rows, hidden, dtype=torch.bfloat16, device=dev)
        self.uniform = torch.empty(rows, device=dev)
        # and what it works in
        self.q = torch.empty(rows, hidden, dtype=torch.int8, device=dev)
        self.x_scale = torch.empty(rows, device=dev)
        self.mask = torch.empty(rows, self.h.W, dtype=torch.int32, device=dev)
        self.logits = torch.empty(rows, V, device=dev)
        self.history = torch.full((rows, max_steps), -1, dtype=torch.int32, device=dev)
        self.length = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.tokens = torch.empty(rows, dtype=torch.int32, device=dev)
        self.logprobs = torch.empty(rows, device=dev)
        self.status = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.temperature = torch.full((rows,), temperature, device=dev)
        self.top_k = torch.full((rows,), top_k, dtype=torch.int32, device=dev)
        self.top_p = torch.full((rows,), top_p, device=dev)
        self.repetition = torch.full((rows,), repetition, device=dev)
        self.head_work = torch.empty(psc.psc_head_work_bytes(rows, V, hidden), dtype=torch.uint8, device=dev)
        self.faults = self.head_work[:4].view(torch.int32)     # of the last projection, on the device
        self.sample_work = torch.empty(psc.psc_sample_work_bytes(rows), dtype=torch.uint8, device=dev)

    def step(self):
        """Everything between a model's last hidden states and the parser's next state."""
        psc = self.psc
        psc.psc_fill_mask(self.h, self.states, self.mask)
        psc.psc_quantize_rows(self.x, self.q, self.x_scale)
        psc.psc_head_logits(self.q, self.x_scale, self.w, self.w_scale, self.logits, bitmask=self.mask,
                            work=self.head_work)
        psc.psc_process_logits(self.logits, history=self.history, history_len=self.length,
                               repetition=self.repetition)
        psc.psc_sample(self.logits, self.uniform, self.tokens, logprobs=self.logprobs, bitmask=self.mask,
                       temperature=self.temperature, top_k=self.top_k, top_p=self.top_p, work=self.sample_work)
        psc.psc_advance(self.h, self.states, self.tokens, self.status)
        self.history.scatter_(1, self.length[:, None].long(), self.tokens[:, None])
        self.length += 1

    def new_inputs(self):
        self.x.normal_(generator=self.gen)
        self.uniform.uniform_(generator=self.gen)


def run(rows: int = 8, steps: int = 40, use_graph: bool = True, seed: int = 0):
    """(workload, tokens [rows, steps], ln probabilities [rows, steps], last statuses [rows]), on the host."""
    import torch
    from workloads import configs
    workload = configs.load(2, batch=1)
    d = Decoder(workload, rows, steps, seed=seed)
    logprobs = torch.empty(steps, rows, device="cuda")
    faults = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = None
    for i in range(steps):
        d.new_inputs()
        if not use_graph or i == 0:
            d.step()                    # the first step sets kernels up, which a capture cannot
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    d.step()
            graph.replay()
        logprobs[i] = d.logprobs
        faults += d.faults
    torch.cuda.synchronize()
    if faults.item():                   # a bounded wait gave up: some logits were not written
        raise RuntimeError(f"psc_head_logits: {faults.item()} blocks gave up")
    return workload, d.history.cpu(), logprobs.t().cpu(), d.status.cpu()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rows", type=int, default=8)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    workload, tokens, logprobs, status = run(a.rows, a.steps)
    for row, lp, st in zip(tokens.tolist(), logprobs, status.tolist()):
        text = b"".join(workload.vocab[t] for t in row if t != workload.eos_id)
        print("%-8s ln p %8.2f  %s" % ("done" if st == 1 else "open" if st == 0 else "status %d" % st, lp.sum(),
                                        text.decode("utf-8", "replace")[:150]))


if __name__ == "__main__":
    main()
