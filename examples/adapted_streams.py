"""Live streams that share one model and one decoding graph, each speaker with a
low-rank adapter of the output layer: hidden rows to words on one GPU.

    python examples/adapted_streams.py

A second of audio at a time, the newest hidden rows of every stream go through
the shared layer and the streams' adapters in one call (Head.project), and
from logits to log-likelihoods in another (loglikes: log-softmax, pdf priors,
acoustic scale), which writes them straight into the streams' frame stores;
Stream.advance decodes them there.  When the streams have ended, a second pass
keeps to the first one's lattices: the pdfs that leave a frame's lattice nodes
are its label mask (Graph.label_masks), and a speaker's likely pdfs get a bias.

The hidden rows, the weights and the graph are synthetic (seeded).
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import synth  # noqa: E402
from paper_1804_03243_amd import wfstdec  # noqa: E402

DEVICE = torch.device("cuda:0")


def make_model(P: int, D: int = 256, G: int = 4, R: int = 8, seed: int = 0):
    """A head of P pdfs over D inputs with G adapters of rank R, and the log priors."""
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    bf16 = lambda t: t.to(torch.bfloat16).to(DEVICE)  # noqa: E731
    head = wfstdec.Head(bf16(3.0 * rnd(P, D) / D ** 0.5), rnd(P).to(DEVICE), bf16(rnd(G, R, D) / D ** 0.5),
                        bf16(0.3 * rnd(G, P, R) / R ** 0.5), torch.full((G,), 2.0, device=DEVICE))
    return head, torch.log_softmax(0.5 * rnd(P), 0).to(DEVICE)


def stream_pass(graph, head, log_prior, hidden, adapters, decoding, chunk: int = 32):
    """Decodes the streams' hidden rows [T_i, D] as they arrive, `chunk` rows of
    each at a time; adapters[i] is stream i's (negative: none)."""
    B, T = len(hidden), [len(h) for h in hidden]
    stream = wfstdec.Stream(graph, B, max(T), *decoding)
    stores = stream.frames.view(-1, graph.num_pdfs)
    for t0 in range(0, max(T), chunk):
        n = [min(chunk, max(0, t - t0)) for t in T]
        rows = torch.cat([h[t0:t0 + k] for h, k in zip(hidden, n)])
        of = np.repeat(np.arange(B), n)
        to = np.concatenate([i * stream.max_T + t0 + np.arange(k) for i, k in enumerate(n)])
        logits = head.project(rows, torch.from_numpy(np.asarray(adapters, np.int32)[of]).to(DEVICE))
        wfstdec.loglikes(logits, scale=0.8, log_prior=log_prior, out=stores,
                         out_row=torch.from_numpy(to.astype(np.int32)).to(DEVICE))
        stream.advance(n)
    return stream.end(), stream


def second_pass(graph, loglikes, first, biases, decoding):
    """Decodes the log-likelihoods [T, P] again within the first pass's lattice,
    the labels of `biases` (zero-based pdfs and values) preferred."""
    T = len(loglikes)
    offsets = np.searchsorted(first.nodes["t"], np.arange(T + 1)).astype(np.int64)  # nodes of frames 0..T-1
    states = np.ascontiguousarray(first.nodes["state"])
    mask = graph.label_masks(torch.from_numpy(offsets).to(DEVICE), torch.from_numpy(states).to(DEVICE))
    pdfs, values = biases
    bias = (torch.tensor([0, len(pdfs)], device=DEVICE), torch.tensor(pdfs, dtype=torch.int32, device=DEVICE),
            torch.tensor(values, dtype=torch.float32, device=DEVICE))
    request = torch.zeros(T, dtype=torch.int32, device=DEVICE)
    again = wfstdec.loglikes(loglikes, normalize=False, mask=mask, bias=bias, request=request)
    return wfstdec.decode(graph, again, *decoding)


def main():
    cfg = synth.workload("tiny_10k")
    graph = wfstdec.Graph(synth.make_graph(cfg), cfg["P"], str(DEVICE))
    decoding = (cfg["beam"], cfg["max_active"], cfg["lattice_beam"])
    head, log_prior = make_model(cfg["P"])
    gen = torch.Generator().manual_seed(1)
    hidden = [torch.randn((t, head.D), generator=gen).to(torch.bfloat16).to(DEVICE) for t in (150, 97, 64, 200)]
    results, stream = stream_pass(graph, head, log_prior, hidden, [2, -1, 0, 2], decoding)
    for i, r in enumerate(results):
        s = second_pass(graph, stream.frames[i, :stream.T[i]], r, ([3, 141], [0.5, 0.25]), decoding)
        print(f"stream {i}: {stream.T[i]} frames, {len(r.words)} words, cost {float(r.cost):.2f}, "
              f"{len(r.links)} lattice links; second pass {len(s.words)} words, cost {float(s.cost):.2f}")


if __name__ == "__main__":
    main()
