"""Fits a shared output layer to the labels that a first pass decodes, and serves it in
four bits a weight: hidden rows to words on one GPU.

    python examples/fit_output_layer.py

A first pass decodes utterances with the layer as it is (Head.project, loglikes,
decode).  Every frame's most likely link of the lattice names its label and how
sure the lattice is of it; frames that it is not sure of have no label.  Steps of
gradient descent follow: losses and gradients straight from the hidden rows
(cross_entropy_grads), clipped by their norm into 32-bit copies (clip_gradients),
against weights held in 32 bits.  The fitted layer is then held in four bits a
weight (micro, MicroHead) and decodes the utterances again.

The hidden rows, the weights and the graph are synthetic (seeded).
"""
from __future__ import annotations

import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import synth  # noqa: E402
from paper_1804_03243_amd import wfstdec  # noqa: E402

DEVICE = torch.device("cuda:0")


def first_pass_labels(result, T: int, least: float = 0.5):
    """(labels int32 [T], confidences float32 [T]) of a decode's lattice: the pdf of each
    frame's link of the highest posterior; -1 and 0 where that is below `least`."""
    links = result.links[result.links["ilabel"] > 0]
    order = np.lexsort((links["arc_id"], -links["posterior"], links["t"]))
    frames, first = np.unique(links["t"][order], return_index=True)
    best = links[order][first]
    label, sure = np.full(T, -1, np.int32), np.zeros(T, np.float32)
    keep = best["posterior"] >= least
    label[frames[keep] - 1], sure[frames[keep] - 1] = best["ilabel"][keep] - 1, best["posterior"][keep]
    return torch.from_numpy(label).to(DEVICE), torch.from_numpy(sure).to(DEVICE)


class Layer:
    """The weights of a step: 32-bit masters and the 16-bit copy that products read."""

    def __init__(self, weight, bias):
        self.master, self.bias = weight.float(), bias.clone()
        self.weight = weight.clone()
        self.grads = [torch.empty_like(self.master), torch.empty_like(self.bias)]  # clipped, in 32 bits

    def step(self, hidden, target, grad, rate: float, max_norm: float):
        """One step; returns the rows' losses and the gradients' norm, both on the device."""
        loss, _, d_weight, d_bias = wfstdec.cross_entropy_grads(hidden, self.weight, target, self.bias, grad)
        norm = wfstdec.clip_gradients([d_weight, d_bias], max_norm, out=self.grads)
        self.master -= rate * self.grads[0]
        self.bias -= rate * self.grads[1]
        self.weight.copy_(self.master)
        return loss, norm


def decode_all(graph, head, log_prior, hidden, decoding):
    loglikes = [wfstdec.loglikes(head.project(h), scale=0.8, log_prior=log_prior) for h in hidden]
    return wfstdec.decode_batch(graph, loglikes, *decoding), loglikes


def main():
    cfg = synth.workload("tiny_10k")
    graph = wfstdec.Graph(synth.make_graph(cfg), cfg["P"], str(DEVICE))
    decoding = (cfg["beam"], cfg["max_active"], cfg["lattice_beam"])
    gen = torch.Generator().manual_seed(0)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    P, D = cfg["P"], 256
    weight = (3.0 * rnd(P, D) / math.sqrt(D)).to(torch.bfloat16).to(DEVICE)
    bias, log_prior = rnd(P).to(DEVICE), torch.log_softmax(0.5 * rnd(P), 0).to(DEVICE)
    hidden = [rnd(t, D).to(torch.bfloat16).to(DEVICE) for t in (150, 97, 64)]
    first, _ = decode_all(graph, wfstdec.Head(weight, bias), log_prior, hidden, decoding)
    labels = [first_pass_labels(r, len(h)) for r, h in zip(first, hidden)]
    rows, target = torch.cat(hidden), torch.cat([t for t, _ in labels])
    grad = torch.cat([c for _, c in labels]) / max(1, int((target >= 0).sum()))
    layer = Layer(weight, bias)
    for i in range(5):
        loss, norm = layer.step(rows, target, grad, rate=0.5, max_norm=1.0)
        print(f"step {i}: loss {float((loss * grad).sum()):.4f}, norm {float(norm):.4f}")
    small = wfstdec.MicroHead(wfstdec.micro(layer.weight), layer.bias)
    again, _ = decode_all(graph, small, log_prior, hidden, decoding)
    for i, (a, b) in enumerate(zip(first, again)):
        print(f"utterance {i}: {len(a.words)} words, cost {float(a.cost):.2f}; fitted, in four bits: {len(b.words)} words, cost {float(b.cost):.2f}")


if __name__ == "__main__":
    main()
