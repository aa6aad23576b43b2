"""The example's path: projection, log-likelihoods into the frame stores, streaming
decode and second pass, against the same log-likelihoods decoded as a whole."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import plain_scores as plain
import synth

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("adapted_streams", os.path.join(ROOT, "examples", "adapted_streams.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("chunk", [1, 32, 500])
def test_streams_equal_whole_decodes(example, chunk):
    wf = example.wfstdec
    cfg = synth.workload("tiny_10k")
    graph = wf.Graph(synth.make_graph(cfg), cfg["P"])
    decoding = (cfg["beam"], cfg["max_active"], cfg["lattice_beam"])
    head, prior = example.make_model(cfg["P"])
    gen = torch.Generator().manual_seed(2)
    hidden = [torch.randn((t, head.D), generator=gen).to(torch.bfloat16).to("cuda:0") for t in (40, 17, 66)]
    adapters = [1, -1, 3]
    results, stream = example.stream_pass(graph, head, prior, hidden, adapters, decoding, chunk)
    weight, bias, a, b, scale = (t.cpu() for t in head._kept)
    for i, (h, g) in enumerate(zip(hidden, adapters)):
        ad = torch.full((len(h),), g, dtype=torch.int32)
        logits, bound = plain.project(h.cpu(), weight, bias, a, b, scale, ad)
        want, slack = plain.loglikes(logits, scale=0.8, log_prior=prior.cpu())
        # a logit's error reaches its own value and, at most as much again, the row's sum
        slack = slack + 0.8 * (bound + bound.max(1, keepdim=True).values)
        plain.close(stream.frames[i, :len(h)], want, slack)
    whole = wf.decode_batch(graph, [stream.frames[i, :len(h)].contiguous() for i, h in enumerate(hidden)], *decoding)
    for r, w in zip(results, whole):
        assert r.cost == w.cost and list(r.words) == list(w.words) and np.array_equal(r.links["arc_id"], w.links["arc_id"])


def test_second_pass_prefers_the_biased_labels(example):
    wf = example.wfstdec
    cfg = synth.workload("tiny_10k")
    graph = wf.Graph(synth.make_graph(cfg), cfg["P"])
    decoding = (cfg["beam"], cfg["max_active"], cfg["lattice_beam"])
    L = torch.from_numpy(synth.make_loglikes(cfg)[:60]).to("cuda:0")
    first = wf.decode(graph, L, *decoding)
    same = example.second_pass(graph, L, first, ([], []), decoding)
    assert same.cost == first.cost and list(same.words) == list(first.words)
    pdf = int(first.links["ilabel"][first.links["ilabel"] > 0][0]) - 1
    better = example.second_pass(graph, L, first, ([pdf], [1.0]), decoding)
    assert better.cost <= first.cost


def test_advance_refuses_other_counts(example):
    wf = example.wfstdec
    cfg = synth.workload("tiny_10k")
    graph = wf.Graph(synth.make_graph(cfg), cfg["P"])
    s = wf.Stream(graph, 2, 10, cfg["beam"], cfg["max_active"], cfg["lattice_beam"])
    with pytest.raises(ValueError):
        s.advance([1])
    with pytest.raises(wf.WdError):
        s.advance([11, 0])
    assert s.T == [0, 0]


def test_advance_waits_for_rows_of_another_stream(example):
    """Rows that the caller's stream is still to write are decoded after it has."""
    wf = example.wfstdec
    cfg = synth.workload("tiny_10k")
    graph = wf.Graph(synth.make_graph(cfg), cfg["P"])
    decoding = (cfg["beam"], cfg["max_active"], cfg["lattice_beam"])
    L = torch.from_numpy(synth.make_loglikes(cfg)[:40]).to("cuda:0")
    s = wf.Stream(graph, 1, 40, *decoding)
    s.frames.zero_()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        torch.cuda._sleep(100_000_000)  # (some tens of milliseconds)
        s.frames[0].copy_(L)
        s.advance([40])
    r, w = s.end()[0], wf.decode(graph, L, *decoding)
    assert r.cost == w.cost and list(r.words) == list(w.words) and np.array_equal(r.links["arc_id"], w.links["arc_id"])
