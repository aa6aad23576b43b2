"""The example's path: first-pass labels, a step of losses, gradients, clipping and
weights, the fitted layer in four bits and its decode, each against the plain forms."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import plain_fit
import plain_scores as plain
import synth

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("fit_output_layer", os.path.join(ROOT, "examples", "fit_output_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.fixture(scope="module")
def setting(example):
    wf = example.wfstdec
    cfg = synth.workload("tiny_10k")
    graph = wf.Graph(synth.make_graph(cfg), cfg["P"])
    gen = torch.Generator().manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    P, D = cfg["P"], 64
    return dict(wf=wf, graph=graph, decoding=(cfg["beam"], cfg["max_active"], cfg["lattice_beam"]), P=P,
                weight=(3.0 * rnd(P, D) / D ** 0.5).to(BF16).cuda(), bias=rnd(P).cuda(), prior=torch.log_softmax(0.5 * rnd(P), 0).cuda(),
                hidden=[rnd(t, D).to(BF16).cuda() for t in (40, 23)])


def test_labels_are_of_the_lattice(example, setting):
    s = setting
    results, _ = example.decode_all(s["graph"], s["wf"].Head(s["weight"], s["bias"]), s["prior"], s["hidden"], s["decoding"])
    for r, h in zip(results, s["hidden"]):
        label, sure = example.first_pass_labels(r, len(h))
        for t in range(len(h)):
            at = r.links[(r.links["t"] == t + 1) & (r.links["ilabel"] > 0)]
            best = at["posterior"].max()
            if best < 0.5:
                assert int(label[t]) == -1 and float(sure[t]) == 0
            else:
                assert int(label[t]) + 1 in at["ilabel"][at["posterior"] == best] and float(sure[t]) == np.float32(best)


@pytest.mark.parametrize("max_norm", [0.05, 1e6])
def test_a_step_and_the_layer_in_four_bits(example, setting, max_norm):
    s = setting
    wf, rows = s["wf"], torch.cat(s["hidden"])
    target = torch.randint(-1, s["P"], (len(rows),), generator=torch.Generator().manual_seed(6), dtype=torch.int32).cuda()
    grad = torch.full((len(rows),), 1.0 / len(rows)).cuda()
    layer = example.Layer(s["weight"], s["bias"])
    loss, norm = layer.step(rows, target, grad, 0.5, max_norm)
    want = plain_fit.cross_entropy(rows.cpu(), s["weight"].cpu(), target.cpu(), s["bias"].cpu(), grad.cpu())
    plain.close(loss, want["loss"], want["bounds"]["loss"])
    # the norm and the clipped gradients of the gradients that were formed (within their bounds of the exact ones)
    _, _, dw, db = wf.cross_entropy_grads(rows, s["weight"], target, s["bias"], grad)
    plain.close(dw, want["dweight"], want["bounds"]["dweight"])
    plain.close(db, want["dbias"], want["bounds"]["dbias"])
    exact, scaled = plain_fit.clip([dw.cpu(), db.cpu()], max_norm)
    assert abs(float(norm) - exact) <= 2 * plain.EPS * exact
    for g, t in zip(layer.grads, scaled):
        plain.close(g, t, 3.1 * plain.EPS * t.abs() + 2.0 ** -150)
    # 32-bit masters: the product's rounding and the difference's
    m = s["weight"].cpu().double() - 0.5 * layer.grads[0].cpu().double()
    plain.close(layer.master, m, 2 * plain.EPS * (m.abs() + layer.grads[0].cpu().double().abs()))
    assert torch.equal(layer.weight, layer.master.to(BF16))
    # in four bits
    held = wf.micro(layer.weight)
    codes, scales = plain_fit.micro(layer.weight.cpu())
    W = plain_fit.micro_values(codes, scales)
    plain.close(held.values(), W, torch.zeros_like(W))
    X = plain_fit.micro_values(*plain_fit.micro(rows.cpu()))
    logits = wf.MicroHead(held, layer.bias).project(rows)
    z = X @ W.T + layer.bias.cpu().double()
    slack = (X.shape[1] + 8) * plain.EPS * (X.abs() @ W.abs().T + layer.bias.cpu().double().abs()) + plain.EPS * z.abs()
    plain.close(logits, z, slack)


def test_the_decode_of_the_fitted_layer(example, setting):
    """Decoded from the four-bit layer's logits as from the same log-likelihoods by themselves."""
    s = setting
    wf = s["wf"]
    head = wf.MicroHead(wf.micro(s["weight"]), s["bias"])
    results, loglikes = example.decode_all(s["graph"], head, s["prior"], s["hidden"], s["decoding"])
    for r, l, h in zip(results, loglikes, s["hidden"]):
        want, slack = plain.loglikes(head.project(h).cpu(), scale=0.8, log_prior=s["prior"].cpu())
        plain.close(l, want, slack)
        one = wf.decode(s["graph"], l.clone(), *s["decoding"])
        assert r.cost == one.cost and list(r.words) == list(one.words) and np.array_equal(r.links["arc_id"], one.links["arc_id"])


def test_captured_step(example, setting):
    """A whole step in a graph, replayed against eager steps."""
    s = setting
    rows = torch.cat(s["hidden"])
    target = torch.randint(0, s["P"], (len(rows),), generator=torch.Generator().manual_seed(7), dtype=torch.int32).cuda()
    grad = torch.full((len(rows),), 1.0 / len(rows)).cuda()
    eager, layer = example.Layer(s["weight"], s["bias"]), example.Layer(s["weight"], s["bias"])
    example.Layer(s["weight"], s["bias"]).step(rows, target, grad, 0.5, 0.1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, norm = layer.step(rows, target, grad, 0.5, 0.1)
    for _ in range(4):
        graph.replay()
        want, want_norm = eager.step(rows, target, grad, 0.5, 0.1)
        torch.cuda.synchronize()
        assert torch.equal(loss, want) and torch.equal(norm, want_norm)
        assert torch.equal(layer.master, eager.master) and torch.equal(layer.bias, eager.bias) and torch.equal(layer.weight, eager.weight)


def test_example_runs(example, capsys):
    example.main()
    assert capsys.readouterr().out.count("\n") == 8
