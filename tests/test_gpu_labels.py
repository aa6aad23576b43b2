"""Label masks from the decoding graph (Graph.label_masks, wd_label_masks)
against a plain implementation, exactly; and the second pass they are for."""
import numpy as np
import pytest
import torch

import plain_scores as plain
import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def wf():
    from paper_1804_03243_amd import wfstdec
    assert torch.cuda.is_available()
    wfstdec.lib()
    return wfstdec


def wide_graph(S, A, P, seed, hub=0):
    """Random graph whose first state has `hub` further arcs."""
    rng = np.random.default_rng(seed)
    src = np.sort(np.concatenate([rng.integers(0, S, A), np.zeros(hub, np.int64)]))
    n = len(src)
    eps = (rng.random(n) < 0.2) & (src < S - 1)
    dst = np.where(eps, src + 1 + (rng.random(n) * (S - 1 - src)).astype(np.int64), rng.integers(0, S, n))
    return dict(num_states=S, start_state=0, row_ptr=np.concatenate([[0], np.cumsum(np.bincount(src, minlength=S))]).astype(np.uint32),
                dst=np.minimum(dst, S - 1).astype(np.uint32), ilabel=np.where(eps, 0, rng.integers(1, P + 1, n)).astype(np.int32),
                olabel=np.zeros(n, np.int32), weight=np.ones(n, np.float32))


def check(wf, graph, g, P, offsets, states):
    got = graph.label_masks(torch.from_numpy(offsets).to(DEV), torch.from_numpy(states).to(DEV))
    assert got.dtype == torch.int32
    assert np.array_equal(got.cpu().numpy(), plain.label_masks(g, P, offsets, states))


@pytest.mark.parametrize("S,A,P,hub", [(1, 0, 1, 0), (5, 9, 31, 0), (50, 200, 32, 0), (300, 900, 33, 500), (4000, 9000, 6000, 3000),
                                       (2000, 9000, 100_003, 70), (500, 5000, 700_001, 100)])
@pytest.mark.parametrize("rows,most", [(1, 0), (1, 1), (3, 40), (70, 5), (500, 30), (2, 9000)])
def test_sizes(wf, S, A, P, hub, rows, most):
    g = wide_graph(S, A, P, S + A, hub) if A else dict(num_states=1, start_state=0, row_ptr=np.zeros(2, np.uint32),
                                                       dst=np.zeros(0, np.uint32), ilabel=np.zeros(0, np.int32),
                                                       olabel=np.zeros(0, np.int32), weight=np.zeros(0, np.float32))
    graph = wf.Graph(g, P)
    rng = np.random.default_rng([rows, most])
    counts = rng.integers(0, most + 1, rows)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    states = rng.integers(0, S, int(offsets[-1])).astype(np.int32)
    check(wf, graph, g, P, offsets, states)
    if len(states) > 3:  # states that the graph does not have, repeats
        states[:3] = [-1, S, 2 ** 31 - 1]
        states[-1] = states[-2]
        check(wf, graph, g, P, offsets, states)


def test_offsets_outside_the_list(wf):
    g = wide_graph(40, 200, 90, 1)
    graph = wf.Graph(g, 90)
    states = np.arange(30, dtype=np.int32)
    check(wf, graph, g, 90, np.array([-4, 5, 3, 29, 100, 2 ** 40], np.int64), states)


def test_output_rows_empty_call_and_other_stream(wf):
    g = wide_graph(40, 200, 90, 1)
    graph = wf.Graph(g, 90)
    offsets, states = np.array([0, 4, 9], np.int64), np.arange(9, dtype=np.int32)
    wide = torch.full((4, 8), 7, dtype=torch.int32, device=DEV)
    out = wide[1:3, 2:6]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o, t = torch.from_numpy(offsets).to(DEV), torch.from_numpy(states).to(DEV)
        assert graph.label_masks(o, t, out=out) is out
    s.synchronize()
    assert np.array_equal(wide[1:3, 2:5].cpu().numpy(), plain.label_masks(g, 90, offsets, states))
    wide[1:3, 2:5] = 7
    assert bool((wide == 7).all())
    assert tuple(graph.label_masks(o[:1], t).shape) == (0, 3)
    for bad in ((o.int(), t), (o, t.long()), (o.cpu(), t), (o[:0], t)):
        with pytest.raises(ValueError):
            graph.label_masks(*bad)
    with pytest.raises(ValueError):
        graph.label_masks(o, t, out=torch.empty((2, 2), dtype=torch.int32, device=DEV))


def test_second_pass_within_a_first_pass_lattice(wf):
    """Masks from a lattice's nodes keep exactly the pdfs of its links, and a decode
    of the masked log-likelihoods finds the same best path."""
    cfg = synth.workload("tiny_10k")
    g, L = synth.make_graph(cfg), synth.make_loglikes(cfg)[:80]
    graph = wf.Graph(g, cfg["P"])
    x = torch.from_numpy(L).to(DEV)
    r = wf.decode(graph, x, cfg["beam"], cfg["max_active"], cfg["lattice_beam"])
    T = len(L)
    offsets = np.searchsorted(r.nodes["t"], np.arange(T + 1)).astype(np.int64)
    m = graph.label_masks(torch.from_numpy(offsets).to(DEV), torch.from_numpy(np.ascontiguousarray(r.nodes["state"])).to(DEV))
    bits = np.unpackbits(m.cpu().numpy().astype("<i4").view(np.uint8).reshape(T, -1), axis=1, bitorder="little")
    for l in r.links[r.links["ilabel"] > 0]:
        assert bits[l["t"] - 1, l["ilabel"] - 1]
    y = wf.loglikes(x, normalize=False, mask=m)
    assert torch.equal(y[y > -float("inf")], x[y > -float("inf")])
    again = wf.decode(graph, y, cfg["beam"], cfg["max_active"], cfg["lattice_beam"])
    assert again.cost == r.cost and list(again.words) == list(r.words)


def test_graph_on_the_current_device(wf):
    """A graph made on "cuda" takes tensors of the device that it is on."""
    g = wide_graph(40, 200, 90, 1)
    check(wf, wf.Graph(g, 90, "cuda"), g, 90, np.array([0, 4, 9], np.int64), np.arange(9, dtype=np.int32))


def test_more_rows_than_a_launch_takes(wf):
    """Rows beyond 2^32 threads of the kernel for long sets, in one call."""
    S, P, N = 500, 90, (1 << 22) + 2
    g = wide_graph(S, 1500, P, 7)
    graph = wf.Graph(g, P)
    n_states = 513 * N  # (most of the list is past the last row's end)
    states = torch.empty(n_states, dtype=torch.int32, device=DEV)
    states[:2 * N] = torch.randint(0, S, (2 * N,), generator=torch.Generator(DEV).manual_seed(8), device=DEV, dtype=torch.int32)
    offsets = 2 * torch.arange(N + 1, device=DEV)
    got = graph.label_masks(offsets, states)
    bits = torch.from_numpy(plain.label_masks(g, P, np.arange(S + 1), np.arange(S))).to(DEV)  # of each state alone
    want = bits[states[:2 * N:2].long()] | bits[states[1:2 * N:2].long()]
    assert torch.equal(got, want)


@pytest.mark.parametrize("S,A,P,hub", [(30_000, 90_000, 3000, 400), (30_000, 90_000, 120_000, 50), (30_000, 120_000, 500_000, 9)])
@pytest.mark.parametrize("rows,most", [(2, 30_000), (1, 40_000), (5, 70_000)])
def test_several_workgroups_a_row(wf, S, A, P, hub, rows, most):
    """Sets of 8192 states and more on average: parts of a row joined in memory."""
    g = wide_graph(S, A, P, S + P, hub)
    graph = wf.Graph(g, P)
    rng = np.random.default_rng([rows, most, P])
    counts = rng.integers(most // 2, most + 1, rows)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    states = rng.integers(0, S // 3, int(offsets[-1])).astype(np.int32)  # (many labels of many states, others of none)
    assert len(states) // rows >= 8192
    wide = torch.full((rows, (P + 31) // 32 + 3), 7, dtype=torch.int32, device=DEV)
    out = wide[:, :(P + 31) // 32]
    graph.label_masks(torch.from_numpy(offsets).to(DEV), torch.from_numpy(states).to(DEV), out=out)
    assert np.array_equal(out.cpu().numpy(), plain.label_masks(g, P, offsets, states))
    assert bool((wide[:, (P + 31) // 32:] == 7).all())
