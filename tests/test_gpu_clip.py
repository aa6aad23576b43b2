"""The norm over many gradients and their clipping (clip_gradients, wd_clip_gradients)
against a plain 64-bit implementation: types, sizes from one value to several chunks,
more tensors than a launch takes, odd addresses, outputs apart, values that are not
finite, captured graphs, refusals."""
import math

import pytest
import torch

import plain_fit as plain
from plain_scores import EPS, rounding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def wf():
    from paper_1804_03243_amd import wfstdec
    assert torch.cuda.is_available()
    wfstdec.lib()
    return wfstdec


def make(sizes, dtype, seed=0):
    """Values of different sizes; a list of types is gone round."""
    gen = torch.Generator().manual_seed(seed)
    types = dtype if isinstance(dtype, list) else [dtype]
    return [(torch.randn(n, generator=gen) * 2.0 ** (i % 7 - 3)).to(types[i % len(types)]) for i, n in enumerate(sizes)]


def check(norm, got, tensors, max_norm):
    want, scaled = plain.clip(tensors, max_norm)
    # (the sum in 64 bits; one rounding of its root)
    assert norm.dtype is F32 and norm.dim() == 0 and abs(float(norm) - want) <= 2 * EPS * want
    for g, t in zip(got, scaled):
        rel, least = rounding(g.dtype)
        # the factor's rounding, the product's, the type's
        assert bool(((g.cpu().double() - t).abs() <= (rel + 2.1 * EPS) * t.abs() + least).all())


SIZES = [[1], [3], [7, 0, 9], [255, 256, 257, 1], [16384], [16383, 16385], [100_003, 5], list(range(1, 66)), [1000] * 64, [33] * 200]


@pytest.mark.parametrize("dtype", [F32, F16, BF16, [F32, BF16, F16]])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("share", [0.3, 1.7])
def test_in_place(wf, dtype, sizes, share):
    tensors = make(sizes, dtype, seed=len(sizes))
    max_norm = share * plain.clip(tensors, 1.0)[0]
    on = [t.to(DEV) for t in tensors]
    norm = wf.clip_gradients(on, max_norm)
    check(norm, on, tensors, max_norm)
    if share > 1:
        assert all(torch.equal(a.cpu(), b) for a, b in zip(on, tensors))


@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, BF16), ([F32, BF16], F32)])
@pytest.mark.parametrize("share", [0.3, 1.7])
def test_into_other_tensors(wf, dtype, out, share):
    tensors = make([5, 16384, 40_001, 1], dtype, seed=3)
    max_norm = share * plain.clip(tensors, 1.0)[0]
    on, to = [t.to(DEV) for t in tensors], [torch.full(t.shape, 7.0, dtype=out, device=DEV) for t in tensors]
    check(wf.clip_gradients(on, max_norm, out=to), to, tensors, max_norm)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(on, tensors))
    # in place and apart in one call
    both = [on[0], to[1], on[2], to[3]]
    check(wf.clip_gradients(on, max_norm, out=both), both, tensors, max_norm)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first", [0, 1, 3])
def test_parts_of_tensors(wf, dtype, first):
    """Tensors that begin at odd elements of one buffer; what stands between them stays."""
    tensors = make([700, 33, 16400], dtype, seed=4)
    buf = torch.full((20_000,), 7.0, dtype=dtype, device=DEV)
    views, at = [], first
    for t in tensors:
        views.append(buf[at:at + len(t)].copy_(t.to(DEV)))
        at += len(t) + 5
    check(wf.clip_gradients(views, 1.0), views, tensors, 1.0)
    for v in views:
        v.fill_(7.0)
    assert bool((buf == 7.0).all())


def test_shapes_and_many_values(wf):
    """Matrices, and more chunks than a launch has workgroups."""
    tensors = [t.view(-1, 8) for t in make([8 * 5_000_000, 8 * 3], BF16, seed=5)]
    on = [t.to(DEV) for t in tensors]
    check(wf.clip_gradients(on, 2.0), on, tensors, 2.0)


def test_extreme_values(wf):
    for v in (1e30, 3e38, 1e-30, 1e-45):  # squares that 32 bits do not hold
        t = torch.tensor([v, -v, 0.0, v], dtype=F32)
        on = [t.to(DEV)]
        norm = wf.clip_gradients(on, v)
        want, scaled = plain.clip([t], float(v))
        assert abs(float(norm) - want) <= 2 * EPS * want + 2 ** -150 or want > 3.4e38 and float(norm) == math.inf
        assert bool(((on[0].cpu().double() - scaled[0]).abs() <= 3.1 * EPS * scaled[0].abs() + 2.0 ** -150).all())


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(wf, bad):
    tensors = make([1000, 20_000], BF16, seed=6)
    tensors[1][77] = bad
    on, to = [t.to(DEV) for t in tensors], [torch.zeros(t.shape, device=DEV) for t in tensors]
    norm = float(wf.clip_gradients(on, 1.0))
    assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
    assert all(torch.equal(a.cpu().view(torch.int16), b.view(torch.int16)) for a, b in zip(on, tensors))
    wf.clip_gradients(on, 1.0, out=to)
    assert all(torch.equal(torch.nan_to_num(a.cpu()), torch.nan_to_num(b.float())) for a, b in zip(to, tensors))


def test_limits(wf):
    tensors = make([100, 200], F32, seed=7)
    on = [t.to(DEV) for t in tensors]
    check(wf.clip_gradients(on, math.inf), on, tensors, math.inf)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(on, tensors))
    check(wf.clip_gradients(on, 0.0), on, tensors, 0.0)
    assert not any(t.any() for t in on)
    assert float(wf.clip_gradients(on, 0.0)) == 0.0
    assert float(wf.clip_gradients([torch.empty(0, device=DEV)], 1.0)) == 0.0


def test_same_bits_every_time(wf):
    tensors = make([100_000, 7, 50_000], F32, seed=8)
    norms = {float(wf.clip_gradients([t.to(DEV) for t in tensors], math.inf)) for _ in range(5)}
    assert len(norms) == 1


def test_captured(wf):
    """Two captured calls replayed several times on new values, eager ones between them."""
    sizes = [[40_000, 3], [17] * 100]
    on = [[torch.zeros(n, device=DEV) for n in s] for s in sizes]
    to = [[torch.zeros(n, dtype=BF16, device=DEV) for n in s] for s in sizes]
    wf.clip_gradients(on[0], 1.0)
    torch.cuda.synchronize()
    graphs, norms = [], []
    for i in (0, 1):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norms.append(wf.clip_gradients(on[i], 1.5, out=to[i]))
        graphs.append(graph)
    for turn in range(4):
        tensors = [make(s, F32, seed=20 + turn) for s in sizes]
        for i in (0, 1):
            for a, b in zip(on[i], tensors[i]):
                a.copy_(b)
            graphs[i].replay()
        if turn % 2:
            wf.clip_gradients([on[0][0].clone()], 2.0)
            torch.cuda.synchronize()
        for i in (0, 1):
            check(norms[i], to[i], tensors[i], 1.5)


def test_another_stream(wf):
    tensors = make([50_000], F32, seed=9)
    on = [torch.zeros(50_000, device=DEV)]
    src = tensors[0].to(DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
        on[0].copy_(src)
        norm = wf.clip_gradients(on, 1.0)
    s.synchronize()
    check(norm, on, tensors, 1.0)


def test_refusals(wf):
    t = torch.ones(100, device=DEV)
    for bad in (lambda: wf.clip_gradients([], 1.0), lambda: wf.clip_gradients([t.cpu()], 1.0), lambda: wf.clip_gradients([t.double()], 1.0),
                lambda: wf.clip_gradients([t[::2]], 1.0), lambda: wf.clip_gradients([t], 1.0, out=[]),
                lambda: wf.clip_gradients([t.clone().requires_grad_()], 1.0), lambda: wf.clip_gradients([t], 1.0, out=[t.clone().requires_grad_()]),
                lambda: wf.clip_gradients([t], 1.0, out=[t[:50]]), lambda: wf.clip_gradients([t], 1.0, out=[t.int()])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: wf.clip_gradients([t, t], 1.0), lambda: wf.clip_gradients([t[:60], t[50:]], 1.0),
                lambda: wf.clip_gradients([t[:50]], 1.0, out=[t[25:75]]), lambda: wf.clip_gradients([t[:50], t[50:]], 1.0, out=[t[50:], t[:50]]),
                lambda: wf.clip_gradients([t], -1.0), lambda: wf.clip_gradients([t], math.nan)):
        with pytest.raises(wf.WdError, match="WD_EINVAL"):
            bad()
    assert bool((t == 1).all())
    # read twice, written apart: no harm
    a, b = torch.empty(100, device=DEV), torch.empty(100, device=DEV)
    assert abs(float(wf.clip_gradients([t, t], math.inf, out=[a, b])) - math.sqrt(200)) < 1e-5
    assert torch.equal(a, t) and torch.equal(b, t)
