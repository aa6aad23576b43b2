"""Logits to log-likelihoods (loglikes, wd_loglikes) against a plain 64-bit
implementation, within the bounds of 32-bit sums: types, lengths, penalties,
biases and masks, rows left empty, infinities and NaN."""
import numpy as np
import pytest
import torch

import plain_scores as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
INF = float("inf")


@pytest.fixture(scope="module")
def wf():
    from paper_1804_03243_amd import wfstdec
    assert torch.cuda.is_available()
    wfstdec.lib()
    return wfstdec


def lists(rng, Q, most, V, wild=True):
    counts = rng.integers(0, most + 1, Q)
    counts[rng.random(Q) < 0.2] = 0
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    ids = (V * rng.random(int(off[-1])) ** 2).astype(np.int32)
    if wild and len(ids) > 4:  # labels outside the row
        ids[rng.integers(0, len(ids), 3)] = [-1, V, 2 ** 31 - 1]
    return torch.from_numpy(off), torch.from_numpy(ids)


def make(N, V, dtype, seed=0, Q=None, history=0, biases=0, masks=0, prior=False):
    rng = np.random.default_rng([seed, N, V])
    gen = torch.Generator().manual_seed(seed + N + V)
    Q = Q or max(1, N // 2)
    d = dict(logits=(torch.randn((N, V), generator=gen) * 4).to(dtype),
             request=torch.from_numpy(rng.integers(-1, Q + 1, N).astype(np.int32)))
    if prior:
        d["log_prior"] = torch.log_softmax(torch.randn(V, generator=gen) * 2, 0)
    if history:
        d["history"] = lists(rng, Q, history, V)
        d["repetition"] = torch.rand(Q, generator=gen) + 0.6
        d["presence"] = torch.randn(Q, generator=gen)
        d["frequency"] = torch.rand(Q, generator=gen) * 0.3
    if biases:
        off, ids = lists(rng, Q, biases, V)
        d["bias"] = (off, ids, torch.randn(len(ids), generator=gen) * 3)
    if masks:
        keep = rng.random((masks, (V + 31) // 32 * 32)) < 0.5
        keep[0] = False  # a mask that leaves nothing
        d["mask"] = torch.from_numpy(np.packbits(keep, axis=1, bitorder="little").view("<i4").copy())
        d["mask_of"] = torch.from_numpy(rng.integers(-1, masks + 1, N).astype(np.int32))
    return d


def call(wf, d, **more):
    on = {k: tuple(t.to(DEV) for t in v) if isinstance(v, tuple) else v.to(DEV) if torch.is_tensor(v) else v
          for k, v in d.items()}
    return wf.loglikes(**on, **more)


def check(wf, d):
    y = call(wf, d)
    want, bound = plain.loglikes(**d)
    plain.close(y, want, bound)
    return y


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("N,V", [(1, 1), (2, 3), (3, 31), (2, 32), (5, 33), (4, 255), (3, 500), (2, 1023), (3, 3001),
                                 (2, 8191), (2, 8192), (2, 8193), (3, 16385), (2, 30000), (1, 32769), (1, 70001)])
def test_lengths(wf, dtype, normalize, N, V):
    d = make(N, V, dtype, history=50, biases=20, masks=3, prior=True)
    check(wf, dict(d, normalize=normalize, scale=0.7))


@pytest.mark.parametrize("part", ["plain", "history", "biases", "masks", "prior"])
@pytest.mark.parametrize("N,V", [(7, 200), (40, 6001), (3, 40001), (300, 64)])
def test_parts(wf, part, N, V):
    kw = {"plain": {}, "history": dict(history=300), "biases": dict(biases=100), "masks": dict(masks=4),
          "prior": dict(prior=True)}[part]
    check(wf, make(N, V, BF16, seed=1, **kw))


@pytest.mark.parametrize("V", [700, 20000, 50000])
def test_long_histories_and_repeated_biases(wf, V):
    """Histories longer than the row, one label over and over, biases given twice."""
    d = make(4, V, F32, seed=2, Q=3)
    ids = torch.cat([torch.full((30000,), 5, dtype=torch.int32), torch.arange(20000, dtype=torch.int32) % V])
    d["request"] = torch.tensor([0, 1, 2, 0], dtype=torch.int32)
    d["history"] = (torch.tensor([0, 50000, 50000, 50000]), ids)
    d["frequency"] = torch.full((3,), 1e-4)
    d["repetition"] = torch.full((3,), 1.3)
    d["bias"] = (torch.tensor([0, 2, 2000, 2003]), torch.arange(2003, dtype=torch.int32) % 90,
                 torch.randn(2003, generator=torch.Generator().manual_seed(3)))
    check(wf, d)


def test_only_some_penalties(wf):
    d = make(6, 300, F32, seed=3, history=40)
    for keep in ("repetition", "presence", "frequency"):
        check(wf, {k: v for k, v in d.items() if k not in ("repetition", "presence", "frequency") or k == keep})


@pytest.mark.parametrize("V", [90, 9000, 40000])
def test_rows_without_anything_left(wf, V):
    """Masks that leave nothing, rows of -inf, the type's lowest value as a mask."""
    d = make(6, V, F32, seed=4)
    z = d["logits"]
    z[1] = -INF
    z[2] = torch.finfo(F32).min
    z[3, : V // 2] = torch.finfo(F32).min
    z[4, 1:] = -INF
    d["mask"] = torch.full((6, (V + 31) // 32), -1, dtype=torch.int32)
    d["mask"][0] = 0
    y = check(wf, d)
    assert bool((y[:2] == -INF).all()) and float(y[4, 0]) == 0.0


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("V", [90, 9000, 40000])
def test_nan_and_infinities(wf, dtype, V):
    """In masked places they are not seen; elsewhere the row is NaN but for its masked places."""
    d = make(6, V, dtype, seed=5)
    z = d["logits"]
    d["mask"] = torch.full((6, (V + 31) // 32), -1, dtype=torch.int32)
    d["mask"][:4, 0] = ~0b111
    z[0, 0], z[1, 1], z[2, 2], z[3, 40], z[4, 50], z[5, 7] = float("nan"), INF, -INF, float("nan"), INF, -INF
    y = check(wf, d)
    assert torch.isfinite(y[:3, 3:]).all() and torch.isnan(y[3, 3:]).all() and torch.isnan(y[4]).all()
    check(wf, dict(d, normalize=False))


@pytest.mark.parametrize("first", [0, 1, 2, 5])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_alignment(wf, dtype, first):
    N, V = 9, 1234
    d = make(N, V, dtype, seed=6, masks=3, prior=True)
    wide = torch.full((N, V + 11), float("nan"), dtype=dtype, device=DEV)
    wide[:, first:first + V] = d["logits"].to(DEV)
    owide = torch.full((N + 2, V + 7), 3.0, device=DEV)
    out = owide[1:N + 1, first:first + V]
    assert call(wf, dict(d, logits=wide[:, first:first + V]), out=out) is out
    plain.close(out, *plain.loglikes(**d))
    owide[1:N + 1, first:first + V] = 3.0
    assert bool((owide == 3.0).all())


@pytest.mark.parametrize("V", [300, 9001, 40000])
def test_output_rows_and_in_place(wf, V):
    N = 7
    d = make(N, V, F32, seed=7, history=20)
    want, bound = plain.loglikes(**d)
    store = torch.full((12, V), 5.0, device=DEV)
    to = torch.tensor([11, 0, -1, 5, 12, 3, 7], dtype=torch.int32)
    call(wf, d, out=store, out_row=to.to(DEV))
    used = [(n, int(r)) for n, r in enumerate(to) if 0 <= r < 12]
    for n, r in used:
        plain.close(store[r:r + 1], want[n:n + 1], bound[n:n + 1])
    rest = [r for r in range(12) if r not in {r for _, r in used}]
    assert bool((store[rest] == 5.0).all())
    z = d["logits"].to(DEV).clone()
    call(wf, dict(d, logits=z), out=z)
    plain.close(z, want, bound)


def test_defaults_of_request_and_mask(wf):
    """Without request and mask_of row n is request n and has mask n."""
    d = make(6, 100, F32, seed=8, Q=4, history=30, masks=5)
    for k in ("request", "mask_of"):
        del d[k]
    check(wf, d)


def test_offsets_outside_their_lists(wf):
    """Offsets that decrease or pass the lists are clamped, never followed."""
    d = make(4, 100, F32, seed=9, Q=4, history=10, biases=10)
    n, m = len(d["history"][1]), len(d["bias"][1])
    d["request"] = torch.arange(4, dtype=torch.int32)
    d["history"] = (torch.tensor([-5, 3, 1, n + 100, 2 ** 40]), d["history"][1])
    d["bias"] = (torch.tensor([0, m, m + 7, 2, -9]), *d["bias"][1:])
    check(wf, d)


def test_many_rows_and_determinism(wf):
    d = make(3000, 501, BF16, seed=10, history=30, biases=9, masks=20, prior=True)
    y = check(wf, d)
    assert torch.equal(y.view(torch.int32), call(wf, d).view(torch.int32))


@pytest.mark.parametrize("V", [300, 20000, 50000])
def test_empty_other_stream_and_graph_replays(wf, V):
    d = make(8, V, F32, seed=11, history=30, biases=9, masks=4)
    on = {k: tuple(t.to(DEV) for t in v) if isinstance(v, tuple) else v.to(DEV) for k, v in d.items()}
    assert tuple(wf.loglikes(on["logits"][:0]).shape) == (0, V)
    want = wf.loglikes(**on)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = wf.loglikes(**on)
    s.synchronize()
    assert torch.equal(y, want)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wf.loglikes(**on, out=out)
    for k in range(4):
        on["logits"].copy_(torch.roll(d["logits"], k, 0).to(DEV))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, wf.loglikes(**on))


def test_rows_beyond_32_bit_offsets(wf):
    N, V, ld = 40, 200, 1 << 26
    d = make(N, V, BF16, seed=12, masks=3)
    wide = torch.empty((N, ld), dtype=BF16, device=DEV)
    wide[:, :V] = d["logits"].to(DEV)
    owide = torch.empty((N, ld), dtype=F32, device=DEV)
    out = call(wf, dict(d, logits=wide[:, :V]), out=owide[:, :V])
    plain.close(out, *plain.loglikes(**d))


def test_refusals(wf):
    d = make(5, 64, F32, Q=3, history=10, biases=10, masks=2, prior=True)
    z = d["logits"].to(DEV)
    on = {k: tuple(t.to(DEV) for t in v) if isinstance(v, tuple) else v.to(DEV) for k, v in d.items()}
    for bad in (z.double(), z.cpu(), z[0], z.t()):
        with pytest.raises((ValueError, RuntimeError)):
            wf.loglikes(bad, out=torch.empty((5, 64), device=DEV))
    for k, bad in (("log_prior", on["log_prior"][:3]), ("log_prior", on["log_prior"].half()), ("request", on["request"].long()),
                   ("request", on["request"][:2]), ("mask", on["mask"][:, :1]), ("mask", on["mask"].long()),
                   ("repetition", on["repetition"][:1]), ("history", on["history"][:1]), ("bias", on["bias"][:2]),
                   ("history", (on["history"][0].int(), on["history"][1])), ("out", torch.empty((5, 63), device=DEV)),
                   ("out", torch.empty((4, 64), device=DEV)), ("out_row", on["request"])):
        with pytest.raises(ValueError):
            wf.loglikes(**dict(on, **{k: bad}))
    with pytest.raises(ValueError):
        wf.loglikes(z, mask_of=on["mask_of"])
    with pytest.raises(ValueError):
        wf.loglikes(z, repetition=on["repetition"])
    for scale in (0.0, -1.0, INF, float("nan")):
        with pytest.raises(wf.WdError):
            wf.loglikes(z, scale=scale)


@pytest.mark.parametrize("V", [700, 20000, 50000])
@pytest.mark.parametrize("most", ["history", "biases", "both"])
def test_lists_beyond_16_bits(wf, V, most):
    """Histories and bias lists of more than 65535 entries, one label more often than that."""
    d = make(3, V, F32, seed=20, Q=2)
    d["request"] = torch.tensor([0, 1, 0], dtype=torch.int32)
    gen = torch.Generator().manual_seed(21)
    n = 70000 if most in ("history", "both") else 300
    ids = torch.randint(0, V, (n + 66000 * (n > 65536),), generator=gen, dtype=torch.int32)
    ids[n:] = 7
    d["history"] = (torch.tensor([0, len(ids) - 3, len(ids)]), ids)
    d["frequency"] = torch.full((2,), 1e-4)
    m = 70001 if most in ("biases", "both") else 200
    d["bias"] = (torch.tensor([0, m - 5, m]), torch.randint(0, V, (m,), generator=gen, dtype=torch.int32),
                 torch.randn(m, generator=gen))
    check(wf, d)


def test_more_rows_than_a_launch_takes(wf):
    """Rows beyond 2^32 threads, in one call."""
    N, V = (1 << 24) + 3, 2
    z = torch.randn((N, V), generator=torch.Generator(DEV).manual_seed(30), device=DEV)
    prior = torch.tensor([-0.5, -1.5], device=DEV)
    y = wf.loglikes(z, log_prior=prior, scale=0.5)
    want = 0.5 * (torch.log_softmax(z.double(), 1) - prior.double())
    # (three roundings of values below 16, those of the sum and the logarithm, halved)
    assert float((y.double() - want).abs().max()) <= 64 * 2.0 ** -24


def test_gradients_are_refused_not_lost(wf):
    d = make(5, 64, F32, Q=3, history=10, biases=10, prior=True)
    on = {k: tuple(t.to(DEV) for t in v) if isinstance(v, tuple) else v.to(DEV) for k, v in d.items()}
    want = wf.loglikes(**on)
    for k in ("logits", "log_prior", "repetition", "presence", "frequency"):
        with pytest.raises(ValueError, match="no backward"):
            wf.loglikes(**dict(on, **{k: on[k].clone().requires_grad_()}))
    with pytest.raises(ValueError, match="no backward"):
        wf.loglikes(**dict(on, bias=(*on["bias"][:2], on["bias"][2].clone().requires_grad_())))
    with torch.no_grad():
        assert torch.equal(wf.loglikes(**dict(on, logits=on["logits"].clone().requires_grad_())), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,V", [(13500, 5001), (2000, 33555)])
def test_outputs_past_the_caches(wf, dtype, N, V):
    """256 MB of outputs and more, rows that do not end at a whole store."""
    z = (torch.randn((N, V), generator=torch.Generator(DEV).manual_seed(31), device=DEV) * 3).to(dtype)
    prior = torch.log_softmax(torch.randn(V, generator=torch.Generator(DEV).manual_seed(32), device=DEV), 0)
    assert N * V * 4 >= 256 << 20
    y = wf.loglikes(z, log_prior=prior, scale=0.9)
    for n0 in range(0, N, 1000):
        x = z[n0:n0 + 1000].double()
        want = 0.9 * (torch.log_softmax(x, 1) - prior.double())
        # |x - max|, the sum's logarithm and the prior are below 64 together, each rounded
        # three times; the sum is of V terms over 64 lanes
        bound = 0.9 * (64 * 4 + V / 64 + 128) * plain.EPS
        assert float((y[n0:n0 + 1000].double() - want).abs().max()) <= bound


def test_lists_of_no_request(wf):
    """Offsets of one entry are lists of no request: an empty batch's, and rows without one."""
    d = make(4, 70, F32, seed=33, masks=2, prior=True)
    none, ids = torch.zeros(1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32)
    lists_ = dict(history=(none, ids), bias=(none, ids, torch.zeros(0)), repetition=torch.zeros(0), presence=torch.zeros(0),
                  frequency=torch.zeros(0))
    check(wf, dict(d, **lists_))
    empty = dict(d, logits=d["logits"][:0], request=d["request"][:0], mask_of=d["mask_of"][:0], **lists_)
    assert tuple(call(wf, empty).shape) == (0, 70)
    for bad in (dict(history=(none[:0], ids)), dict(bias=(none[:0], ids, torch.zeros(0)))):
        with pytest.raises(ValueError):
            call(wf, dict(d, **bad))


@pytest.mark.parametrize("given", [True, False])
def test_requests_and_masks_of_later_launches(wf, given):
    """Rows beyond the first launch keep their own request, mask and output row."""
    N, V, Q = (1 << 24) + 40, 3, (1 << 24) + 30  # (the last ten rows have no request and no mask of their own)
    gen = torch.Generator(DEV).manual_seed(34)
    z = torch.randn((N, V), generator=gen, device=DEV)
    off = torch.arange(Q + 1, device=DEV)  # (a label each)
    ids = torch.randint(0, V, (Q,), generator=gen, device=DEV, dtype=torch.int32)
    presence, values = torch.rand(Q, generator=gen, device=DEV), torch.randn(Q, generator=gen, device=DEV)
    mask = torch.randint(1, 8, (Q, 1), generator=gen, device=DEV, dtype=torch.int32)
    kw = {}
    if given:
        kw = dict(request=torch.arange(N, device=DEV, dtype=torch.int32), mask_of=torch.arange(N, device=DEV, dtype=torch.int32),
                  out_row=torch.arange(N - 1, -1, -1, device=DEV, dtype=torch.int32), out=torch.empty((N, V), device=DEV))
    y = wf.loglikes(z, normalize=False, history=(off, ids), presence=presence, bias=(off, ids, values), mask=mask, **kw)
    y = y.flip(0) if given else y
    want = z.clone()  # (in 32 bits: the presence off, then the bias on, each rounded once)
    at = ids.long()[:, None]
    want[:Q] = want[:Q].scatter(1, at, (want[:Q].gather(1, at) - presence[:, None]) + values[:, None])
    keep = (mask >> torch.arange(V, device=DEV)) & 1
    want[:Q] = torch.where(keep == 1, want[:Q], torch.full((), -INF, device=DEV))
    assert torch.equal(y, want)
