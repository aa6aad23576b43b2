"""Cross entropy straight from hidden rows and its gradients (cross_entropy,
cross_entropy_grads, wd_cross_entropy*) against a plain 64-bit implementation,
within the bounds of 32-bit sums and one rounding of dz: types, odd sizes,
strides, rows without labels, infinities beside them, pieces, captured graphs."""
import math

import pytest
import torch

import plain_fit as plain
from plain_scores import close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def wf():
    from paper_1804_03243_amd import wfstdec
    assert torch.cuda.is_available()
    wfstdec.lib()
    return wfstdec


def make(N, D, P, dtype, seed=0, sure=2.0):
    """Rows that lean towards their labels; some labels outside the range."""
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    weight = (2.0 * rnd(P, D) / D ** 0.5).to(dtype)
    target = torch.randint(0, P, (N,), generator=gen, dtype=torch.int32)
    x = (rnd(N, D) + sure * weight[target.long()].float()).to(dtype)
    target[torch.rand(N, generator=gen) < 0.15] = -1
    target[torch.rand(N, generator=gen) < 0.05] = P
    return dict(x=x, weight=weight, target=target, bias=rnd(P), grad=torch.rand(N, generator=gen) / N)


def on(d):
    return {k: v.to(DEV) for k, v in d.items()}


def check(got, d, names=("loss", "dx", "dweight", "dbias")):
    want = plain.cross_entropy(d["x"], d["weight"], d["target"], d.get("bias"), d.get("grad"))
    for v, name in zip(got, names):
        close(v, want[name], want["bounds"][name])


def both(wf, d):
    g = on(d)
    got = wf.cross_entropy_grads(g["x"], g["weight"], g["target"], g.get("bias"), g.get("grad"))
    names = ("loss", "dx", "dweight", "dbias") if "bias" in d else ("loss", "dx", "dweight")
    check(got[:len(names)], d, names)
    loss = wf.cross_entropy(g["x"], g["weight"], g["target"], g.get("bias"))
    assert torch.equal(loss, got[0])
    return got


SIZES = [(1, 1, 1), (1, 8, 5), (2, 64, 16), (3, 100, 63), (15, 31, 64), (16, 32, 65), (17, 129, 257), (64, 512, 500),
         (65, 72, 300), (100, 1000, 77), (129, 200, 129), (200, 64, 1000), (300, 320, 520), (520, 128, 2049), (1, 64, 5000),
         (1500, 72, 40), (700, 96, 1264)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N,D,P", SIZES)
def test_sizes(wf, dtype, N, D, P):
    both(wf, make(N, D, P, dtype, seed=N + D))


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_tiles_of_every_size(wf, dtype):
    """Products that take the largest tiles and the middle ones, each with ragged ends."""
    both(wf, make(4099, 72, 4104, dtype, seed=1))
    both(wf, make(2000, 104, 1801, dtype, seed=2))


def on_gpu(d, got):
    """The same checks, the 64-bit products on the GPU (for sizes that the CPU takes long for)."""
    x, w = d["x"].double(), d["weight"].double()
    N, (P, D) = len(x), w.shape
    has = (d["target"] >= 0) & (d["target"] < P)
    label = d["target"].long().clamp(0, P - 1)[:, None]
    z = x @ w.T + d["bias"].double()
    err = (D + 8) * plain.EPS * (x.abs() @ w.abs().T + d["bias"].double().abs()).amax(1)
    loss = torch.where(has, torch.logsumexp(z, 1) - z.gather(1, label)[:, 0], 0.0)
    lerr = 3 * err + (P / 64 + 64) * plain.EPS + 16 * plain.EPS * z.abs().amax(1)
    close(got[0], loss.cpu(), (lerr + plain.EPS * loss).cpu())
    top = z.amax(1, keepdim=True)
    dz = torch.exp(z.sub_(top))
    dz /= dz.sum(1, keepdim=True)
    dz.scatter_add_(1, label, -torch.ones(label.shape, dtype=torch.float64, device=DEV))
    dz *= torch.where(has, d["grad"].double(), 0.0)[:, None]
    rel, least = plain.rounding(d["x"].dtype)
    least = least * 2.0 ** -13 * float(d["grad"].max()) if d["x"].dtype is F16 else least
    # (an error of a probability is at most that of its logit and of the sum, relative to it; near the label's 1 it is
    # as much of 1 - p as of p)
    slack = dz.abs().mul_(rel).add_(least)
    more = (lerr + 2 * err)[:, None] * torch.where(has, d["grad"].double(), 0.0)[:, None]
    for v, want, bound in ((got[1], dz @ w, slack @ w.abs() + 2 * more * w.abs().amax(0) + (P + 16) * plain.EPS * (dz.abs() @ w.abs())),
                           (got[2], dz.T @ x, slack.T @ x.abs() + dz.abs().T @ (x.abs() * (lerr + 2 * err)[:, None])
                            + label_slack(d, label, more, x) + (N + 16) * plain.EPS * (dz.abs().T @ x.abs()))):
        close(v, want.cpu(), (bound * (1 + rel) + rel * want.abs() + plain.rounding(v.dtype)[1]).cpu())
    be = dz.abs().T @ (lerr + 2 * err) + label_slack(d, label, more, torch.ones((N, 1), dtype=torch.float64, device=DEV))[:, 0]
    close(got[3], dz.sum(0).cpu(), (be + (N + 16) * plain.EPS * dz.abs().sum(0)).cpu())


def label_slack(d, label, more, x):
    out = torch.zeros((len(d["weight"]), x.shape[1]), dtype=torch.float64, device=DEV)
    return out.index_add_(0, label[:, 0], more * x.abs())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N,D,P", [(2300, 40, 120_001), (300_001, 24, 1001), (70_000, 16, 300), (3, 16, 5_000_000)])
def test_pieces(wf, dtype, N, D, P):
    """Gradients in several pieces of the labels, and of the rows; losses in several launches."""
    d = on(make(N, D, P, dtype, seed=5))
    got = wf.cross_entropy_grads(d["x"], d["weight"], d["target"], d["bias"], d["grad"])
    on_gpu(d, got)


def test_without_bias_and_gradient(wf):
    d = make(90, 64, 200, BF16, seed=3)
    del d["bias"], d["grad"]
    assert both(wf, d)[3] is None
    d = make(90, 64, 200, F16, seed=3)
    del d["grad"]
    both(wf, d)


@pytest.mark.parametrize("N,D", [(5, 64), (70, 64), (5, 60), (300, 72)])
def test_strides_and_alignment(wf, N, D):
    """Rows inside wider tensors, starting at odd elements, NaNs beside them."""
    d = make(N, D, 70, BF16, seed=7)
    g = on(d)
    for first in (0, 1, 3, 8):
        x = torch.full((N, D + 13), math.nan, dtype=BF16, device=DEV)
        x[:, first:first + D] = g["x"]
        w = torch.full((70, D + 9), math.nan, dtype=BF16, device=DEV)
        w[:, first:first + D] = g["weight"]
        check(wf.cross_entropy_grads(x[:, first:first + D], w[:, first:first + D], g["target"], g["bias"], g["grad"]), d)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_rows_left_out_reach_nothing(wf, dtype):
    """Infinities and NaNs in rows without a label or with gradient 0."""
    d = make(300, 64, 90, dtype, seed=11)
    d["target"][:20] = -1
    d["target"][20:40] = 3
    d["grad"][20:40] = 0.0
    d["x"][:10] = math.nan
    d["x"][10:20] = math.inf
    d["x"][20:30] = -math.inf
    d["x"][30:40] = math.nan
    g = on(d)
    loss, dx, dw, db = wf.cross_entropy_grads(g["x"], g["weight"], g["target"], g["bias"], g["grad"])
    assert bool((loss[:20] == 0).all()) and bool((dx[:40] == 0).all())
    assert bool(torch.isnan(loss[20:40]).all())
    d["x"][:40] = 0.0  # what stands there does not matter
    d["target"][20:40] = -1
    loss[20:40] = 0.0
    check((loss, dx, dw, db), d)


def test_nan_rows_with_labels_show(wf):
    d = make(100, 64, 90, BF16, seed=12)
    d["target"][:] = 5
    d["x"][7] = math.nan
    g = on(d)
    loss, dx, dw, db = (t.cpu() for t in wf.cross_entropy_grads(g["x"], g["weight"], g["target"], g["bias"], g["grad"]))
    assert bool(torch.isnan(loss[7])) and bool(torch.isfinite(loss[torch.arange(100) != 7]).all())
    assert bool(torch.isnan(dx[7]).all()) and bool(torch.isfinite(dx[torch.arange(100) != 7]).all())
    assert bool(torch.isnan(dw).all()) and bool(torch.isnan(db).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_labels_switched_off(wf, dtype):
    """Biases of -inf: no probability, no gradient; a label there costs +inf."""
    d = make(80, 64, 150, dtype, seed=13)
    off = torch.arange(150) % 3 == 0
    d["bias"][off] = -math.inf
    d["target"][:] = torch.where(torch.arange(80) < 70, 1, 3).int()
    got = both(wf, d)
    assert bool(torch.isinf(got[0][70:]).all())
    d["target"][:] = 1
    got = both(wf, d)
    assert bool((got[2].cpu()[off] == 0).all())


@pytest.mark.parametrize("P", [5, 64, 300])
def test_rows_without_any_logit(wf, P):
    d = make(40, 32, P, BF16, seed=14)
    d["bias"][:] = -math.inf
    d["target"][:] = 1
    d["target"][:5] = -1
    loss, dx, dw, db = (t.cpu() for t in wf.cross_entropy_grads(*(on(d)[k] for k in ("x", "weight", "target", "bias", "grad"))))
    assert bool((loss[:5] == 0).all()) and bool((loss[5:] == math.inf).all())
    assert not dx.any() and not dw.any() and not db.any()


def test_no_rows(wf):
    d = on(make(4, 32, 10, BF16))
    loss, dx, dw, db = wf.cross_entropy_grads(d["x"][:0], d["weight"], d["target"][:0], d["bias"], d["grad"][:0])
    assert loss.numel() == 0 and dx.shape == (0, 32) and not dw.any() and not db.any() and dw.shape == (10, 32)
    assert wf.cross_entropy(d["x"][:0], d["weight"], d["target"][:0]).shape == (0,)


@pytest.mark.parametrize("scale", [1e-30, 1e-8, 1.0, 1e6])
def test_half_precision_keeps_small_gradients(wf, scale):
    """Gradients far below half precision's range, and probabilities far below the largest.
    (Sizes whose outputs are half precision's normal numbers or its zeros: the bound counts both.)"""
    d = make(60, 64, 300, F16, seed=15, sure=4.0)
    d["grad"] = d["grad"] * scale
    if scale > 1:
        d["x"], d["weight"] = d["x"] / 16, d["weight"] / 16
    both(wf, d)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_gradients_against_differences(wf, dtype):
    """The gradients predict how the loss changes along a direction."""
    d = make(50, 64, 120, dtype, seed=16)
    g = on(d)
    loss, dx, dw, db = wf.cross_entropy_grads(g["x"], g["weight"], g["target"], g["bias"], g["grad"])
    gen = torch.Generator().manual_seed(1)
    for what, slope in (("x", dx), ("weight", dw), ("bias", db)):
        v = torch.randn(d[what].shape, generator=gen, dtype=torch.float64)
        h = 1e-4
        total = []
        for s in (1, -1):
            at = {k: d[k].double() + (s * h * v if k == what else 0) for k in ("x", "weight", "bias")}
            z = at["x"] @ at["weight"].T + at["bias"]
            has = (d["target"] >= 0) & (d["target"] < 120)
            t = d["target"].long().clamp(0, 119)
            each = torch.logsumexp(z, 1) - z[torch.arange(50), t]
            total.append(float((each * d["grad"].double() * has).sum()))
        want = (total[0] - total[1]) / (2 * h)
        slack = plain.cross_entropy(**d)["bounds"][{"x": "dx", "weight": "dweight", "bias": "dbias"}[what]]
        # (the second difference's error: h^2 / 6 times a third derivative of the order of |v|^3 of the logits' change)
        assert abs(float((slope.cpu().double() * v).sum()) - want) <= float((slack * v.abs()).sum()) + 1e-5


@pytest.mark.parametrize("N,P", [(3, 50), (200, 700)])
def test_autograd(wf, N, P):
    d = make(N, 40, P, BF16, seed=17)
    g = on(d)
    x, w, b = (g[k].clone().requires_grad_() for k in ("x", "weight", "bias"))
    h = x * 1.0  # (a row with a history)
    loss = wf.cross_entropy(h, w, g["target"], b)
    (loss * g["grad"]).sum().backward()
    check((loss, x.grad, w.grad, b.grad), d)
    # a part of the gradients
    w.grad = None
    wf.cross_entropy(g["x"], w, g["target"], g["bias"]).sum().backward()
    check((w.grad,), {k: v for k, v in d.items() if k != "grad"}, ("dweight",))
    with torch.no_grad():
        assert not wf.cross_entropy(x, w, g["target"], b).requires_grad
    twice = torch.autograd.grad(wf.cross_entropy(x, w, g["target"], b).sum(), w, create_graph=True)[0]
    with pytest.raises(RuntimeError):
        twice.float().sum().backward()


def test_an_adapter_is_more_columns(wf):
    """W x + s B (A x) is [W, s B] [x; A x]: gradients of A and B through autograd."""
    N, D, P, R = 120, 64, 90, 8
    d = make(N, D, P, BF16, seed=18)
    g = on(d)
    gen = torch.Generator().manual_seed(2)
    A, B = ((0.3 * torch.randn(s, generator=gen)).to(BF16).to(DEV).requires_grad_() for s in ((R, D), (P, R)))
    u = (g["x"].float() @ A.float().T).to(BF16)
    loss = wf.cross_entropy(torch.cat([g["x"], u], 1), torch.cat([g["weight"], 0.5 * B], 1), g["target"], g["bias"])
    (loss * g["grad"]).sum().backward()
    e = dict(d, x=torch.cat([d["x"], u.detach().cpu()], 1), weight=torch.cat([d["weight"], 0.5 * B.detach().cpu()], 1))
    want = plain.cross_entropy(**e)
    close(loss, want["loss"], want["bounds"]["loss"])
    # (two more roundings: of 0.5 B's gradient, exact, and of u's on its way to A)
    close(B.grad, 0.5 * want["dweight"][:, D:], 0.5 * want["bounds"]["dweight"][:, D:])
    wa = want["dx"][:, D:].T @ d["x"].double()
    ba = want["bounds"]["dx"][:, D:].T @ d["x"].double().abs()
    close(A.grad, wa, ba + 2 ** -8 * wa.abs() + (N + 8) * 2 ** -24 * (want["dx"][:, D:].abs().T @ d["x"].double().abs()) + 1e-30)


def test_same_bits_every_time(wf):
    d = on(make(700, 128, 900, BF16, seed=19))
    first = wf.cross_entropy_grads(d["x"], d["weight"], d["target"], d["bias"], d["grad"])
    for _ in range(3):
        again = wf.cross_entropy_grads(d["x"], d["weight"], d["target"], d["bias"], d["grad"])
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_another_stream(wf):
    d = make(400, 64, 500, BF16, seed=20)
    g = on(d)
    x = torch.zeros_like(g["x"])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
        x.copy_(g["x"])
        got = wf.cross_entropy_grads(x, g["weight"], g["target"], g["bias"], g["grad"])
    s.synchronize()
    check(got, d)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_captured_step(wf, dtype):
    """Two captured steps replayed several times, with eager work between them."""
    sets = [make(n, 64, p, dtype, seed=21 + n) for n, p in ((150, 300), (70, 900))]
    gs = [on(d) for d in sets]
    call = lambda g: wf.cross_entropy_grads(g["x"], g["weight"], g["target"], g["bias"], g["grad"])  # noqa: E731
    eager = [call(g) for g in gs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for g in gs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(g))
        graphs.append(graph)
    for turn in range(4):
        for i in (0, 1):
            for o in outs[i]:
                o.fill_(7.0)
            graphs[i].replay()
            if turn % 2:
                call(gs[1 - i])
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], eager[i]))
    # new inputs in the same places
    new = make(150, 64, 300, dtype, seed=99)
    for k, v in new.items():
        gs[0][k].copy_(v)
    graphs[0].replay()
    torch.cuda.synchronize()
    check(outs[0], new)


def test_autograd_under_capture_is_refused(wf):
    g = on(make(10, 32, 20, BF16))
    w = g["weight"].clone().requires_grad_()
    loss = wf.cross_entropy(g["x"], w, g["target"], g["bias"])
    graph = torch.cuda.CUDAGraph()
    a = torch.zeros(1, device=DEV)
    with torch.cuda.graph(graph):
        a += 1
        with pytest.raises(ValueError, match="captured"):
            wf.cross_entropy(g["x"], w, g["target"], g["bias"])
    loss.sum().backward()
    assert w.grad is not None


def test_refusals(wf):
    d = on(make(10, 32, 20, BF16))
    x, w, t, b = d["x"], d["weight"], d["target"], d["bias"]
    for bad in (lambda: wf.cross_entropy(x.float(), w, t, b), lambda: wf.cross_entropy(x.float(), w.float(), t, b),
                lambda: wf.cross_entropy(x.half(), w, t, b), lambda: wf.cross_entropy(x, w, t.long(), b),
                lambda: wf.cross_entropy(x, w, t[:9], b), lambda: wf.cross_entropy(x, w, t, b.to(BF16)),
                lambda: wf.cross_entropy(x, w[:, :31], t, b), lambda: wf.cross_entropy(x.T, w, t, b),
                lambda: wf.cross_entropy(x, w, None, b), lambda: wf.cross_entropy(x.cpu(), w, t, b),
                lambda: wf.cross_entropy(x, w, t, b[:19]), lambda: wf.cross_entropy_grads(x, w, t, b, d["grad"].to(BF16)),
                lambda: wf.cross_entropy_grads(x, w, t, b, d["grad"][:9])):
        with pytest.raises(ValueError):
            bad()


def test_blocks_of_rows(wf):
    """Losses in several launches, the last of a few rows (other tiles than the others')."""
    N, D, P = 4096 * 2 + 40, 16, 140_001  # (blocks of 4096 rows)
    d = on(make(N, D, P, BF16, seed=8))
    loss = wf.cross_entropy(d["x"], d["weight"], d["target"], d["bias"])
    has = (d["target"] >= 0) & (d["target"] < P)
    for a in range(0, N, 2048):
        r = slice(a, min(a + 2048, N))
        z = d["x"][r].double() @ d["weight"].double().T + d["bias"].double()
        err = (D + 8) * plain.EPS * (d["x"][r].double().abs() @ d["weight"].double().abs().T + d["bias"].double().abs()).amax(1)
        want = torch.where(has[r], torch.logsumexp(z, 1) - z.gather(1, d["target"][r].long().clamp(0, P - 1)[:, None])[:, 0], 0.0)
        slack = 3 * err + (P / 64 + 64) * plain.EPS + 16 * plain.EPS * z.abs().amax(1) + plain.EPS * want
        close(loss[r], want.cpu(), slack.cpu())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N", [1, 2, 64])
def test_few_rows_are_rounded_once(wf, dtype, N):
    """Up to 64 rows dz has two terms: the gradients are those of exact ones rounded, but for
    32-bit sums and what two terms leave (2^-17 of a value in bfloat16, 2^-22 in half precision)."""
    d = make(N, 96, 200, dtype, seed=31 + N)
    d["target"][0] = 7
    d["x"][0] *= 0.25  # (not sure of its label)
    g = on(d)
    want = plain.cross_entropy(**d)
    got = wf.cross_entropy_grads(g["x"], g["weight"], g["target"], g["bias"], g["grad"])
    rel, least = plain.rounding(dtype)
    terms = {BF16: 2.0 ** -16, F16: 2.0 ** -21}[dtype]
    z = d["x"].double() @ d["weight"].double().T + d["bias"].double()
    p = torch.softmax(z, 1)
    # (a logit's 32-bit error, the sum's and the exponential's, relative to each probability)
    logit = (104 * plain.EPS * (d["x"].double().abs() @ d["weight"].double().abs().T + d["bias"].double().abs())).amax(1, keepdim=True)
    dz = (4 * logit + 96 * plain.EPS + 8 * plain.EPS * (z.amax(1, keepdim=True) - z).abs()) * p * d["grad"].double()[:, None]
    size = (p * d["grad"].double()[:, None])
    has = (d["target"] >= 0) & (d["target"] < 200)
    size[has, d["target"][has].long()] += d["grad"].double()[has]
    for v, k, err in ((got[1], "dx", (dz + (terms + 500 * plain.EPS) * size) @ d["weight"].double().abs()),
                      (got[2], "dweight", (dz + (terms + 500 * plain.EPS) * size).T @ d["x"].double().abs())):
        small = 2.0 ** -38 * float(d["grad"].max()) * 300 * 8 if dtype is F16 else 0.0  # (what half precision's second term cannot hold)
        close(v, want[k], err * (1 + rel) + rel * want[k].abs() + least + small)
