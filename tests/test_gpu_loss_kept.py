"""Gradients of wide layers formed together with their losses, whose exponentials are held
in 20 bits on the way (cross_entropy_grads of more than 64 rows and 512 columns or more),
against a plain 64-bit implementation: sizes at every border of the tiles, masks, infinities,
rows that are sure of a label, several launches, captured graphs."""
import math

import pytest
import torch

import plain_fit as plain
from test_gpu_loss import both, check, make, on, on_gpu, wf  # noqa: F401

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16
FIELDS = ("x", "weight", "target", "bias", "grad")


def grads(wf, d):
    return wf.cross_entropy_grads(*(d.get(k) for k in FIELDS))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N,D,P", [(65, 512, 1), (66, 520, 63), (64, 512, 100), (100, 777, 65), (129, 512, 64), (80, 1000, 513), (200, 513, 1025),
                                   (300, 2050, 40), (257, 512, 575), (1030, 512, 131)])
def test_sizes(wf, dtype, N, D, P):  # noqa: F811
    both(wf, make(N, D, P, dtype, seed=N + D))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N,D,P", [(2000, 520, 1801), (4099, 512, 4104), (9000, 512, 70), (4 * 4096 + 70, 512, 4100), (4300, 512, 131_100)])
def test_larger_tiles_and_several_launches(wf, dtype, N, D, P):  # noqa: F811
    d = on(make(N, D, P, dtype, seed=1))
    on_gpu(d, grads(wf, d))


def test_more_than_is_kept(wf):  # noqa: F811
    """Above the bytes that are kept, the logits are formed again."""
    d = on(make(17_000, 512, 131_200, BF16, seed=2))
    got = grads(wf, d)
    sub = slice(0, 17_000, 200)
    part = dict(d, **{k: d[k][sub].contiguous() for k in ("x", "target", "grad")})
    alone = grads(wf, part)
    # rows' own gradients do not hang on the others'; both roundings of dz, and of dx
    slack = 4 * 2.0 ** -8 * (alone[1].float().norm() + 1e-30)
    assert float((got[1][sub].float() - alone[1].float()).norm()) <= float(slack)
    assert float((got[0][sub] - alone[0]).abs().max()) <= 1e-4
    assert all(bool(torch.isfinite(t.float()).all()) for t in got)


def test_without_bias_and_gradient(wf):  # noqa: F811
    for dtype in (BF16, F16):
        d = make(90, 512, 200, dtype, seed=3)
        del d["bias"], d["grad"]
        assert both(wf, d)[3] is None


@pytest.mark.parametrize("first", [0, 1, 8])
def test_strides_and_alignment(wf, first):  # noqa: F811
    d = make(70, 517, 130, BF16, seed=7)
    g = on(d)
    x = torch.full((70, 517 + 13), math.nan, dtype=BF16, device=DEV)
    x[:, first:first + 517] = g["x"]
    w = torch.full((130, 517 + 9), math.nan, dtype=BF16, device=DEV)
    w[:, first:first + 517] = g["weight"]
    check(wf.cross_entropy_grads(x[:, first:first + 517], w[:, first:first + 517], g["target"], g["bias"], g["grad"]), d)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_rows_left_out_reach_nothing(wf, dtype):  # noqa: F811
    d = make(300, 512, 90, dtype, seed=11)
    d["target"][:20] = -1
    d["target"][20:40] = 3
    d["grad"][20:40] = 0.0
    d["x"][:10], d["x"][10:20], d["x"][20:30], d["x"][30:40] = math.nan, math.inf, -math.inf, math.nan
    loss, dx, dw, db = grads(wf, on(d))
    assert bool((loss[:20] == 0).all()) and bool((dx[:40] == 0).all()) and bool(torch.isnan(loss[20:40]).all())
    d["x"][:40] = 0.0  # what stands there does not matter
    d["target"][20:40] = -1
    loss[20:40] = 0.0
    check((loss, dx, dw, db), d)


def test_nan_and_infinite_rows_with_labels_show(wf):  # noqa: F811
    for value, where in ((math.nan, slice(None)), (math.inf, slice(0, 1))):
        d = make(100, 512, 90, BF16, seed=12)
        d["target"][:] = 5
        d["x"][7, where] = value
        loss, dx, dw, db = (t.cpu() for t in grads(wf, on(d)))
        rest = torch.arange(100) != 7
        assert bool(torch.isnan(loss[7])) and bool(torch.isfinite(loss[rest]).all())
        assert bool(torch.isnan(dx[7]).all()) and bool(torch.isfinite(dx[rest]).all())
        assert bool(torch.isnan(dw).all()) and bool(torch.isnan(db).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_labels_switched_off(wf, dtype):  # noqa: F811
    """Biases of -inf, of a whole block of labels too: no probability, no gradient; a label there costs +inf."""
    d = make(80, 512, 250, dtype, seed=13)
    off = (torch.arange(250) % 3 == 0) | ((torch.arange(250) >= 64) & (torch.arange(250) < 128))
    d["bias"][off] = -math.inf
    d["target"][:] = torch.where(torch.arange(80) < 70, 1, 100).int()
    got = both(wf, d)
    assert bool(torch.isinf(got[0][70:]).all())
    d["target"][:] = 1
    got = both(wf, d)
    assert bool((got[2].cpu()[off] == 0).all()) and bool((got[3].cpu()[off] == 0).all())


def test_rows_without_any_logit(wf):  # noqa: F811
    d = make(80, 512, 300, BF16, seed=14)
    d["bias"][:] = -math.inf
    d["target"][:], d["target"][:5] = 1, -1
    loss, dx, dw, db = (t.cpu() for t in grads(wf, on(d)))
    assert bool((loss[:5] == 0).all()) and bool((loss[5:] == math.inf).all())
    assert not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("sure", [0.0, 6.0, 20.0])
def test_rows_that_are_sure(wf, dtype, sure):  # noqa: F811
    """Logits that lean towards the label until hardly anything is left of the others, and
    towards a wrong one."""
    d = make(200, 512, 300, dtype, seed=15, sure=sure)
    d["target"][:50] = (d["target"][:50] + 1) % 300
    both(wf, d)


@pytest.mark.parametrize("scale", [1e-30, 1e-8, 1.0])
def test_half_precision_keeps_small_gradients(wf, scale):  # noqa: F811
    for N in (80, 4200):  # (the power of two in a launch of its own, and not)
        d = make(N, 512, 70, F16, seed=16, sure=3.0)
        d["grad"] = d["grad"] * scale
        both(wf, d)


def test_dbias_is_of_32_bits(wf):  # noqa: F811
    """The labels' own gradients do not carry the exponentials' 20 bits into db: 2^-20 of its norm."""
    d = make(3000, 512, 200, BF16, seed=17)
    want = plain.cross_entropy(**d)["dbias"]
    off = grads(wf, on(d))[3].cpu().double() - want
    assert float(off.norm() / want.norm()) < 2.0 ** -20


def test_same_bits_and_captured(wf):  # noqa: F811
    sets = [make(n, 512, p, BF16, seed=21 + n) for n, p in ((150, 300), (700, 900))]
    gs = [on(d) for d in sets]
    eager = [grads(wf, g) for g in gs]
    assert all(torch.equal(a, b) for g, e in zip(gs, eager) for a, b in zip(grads(wf, g), e))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for g in gs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(grads(wf, g))
        graphs.append(graph)
    for turn in range(4):
        for i in (0, 1):
            for o in outs[i]:
                o.fill_(7.0)
            graphs[i].replay()
            if turn % 2:
                grads(wf, gs[1 - i])
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], eager[i]))


def test_parts_of_the_gradients(wf):  # noqa: F811
    """Each gradient alone is what it is with the others; the losses may be left out."""
    d = on(make(90, 512, 150, BF16, seed=22))
    want = grads(wf, d)
    for wanted in ((True, False, False), (False, True, False), (False, False, True)):
        a = wf._loss_args(d["x"], d["weight"], d["target"], d["bias"])
        got = wf._loss_grads(a, d["x"], d["weight"], d["bias"], None, None, d["grad"], wanted)
        for g, w, is_wanted in zip(got, want[1:], wanted):
            if is_wanted:
                assert float((g.float() - w.float()).norm()) <= 2.0 ** -7 * float(w.float().norm())
            else:
                assert g is None


@pytest.mark.parametrize("N,P", [(300, 4_194_000), (300_000, 5000)])
def test_as_far_as_is_kept(wf, N, P):  # noqa: F811
    """Close to the most that is kept: as with the logits formed again, but for the roundings."""
    gen = torch.Generator(DEV).manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=gen, device=DEV)  # noqa: E731
    w, x = (rnd(P, 512) / 10).to(BF16), rnd(N, 512).to(BF16)
    t, g = torch.randint(-1, P, (N,), generator=gen, device=DEV, dtype=torch.int32), torch.rand(N, device=DEV) / N
    loss, dx, dw, db = wf.cross_entropy_grads(x, w, t, None, g)
    a = wf._loss_args(x, w, t, None)
    stats = torch.empty((N, 2), device=DEV)
    assert torch.equal(wf._loss(a, x.device, stats), loss)
    ex, ew, _ = wf._loss_grads(a, x, w, None, stats, None, g, (True, True, True))
    for v, e in ((dx, ex), (dw, ew)):
        assert bool(torch.isfinite(v).all())
        # (each within two roundings, of dz and its own, of the same values)
        assert float((v.float() - e.float()).norm()) <= 4 * 2.0 ** -8 * float(e.float().norm())
