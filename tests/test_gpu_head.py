"""Projection with low-rank adapters (Head.project, wd_project) against a plain
64-bit implementation, within the bounds of 32-bit sums: types, odd sizes,
strides, ranks, rows of many adapters in any order, infinities beside them."""
import pytest
import torch

import plain_scores as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def wf():
    from paper_1804_03243_amd import wfstdec
    assert torch.cuda.is_available()
    wfstdec.lib()
    return wfstdec


def make(N, D, P, G, R, dtype, seed=0, adapters="mixed"):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    d = dict(x=rnd(N, D).to(dtype), weight=(rnd(P, D) / D ** 0.5).to(dtype), bias=rnd(P))
    if G:
        d.update(a=(rnd(G, R, D) / D ** 0.5).to(dtype), b=(rnd(G, P, R) / R ** 0.5).to(dtype),
                 scale=torch.rand(G, generator=gen) + 0.5)
        if adapters == "mixed":  # any order, some without, some out of range
            d["adapter"] = torch.randint(-2, G + 1, (N,), generator=gen, dtype=torch.int32)
        elif adapters == "runs":
            d["adapter"] = (torch.arange(N) * G // max(N, 1)).to(torch.int32)
        else:
            d["adapter"] = (torch.arange(N) % G).to(torch.int32)
    return d


def head_of(wf, d):
    on = lambda k: d[k].to(DEV) if k in d else None  # noqa: E731
    return wf.Head(on("weight"), on("bias"), on("a"), on("b"), on("scale"))


def check(wf, d, out_dtype=F32):
    y = head_of(wf, d).project(d["x"].to(DEV), d["adapter"].to(DEV) if "adapter" in d else None, out_dtype=out_dtype)
    want, bound = plain.project(d["x"], d["weight"], d.get("bias"), d.get("a"), d.get("b"), d.get("scale"),
                                d.get("adapter"), out_dtype)
    plain.close(y, want, bound)
    return y


@pytest.mark.parametrize("dtype,same", [(BF16, False), (F16, False), (BF16, True), (F16, True)])
@pytest.mark.parametrize("N,D,P,G,R", [
    (1, 1, 1, 1, 1), (1, 8, 5, 2, 3), (2, 64, 16, 1, 8), (3, 100, 63, 3, 7), (15, 32, 64, 4, 16), (16, 31, 65, 16, 2),
    (17, 129, 257, 5, 17), (33, 512, 500, 33, 8), (64, 256, 130, 64, 16), (65, 72, 300, 7, 12), (100, 1000, 77, 9, 33),
    (129, 200, 129, 3, 64), (200, 64, 1000, 200, 4), (300, 320, 520, 6, 128), (520, 128, 513, 40, 16), (700, 96, 264, 2, 5),
])
def test_sizes(wf, dtype, same, N, D, P, G, R):
    check(wf, make(N, D, P, G, R, dtype, seed=N + D), dtype if same else F32)


@pytest.mark.parametrize("adapters", ["runs", "cycle", "mixed"])
@pytest.mark.parametrize("N", [40, 260, 1030])
def test_orders_of_adapters(wf, adapters, N):
    check(wf, make(N, 128, 192, 13, 16, BF16, seed=N, adapters=adapters))


@pytest.mark.parametrize("N", [1, 20, 300])
def test_without_adapters_bias_or_scale(wf, N):
    d = make(N, 96, 130, 0, 0, F16, seed=N)
    del d["bias"]
    check(wf, d)
    d = make(N, 96, 130, 3, 8, F16, seed=N)
    del d["scale"]
    check(wf, d)
    none = dict(d, adapter=torch.full((N,), -1, dtype=torch.int32))
    y = check(wf, none)
    z = head_of(wf, d).project(d["x"].to(DEV))  # no adapter given: the shared layer
    assert torch.equal(y, z)


def test_large_problem_many_tiles(wf):
    """Rows and outputs beyond several tiles of every size, against 64 bits on the GPU."""
    N, D, P, G, R = 4099, 328, 2056, 11, 24
    d = make(N, D, P, G, R, BF16, seed=3, adapters="runs")
    y = head_of(wf, d).project(d["x"].to(DEV), d["adapter"].to(DEV)).cpu().double()
    X, W = d["x"].double(), d["weight"].double()
    want = X @ W.T + d["bias"].double()
    mag = X.abs() @ W.abs().T + d["bias"].double().abs()
    low = torch.zeros(N, P, dtype=torch.float64)
    for g in range(G):
        r = d["adapter"] == g
        low[r] = float(d["scale"][g]) * ((X[r].abs() @ d["a"][g].double().abs().T) @ d["b"][g].double().abs().T)
        want[r] += float(d["scale"][g]) * ((X[r] @ d["a"][g].double().T) @ d["b"][g].double().T)
    bound = (D + 8) * plain.EPS * mag + ((D + 2 * R + 16) * plain.EPS + 2.0 ** -16) * low + plain.EPS * want.abs()
    plain.close(y, want, bound)


@pytest.mark.parametrize("N,D", [(5, 64), (70, 64), (5, 60), (300, 72)])
def test_strides_and_alignment(wf, N, D):
    """Rows inside wider tensors, starting at odd elements; columns beside the output stay."""
    P, G, R = 70, 3, 6
    d = make(N, D, P, G, R, BF16, seed=7)
    for first in (0, 1, 3, 8):
        wide = torch.full((N, D + 13), float("nan"), dtype=BF16, device=DEV)
        wide[:, first:first + D] = d["x"].to(DEV)
        wwide = torch.full((P, D + 9), float("nan"), dtype=BF16, device=DEV)
        wwide[:, first:first + D] = d["weight"].to(DEV)
        head = wf.Head(wwide[:, first:first + D], d["bias"].to(DEV), d["a"].to(DEV), d["b"].to(DEV), d["scale"].to(DEV))
        for dtype in (F32, BF16):
            owide = torch.full((N + 2, P + 5), 7.0, dtype=dtype, device=DEV)
            out = owide[1:N + 1, first % 4:first % 4 + P]
            assert head.project(wide[:, first:first + D], d["adapter"].to(DEV), out=out) is out
            want, bound = plain.project(d["x"], d["weight"], d["bias"], d["a"], d["b"], d["scale"], d["adapter"], dtype)
            plain.close(out, want, bound)
            owide[1:N + 1, first % 4:first % 4 + P] = 7.0
            assert bool((owide == 7.0).all())


@pytest.mark.parametrize("N", [6, 40, 300])
def test_other_rows_adapters_do_not_reach_a_row(wf, N):
    """Infinite and NaN adapters: only the rows that use them see them."""
    d = make(N, 64, 80, 4, 8, BF16, seed=11)
    d["b"][1] = float("inf")
    d["a"][2] = float("nan")
    y = head_of(wf, d).project(d["x"].to(DEV), d["adapter"].to(DEV)).cpu()
    hit = (d["adapter"] == 1) | (d["adapter"] == 2)
    want, bound = plain.project(d["x"], d["weight"], d["bias"], d["a"], d["b"], d["scale"], d["adapter"])
    plain.close(y[~hit], want[~hit], bound[~hit])
    assert not torch.isfinite(y[hit]).any()
    x = d["x"].clone()
    x[N // 2] = float("inf")  # nor does a row reach another row
    z = head_of(wf, d).project(x.to(DEV), d["adapter"].to(DEV)).cpu()
    rest = (torch.arange(N) != N // 2) & ~hit
    assert torch.equal(z[rest], y[rest])
    assert not torch.isfinite(z[N // 2]).any()


@pytest.mark.parametrize("N", [3, 50, 280])
def test_half_precision_low_rank_beyond_its_range(wf, N):
    """A_g x above 65504 and far below 2^-24: held with the row's exponent."""
    d = make(N, 64, 48, 4, 8, F16, seed=5)
    d["a"][0] *= 3000.0
    d["x"][: N // 2] *= 100.0
    d["b"][0] /= 3000.0
    d["scale"][1] = 1e-9
    d["scale"][2] = 1e6
    d["b"][2] *= 1e-3
    check(wf, d)


def test_weights_changed_in_place_and_repeated_calls(wf):
    d = make(40, 64, 96, 3, 8, BF16, seed=9)
    head, x, g = head_of(wf, d), d["x"].to(DEV), d["adapter"].to(DEV)
    y = head.project(x, g)
    assert torch.equal(y, head.project(x, g))
    head._kept[0].mul_(2.0)
    head._kept[3].mul_(2.0)
    d["weight"], d["b"] = d["weight"] * 2, d["b"] * 2
    want, bound = plain.project(d["x"], d["weight"], d["bias"], d["a"], d["b"], d["scale"], d["adapter"])
    plain.close(head.project(x, g), want, bound)


def test_empty_and_other_stream(wf):
    d = make(30, 64, 96, 3, 8, BF16, seed=2)
    head = head_of(wf, d)
    x, g = d["x"].to(DEV), d["adapter"].to(DEV)
    assert tuple(head.project(x[:0], g[:0]).shape) == (0, 96)
    want = head.project(x, g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = head.project(x, g)
    s.synchronize()
    assert torch.equal(y, want)


def test_rows_beyond_32_bit_offsets(wf):
    """Rows and outputs whose element offsets pass 2^31."""
    N, D, P, ld = 40, 64, 96, 1 << 26
    d = make(N, D, P, 3, 8, BF16, seed=4)
    wide = torch.empty((N, ld), dtype=BF16, device=DEV)
    wide[:, :D] = d["x"].to(DEV)
    owide = torch.empty((N, ld), dtype=BF16, device=DEV)
    out = head_of(wf, d).project(wide[:, :D], d["adapter"].to(DEV), out=owide[:, :P])
    want, bound = plain.project(d["x"], d["weight"], d["bias"], d["a"], d["b"], d["scale"], d["adapter"], BF16)
    plain.close(out, want, bound)


def test_graph_capture_replays(wf):
    """Recorded into a graph and replayed with new rows: the eager result each time."""
    d = make(64, 128, 160, 5, 8, BF16, seed=6)
    head, x, g = head_of(wf, d), d["x"].to(DEV), d["adapter"].to(DEV)
    out = torch.empty((64, 160), device=DEV)
    head.project(x, g, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        head.project(x, g, out=out)
    for k in range(4):
        x.copy_(torch.roll(d["x"], k, 0).to(DEV))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, head.project(x, g))


def test_refusals(wf):
    d = make(8, 64, 32, 3, 8, BF16)
    on = {k: v.to(DEV) for k, v in d.items()}
    head = head_of(wf, d)
    for bad in (on["x"].float(), on["x"][:, :60], on["x"].cpu(), on["x"].t(), on["x"][0]):
        with pytest.raises(ValueError):
            head.project(bad)
    for bad in (on["adapter"].long(), on["adapter"][:5], d["adapter"]):
        with pytest.raises(ValueError):
            head.project(on["x"], bad)
    with pytest.raises(ValueError):
        head.project(on["x"], out_dtype=F16)
    with pytest.raises(ValueError):
        head.project(on["x"], out=torch.empty((8, 31), device=DEV))
    with pytest.raises(ValueError):
        wf.Head(on["weight"].float())
    with pytest.raises(ValueError):
        wf.Head(on["weight"], on["bias"][:5])
    with pytest.raises(ValueError):
        wf.Head(on["weight"], None, on["a"])
    with pytest.raises(ValueError):
        wf.Head(on["weight"], None, on["a"], on["b"][:, :5])
    with pytest.raises(wf.WdError):
        wf.Head(on["weight"], None, torch.zeros((1, 129, 64), dtype=BF16, device=DEV),
                torch.zeros((1, 32, 129), dtype=BF16, device=DEV))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("run", [1000, 70, 33, 5])
@pytest.mark.parametrize("N,P,R", [(1300, 1000, 16), (8300, 2100, 8), (8300, 2100, 40), (8300, 2100, 12)])
def test_runs_of_adapters_in_large_tiles(wf, dtype, run, N, P, R):
    """Tiles of one, two, several and many adapters, with rows of none between; the same
    rows come out where another adapter is infinite."""
    D, G = 72, 40
    d = make(N, D, P, G, R, dtype, seed=run + R, adapters="runs")
    d["adapter"] = ((torch.arange(N) // run) % (G + 1)).to(torch.int32)  # (G: out of range, none)
    head = head_of(wf, d)
    x, g = d["x"].to(DEV), d["adapter"].to(DEV)
    y = head.project(x, g)
    X, W = d["x"].double().to(DEV), d["weight"].double().to(DEV)
    want = X @ W.T + d["bias"].double().to(DEV)
    mag = X.abs() @ W.abs().T + d["bias"].double().abs().to(DEV)
    low = torch.zeros_like(want)
    for k in range(G):
        r = g == k
        A, B, s = d["a"][k].double().to(DEV), d["b"][k].double().to(DEV), float(d["scale"][k])
        low[r] = s * ((X[r].abs() @ A.abs().T) @ B.abs().T)
        want[r] += s * ((X[r] @ A.T) @ B.T)
    bound = (D + 8) * plain.EPS * mag + ((D + 2 * R + 16) * plain.EPS + 2.0 ** -16) * low + plain.EPS * want.abs()
    off = (y.double() - want).abs() - bound
    assert float(off.max()) <= 0
    head._kept[3][3] = float("inf")
    z = head.project(x, g)
    hit = g == 3
    assert not torch.isfinite(z[hit]).any()
    off = (z[~hit].double() - want[~hit]).abs() - bound[~hit]
    assert float(off.max()) <= 0


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N,D,P,G,R", [
    (1, 3, 40, 2, 2), (40, 3, 1, 2, 2), (1, 7, 1, 1, 1), (300, 7, 90, 1, 1), (30, 2, 300, 3, 1), (70, 200, 1, 2, 3), (600, 90, 7, 1, 1),
    (1, 9, 1, 1, 1), (9, 9, 9, 1, 1), (3, 15, 17, 1, 9), (90, 17, 3, 2, 2), (530, 8, 33, 1, 1), (700, 33, 10, 1, 15), (90, 9, 1, 90, 9),
])
def test_small_arrays_and_their_last_elements(wf, dtype, N, D, P, G, R):
    """Arrays of less than a load, and those whose last rows end inside one."""
    check(wf, make(N, D, P, G, R, dtype, seed=N + D + P), F32)


@pytest.mark.parametrize("N,D,P,G,R", [(66, 300, 700, 66, 9), (128, 512, 1000, 20, 16), (250, 1133, 500, 250, 38), (500, 96, 200, 60, 5)])
def test_blocks_of_rows_of_many_adapters(wf, N, D, P, G, R):
    d = make(N, D, P, G, R, BF16, seed=N + R)
    y = check(wf, d)
    d["b"][int(d["adapter"][N - 1])] = float("inf")  # only its own rows change
    z = head_of(wf, d).project(d["x"].to(DEV), d["adapter"].to(DEV))
    same = d["adapter"] != d["adapter"][N - 1]
    assert torch.equal(y.cpu()[same], z.cpu()[same])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("G", [0, 1, 3])
@pytest.mark.parametrize("N,D,P", [(2, 1, 40), (7, 1, 3), (8, 1, 3), (2, 3, 40), (3, 2, 7), (4, 2, 7), (40, 1, 5), (40, 3, 2),
                                   (5, 1, 8), (2, 4, 2), (2, 5, 1), (300, 1, 2), (600, 2, 3)])
def test_arrays_that_end_before_a_load_does(wf, dtype, G, N, D, P):
    """Rows and weights of fewer than eight elements in all, and of just as many."""
    check(wf, make(N, D, P, G, 2, dtype, seed=N + D + P), F32)


def test_parameters_given_other_memory(wf):
    """A head reads the memory that it was made with, also when the module's parameters
    have moved on and nobody else holds it."""
    d = make(40, 64, 96, 3, 8, BF16, seed=12)
    layer = torch.nn.Linear(64, 96).to(BF16).to(DEV)
    layer.weight.data.copy_(d["weight"])
    params = {k: torch.nn.Parameter(d[k].to(DEV)) for k in ("bias", "a", "b", "scale")}
    head = wf.Head(layer.weight, *(params[k] for k in ("bias", "a", "b", "scale")))
    layer.half()
    for p in params.values():
        p.data = torch.zeros_like(p.data)
    taken = [torch.full((k,), float("nan"), dtype=BF16, device=DEV) for k in (96 * 64, 3 * 8 * 64, 3 * 96 * 8, 2 * 96, 2 * 3)
             for _ in range(4)]  # (memory that was given back would be taken by these)
    y = head.project(d["x"].to(DEV), d["adapter"].to(DEV))
    plain.close(y, *plain.project(d["x"], d["weight"], d["bias"], d["a"], d["b"], d["scale"], d["adapter"]))
    del taken


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_more_rows_than_a_launch_takes(wf, dtype):
    """Rows whose 16-row tiles would be 2^32 threads, in one call."""
    N, D, P, G, R = (1 << 28) + 21, 8, 2, 3, 3
    d = make(4096, D, P, G, R, dtype, seed=13)
    x = d["x"].to(DEV).repeat(N // 4096 + 1, 1)[:N]
    g = d["adapter"].to(DEV).repeat(N // 4096 + 1)[:N]
    y = head_of(wf, d).project(x, g, out_dtype=dtype)
    want, bound = plain.project(d["x"], d["weight"], d["bias"], d["a"], d["b"], d["scale"], d["adapter"], dtype)
    plain.close(y[:4096], want, bound)
    for n0 in range(4096, N, 4096):  # (the rows repeat)
        if n0 % (1 << 26) == 0 or N - n0 < 8192:
            plain.close(y[n0:n0 + 4096], want[:N - n0], bound[:N - n0])
    assert torch.equal(y[4096:1 << 27].view(-1, 4096, P), y[:4096].expand((1 << 27) // 4096 - 1, 4096, P))
    assert torch.equal(y[1 << 27:1 << 28].view(-1, 4096, P), y[:4096].expand((1 << 27) // 4096, 4096, P))


def test_gradients_are_refused_not_lost(wf):
    d = make(8, 64, 32, 3, 8, BF16)
    head, x = head_of(wf, d), d["x"].to(DEV)
    y = head.project(x)
    p = torch.nn.Parameter(x.clone())
    for call in (lambda: head.project(p), lambda: head.project(p * 2), lambda: head.project(x, out=torch.nn.Parameter(y.clone()))):
        with pytest.raises(ValueError, match="no backward"):
            call()
    with torch.no_grad():
        assert torch.equal(head.project(p), y)
    assert torch.equal(head.project(p.detach()), y)
    # (weights are taken detached)
    assert torch.equal(wf.Head(torch.nn.Parameter(d["weight"].to(DEV)), d["bias"].to(DEV)).project(x), y)


@pytest.mark.parametrize("dtype,same", [(BF16, False), (F16, False), (BF16, True)])
@pytest.mark.parametrize("N,D,P,R,run", [(3, 64, 80, 8, 1), (10, 64, 80, 12, 3), (60, 72, 130, 40, 20), (200, 64, 96, 8, 200), (200, 64, 96, 40, 64),
                                         (300, 333, 70, 5, 300), (700, 64, 1000, 16, 256), (700, 64, 1000, 9, 30), (700, 64, 1000, 96, 100),
                                         (8300, 72, 2100, 16, 1000), (8300, 72, 2100, 70, 1000), (1300, 77, 2100, 12, 700)])
def test_own_adapters_infinities(wf, dtype, same, N, D, P, R, run):
    """Infinite weights of a row's own adapter: the formula's infinities, not NaN."""
    G = 4
    d = make(N, D, P, G, R, dtype, seed=N + R, adapters="runs")
    d["adapter"] = ((torch.arange(N) // run) % (G + 1)).to(torch.int32)
    gen = torch.Generator().manual_seed(N)
    for k, v in enumerate([float("inf"), float("-inf"), float("inf")]):
        at = torch.randint(0, G, (5,), generator=gen), torch.randint(0, P, (5,), generator=gen), torch.randint(0, R, (5,), generator=gen)
        d["b"][at] = v
    d["b"][0, P // 2, R - 1] = float("inf")
    check(wf, d, dtype if same else F32)


@pytest.mark.parametrize("adapters", ["runs", "mixed"])
@pytest.mark.parametrize("N,D,P,R", [(10, 16, 48, 8), (100, 16, 96, 12), (400, 24, 300, 8), (700, 16, 96, 8), (1300, 24, 1000, 20),
                                     (8300, 16, 2100, 8)])
def test_half_precision_ranks_far_below_the_others(wf, adapters, N, D, P, R):
    """Single ranks of A scaled down and the same columns of B up: their A x is held
    to 16 bits of its own, not of the row's largest."""
    d = make(N, D, P, 3, R, F16, seed=N + D, adapters=adapters)
    for r, by in ((1, 12), (4, 9), (R - 1, 13)):
        d["a"][:, r] *= 2.0 ** -by
        d["b"][:, :, r] *= 2.0 ** by
    check(wf, d)


def check_on_gpu(wf, d, out_dtype=F32):
    """As check(), in 64 bits on the GPU, for rows of sorted adapters."""
    dev = {k: v.to(DEV) for k, v in d.items()}
    y = head_of(wf, d).project(dev["x"], dev["adapter"], out_dtype=out_dtype)
    X, W, R = dev["x"].double(), dev["weight"].double(), d["a"].shape[1]
    rel, least = plain.rounding(out_dtype)
    worst = 0.0
    for g in range(-1, d["a"].shape[0]):
        rows = torch.nonzero(dev["adapter"] == g)[:, 0]
        for r in rows.split(4096) if len(rows) else ():
            want = X[r] @ W.T + dev["bias"].double()
            err = (X.shape[1] + 8) * plain.EPS * (X[r].abs() @ W.abs().T + dev["bias"].double().abs())
            if g >= 0:
                A, B, s = dev["a"][g].double(), dev["b"][g].double(), float(d["scale"][g])
                u, um = s * (X[r] @ A.T), s * (X[r].abs() @ A.abs().T)
                want += u @ B.T
                err += ((X.shape[1] + 2 * R + 16) * plain.EPS * um + 2.0 ** -16 * u.abs()) @ B.abs().T
            off = (y[r].double() - want).abs() - (err * (1 + rel) + rel * want.abs() + least)
            worst = max(worst, float(off.max()))
    assert worst <= 0.0
    return y


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("run", [2000, 700, 41])
@pytest.mark.parametrize("N,D,P,R", [(2000, 333, 1600, 11), (300, 333, 70, 5), (2000, 1027, 1601, 16), (150, 777, 500, 40)])
def test_unaligned_rows_of_many_steps(wf, dtype, run, N, D, P, R):
    """Widths that are no multiple of eight, in tiles of 64 and of 128: the rows of
    later steps go through registers while earlier ones are multiplied."""
    d = make(N, D, P, 3, R, dtype, seed=N + D, adapters="runs")
    d["adapter"] = ((torch.arange(N) // run + 1) % 4 - 1).to(torch.int32)
    check_on_gpu(wf, d)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("run", [5000, 900, 90, 7])
@pytest.mark.parametrize("N,D,P,R", [(2500, 128, 1300, 65), (2500, 136, 1300, 100), (4500, 64, 4200, 128), (4500, 72, 4100, 81)])
def test_ranks_above_64_in_large_tiles(wf, dtype, run, N, D, P, R):
    d = make(N, D, P, 3, R, dtype, seed=N + R, adapters="runs")
    d["adapter"] = ((torch.arange(N) // run + 1) % 4 - 1).to(torch.int32)
    check_on_gpu(wf, d)


@pytest.mark.parametrize("dtype,out", [(BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)])
@pytest.mark.parametrize("D", [72, 77])
@pytest.mark.parametrize("P", [8001, 8004])
def test_outputs_past_the_caches(wf, dtype, out, D, P):
    """256 MB of outputs and more, rows that do not end at a whole store."""
    N = 17003 if out is not F32 else 8503
    d = make(N, D, P, 3, 8, dtype, seed=N + P, adapters="runs")
    d["adapter"] = ((torch.arange(N) // 1500 + 1) % 4 - 1).to(torch.int32)
    assert N * P * (4 if out is F32 else 2) >= 256 << 20
    check_on_gpu(wf, d, out)
