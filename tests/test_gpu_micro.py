"""Microscaled 4-bit matrices and the output layer that holds its weights so (micro,
Micro.values, MicroHead, wd_micro_*): codes, scales and values equal to the
definition's, products within the bound of 32-bit sums."""
import math

import pytest
import torch

import plain_fit as plain
from plain_scores import EPS, close, rounding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def wf():
    from paper_1804_03243_amd import wfstdec
    assert torch.cuda.is_available()
    wfstdec.lib()
    return wfstdec


def codes_of(m):
    """(codes [rows, D], scale bytes [rows, ceil(D/32)]) of a Micro, by its layout."""
    c = m.codes.cpu().long()
    both = torch.stack([c & 15, c >> 4], 2).view(m.rows, -1)
    assert not both[:, m.D:].any()
    b = torch.arange((m.D + 31) // 32)
    at = b // 16 * 16 + b % 4 * 4 + b // 4 % 4
    scales = m.scales.cpu().long()
    rest = torch.ones(scales.shape[1], dtype=torch.bool)
    rest[at] = False
    assert not scales[:, rest].any()
    return both[:, :m.D], scales[:, at]


def check(wf, x, on=None):
    m = wf.micro(x.to(DEV) if on is None else on)
    codes, scales = codes_of(m)
    want, wscales = plain.micro(x)
    assert torch.equal(scales, wscales) and torch.equal(codes, want)
    values = plain.micro_values(want, wscales)
    for dtype in (BF16, F32):
        v = m.values(dtype)
        assert v.dtype is dtype
        close(v, values, torch.zeros_like(values))
    return m


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,D", [(1, 1), (1, 31), (2, 32), (3, 33), (5, 64), (2, 500), (3, 512), (2, 520), (1, 1000), (33, 7), (4, 1064)])
def test_codes(wf, dtype, rows, D):
    gen = torch.Generator().manual_seed(rows + D)
    x = torch.randn((rows, D), generator=gen) * torch.exp(2 * torch.randn((rows, 1), generator=gen))
    check(wf, x.to(dtype))


def test_every_border(wf):
    """All values between the codes, ties among them, at several powers of two."""
    steps = torch.arange(-64, 65) / 8.0
    x = torch.stack([torch.cat([s, torch.full((160 - 129,), 7.5)]) for s in (steps, steps)])  # (a block's largest below 8)
    for power in (0, 5, -9, 100, -100):
        check(wf, x * 2.0 ** power)
        check(wf, (x * 2.0 ** power).to(BF16))


def test_extreme_values(wf):
    x = torch.zeros(12, 64)
    x[1, 3] = 2.0 ** -149
    x[2, :4] = torch.tensor([2.0 ** -127, 2.0 ** -128, 2.0 ** -129, -(2.0 ** -128)])
    x[3, :4] = torch.tensor([2.0 ** -124, 2.0 ** -126, 2.0 ** -127, 1.5 * 2.0 ** -127])
    x[4, :3] = torch.tensor([3.4e38, -1e38, 1e30])
    x[5, 0], x[6, 40], x[7, 1] = math.inf, -math.inf, math.nan
    x[8, :2] = torch.tensor([1.0, -1e-30])
    x[9] = -0.0
    x[10, :2] = torch.tensor([7.0, 8.0])
    x[11, :2] = torch.tensor([-7.999, 0.25])
    check(wf, x)
    check(wf, x.to(BF16))
    check(wf, x[5:].to(F16))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(wf, dtype):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((9, 100), generator=gen).to(dtype)
    for first in (0, 1, 3):
        wide = torch.full((9, 111), math.nan, dtype=dtype, device=DEV)
        wide[:, first:first + 100] = x.to(DEV)
        check(wf, x, wide[:, first:first + 100])


def test_large_matrix(wf):
    """More values than a launch has threads, against elementary operations."""
    x = (torch.randn((70_000, 1000), generator=torch.Generator(DEV).manual_seed(1), device=DEV)).to(BF16)
    got = wf.micro(x).values()
    v = torch.nn.functional.pad(x.double(), (0, 24)).view(70_000, 32, 32)
    unit = torch.exp2(torch.floor(torch.log2(v.abs().amax(2, keepdim=True))) - 2)
    y = v / unit
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    want = (torch.clamp(torch.round(y / step) * step, -6, 6) * unit).view(70_000, -1)[:, :1000]
    assert torch.equal(got.double(), want)


def project(wf, x, w, bias, out_dtype=F32, out=None, rows=None):
    head = wf.MicroHead(wf.micro(w.to(DEV)), None if bias is None else bias.to(DEV))
    y = head.project(x.to(DEV) if rows is None else rows, out=out, out_dtype=out_dtype)
    X, W = plain.micro_values(*plain.micro(x)), plain.micro_values(*plain.micro(w))
    want, mag = X @ W.T, X.abs() @ W.abs().T
    if bias is not None:
        want, mag = want + bias.double(), mag + bias.double().abs()
    rel, least = rounding(out_dtype)
    err = (x.shape[1] + 8) * EPS * mag
    close(y, want, err * (1 + rel) + rel * want.abs() + least)
    return y


@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F16), (F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("N,D,P", [(1, 1, 1), (1, 8, 5), (2, 64, 16), (3, 100, 63), (16, 31, 65), (17, 129, 257), (33, 520, 40), (64, 256, 130),
                                   (65, 72, 300), (40, 1100, 77), (129, 200, 129), (200, 64, 300)])
def test_products(wf, dtype, out, N, D, P):
    gen = torch.Generator().manual_seed(N + D)
    project(wf, torch.randn((N, D), generator=gen).to(dtype), torch.randn((P, D), generator=gen).to(dtype) / D ** 0.5,
            torch.randn(P, generator=gen), out)


@pytest.mark.parametrize("N,D,P", [(5000, 328, 2056), (300, 1100, 6000), (1, 512, 100_000), (64, 96, 30_000), (2100, 72, 2100),
                                   (20, 200, 20_001), (8, 1100, 4001), (9, 600, 4001), (32, 2000, 17_000), (6500, 40, 15_000)])
def test_large_products(wf, N, D, P):
    """Tiles of every size, against 64 bits on the GPU."""
    gen = torch.Generator(DEV).manual_seed(N)
    x = torch.randn((N, D), generator=gen, device=DEV).to(BF16)
    w = wf.micro(torch.randn((P, D), generator=gen, device=DEV))
    bias = torch.randn(P, generator=gen, device=DEV)
    X, W = wf.micro(x).values(F32).double(), w.values(F32).double()
    want, mag = X @ W.T + bias.double(), X.abs() @ W.abs().T + bias.double().abs()
    for dtype in (F32, BF16):
        y = wf.MicroHead(w, bias).project(x, out_dtype=dtype)
        rel, least = rounding(dtype)
        close(y, want.cpu(), ((D + 8) * EPS * mag * (1 + rel) + rel * want.abs() + least).cpu())


@pytest.mark.parametrize("N", [3, 70, 300])
def test_output_strides(wf, N):
    """Columns and rows beside the output stay."""
    gen = torch.Generator().manual_seed(5)
    x, w = torch.randn((N, 64), generator=gen).to(BF16), torch.randn((70, 64), generator=gen)
    for dtype in (F32, BF16):
        for first in (0, 1, 3):
            wide = torch.full((N + 2, 75), 7.0, dtype=dtype, device=DEV)
            out = wide[1:N + 1, first:first + 70]
            assert project(wf, x, w, None, dtype, out) is out
            out.fill_(7.0)
            assert bool((wide == 7.0).all())


@pytest.mark.parametrize("N", [5, 80, 300])
def test_values_that_are_not_finite(wf, N):
    """Rows and outputs of such values are NaN, the others as without them."""
    gen = torch.Generator().manual_seed(6)
    x, w = torch.randn((N, 200), generator=gen), torch.randn((150, 200), generator=gen)
    x[2, 190], w[7, 3], w[149, 100] = math.inf, math.nan, -math.inf
    y = wf.MicroHead(wf.micro(w.to(DEV))).project(x.to(DEV)).cpu()
    X, W = plain.micro_values(*plain.micro(x)), plain.micro_values(*plain.micro(w))
    want, mag = X @ W.T, torch.nan_to_num(X).abs() @ torch.nan_to_num(W).abs().T
    want[2], want[:, 7], want[:, 149] = math.nan, math.nan, math.nan
    close(y, want, 208 * EPS * mag + EPS * torch.nan_to_num(want).abs())


def test_no_rows(wf):
    head = wf.MicroHead(wf.micro(torch.ones((10, 40), device=DEV)))
    assert head.project(torch.ones((0, 40), device=DEV)).shape == (0, 10)
    assert wf.micro(torch.ones((0, 40), device=DEV)).values().shape == (0, 40)


def test_weights_changed_in_place_are_read(wf):
    w = wf.micro(torch.ones((10, 40), device=DEV))
    head = wf.MicroHead(w)
    x = torch.ones((3, 40), device=DEV)
    assert bool((head.project(x) == 40).all())
    other = wf.micro(2 * torch.ones((10, 40), device=DEV))
    w.codes.copy_(other.codes)
    w.scales.copy_(other.scales)
    assert bool((head.project(x) == 80).all())
    again = wf.Micro(w.codes.clone(), w.scales.clone(), 40)
    assert torch.equal(again.values(), w.values())


def test_captured(wf):
    gen = torch.Generator(DEV).manual_seed(7)
    x = [torch.randn((n, 96), generator=gen, device=DEV).to(BF16) for n in (5, 200)]
    head = wf.MicroHead(wf.micro(torch.randn((300, 96), generator=gen, device=DEV)))
    eager = [head.project(v) for v in x]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for v in x:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(head.project(v))
        graphs.append(graph)
    for turn in range(4):
        for i in (0, 1):
            outs[i].fill_(7.0)
            graphs[i].replay()
        if turn % 2:
            head.project(x[0])
            torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))


def test_another_stream(wf):
    gen = torch.Generator(DEV).manual_seed(8)
    src = torch.randn((50, 96), generator=gen, device=DEV)
    head = wf.MicroHead(wf.micro(torch.randn((300, 96), generator=gen, device=DEV)))
    want = head.project(src)
    x = torch.zeros_like(src)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
        x.copy_(src)
        got = head.project(x)
    s.synchronize()
    assert torch.equal(got, want)


def test_refusals(wf):
    x = torch.ones((4, 40), device=DEV)
    m = wf.micro(x)
    head = wf.MicroHead(m)
    for bad in (lambda: wf.micro(x.double()), lambda: wf.micro(x[0]), lambda: wf.micro(x.T), lambda: wf.micro(x.clone().requires_grad_()),
                lambda: m.values(F16), lambda: wf.MicroHead(x), lambda: wf.MicroHead(m, torch.ones(5, device=DEV)),
                lambda: head.project(x[:, :39]), lambda: head.project(x, out_dtype=torch.int32), lambda: head.project(x.cpu()),
                lambda: head.project(x.clone().requires_grad_()), lambda: head.project(x, out=torch.empty((4, 5), device=DEV)),
                lambda: wf.Micro(m.codes, m.scales, 100), lambda: wf.Micro(m.codes[:3], m.scales, 40), lambda: wf.Micro(m.codes.int(), m.scales, 40)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("N", [3, 40, 300])
@pytest.mark.parametrize("power", [0, 60, -60, 100])
def test_products_of_far_apart_sizes(wf, N, power):
    """Rows and weights whose powers of two cancel in the product."""
    gen = torch.Generator().manual_seed(9)
    x, w = torch.randn((N, 130), generator=gen) * 2.0 ** power, torch.randn((100, 130), generator=gen) * 2.0 ** -power
    project(wf, x, w, None)
