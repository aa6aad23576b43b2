"""Argument checks of the operators that fit the output layer and hold it in four bits,
at the C ABI: they come before any device work, so no GPU is needed and the pointers
are never followed."""
import ctypes
import math
import os

import pytest

from paper_1804_03243_amd import build, wfstdec as wf


@pytest.fixture(scope="module", autouse=True)
def library():
    if not os.path.exists(wf.LIB_PATH):
        build.build()
    return wf.lib()


P = 0x10000  # an aligned address that nothing reads


def loss(**kw):
    d = dict(N=5, D=64, P=100, type=wf.WD_BF16, x=P, x_ld=64, weight=P, weight_ld=64, bias=P, target=P, loss=P, stats=P, grad=P,
             dx=P, dx_ld=64, dweight=P, dweight_ld=64, dbias=P)
    return wf.wd_loss_args(**{**d, **kw})


BAD = [dict(N=-1), dict(N=1 << 31), dict(D=0), dict(D=1 << 22), dict(P=0), dict(P=1 << 24), dict(type=wf.WD_F32), dict(type=9), dict(x_ld=63),
       dict(weight_ld=63), dict(weight=None), dict(x=None), dict(target=None), dict(x=P + 1), dict(weight=P + 1), dict(bias=P + 2),
       dict(target=P + 2), dict(loss=P + 2), dict(stats=P + 4)]
BAD_GRADS = [dict(dx_ld=63), dict(dweight_ld=63), dict(dx=None, dweight=None, dbias=None), dict(grad=P + 2), dict(dx=P + 1),
             dict(dweight=P + 1), dict(dbias=P + 2), dict(N=(1 << 19) + 1, P=(1 << 19) + 1)]


@pytest.mark.parametrize("bad", BAD + [dict(loss=None, stats=None)])
def test_losses(bad):
    for call in (lambda a: wf.wd_cross_entropy_workspace_bytes(a), lambda a: wf.wd_cross_entropy(a, P, 1 << 40, 0)):
        with pytest.raises(wf.WdError, match="WD_EINVAL"):
            call(loss(**bad))


@pytest.mark.parametrize("bad", BAD + BAD_GRADS)
def test_loss_gradients(bad):
    for call in (lambda a: wf.wd_cross_entropy_grads_workspace_bytes(a), lambda a: wf.wd_cross_entropy_grads(a, P, 1 << 40, 0)):
        with pytest.raises(wf.WdError, match="WD_EINVAL"):
            call(loss(**bad))


def test_loss_workspaces():
    for need, call in ((wf.wd_cross_entropy_workspace_bytes(loss()), wf.wd_cross_entropy),
                       (wf.wd_cross_entropy_grads_workspace_bytes(loss()), wf.wd_cross_entropy_grads)):
        assert need > 0
        for ws, n in ((None, need), (P, need - 1), (P + 4, need)):
            with pytest.raises(wf.WdError, match="workspace"):
                call(loss(), ws, n, 0)
    wf.wd_cross_entropy(loss(N=0, x=None, target=None, loss=None, stats=None), None, 0, 0)
    # what the workspace holds does not grow with rows times labels
    sizes = [wf.wd_cross_entropy_grads_workspace_bytes(loss(N=n, P=p)) for n, p in ((1 << 16, 1 << 14), (1 << 20, 1 << 14), (1 << 14, 1 << 20))]
    assert all(s < (1 << 31) for s in sizes)
    assert wf.wd_cross_entropy_workspace_bytes(loss(N=1 << 20, P=1 << 17)) < 1 << 26
    # (without stats the gradients may keep 2.6 bytes of each logit, up to 5.3 GB)
    need = lambda **kw: wf.wd_cross_entropy_grads_workspace_bytes(loss(stats=None, D=512, x_ld=512, weight_ld=512, dx_ld=512, dweight_ld=512, **kw))  # noqa: E731
    assert 1 << 31 < need(N=1 << 15, P=1 << 15) < 2.7 * 2 ** 30 + (1 << 30)
    assert all(need(N=n, P=p) < 7 * 2 ** 30 for n, p in ((1 << 16, 1 << 15), (1 << 17, 1 << 15), (1 << 14, 1 << 18), (1 << 19, 1 << 14)))
    # nothing is kept of outputs that a tile's offsets would not reach, or of very many rows
    assert need(N=500, P=(1 << 22) - 64) > 1 << 32 > need(N=500, P=1 << 22)
    assert need(N=1 << 24, P=64) < need(N=1 << 22, P=64) * 4


def clip(tensors, n=None, max_norm=1.0, norm=P, ws=P, ws_bytes=1 << 30):
    rows = [dict(dict(data=P * (2 + i), n=100, out=None, type=wf.WD_F32, out_type=0), **t) for i, t in enumerate(tensors)]
    table = (wf.wd_gradient * max(len(rows), 1))(*[wf.wd_gradient(**r) for r in rows])
    wf.wd_clip_gradients(table, len(rows) if n is None else n, max_norm, norm, ws, ws_bytes, 0)


@pytest.mark.parametrize("tensors", [[dict(n=-1)], [dict(n=2 ** 41)], [dict(type=3)], [dict(type=-1)], [dict(out=P * 9, out_type=7)], [dict(data=None)],
                                     [dict(data=P + 2)], [dict(data=P + 1, type=wf.WD_BF16)], [dict(out=P * 9 + 1, out_type=wf.WD_F16)],
                                     [dict(data=P * 2), dict(data=P * 2)], [dict(data=P * 2), dict(data=P * 2 + 396)],
                                     [dict(data=P * 2, out=P * 2 + 4)], [dict(data=P * 2, out=P * 2, out_type=wf.WD_BF16)],
                                     [dict(data=P * 2, out=P * 5), dict(data=P * 3, out=P * 5)], [dict(data=P * 2, out=P * 3), dict(data=P * 3, out=P * 2)],
                                     [dict(data=P)], [dict(data=P * 2, out=P * 3), dict(data=P * 3 + 200)]])
def test_clipping(tensors):
    with pytest.raises(wf.WdError, match="WD_EINVAL"):
        clip(tensors)


def test_clipping_arguments():
    for kw in (dict(n=-1), dict(n=(1 << 24) + 1), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(norm=None), dict(norm=P + 2), dict(ws=None),
               dict(ws=P + 4), dict(ws_bytes=16)):
        with pytest.raises(wf.WdError, match="WD_EINVAL"):
            clip([dict()], **kw)
    with pytest.raises(wf.WdError):
        wf.wd_clip_gradients(None, 3, 1.0, P, P, 1 << 20, 0)
    with pytest.raises(wf.WdError):
        wf.wd_clip_workspace_bytes(-1)
    assert wf.wd_clip_workspace_bytes(0) > 0


def micro(**kw):
    return wf.wd_micro(**{**dict(rows=100, D=64, codes=P, scales=P), **kw})


BAD_MICRO = [dict(rows=-1), dict(rows=1 << 31), dict(D=0), dict(D=1 << 22), dict(codes=None), dict(scales=None), dict(codes=P + 8), dict(scales=P + 8)]


@pytest.mark.parametrize("bad", BAD_MICRO)
def test_micro_matrices(bad):
    for call in (lambda m: wf.wd_micro_quantize(P, wf.WD_F32, 64, m, 0), lambda m: wf.wd_micro_values(m, P, wf.WD_F32, 64, 0),
                 lambda m: wf.wd_micro_project_workspace_bytes(m, 5), lambda m: project(m)):
        with pytest.raises(wf.WdError, match="WD_EINVAL"):
            call(micro(**bad))


def project(m=None, **kw):
    d = dict(bias=P, x=P, type=wf.WD_BF16, x_ld=64, N=5, out=P, out_type=wf.WD_F32, out_ld=100, ws=P, ws_bytes=1 << 20, stream=0)
    d.update(kw)
    wf.wd_micro_project(m or micro(), *d.values())


@pytest.mark.parametrize("bad", [dict(bias=P + 2), dict(x=None), dict(x=P + 1), dict(type=5), dict(x_ld=63), dict(N=-1), dict(N=1 << 31), dict(out=None),
                                 dict(out=P + 2), dict(out_type=-1), dict(out_ld=99), dict(ws=None), dict(ws=P + 4), dict(ws_bytes=100)])
def test_micro_products(bad):
    with pytest.raises(wf.WdError, match="WD_EINVAL"):
        project(**bad)


def test_micro_arguments():
    for m in (micro(rows=0), micro(rows=1 << 24)):
        with pytest.raises(wf.WdError, match="outputs"):
            wf.wd_micro_project_workspace_bytes(m, 5)
    for args in ((None, wf.WD_F32, 64), (P, 3, 64), (P, wf.WD_F32, 63), (P + 2, wf.WD_F32, 64), (P + 1, wf.WD_F16, 64)):
        with pytest.raises(wf.WdError, match="WD_EINVAL"):
            wf.wd_micro_quantize(*args, micro(), 0)
    for args in ((None, wf.WD_F32, 64), (P, wf.WD_F16, 64), (P, wf.WD_F32, 63), (P + 2, wf.WD_F32, 64)):
        with pytest.raises(wf.WdError, match="WD_EINVAL"):
            wf.wd_micro_values(micro(), *args, 0)
    for rows, D in ((-1, 5), (5, 0), (5, 1 << 22)):
        with pytest.raises(wf.WdError, match="WD_EINVAL"):
            wf.wd_micro_bytes(rows, D)
    assert wf.wd_micro_bytes(3, 1) == (48, 48) and wf.wd_micro_bytes(10, 513) == (10 * 17 * 16, 10 * 32)
    wf.wd_micro_quantize(None, wf.WD_F32, 64, micro(rows=0, codes=None, scales=None), 0)
    project(N=0, x=None, out=None, ws=None)


def test_null_arguments():
    L, n = wf.lib(), ctypes.c_size_t()
    for f in (L.wd_cross_entropy_workspace_bytes, L.wd_cross_entropy_grads_workspace_bytes):
        assert f(None, ctypes.byref(n)) == wf.WD_EINVAL and f(ctypes.byref(loss()), None) == wf.WD_EINVAL
    assert L.wd_cross_entropy(None, None, 0, None) == wf.WD_EINVAL and L.wd_cross_entropy_grads(None, None, 0, None) == wf.WD_EINVAL
    assert L.wd_clip_workspace_bytes(1, None) == wf.WD_EINVAL
    assert L.wd_micro_bytes(1, 1, None, ctypes.byref(n)) == wf.WD_EINVAL
    assert L.wd_micro_project_workspace_bytes(ctypes.byref(micro()), 1, None) == wf.WD_EINVAL
    assert L.wd_micro_project_workspace_bytes(None, 1, ctypes.byref(n)) == wf.WD_EINVAL


def test_structures_match_the_header():
    """Field order and sizes as the C compiler lays the header's structures out."""
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for name, cls in (("wd_loss_args", wf.wd_loss_args), ("wd_gradient", wf.wd_gradient), ("wd_micro", wf.wd_micro)):
        body = "".join(f'printf("%zu ", offsetof({name}, {f}));' for f, _ in cls._fields_)
        with tempfile.TemporaryDirectory() as d:
            c = os.path.join(d, "t.c")
            with open(c, "w") as f:
                f.write(f'#include <stdio.h>\n#include "wfstdec.h"\nint main(void){{{body}printf("%zu", sizeof({name}));return 0;}}\n')
            subprocess.run(["gcc", "-I", os.path.join(root, "include"), "-o", c[:-2], c], check=True)
            got = [int(x) for x in subprocess.run([c[:-2]], capture_output=True, text=True, check=True).stdout.split()]
        assert got == [getattr(cls, f).offset for f, _ in cls._fields_] + [ctypes.sizeof(cls)]
