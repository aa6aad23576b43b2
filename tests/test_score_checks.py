"""Argument checks of the operators that make log-likelihoods, at the C ABI: they
come before any device work, so no GPU is needed and the pointers are never
followed."""
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


def head(**kw):
    d = dict(D=64, P=100, type=wf.WD_BF16, n_adapters=2, rank=8, weight_ld=64, weight=P, bias=P, a=P, b=P, scale=P)
    return wf.wd_head(**{**d, **kw})


@pytest.mark.parametrize("bad", [dict(D=0), dict(P=0), dict(P=1 << 24), dict(type=wf.WD_F32), dict(type=7), dict(weight_ld=63),
                                 dict(weight=None), dict(n_adapters=-1), dict(rank=0), dict(rank=wf.WD_MAX_RANK + 1),
                                 dict(a=None), dict(b=None), dict(weight=P + 1), dict(a=P + 1), dict(bias=P + 2), dict(scale=P + 2)])
def test_heads(bad):
    with pytest.raises(wf.WdError, match="WD_EINVAL"):
        wf.wd_project_workspace_bytes(head(**bad), 5)


def project(h=None, **kw):
    d = dict(x=P, x_ld=64, N=5, adapter=P, out=P, out_ld=100, out_type=wf.WD_F32, ws=P, ws_bytes=1 << 20, stream=0)
    d.update(kw)
    wf.wd_project(h or head(), *d.values())


@pytest.mark.parametrize("bad", [dict(N=-1), dict(N=1 << 31), dict(x_ld=63), dict(out_ld=99), dict(out_type=wf.WD_F16), dict(out_type=9),
                                 dict(x=None), dict(out=None), dict(x=P + 1), dict(out=P + 2), dict(adapter=P + 2), dict(ws=None),
                                 dict(ws=P + 4), dict(ws_bytes=16)])
def test_projections(bad):
    with pytest.raises(wf.WdError, match="WD_EINVAL"):
        project(**bad)


def test_calls_without_work():
    project(N=0, x=None, out=None, ws=None)
    wf.wd_loglikes(scores(N=0, logits=None, out=None), None, 0, 0)
    assert wf.wd_project_workspace_bytes(head(n_adapters=0, rank=0, a=None, b=None), 1000) == 0
    assert wf.wd_loglikes_workspace_bytes(scores()) == 0
    assert wf.wd_loglikes_workspace_bytes(scores(V=100_000, ld=100_000, out_ld=100_000, mask_ld=3125)) > 0
    assert wf.wd_project_workspace_bytes(head(), 1000) >= 1000 * 3 * 8 * 2


def scores(**kw):
    d = dict(N=5, V=64, type=wf.WD_F32, logits=P, ld=64, normalize=1, scale=1.0, n_requests=2, hist_off=P, hist=P, n_hist=9,
             bias_off=P, bias_id=P, bias_val=P, n_bias=9, mask=P, n_masks=2, mask_ld=2, out=P, out_ld=64, out_rows=5)
    return wf.wd_loglikes_args(**{**d, **kw})


@pytest.mark.parametrize("bad", [dict(N=-1), dict(N=1 << 31), dict(V=0), dict(V=1 << 24), dict(type=3), dict(ld=63), dict(out_ld=63),
                                 dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(n_requests=-1),
                                 dict(n_requests=0), dict(n_hist=-1), dict(hist=None), dict(n_bias=-1), dict(n_bias=2 ** 32),
                                 dict(bias_id=None), dict(bias_val=None), dict(n_masks=-1), dict(mask_ld=1), dict(out_rows=4),
                                 dict(out_rows=-1), dict(logits=None), dict(out=None), dict(logits=P + 2), dict(out=P + 2),
                                 dict(log_prior=P + 1), dict(request=P + 2), dict(hist=P + 2), dict(hist_off=P + 4),
                                 dict(bias_off=P + 4), dict(mask=P + 1), dict(mask_of=P + 2), dict(out_row=P + 2)])
def test_scores(bad):
    with pytest.raises(wf.WdError, match="WD_EINVAL"):
        wf.wd_loglikes(scores(**bad), None, 0, 0)


def test_scores_workspace():
    long = dict(V=100_000, ld=100_000, out_ld=100_000, mask_ld=3125)
    need = wf.wd_loglikes_workspace_bytes(scores(**long))
    for ws, n in ((None, need), (P, need - 1), (P + 4, need)):
        with pytest.raises(wf.WdError, match="workspace"):
            wf.wd_loglikes(scores(**long), ws, n, 0)


def test_null_arguments():
    L = wf.lib()
    n = ctypes.c_size_t()
    assert L.wd_project_workspace_bytes(None, 1, ctypes.byref(n)) == wf.WD_EINVAL
    assert L.wd_project_workspace_bytes(ctypes.byref(head()), 1, None) == wf.WD_EINVAL
    assert L.wd_project(None, P, 64, 1, None, P, 100, 0, None, 0, None) == wf.WD_EINVAL
    assert L.wd_loglikes_workspace_bytes(None, ctypes.byref(n)) == wf.WD_EINVAL
    assert L.wd_loglikes_workspace_bytes(ctypes.byref(scores()), None) == wf.WD_EINVAL
    assert L.wd_loglikes(None, None, 0, None) == wf.WD_EINVAL
    assert L.wd_label_masks(None, 1, P, P, 1, P, 1, None) == wf.WD_EINVAL


def test_structures_match_the_header():
    """Field order and sizes as the C compiler lays the header's structures out."""
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for name, cls in (("wd_head", wf.wd_head), ("wd_loglikes_args", wf.wd_loglikes_args)):
        body = "".join(f'printf("%zu ", offsetof({name}, {f}));' for f, _ in cls._fields_)
        with tempfile.TemporaryDirectory() as d:
            c = os.path.join(d, "t.c")
            with open(c, "w") as f:
                f.write(f'#include <stdio.h>\n#include "wfstdec.h"\nint main(void){{{body}printf("%zu", sizeof({name}));return 0;}}\n')
            subprocess.run(["gcc", "-I", os.path.join(root, "include"), "-o", c[:-2], c], check=True)
            got = [int(x) for x in subprocess.run([c[:-2]], capture_output=True, text=True, check=True).stdout.split()]
        assert got == [getattr(cls, f).offset for f, _ in cls._fields_] + [ctypes.sizeof(cls)]
