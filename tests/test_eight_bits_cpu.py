"""The C entry points of the operators in 8 bits refuse bad arguments before anything touches a device, and the
binding refuses tensors that it cannot describe to them.  (No GPU: the pointers are never followed.)"""
import os

import pytest
import torch

from paper_2111_00705_b200 import binding as cd

P = 4096          # an aligned address nobody reads
NAN, INF = float("nan"), float("inf")


def norm(x=P, xs=40, r=P * 2, rs=40, w=P, rows=4, cols=40, eps=1e-6, t=cd.BF16, wt=cd.F32, total=P * 3, ts=40, y=P * 4, ys=40, q=P * 5, qs=40,
         scale=P, kept=P * 6, ks=40, e=P * 7, es=2, rstd=P):
    return cd.lib().cdadam_rms_norm(x, xs, r, rs, w, rows, cols, eps, t, wt, total, ts, y, ys, q, qs, scale, kept, ks, e, es, rstd, None)


def backward(dy=P, dys=40, x=P * 2, xs=40, e=None, es=2, w=P, rstd=P, dt=P * 3, dts=40, rows=4, cols=40, groups=2, t=cd.BF16, wt=cd.F32, gt=cd.F32,
             dx=P * 4, dxs=40, dw=P * 5, dws=40, ws=P * 6, wsb=1 << 40):
    return cd.lib().cdadam_rms_norm_backward(dy, dys, x, xs, e, es, w, rstd, dt, dts, rows, cols, groups, t, wt, gt, dx, dxs, dw, dws, 0, ws,
                                             wsb, None)


def quantize(x=P, xs=40, rows=4, cols=40, t=cd.BF16, q=P * 2, qs=40, scale=P):
    return cd.lib().cdadam_quantize_rows(x, xs, rows, cols, t, q, qs, scale, None)


def dequantize(q=P, qs=40, scale=P, rows=4, cols=40, t=cd.BF16, y=P * 2, ys=40):
    return cd.lib().cdadam_dequantize_rows(q, qs, scale, rows, cols, t, y, ys, None)


def checkpoint(x=P, xs=40, rows=4, cols=40, t=cd.BF16, k=P * 2, ks=40, e=P * 3, es=2):
    return cd.lib().cdadam_checkpoint8(x, xs, rows, cols, t, k, ks, e, es, None)


def restore(k=P * 2, ks=40, e=P * 3, es=2, rows=4, cols=40, t=cd.BF16, x=P, xs=40):
    return cd.lib().cdadam_checkpoint8_restore(k, ks, e, es, rows, cols, t, x, xs, None)


def product(x=P, xs=48, xsc=P, w=P * 2, ws=48, wsc=P, b=P, tokens=4, channels=6, inner=40, t=cd.BF16, bt=cd.F32, y=P * 3, ys=6):
    return cd.lib().cdadam_matmul8(x, xs, xsc, w, ws, wsc, b, tokens, channels, inner, t, bt, y, ys, None)


REFUSED = [
    (norm, dict(t=3)), (norm, dict(wt=-1)), (norm, dict(rows=-1)), (norm, dict(rows=1 << 31)), (norm, dict(cols=0)),
    (norm, dict(cols=cd.MAX_NORM_COLS + 1)), (norm, dict(eps=-1.0)), (norm, dict(eps=NAN)), (norm, dict(eps=INF)),
    (norm, dict(x=None)), (norm, dict(x=P + 1)), (norm, dict(xs=-1)), (norm, dict(xs=(1 << 31) + 1)), (norm, dict(rs=-1)),
    (norm, dict(r=P + 1)), (norm, dict(w=P + 2)), (norm, dict(ts=39)), (norm, dict(ys=39)), (norm, dict(y=P * 3)),
    (norm, dict(total=P, ts=48)), (norm, dict(y=P * 2, ys=48)), (norm, dict(q=None)), (norm, dict(scale=None)), (norm, dict(qs=39)),
    (norm, dict(kept=None)), (norm, dict(e=None)), (norm, dict(ks=39)), (norm, dict(es=1)), (norm, dict(rstd=P + 2)),
    (norm, dict(scale=P + 1)), (norm, dict(total=None, y=None, q=None, scale=None, kept=None, e=None, rstd=None)),
    (backward, dict(t=9)), (backward, dict(gt=5)), (backward, dict(wt=7)), (backward, dict(groups=0)), (backward, dict(groups=3)),
    (backward, dict(groups=65536, rows=65536)), (backward, dict(dx=None, dw=None)), (backward, dict(rstd=None)),
    (backward, dict(dy=None)), (backward, dict(x=None)), (backward, dict(x=None, e=P)), (backward, dict(dxs=39)), (backward, dict(dws=39)),
    (backward, dict(dx=P, dxs=48)), (backward, dict(dx=P * 2, dxs=48)), (backward, dict(dx=P * 3, dxs=48)),
    (backward, dict(dx=P * 2, e=P * 7)), (backward, dict(dts=-1)), (backward, dict(dt=P + 1)), (backward, dict(dw=P + 2)),
    (backward, dict(cols=0)), (backward, dict(es=-1, e=P)), (backward, dict(rstd=P + 2)),
    (quantize, dict(t=4)), (quantize, dict(x=None)), (quantize, dict(q=None)), (quantize, dict(scale=None)), (quantize, dict(qs=39)),
    (quantize, dict(scale=P + 2)), (quantize, dict(cols=0)), (quantize, dict(rows=-3)),
    (dequantize, dict(t=4)), (dequantize, dict(q=None)), (dequantize, dict(y=None)), (dequantize, dict(scale=None)),
    (dequantize, dict(ys=39)), (dequantize, dict(y=P + 1)), (dequantize, dict(qs=-1)),
    (checkpoint, dict(t=4)), (checkpoint, dict(x=None)), (checkpoint, dict(k=None)), (checkpoint, dict(e=None)),
    (checkpoint, dict(ks=39)), (checkpoint, dict(es=1)), (checkpoint, dict(xs=-1)),
    (restore, dict(t=4)), (restore, dict(x=None)), (restore, dict(k=None)), (restore, dict(e=None)), (restore, dict(xs=39)),
    (restore, dict(ks=-1)), (restore, dict(es=-1)),
    (product, dict(t=3)), (product, dict(bt=3)), (product, dict(tokens=-1)), (product, dict(channels=(1 << 30) + 1)), (product, dict(tokens=1 << 31)), (product, dict(inner=0)),
    (product, dict(inner=cd.MAX_INNER + 1, xs=1 << 18, ws=1 << 18)), (product, dict(x=None)), (product, dict(w=None)),
    (product, dict(y=None)), (product, dict(xsc=None)), (product, dict(wsc=None)), (product, dict(x=P + 8)), (product, dict(w=P + 1)),
    (product, dict(xs=40)), (product, dict(ws=56)), (product, dict(xs=32)), (product, dict(ws=32)), (product, dict(ys=5)),
    (product, dict(y=P + 1)), (product, dict(xsc=P + 2)), (product, dict(wsc=P + 1)), (product, dict(b=P + 2)),
    (product, dict(tokens=1 << 30, channels=1 << 30)),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refused_before_anything_is_queued(i):
    f, bad = REFUSED[i]
    assert f(**bad) == cd.ERR_ARG
    assert cd.last_error().startswith("cdadam_")


def test_small_workspace_is_refused():
    need = cd.rms_norm_workspace(4096, 1024, 2)
    assert need > 0
    wide = dict(rows=4096, cols=1024, dys=1024, xs=1024, dts=1024, dxs=1024, dws=1024)
    assert backward(**wide, wsb=need - 1) == cd.ERR_ARG and "workspace" in cd.last_error()
    assert backward(**wide, ws=None) == cd.ERR_ARG
    assert backward(**wide, ws=P + 8) == cd.ERR_ARG
    assert cd.rms_norm_workspace(-1, 8, 1) == cd.rms_norm_workspace(8, 8, 0) == 0


def test_nothing_to_do_is_no_error():
    assert norm(rows=0, x=None, r=None, total=None, y=None) == cd.OK
    assert backward(rows=0, dy=None, x=None, dx=None, dw=None) == cd.OK
    assert quantize(rows=0, x=None, q=None, scale=None) == cd.OK
    assert dequantize(rows=0, y=None, q=None, scale=None) == cd.OK
    assert checkpoint(rows=0, x=None, k=None, e=None) == cd.OK
    assert restore(rows=0, x=None, k=None, e=None) == cd.OK
    assert product(tokens=0, x=None, y=None, xsc=None) == cd.OK
    assert product(channels=0, w=None, y=None, wsc=None) == cd.OK


def test_limits_match_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "cdadam.h")).read()
    for name, value in (("CHECKPOINT_BLOCK", cd.CHECKPOINT_BLOCK), ("MAX_INNER", cd.MAX_INNER)):
        assert "#define CDADAM_%s %d " % (name, value) in text, name


def test_binding_refuses_what_it_cannot_describe():
    x, q, e = torch.zeros(4, 40), torch.zeros(4, 40, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8)
    s = torch.zeros(4)
    for call in (lambda: cd.rms_norm(x), lambda: cd.rms_norm(x.double()), lambda: cd.rms_norm8(x[0]), lambda: cd.rms_norm8(x.t()),
                 lambda: cd.rms_norm_backward(x, x, None, s), lambda: cd.rms_norm_backward(x, (q, e), None, s),
                 lambda: cd.quantize_rows(x), lambda: cd.dequantize_rows(q, s), lambda: cd.checkpoint8(x),
                 lambda: cd.checkpoint8_restore(q, e), lambda: cd.matmul8(q, s, q, s)):
        with pytest.raises(ValueError):
            call()


def test_a_checkpoint_to_write_into_has_aligned_rows():
    kept, exps = cd.checkpoint8_like(torch.zeros(3, 37))
    assert kept.shape == (3, 37) and kept.stride() == (48, 1) and exps.shape == (3, 2)
