"""The operators' C entry points refuse bad arguments before anything touches a device, and the
binding refuses tensors it cannot describe to them.  (No GPU: the pointers are never followed.)"""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd

P = 4096          # an aligned address nobody reads


def norm(x=P, xs=8, w=P, b=P, rows=4, cols=8, eps=1e-5, t=cd.BF16, wt=cd.F32, y=P * 2, ys=8, mean=P, rstd=P):
    return cd.lib().cdadam_layer_norm(x, xs, w, b, rows, cols, eps, t, wt, y, ys, mean, rstd, None)


def norm_backward(dy=P, dys=8, x=P * 2, xs=8, w=P, mean=P, rstd=P, rows=4, cols=8, groups=2, t=cd.BF16, wt=cd.F32, gt=cd.F32,
                  dx=P * 3, dxs=8, dw=P * 4, dws=8, db=P * 5, dbs=8, ws=P * 6, wsb=1 << 40):
    return cd.lib().cdadam_layer_norm_backward(dy, dys, x, xs, w, mean, rstd, rows, cols, groups, t, wt, gt, dx, dxs, dw, dws,
                                               db, dbs, 0, ws, wsb, None)


def logprobs(z=P, zs=16, tok=P, rows=4, vocab=16, t=cd.BF16, it=1, temp=1.0, k=4, lp=P, ent=P, lse=P, ids=P, top=P):
    return cd.lib().cdadam_token_logprobs(z, zs, tok, rows, vocab, t, it, temp, k, lp, ent, lse, ids, top, None)


def logprobs_backward(z=P, zs=16, tok=P, rows=4, vocab=16, t=cd.BF16, it=1, temp=1.0, lse=P, ent=P, dlp=P, dent=P, dz=P * 2,
                      dzs=16):
    return cd.lib().cdadam_token_logprobs_backward(z, zs, tok, rows, vocab, t, it, temp, lse, ent, dlp, dent, dz, dzs, None)


def distill(z=P, zs=16, ids=P, lq=P, rows=4, vocab=16, k=4, t=cd.BF16, it=1, temp=1.0, rest=1, dloss=P, loss=P, dz=P * 2,
            dzs=16):
    return cd.lib().cdadam_distill(z, zs, ids, lq, rows, vocab, k, t, it, temp, rest, dloss, loss, dz, dzs, None)


NAN, INF = float("nan"), float("inf")
REFUSED = [
    (norm, dict(t=3)), (norm, dict(wt=-1)), (norm, dict(rows=-1)), (norm, dict(rows=1 << 31)), (norm, dict(cols=0)),
    (norm, dict(cols=cd.MAX_NORM_COLS + 1)), (norm, dict(eps=-1.0)), (norm, dict(eps=NAN)), (norm, dict(eps=INF)),
    (norm, dict(x=None)), (norm, dict(y=None)), (norm, dict(x=P + 1)), (norm, dict(w=P + 2)), (norm, dict(ys=7)),
    (norm, dict(xs=-8)), (norm, dict(xs=(1 << 31) + 1)), (norm, dict(y=P, ys=16)), (norm, dict(mean=P + 2)),
    (norm_backward, dict(t=9)), (norm_backward, dict(gt=5)), (norm_backward, dict(groups=0)), (norm_backward, dict(groups=3)),
    (norm_backward, dict(groups=65536, rows=65536)), (norm_backward, dict(dx=None, dw=None, db=None)),
    (norm_backward, dict(mean=None)), (norm_backward, dict(rstd=None)), (norm_backward, dict(dy=None)),
    (norm_backward, dict(dxs=4)), (norm_backward, dict(dws=7)), (norm_backward, dict(dbs=0)), (norm_backward, dict(dx=P, dxs=16)),
    (norm_backward, dict(dx=P * 2, dxs=16)), (norm_backward, dict(dw=P + 2)), (norm_backward, dict(cols=0)),
    (logprobs, dict(t=3)), (logprobs, dict(it=2)), (logprobs, dict(vocab=0)), (logprobs, dict(vocab=cd.MAX_VOCAB + 1)),
    (logprobs, dict(rows=-1)), (logprobs, dict(temp=0.0)), (logprobs, dict(temp=-1.0)), (logprobs, dict(temp=NAN)),
    (logprobs, dict(temp=INF)), (logprobs, dict(k=-1)), (logprobs, dict(k=17)), (logprobs, dict(k=129, vocab=200)),
    (logprobs, dict(tok=None)), (logprobs, dict(ids=None)), (logprobs, dict(top=None)), (logprobs, dict(z=None)),
    (logprobs, dict(z=P + 1)), (logprobs, dict(tok=P + 4)), (logprobs, dict(zs=-1)),
    (logprobs_backward, dict(lse=None)), (logprobs_backward, dict(ent=None)), (logprobs_backward, dict(tok=None)),
    (logprobs_backward, dict(dz=None)), (logprobs_backward, dict(dzs=15)), (logprobs_backward, dict(dz=P, dzs=32)),
    (logprobs_backward, dict(temp=1e-5)), (logprobs_backward, dict(t=-1)),
    (distill, dict(k=0)), (distill, dict(k=129)), (distill, dict(loss=None, dz=None)), (distill, dict(dloss=None)),
    (distill, dict(ids=None)), (distill, dict(lq=None)), (distill, dict(dzs=8)), (distill, dict(dz=P, dzs=32)),
    (distill, dict(temp=2e4)), (distill, dict(it=7)), (distill, dict(ids=P + 4)), (distill, dict(lq=P + 2)),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refused_before_anything_is_queued(i):
    f, bad = REFUSED[i]
    assert f(**bad) == cd.ERR_ARG
    assert cd.last_error().startswith("cdadam_")


def test_small_workspace_is_refused():
    need = cd.layer_norm_workspace(4096, 1024, 2)
    if need:
        assert norm_backward(rows=4096, cols=1024, dys=1024, xs=1024, dxs=1024, dws=1024, dbs=1024, wsb=need - 1) == cd.ERR_ARG
        assert "workspace" in cd.last_error()
        assert norm_backward(rows=4096, cols=1024, dys=1024, xs=1024, dxs=1024, dws=1024, dbs=1024, ws=None) == cd.ERR_ARG


def test_no_rows_is_no_error():
    assert norm(rows=0, x=None, y=None) == cd.OK
    assert logprobs(rows=0, z=None, tok=None) == cd.OK
    assert logprobs_backward(rows=0, z=None, dz=None) == cd.OK
    assert distill(rows=0, z=None, ids=None, lq=None, dz=None) == cd.OK


def test_limits_match_the_header():
    import os
    text = open(os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "cdadam.h")).read()
    for name, value in (("MAX_LIST", cd.MAX_LIST), ("MAX_VOCAB", cd.MAX_VOCAB), ("MAX_NORM_COLS", cd.MAX_NORM_COLS)):
        assert "#define CDADAM_%s %d " % (name, value) in text, name


def test_binding_refuses_tensors_on_the_host_and_of_other_types():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        cd.layer_norm(x)
    with pytest.raises(ValueError):
        cd.layer_norm(x.double())
    with pytest.raises(ValueError):
        cd.layer_norm(x[0])
    with pytest.raises(ValueError):
        cd.layer_norm(x.t())
    with pytest.raises(ValueError):
        cd.token_logprobs(x, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        cd.token_logprobs(x, torch.zeros(4, dtype=torch.int16))
    with pytest.raises(ValueError):
        cd.distill(x, torch.zeros(4, dtype=torch.int64), torch.zeros(4))
    with pytest.raises(ValueError):
        cd.distill(x, torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 3))
