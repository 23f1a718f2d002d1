"""The operators' bounded waits: with the limit at 0 every wait for a copy runs out (nothing goes wrong
on the device: the blocks wait a second time, with the default limit, before they go on), and
the outputs say so.  Rows enough that every ring of stages is refilled several times."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_operators import gen, matrix, teacher_list

pytestmark = pytest.mark.gpu


@pytest.fixture
def no_waiting():
    yield lambda: cd.set_operator_wait_limit(0)
    cd.set_operator_wait_limit(-1)


def nan_then_restored(call, no_waiting, nan):
    """call() has NaN outputs under the limit (those that `nan` picks), and its own bits with the default."""
    want = [t.clone() for t in call()]
    no_waiting()
    got = call()
    torch.cuda.synchronize()
    assert all(bool(t.isnan().all()) for t in nan(got))
    cd.set_operator_wait_limit(-1)
    again = call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want))


@pytest.mark.parametrize("rows,cols", [(200000, 96), (60000, 600), (60000, 601), (30000, 1002), (12000, 3000), (9000, 4100),
                                       (6000, 8192), (6000, 8191)])
def test_layer_norm(rows, cols, no_waiting):
    g = gen(rows, cols)
    x, dy = matrix(rows, cols, torch.bfloat16, g), matrix(rows, cols, torch.bfloat16, g)
    w, b = torch.randn(2, cols, generator=g, device="cuda").unbind(0)
    nan_then_restored(lambda: cd.layer_norm(x, w, b), no_waiting, lambda out: out)
    _, mean, rstd = cd.layer_norm(x, w, b)
    nan_then_restored(lambda: cd.layer_norm_backward(dy, x, w, mean, rstd, groups=2), no_waiting, lambda out: out)


@pytest.mark.parametrize("vocab", [40, 1000, 30522, 131072])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_distill(vocab, dtype, no_waiting):
    g = gen(vocab, 81)
    z = matrix(700, vocab, dtype, g)
    ids, lq = teacher_list(700, vocab, 20, g)
    dloss = torch.ones(700, device="cuda")
    dloss[5] = 0.0                                      # a row without a gradient coming in has none
    rows = torch.arange(700, device="cuda") != 5

    def nan(out):
        assert not out[1][5].any()
        return out[0], out[1][rows]
    nan_then_restored(lambda: cd.distill(z, ids, lq, dloss), no_waiting, nan)


def test_the_limit_is_the_threads_own(no_waiting):
    import threading
    x = torch.randn(100, 768, device="cuda")
    want = cd.layer_norm(x)[0].clone()
    no_waiting()
    got = []
    t = threading.Thread(target=lambda: got.append(cd.layer_norm(x)[0]))
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want)
