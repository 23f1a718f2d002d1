"""Layer norm of so many rows that the ring of stages of every group of threads is refilled at least
twice, at both ends of the range of widths of every variant: an SM's rings hold at most 216 KB, all SMs'
together 32 MB, and the rows take 100 MB.  Tolerances as in test_gpu_operators."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_operators import TYPES, check_backward, check_norm, gen, matrix

pytestmark = pytest.mark.gpu

ENDS = [256, 512, 768, 1024, 2048, 4096, 5120, 6144, 8192]      # last widths of a variant
VECTORS = [8] + [v for e in ENDS for v in (e, e + 8)][:-1]      # rows that go by 16 bytes,
PAIRS = [2] + [v for e in ENDS for v in (e - 2, e + 2)][:-1]    # by two elements,
SINGLE = [1] + [v for e in ENDS for v in (e - 1, e + 1)][:-1]   # and one by one


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", VECTORS + PAIRS + SINGLE)
def test_rings_that_are_refilled(cols, dtype):
    dt = TYPES[dtype]
    g = gen(cols, 91)
    rows = 100_000_000 // ((cols * dt.itemsize + 30) // 16 * 16) // 3 * 3
    x, dy = matrix(rows, cols, dt, g, 1.5), matrix(rows, cols, dt, g, 0.1)
    w, b = torch.randn(2, cols, generator=g, device="cuda").unbind(0)
    check_norm(x, w, b)
    check_backward(dy, x, w, 1)
    check_backward(dy, x, None, 3)


@pytest.mark.parametrize("cols,pad", [(768, 8), (1021, 3), (1022, 2), (96, 1), (5000, 1), (8191, 5)])
def test_refilled_rings_of_rows_apart_and_in_place(cols, pad):
    """Row strides that are not the width; what lies between the rows is NaN.  In place: a refill is
    read behind the rows that are written."""
    g = gen(cols, 92)
    rows = 100_000_000 // (2 * cols) // 2 * 2
    x, dy = matrix(rows, cols, torch.bfloat16, g, 1.5, pad, 1), matrix(rows, cols, torch.bfloat16, g, 0.1, 0, 3)
    check_norm(x, None, None)
    check_backward(dy, x, None, 2)
    y, mean, rstd = cd.layer_norm(x)
    dx, dw, db = cd.layer_norm_backward(dy, x, None, mean, rstd, groups=2)
    x2 = matrix(rows, cols, torch.bfloat16, g, 0.0, pad, 1)          # the same alignment: the same order of the sums
    x2.copy_(x)
    assert torch.equal(cd.layer_norm(x2, out=(x2, None, None))[0], y)
    e = [torch.empty_like(t) for t in (dw, db)]
    got = cd.layer_norm_backward(dy, x, None, mean, rstd, groups=2, out=(dy, *e))
    assert all(torch.equal(a, b) for a, b in zip(got, (dx, dw, db)))
