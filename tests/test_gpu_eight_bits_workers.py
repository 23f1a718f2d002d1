"""The norm's gradient for more workers than other tests have, with rows on both sides of where a cluster of eight blocks shares a
worker's: against 64 bits (tolerances of test_gpu_eight_bits), and the same bits every time."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_eight_bits import check_backward
from test_gpu_operators import TYPES, gen, matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,groups", [(10 * 700, 768, 10), (16 * 100, 768, 16), (16 * 900, 768, 16), (16 * 128, 4096, 16), (16 * 600, 4096, 16),
                                              (24 * 300, 2048, 24), (24 * 1000, 760, 24), (12 * 500, 1021, 12), (15 * 300, 8192, 15),
                                              (16 * 64, 8192, 16), (16 * 300, 8192, 16), (36 * 40, 4096, 36)])
def test_workers(rows, cols, groups, dtype):
    g = gen(rows, cols, 163)
    dt = TYPES[dtype]
    x, dy, more = (matrix(rows, cols, dt, g) for _ in range(3))
    w = torch.randn(cols, generator=g, device="cuda")
    for kept in (False, True):
        given, rstd, dx, dw = check_backward(dy, x, w, groups, more, kept)
        again = cd.rms_norm_backward(dy, given, w, rstd, more, groups)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
        alone = cd.rms_norm_backward(dy, given, w, rstd, more, groups, out=(None, torch.empty_like(dw)))[1]
        assert torch.equal(alone, dw)
