"""Layer norm at the ends of binary32's range, on both sides of the width from which rows take another
kernel, against 64 bits.  Tolerances as in test_gpu_operators."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_operators import TYPES, check_backward, check_norm, gen, matrix

pytestmark = pytest.mark.gpu

# rows that go by vectors, by two elements, by one; 96 to 12000 columns
COLS = [96, 98, 99, 1000, 1002, 1001, 4096, 4098, 4099, 8192, 8190, 8191, 10000, 10001, 12000]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_squares_beyond_the_range_of_binary32(cols, dtype):
    g = gen(cols, 61)
    x = matrix(9, cols, TYPES[dtype], g)
    w, b = torch.randn(2, cols, generator=g, device="cuda").unbind(0)
    x[3] *= 1e16                                          # the largest squares that still sum to less than 2^127
    check_norm(x, w, b)
    x[2] *= 1e20
    x[8] *= -1e25
    y, mean, rstd = cd.layer_norm(x, w, b)
    for i in (2, 8):
        assert rstd[i] == 0 and torch.equal(y[i], b.to(x.dtype))
        assert abs(float(mean[i]) - float(x[i].double().mean())) <= 2.0 ** -15 * float(x[i].double().abs().max())
    keep = [0, 1, 3, 4, 5, 6, 7]
    check_norm(x[keep], w, b)
    assert torch.equal(cd.layer_norm(x[keep], w, b)[0], y[keep])
    # such a row's gradient: 0, and nothing of it in dweight
    check_backward(matrix(9, cols, TYPES[dtype], g), x, w)


@pytest.mark.parametrize("cols", COLS)
def test_small_spreads_without_eps(cols):
    """Deviations of 1e-12 around 0: squares of 1e-24, far from 0 and from what is subnormal."""
    g = gen(cols, 62)
    x = matrix(5, cols, torch.float32, g, 1e-12)
    check_norm(x, None, None, 0.0)
