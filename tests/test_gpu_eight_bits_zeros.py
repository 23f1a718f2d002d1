"""Products of 8-bit rows bit for bit: the sign of zero too is that of the documented steps, whatever kernel the numbers of
tokens and channels select.  Zeros come from a sum of 0 with a negative scale, from a scale of 0 with a negative
sum, and from outputs below the type's range; a bias of either zero is added like any other."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_eight_bits import eight, product64
from test_gpu_operators import TYPES, gen

pytestmark = pytest.mark.gpu


def bits(t):
    return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens,channels", [(1, 300), (2, 300), (3, 300), (20, 517), (60, 517), (128, 16500), (200, 300), (300, 4096),
                                             (300, 4099), (513, 2600)])
def test_signs_of_zero(tokens, channels, dtype):
    g = gen(tokens, 157)
    x, w = eight(tokens, 90, g), eight(channels, 90, g)
    x[::3] = 0
    w[1::5] = 0
    xs = torch.rand(tokens, generator=g, device="cuda") - 0.5
    ws = torch.randn(channels, generator=g, device="cuda")
    xs[1::7], ws[2::7], ws[3::7] = 0.0, -0.0, 1e-44
    xs[2::7] = -1e-6
    for bias in (None, 0.0, -0.0, 2.5):
        b = None if bias is None else torch.full((channels,), bias, device="cuda")
        got, want = cd.matmul8(x, xs, w, ws, b, TYPES[dtype]), product64(x, xs, w, ws, b, TYPES[dtype])
        assert bool(((want == 0) & want.signbit()).any()) or bias in (0.0, 2.5)
        wrong = (bits(got) != bits(want)).nonzero()
        assert len(wrong) == 0, (bias, len(wrong), wrong[:3].tolist())
