"""Matrices of one row: their row stride means nothing, whatever it is (the tensor of one row that a program has cut out of
something else brings any), in rows that start on 16 bytes and in rows that start anywhere."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_operators import TYPES, gen, matrix

pytestmark = pytest.mark.gpu

STRIDES = [0, 1, 7, (1 << 31) + 5, (1 << 60) + 3, (1 << 61) - 1, (1 << 62) - 1, (1 << 62) - 2, (1 << 62) + 1, (1 << 63) - 1]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", [1, 5, 40, 1000, 1021, 9001, 17003])
def test_any_stride(cols, dtype):
    g = gen(cols, 151)
    dt = TYPES[dtype]
    w = torch.randn(cols, generator=g, device="cuda")
    for shift in (0, 3):
        x, r, dy = (matrix(1, cols, dt, g, 1.0, 0, shift) for _ in range(3))
        y, total, rstd = cd.rms_norm(x, w, r)
        dx, dw = cd.rms_norm_backward(dy, total, w, rstd, r)
        kept, exps = cd.checkpoint8(x)
        q, scale = cd.quantize_rows(x)
        want = y, total, rstd, dx, dw, kept, exps, q, scale, cd.checkpoint8_restore(kept, exps, dt), cd.dequantize_rows(q, scale, dt)
        for stride in STRIDES:
            def one(t):
                return torch.as_strided(t, (1, cols), (stride, 1), t.storage_offset())

            def out():
                return one(matrix(1, cols, dt, g, 1.0, 0, shift))
            y, total, rstd = cd.rms_norm(one(x), w, one(r), out=(out(), out(), torch.empty(1, device="cuda")))
            dx, dw = cd.rms_norm_backward(one(dy), one(total), w, rstd, one(r), out=(out(), one(torch.empty(1, cols, device="cuda"))))
            kept, exps = cd.checkpoint8(one(x))
            q, scale = cd.quantize_rows(one(x))
            got = (y, total, rstd, dx, dw, kept, exps, q, scale, cd.checkpoint8_restore(one(kept), exps, out=out()),
                   cd.dequantize_rows(one(q), scale, out=out()))
            assert all(torch.equal(a, b) for a, b in zip(got, want)), stride
