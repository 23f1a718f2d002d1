"""Products of many tokens (pairs of SMs) whose rows are longer than a pair's ring of stages, with several tiles to a pair, so that
the ring wraps inside a tile and both sets of sums are used over and over; and outputs of the norm, the checkpoints and
the rows format to rows that start anywhere, exactly."""
import math

import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_eight_bits import check_product, eight, product64, restored64, sum_tol
from test_gpu_operators import TYPES, close, gen, matrix, round_tol

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bias", [None, "f32", "bf16"])
@pytest.mark.parametrize("tokens,channels,inner", [(2049, 5000, 1021), (4100, 8200, 769), (1030, 20011, 4100), (300, 4100, 700), (700, 40000, 1500),
                                                   (2100, 1003, 5001)])
def test_long_rows(tokens, channels, inner, bias, dtype):
    g = gen(tokens, inner, 167)
    check_product(tokens, channels, inner, g, TYPES[dtype], None if bias is None else TYPES[bias])


@pytest.mark.parametrize("inner", [1, 128, 129, 512, 513, 640, 641, 768, 769, 1280, 1281, 1409])
def test_numbers_of_stages(inner):
    """Around whole turns of the ring of five."""
    g = gen(inner, 173)
    for tokens, channels in ((600, 19000), (2400, 3000)):           # 225 and 120 tiles for 74 pairs
        check_product(tokens, channels, inner, g, torch.bfloat16)


def test_many_tiles_of_long_rows():
    check_product(4096, 30001, 4096, gen(25, 179), torch.float16)


def test_the_largest_sums():
    x = torch.full((2100, 131072), -128, dtype=torch.int8, device="cuda")[:, :131071]
    w = torch.full((1003, 131072), -128, dtype=torch.int8, device="cuda")[:, :131071]
    w[1::2] = 127
    one, ones = torch.ones(2100, device="cuda"), torch.ones(1003, device="cuda")
    y = cd.matmul8(x, one, w, ones, dtype=torch.float32)
    assert (y[:, ::2] == 16384 * 131071).all() and (y[:, 1::2] == torch.tensor(-16256 * 131071.0)).all()


@pytest.mark.parametrize("channels", [4096, 4099, 20000])
def test_waits_that_run_out(channels):
    """Up to several tiles a pair; behind it the exact product again."""
    g = gen(channels, 181)
    x, w = eight(1500, 2000, g), eight(channels, 2000, g)
    xs, ws = torch.rand(1500, generator=g, device="cuda") + 0.01, torch.rand(channels, generator=g, device="cuda") + 0.01
    want = product64(x, xs, w, ws, None, torch.bfloat16)
    assert torch.equal(cd.matmul8(x, xs, w, ws), want)
    try:
        cd.set_operator_wait_limit(0)
        got = cd.matmul8(x, xs, w, ws)
        torch.cuda.synchronize()
    finally:
        cd.set_operator_wait_limit(-1)
    # what was waited for in time is right, the rest NaN
    assert bool((got.isnan() | (got == want)).all()) and bool(got.isnan().any())
    assert torch.equal(cd.matmul8(x, xs, w, ws), want)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", [1, 5, 40, 260, 1000, 1021, 4099, 9001, 17003])
def test_outputs_that_start_anywhere(cols, dtype):
    """The sum, restored checkpoints and values of rows are defined exactly; the norm and its gradient once rounded, with
    the tolerances of their other tests."""
    g = gen(cols, 191)
    dt = TYPES[dtype]
    tol = sum_tol(cols)
    for shift, pad in ((0, 0), (1, 0), (0, 1), (3, 2), (8, 8), (5, 7), (4, 4), (2, 5), (7, 3)):
        for rows in (1, 2, 37):
            x, r, dy = (matrix(rows, cols, dt, g, 1.0, pad, shift) for _ in range(3))
            w = torch.randn(cols, generator=g, device="cuda")

            def out():
                return matrix(rows, cols, dt, g, 1.0, shift, pad)
            y, total, rstd = cd.rms_norm(x, w, r, out=(out(), out(), torch.empty(rows, device="cuda")))
            h = (x.float() + r.float()).to(dt)
            assert torch.equal(total, h)
            s = (h.double().square().mean(1, keepdim=True) + 1e-6).rsqrt()
            want = (h.float() * w).double() * s
            close(y, want, want.abs() * (tol + 2.0 ** -22) + round_tol(want, dt), "y")
            kept, exps = cd.checkpoint8(x)
            assert torch.equal(cd.checkpoint8_restore(kept, exps, out=out()).double(), restored64(kept, exps))
            q, scale = cd.quantize_rows(x)
            assert torch.equal(cd.dequantize_rows(q, scale, out=out()), (q.float() * scale[:, None]).to(dt))
            dx = cd.rms_norm_backward(dy, h, w, rstd, r, out=(out(), None))[0]
            s = rstd.double()[:, None]
            g64, xh = dy.double() * w.double(), h.double() * s
            want = s * (g64 - xh * (g64 * xh).mean(1, keepdim=True)) + r.double()
            size = s * (g64.abs() * 2.0 ** -21 + xh.abs() * (g64 * xh).abs().mean(1, keepdim=True) * (tol + 2.0 ** -21))
            close(dx, want, size + r.double().abs() * 2.0 ** -23 + round_tol(want, dt), "dx")


def test_a_captured_product_is_right():
    """Weights quantised right in front of it in the graph, replayed with others; against 64 bits."""
    g = gen(26, 193)
    x, w = torch.randn(1200, 900, generator=g, device="cuda"), torch.randn(4003, 900, generator=g, device="cuda")

    def chain():
        q, s = cd.quantize_rows(x)
        p, t = cd.quantize_rows(w)
        return q, s, p, t, cd.matmul8(q, s, p, t, dtype=torch.float32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, s, p, t, y = chain()
    for scale in (1.0, 3.0, math.pi):
        x.copy_(torch.randn(1200, 900, generator=g, device="cuda") * scale)
        w.copy_(torch.randn(4003, 900, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, product64(q, s, p, t, None, torch.float32))
        # both operands off by half a step at most
        off = 0.5 * s[:, None].double() * w.double().abs().sum(1) + 0.5 * t.double() * (q.double().abs().sum(1) * s.double())[:, None]
        ref = x.double() @ w.double().T
        close(y, ref, off * (1 + 2.0 ** -20) + ref.abs() * 2.0 ** -21)
