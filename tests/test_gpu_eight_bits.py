"""The operators in 8 bits against plain implementations in 64 bits.

Tolerances.  Whole numbers (8-bit rows, checkpoints, their exponents) and sums in the activations' type have to be
equal: their definitions leave no rounding open.  Products of 8-bit rows have to be equal to the documented
binary32 steps on the exact sum.  Elsewhere outputs are rounded once to their type (2^-24, 2^-8 or 2^-11 of the
value), and below that come the sums: at most 32 terms of a row in a thread, then at most 16 + 5 additions, each 2^-24 of a
sum of terms of one sign, is below 53 2^-24 < 2^-18 (rows beyond 16384 columns: 1024 terms, 2^-13.9); a
root's relative error is half its argument's.  SUM = 2^-15 of the sum of magnitudes is allowed (LONG = 2^-13 beyond
16384 columns); a lost or doubled unit of eight columns exceeds it in these rows.
"""
import math

import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_operators import INF, SUM, TYPES, close, gen, matrix, round_tol

pytestmark = pytest.mark.gpu
LONG = 2.0 ** -13


def sum_tol(cols):
    return SUM if cols <= 16384 else LONG


def two_to(e):
    """2^e in 64 bits, exactly (a power function need not be)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def whole(t):
    """t rounded to the nearest integer, to the even one at a half."""
    low = t.floor()
    return low + ((t - low > 0.5) | ((t - low == 0.5) & (low.remainder(2.0) == 1.0)))


def rows64(p):
    """(q, step) of binary32 rows p; q 0 and step NaN where a row is not finite."""
    p = p.double()
    m = p.abs().amax(1)
    fine = m.isfinite()
    t = torch.where(((m > 0) & fine)[:, None], 127.0 * p / m[:, None], 0.0)
    return whole(t).to(torch.int8), torch.where(fine, m / 127.0, math.nan)


def kept64(x):
    """(kept, exponents) of a matrix."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -cols % 32)).unflatten(1, (-1, 32))
    m = v.abs().amax(2, keepdim=True)
    fine = m.isfinite()
    e = torch.where(fine & (m > 0), torch.frexp(torch.where(fine, m, 1.0)).exponent - 7, -126).clamp(min=-126)
    q = whole(v * two_to(-e)).clamp(-127, 127)
    q = torch.where(fine, q, 0.0).flatten(1)[:, :cols]
    return q.to(torch.int8), torch.where(fine, e + 127, 255)[:, :, 0].to(torch.uint8)


def restored64(kept, exponents):
    step = two_to(exponents.long() - 127)
    step = torch.where(exponents == 255, math.nan, step)
    return kept.double() * step.repeat_interleave(32, 1)[:, :kept.shape[1]]


def byte_matrix(rows, cols, pad=0, shift=0, dtype=torch.int8):
    """A matrix of bytes with row stride cols + pad, `shift` bytes behind a 256-byte boundary; 77 around it."""
    buf = torch.full((shift + rows * (cols + pad) + 16,), 77, device="cuda", dtype=dtype)
    return buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols], buf


def untouched(m, buf, shift):
    """Everything around the matrix of byte_matrix still holds 77."""
    around = buf.clone()
    rows, cols, stride = *m.shape, m.stride(0)
    around[shift:shift + rows * stride].view(rows, stride)[:, :cols] = 77
    return bool((around == 77).all())


def check_norm(x, w, residual=None, eps=1e-6, pad=0, shift=0):
    """Both forms of the norm with all their outputs."""
    rows, cols = x.shape
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    h64 = h.double()
    rstd64 = (h64.square().mean(1) + eps).rsqrt()
    p = h.float() if w is None else h.float() * w.float()
    kept = byte_matrix(rows, cols, pad, shift)
    exps = byte_matrix(rows, -(-cols // 32), pad, shift, torch.uint8)
    y, total, rstd = cd.rms_norm(x, w, residual, eps, checkpoint=(kept[0], exps[0]))
    tol = sum_tol(cols)
    close(rstd, rstd64, rstd64 * tol, "rstd")
    want = p.double() * rstd64[:, None]
    close(y, want, want.abs() * (tol + 2.0 ** -22) + round_tol(want, x.dtype), "y")
    if residual is None:
        assert total is None
    else:
        assert torch.equal(total, h), "total"
    for got, ref in zip((kept[0], exps[0]), kept64(h)):
        assert torch.equal(got, ref), "checkpoint"
    assert untouched(*kept, shift) and untouched(*exps, shift)
    q8 = byte_matrix(rows, cols, pad, shift)
    scale = torch.empty(rows, device="cuda")
    rstd8 = torch.empty(rows, device="cuda")
    cd.rms_norm8(x, w, residual, eps, out=(q8[0], scale, None, rstd8))
    q, step = rows64(p)
    assert torch.equal(q8[0], q), ("q", (q8[0] != q).nonzero()[:3])
    assert untouched(*q8, shift) and torch.equal(rstd8, rstd)
    close(scale, step * rstd64, step * rstd64 * (tol + 2.0 ** -22) + 1e-44, "scale")
    return y, total, rstd


COLS = [1, 2, 3, 5, 7, 8, 9, 31, 32, 33, 64, 100, 255, 256, 257, 511, 512, 513, 767, 768, 1000, 1021, 1024, 1032, 1537, 2047, 2048, 2056,
        4096, 4100, 6144, 8191, 8192, 8200, 12288, 16384, 16385, 20000, 33000, 70001]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", COLS)
def test_norm_every_width(cols, dtype):
    g = gen(cols, 11)
    for i, (rows, pad, shift) in enumerate(((1, 0, 0), (5, 0, 0), (3, 8, 0), (9, 3, 0), (7, 0, 1), (2, 16, 16))):
        x = matrix(rows, cols, TYPES[dtype], g, 2.0, pad, shift)
        r = matrix(rows, cols, TYPES[dtype], g, 1.0, shift, pad) if i % 2 else None
        w = torch.randn(cols + 8, generator=g, device="cuda")
        check_norm(x, w[8 - i % 4:][:cols], r, 1e-6, pad, shift)
    check_norm(x, None)


@pytest.mark.parametrize("wtype", list(TYPES))
@pytest.mark.parametrize("dtype", list(TYPES))
def test_norm_weight_types(dtype, wtype):
    g = gen(3, 17)
    for cols in (768, 1021, 5000, 17000):
        x = matrix(9, cols, TYPES[dtype], g)
        check_norm(x, torch.randn(cols, generator=g, device="cuda").to(TYPES[wtype]))


def test_norm_many_rows_of_every_shape():
    g = gen(5, 23)
    for rows, cols in ((70000, 8), (9001, 96), (4097, 768), (2049, 1021), (1500, 4096), (700, 16384), (149, 20000)):
        x = matrix(rows, cols, torch.bfloat16, g)
        check_norm(x, torch.randn(cols, generator=g, device="cuda"), matrix(rows, cols, torch.bfloat16, g))


@pytest.mark.parametrize("cols", [40, 1000, 17000])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_norm_in_place_and_broadcast_residual(dtype, cols):
    g = gen(cols, 29)
    dt = TYPES[dtype]
    x, r, w = matrix(37, cols, dt, g), matrix(37, cols, dt, g), torch.randn(cols, generator=g, device="cuda")
    y, total, rstd = cd.rms_norm(x, w, r)
    a, b = x.clone(), r.clone()
    cd.rms_norm(a, w, b, out=(b, a, None))              # the sum over x, the output over the residual
    assert torch.equal(a, total) and torch.equal(b, y)
    a, b = x.clone(), r.clone()
    cd.rms_norm(a, w, b, out=(a, b, None))              # the other way round
    assert torch.equal(b, total) and torch.equal(a, y)
    a = x.clone()
    assert torch.equal(cd.rms_norm(a, w, r, out=(a, None, None))[0], y)
    row = r[:1].expand(37, cols)
    got = cd.rms_norm(x, w, row)
    want = cd.rms_norm(x, w, row.contiguous())
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("cols", [300, 17000])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_norm_rows_without_size_and_not_finite(dtype, cols):
    g = gen(4, 31)
    x = matrix(7, cols, TYPES[dtype], g)
    x[0] = 0.0
    x[1] = 0.0
    x[1, 7] = 1e-7
    x[2] *= 1e-3
    x[3] = 1.0
    check_norm(x, None)
    check_norm(x, torch.randn(cols, generator=g, device="cuda"))
    x[4, 17], x[5, 3], x[6, cols - 1] = math.nan, INF, -INF
    kept = cd.checkpoint8_like(x)
    y, _, rstd = cd.rms_norm(x, checkpoint=kept)
    q, scale, _, _ = cd.rms_norm8(x)
    assert y[4].isnan().all() and rstd[4].isnan() and rstd[5] == 0 and rstd[6] == 0
    assert y[5, 3].isnan() and y[6, cols - 1].isnan() and y[5:].isnan().sum() == 2 and not y[5, :3].any()
    assert scale[4:].isnan().all() and not q[4:].any() and scale[:4].isfinite().all()
    for got, ref in zip(kept, kept64(x)):
        assert torch.equal(got, ref)


def test_norm_squares_beyond_binary32():
    x = torch.full((2, 64), 1e30, device="cuda")
    x[1] = 1.0
    y, _, rstd = cd.rms_norm(x)
    assert rstd[0] == 0 and not y[0].any() and y[1].allclose(torch.ones(64, device="cuda"))
    q, scale, _, _ = cd.rms_norm8(x)
    assert scale[0] == 0 and (q == 127).all()


# ---------------------------------------------------------------------------------------------
# rows and checkpoints
# ---------------------------------------------------------------------------------------------
def check_rows(x):
    q, scale = cd.quantize_rows(x)
    rq, step = rows64(x.float())
    assert torch.equal(q, rq), (q != rq).nonzero()[:3]
    close(scale, step, step * 2.0 ** -24 + 2.0 ** -149, "scale")
    for dtype in TYPES.values():
        got = cd.dequantize_rows(q, scale, dtype)
        assert torch.equal(got.nan_to_num(7.0), (q.float() * scale[:, None]).to(dtype).nan_to_num(7.0))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_at_halves(dtype):
    """Rows whose quotients are next to a half or on it: half the largest, odd multiples of the largest / 254."""
    g = gen(6, 37)
    dt = TYPES[dtype]
    m = torch.rand(64, 1, generator=g, device="cuda") * 3 + 0.1
    m[:8] = torch.tensor([127.0, 254.0, 63.5, 1.0, 0.5, 31.75, 2.0 ** -10, 508.0], device="cuda")[:, None]
    k = torch.randint(-127, 127, (64, 500), generator=g, device="cuda")
    x = ((2 * k + 1).double() * m.double() / 254).float()
    near = torch.randint(-2, 3, x.shape, generator=g, device="cuda").int()
    x = (x.view(torch.int32) + near).view(torch.float32)
    x = torch.minimum(torch.maximum(x, -m), m)
    x[:, :1], x[:, 1:2], x[:, 2:3] = m, m / 2, -m / 2
    check_rows(x.to(dt))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_every_size(dtype):
    g = gen(7, 41)
    for e in (-149, -140, -127, -120, -100, -20, 0, 15, 100, 126):
        x = (torch.randn(5, 333, generator=g, device="cuda").clamp(-1.9, 1.9).double() * 2.0 ** e).to(TYPES[dtype])
        if x.isfinite().all():
            check_rows(x)
    x = torch.zeros(4, 50, device="cuda", dtype=TYPES[dtype])
    x[1, 3], x[2, 4], x[3, 5] = math.nan, INF, -0.0
    check_rows(x)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", [1, 7, 8, 31, 32, 33, 63, 100, 1000, 1021, 4096, 70001])
def test_checkpoint_and_back(cols, dtype):
    g = gen(cols, 43)
    dt = TYPES[dtype]
    for rows, pad, shift in ((1, 0, 0), (6, 0, 0), (33, 3, 1), (9, 8, 8)):
        x = matrix(rows, cols, dt, g, 3.0, pad, shift)
        x *= torch.rand(rows, 1, generator=g, device="cuda").to(dt) * 4
        kept, exps = byte_matrix(rows, cols, pad, shift), byte_matrix(rows, -(-cols // 32), pad, shift, torch.uint8)
        cd.checkpoint8(x, out=(kept[0], exps[0]))
        for got, ref in zip((kept[0], exps[0]), kept64(x)):
            assert torch.equal(got, ref)
        assert untouched(*kept, shift) and untouched(*exps, shift)
        want = restored64(kept[0], exps[0])
        back = cd.checkpoint8_restore(kept[0], exps[0], out=matrix(rows, cols, dt, g, 1.0, pad, shift))
        assert torch.equal(back.double(), want)                            # exact in the type it was kept from
        assert torch.equal(cd.checkpoint8_restore(kept[0], exps[0], torch.bfloat16).double(), want)    # and in bfloat16
        step = two_to(exps[0].long() - 127).repeat_interleave(32, 1)[:, :cols]
        off = (want - x.double()).abs()
        assert bool((off <= torch.where(x.double().abs() > 127 * step, step, step / 2)).all())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_checkpoint_of_every_size(dtype):
    g = gen(8, 47)
    dt = TYPES[dtype]
    rows = [(torch.randn(70, generator=g, device="cuda").clamp(-1.9, 1.9).double() * 2.0 ** e).to(dt) for e in range(-150, 128, 3)]
    rows += [torch.full((70,), v, device="cuda").to(dt) for v in (0.0, torch.finfo(dt).max, torch.finfo(dt).min, torch.finfo(dt).tiny, 127.5, 0.99)]
    x = torch.stack([r for r in rows if r.isfinite().all()])
    kept, exps = cd.checkpoint8(x)
    for got, ref in zip((kept, exps), kept64(x)):
        assert torch.equal(got, ref)
    assert torch.equal(cd.checkpoint8_restore(kept, exps, dt).double(), restored64(kept, exps))
    x = torch.ones(3, 100, device="cuda", dtype=dt)
    x[0, 40], x[1, 99], x[2, 0] = math.nan, INF, -INF
    kept, exps = cd.checkpoint8(x)
    assert exps.tolist() == [[121, 255, 121, 121], [121, 121, 121, 255], [255, 121, 121, 121]]
    back = cd.checkpoint8_restore(kept, exps, dt)
    assert back.isnan().sum() == 32 + 4 + 32 and (back[~back.isnan()] == 1).all()


# ---------------------------------------------------------------------------------------------
# gradient of the norm
# ---------------------------------------------------------------------------------------------
def check_backward(dy, x, w, groups=1, dtotal=None, checkpoint=False, **kw):
    rows, cols = dy.shape
    rstd = (x.double().square().mean(1) + 1e-6).rsqrt().float()
    if checkpoint:
        given = cd.checkpoint8(x)
        x64 = restored64(*given)
    else:
        given, x64 = x, x.double()
    s = rstd.double()[:, None]
    g64, xh = dy.double() * (1.0 if w is None else w.double()), x64 * s
    want = s * (g64 - xh * (g64 * xh).mean(1, keepdim=True)) + (0.0 if dtotal is None else dtotal.double())
    tol = sum_tol(cols)
    size = s * (g64.abs() * 2.0 ** -21 + xh.abs() * (g64 * xh).abs().mean(1, keepdim=True) * (tol + 2.0 ** -21))
    size = size + (0.0 if dtotal is None else dtotal.double().abs() * 2.0 ** -23)
    each = (dy.double() * xh).view(groups, -1, cols)
    dx, dw = cd.rms_norm_backward(dy, given, w, rstd, dtotal, groups, **kw)
    close(dx, want, size + round_tol(want, dy.dtype), "dx")
    close(dw, each.sum(1), each.abs().sum(1) * SUM + round_tol(each.sum(1), dw.dtype), "dweight")
    return given, rstd, dx, dw


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", COLS)
def test_backward_every_width(cols, dtype):
    g = gen(cols, 53)
    dt = TYPES[dtype]
    for i, (rows, groups, pad, shift) in enumerate(((1, 1, 0, 0), (12, 3, 0, 0), (10, 2, 8, 0), (9, 1, 3, 0), (8, 8, 0, 1), (77, 7, 0, 0))):
        x, dy = matrix(rows, cols, dt, g, 2.0, pad, shift), matrix(rows, cols, dt, g, 1.0, shift, pad)
        w = torch.randn(cols + 8, generator=g, device="cuda")[8 - i % 4:][:cols]
        dt_ = matrix(rows, cols, dt, g, 1.0, pad, shift) if i % 2 else None
        check_backward(dy, x, w, groups, dt_)
        check_backward(dy, x, w if i else None, groups, dt_, checkpoint=True)


def test_backward_many_rows():
    g = gen(9, 59)
    for rows, cols, groups in ((70000, 8, 7), (40000, 96, 1), (9000, 768, 8), (6001, 1021, 1), (4096, 4096, 2), (2400, 8192, 1), (3000, 16384, 3)):
        x, dy = matrix(rows, cols, torch.bfloat16, g), matrix(rows, cols, torch.bfloat16, g)
        w = torch.randn(cols, generator=g, device="cuda")
        for kept in (False, True):
            check_backward(dy, x, w, groups, dy if kept else None, checkpoint=kept)


@pytest.mark.parametrize("gtype", list(TYPES))
@pytest.mark.parametrize("cols", [100, 1024, 17000])
def test_backward_into_slices_and_accumulated(cols, gtype):
    g = gen(cols, 61)
    x, dy = matrix(600, cols, torch.float32, g), matrix(600, cols, torch.float32, g)
    w = torch.randn(cols, generator=g, device="cuda")
    grads = torch.full((3, 2 * cols + 5), 9.0, device="cuda").to(TYPES[gtype])
    _, rstd, dx, dw = check_backward(dy, x, w, 3)
    slice_ = grads[:, cols:2 * cols]
    cd.rms_norm_backward(dy, x, w, rstd, groups=3, out=(None, slice_))
    assert torch.equal(slice_, dw.to(slice_.dtype)) and (grads[:, :cols] == 9).all() and (grads[:, 2 * cols:] == 9).all()
    before = slice_.clone()
    cd.rms_norm_backward(dy, x, w, rstd, groups=3, out=(None, slice_), accumulate=True)
    assert torch.equal(slice_, (before.float() + dw).to(slice_.dtype))


@pytest.mark.parametrize("cols", [40, 1000, 17000])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_backward_in_place_and_selected_outputs(dtype, cols):
    g = gen(cols, 67)
    dt = TYPES[dtype]
    x, dy, more = (matrix(300, cols, dt, g) for _ in range(3))
    w = torch.randn(cols, generator=g, device="cuda")
    for kept in (False, True):
        given, rstd, dx, dw = check_backward(dy, x, w, 1, more, kept)
        for target in range(2 if kept else 3):
            a, b = dy.clone(), more.clone()
            c = given if kept else x.clone()
            out = (a, b, c)[target]
            got = cd.rms_norm_backward(a, c, w, rstd, b, out=(out, torch.empty_like(dw)))
            assert torch.equal(out, dx) and torch.equal(got[1], dw)
        assert torch.equal(cd.rms_norm_backward(dy, given, w, rstd, more, out=(torch.empty_like(dy), None))[0], dx)
        assert torch.equal(cd.rms_norm_backward(dy, given, w, rstd, more, out=(None, torch.empty_like(dw)))[1], dw)
        again = cd.rms_norm_backward(dy, given, w, rstd, more)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    row = dy[:1].expand(300, cols)
    got, want = cd.rms_norm_backward(row, x, w, rstd), cd.rms_norm_backward(row.contiguous(), x, w, rstd)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("cols", [40, 1000, 1021, 9000, 17000])
def test_backward_from_a_checkpoint_that_starts_anywhere(cols):
    g = gen(cols, 137)
    x, dy = matrix(50, cols, torch.bfloat16, g), matrix(50, cols, torch.bfloat16, g)
    given, rstd, dx, dw = check_backward(dy, x, None, 5, None, True)
    for pad, shift in ((3, 1), (8, 4), (16, 0)):
        kept, exps = byte_matrix(50, cols, pad, shift)[0], byte_matrix(50, -(-cols // 32), pad, shift, torch.uint8)[0]
        kept.copy_(given[0])
        exps.copy_(given[1])
        got = cd.rms_norm_backward(dy, (kept, exps), None, rstd, groups=5)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw)


def test_backward_of_the_most_groups():
    g = gen(22, 139)
    x, dy = matrix(2 * 65535, 8, torch.float32, g), matrix(2 * 65535, 8, torch.float32, g)
    check_backward(dy, x, None, 65535)
    check_backward(dy, x, None, 65535, checkpoint=True)
    x, dy = matrix(65535, 16400, torch.bfloat16, g), matrix(65535, 16400, torch.bfloat16, g)
    rstd = torch.ones(65535, device="cuda")
    dw = torch.empty(65535, 16400, dtype=torch.bfloat16, device="cuda")
    cd.rms_norm_backward(dy, x, None, rstd, groups=65535, out=(None, dw))
    for a in range(0, 65535, 8192):
        want = dy[a:a + 8192].float() * x[a:a + 8192].float()
        assert torch.equal(dw[a:a + 8192], want.bfloat16())


def test_single_outputs_of_the_norm():
    """Through the C entry point, each output alone and all of them."""
    g = gen(23, 149)
    x, r = (torch.randn(33, 520, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(520, generator=g, device="cuda")
    kept = cd.checkpoint8_like(x)
    y, total, rstd = cd.rms_norm(x, w, r, checkpoint=kept)
    q, scale, _, _ = cd.rms_norm8(x, w, r)
    want = {"total": total, "y": y, "q": q, "scale": scale, "kept": kept[0], "exponents": kept[1], "rstd": rstd}
    for names in (("total",), ("y",), ("q", "scale"), ("kept", "exponents"), ("rstd",), tuple(want)):
        got = {n: torch.zeros_like(want[n], memory_format=torch.contiguous_format) for n in names}
        p = {n: got[n].data_ptr() if n in got else None for n in want}
        code = cd.lib().cdadam_rms_norm(x.data_ptr(), 520, r.data_ptr(), 520, w.data_ptr(), 33, 520, 1e-6, cd.BF16, cd.F32, p["total"], 520,
                                        p["y"], 520, p["q"], 520, p["scale"], p["kept"], 520, p["exponents"], 17, p["rstd"],
                                        torch.cuda.current_stream().cuda_stream)
        assert code == cd.OK and all(torch.equal(got[n], want[n]) for n in names), names


def test_backward_without_rows():
    e = torch.empty(0, 70, device="cuda")
    dw = torch.full((2, 70), 5.0, device="cuda")
    cd.rms_norm_backward(e, e, None, torch.empty(0, device="cuda"), groups=2, out=(e, dw))
    assert not dw.any()
    cd.rms_norm_backward(e, cd.checkpoint8(e), None, torch.empty(0, device="cuda"), out=(e, dw[:1].fill_(3.0)), accumulate=True)
    assert (dw[0] == 3).all()


def test_backward_against_differences():
    """Central differences of the forward kernel along a direction, step 2^-7: the third derivative's term is below
    2^-14 of the gradient's size here, the rounding of y (2^-24 of up to 4 for 12 x 96 terms, over the step) below 2^-12."""
    g = gen(10, 71)
    x, r, c, c2, d = (torch.randn(12, 96, generator=g, device="cuda") for _ in range(5))
    w, dw_ = torch.randn(2, 96, generator=g, device="cuda").unbind(0)

    def f(t):
        y, total, _ = cd.rms_norm(x + t * d, w + t * dw_, r)
        return float((y.double() * c.double()).sum() + (total.double() * c2.double()).sum())
    _, total, rstd = cd.rms_norm(x, w, r)
    dx, dw = cd.rms_norm_backward(c, total, w, rstd, c2)
    h = 2.0 ** -7
    slope = (f(h) - f(-h)) / (2 * h)
    want = float((dx.double() * d.double()).sum() + (dw[0].double() * dw_.double()).sum())
    size = float((dx.double() * d.double()).abs().sum() + (dw[0].double() * dw_.double()).abs().sum())
    assert abs(slope - want) <= size * 2.0 ** -10, (slope, want, size)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", [1, 5, 40, 260, 1000, 1021, 4099, 9001, 17003])
def test_nothing_around_the_rows_is_written(cols, dtype):
    """Every output of the activations' type into rows that start anywhere, on buffers of NaN; inputs likewise, so that a
    value from outside a row would show."""
    g = gen(cols, 131)
    dt = TYPES[dtype]
    for shift, pad in ((0, 0), (1, 0), (0, 1), (3, 2), (8, 8), (5, 7), (4, 4)):
        for rows in (1, 2, 37):
            x, r, dy = (matrix(rows, cols, dt, g, 1.0, pad, shift) for _ in range(3))
            w = torch.randn(cols, generator=g, device="cuda")

            def out():
                buf = torch.full((shift + rows * (cols + pad) + 40,), math.nan, device="cuda").to(dt)
                return buf, torch.as_strided(buf, (rows, cols), (cols + pad, 1), shift)
            want = cd.rms_norm(x.contiguous(), w, r.contiguous())
            kept = cd.checkpoint8(x)
            q, scale = cd.quantize_rows(x)
            dwant = cd.rms_norm_backward(dy.contiguous(), x.contiguous(), w, want[2], r.contiguous())
            for buf, view, expected, call in (
                    (*out(), want[0], lambda v: cd.rms_norm(x, w, r, out=(v, None, None))),
                    (*out(), want[1], lambda v: cd.rms_norm(x, w, r, out=(None, v, None))),
                    (*out(), dwant[0], lambda v: cd.rms_norm_backward(dy, x, w, want[2], r, out=(v, None))),
                    (*out(), cd.checkpoint8_restore(*kept, dtype=dt), lambda v: cd.checkpoint8_restore(*kept, out=v)),
                    (*out(), cd.dequantize_rows(q, scale, dt), lambda v: cd.dequantize_rows(q, scale, out=v))):
                call(view)
                close(view, expected.double(), expected.double().abs() * 2.0 ** -6 + 1e-3)
                assert (~buf.isnan()).sum() == rows * cols     # a gradient may be beyond binary16: infinite, not NaN


# ---------------------------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------------------------
def eight(rows, inner, g, pad=0, low=-127):
    """8-bit rows 16-byte aligned, what lies behind a row's end is 77."""
    stride = -(-inner // 16) * 16 + pad
    m = torch.full((rows, stride), 77, dtype=torch.int8, device="cuda")[:, :inner]
    m.copy_(torch.randint(low, 128, (rows, inner), generator=g, device="cuda"))
    return m


def product64(x, xs, w, ws, bias, dtype):
    """The documented binary32 steps on the exact sum."""
    y = (x.double() @ w.double().T).float() * xs[:, None] * ws
    return (y if bias is None else y + bias.float()).to(dtype)


def check_product(tokens, channels, inner, g, dtype=torch.float32, bias=None, pad=0, y_pad=0):
    x, w = eight(tokens, inner, g, pad), eight(channels, inner, g, pad)
    xs, ws = torch.rand(tokens, generator=g, device="cuda") + 0.01, torch.randn(channels, generator=g, device="cuda") * 0.01
    b = None if bias is None else torch.randn(channels, generator=g, device="cuda").to(bias)
    out = matrix(tokens, channels, dtype, g, 1.0, y_pad, y_pad)
    rest = torch.as_strided(out, (tokens, channels + y_pad), (channels + y_pad, 1))
    got = cd.matmul8(x, xs, w, ws, b, out=out)
    want = product64(x, xs, w, ws, b, dtype)
    assert torch.equal(got, want), ((got != want).nonzero()[:4], float((got - want).abs().max()))
    if y_pad:
        assert rest[:, channels:].isnan().all()


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 200, 256, 257, 300, 513])
def test_product_every_number_of_tokens(tokens):
    g = gen(tokens, 73)
    for channels, inner in ((1, 1), (5, 16), (127, 100), (128, 128), (129, 1021), (300, 129), (1000, 768), (333, 4100)):
        check_product(tokens, channels, inner, g)


@pytest.mark.parametrize("inner", [1, 2, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 255, 256, 257, 511, 1000, 1024, 5001, 16384, 131071])
def test_product_every_length(inner):
    g = gen(inner, 79)
    for tokens, channels in ((1, 70), (3, 129), (8, 513), (9, 128), (40, 257), (130, 300), (300, 259)):
        check_product(tokens, channels, inner, g)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("bias", [None] + list(TYPES))
def test_product_types_bias_and_strides(dtype, bias):
    g = gen(12, 83)
    for tokens, channels, inner in ((1, 500, 768), (6, 333, 100), (20, 130, 512), (100, 1000, 260), (700, 515, 384), (300, 9500, 96)):
        check_product(tokens, channels, inner, g, TYPES[dtype], None if bias is None else TYPES[bias], pad=32, y_pad=3)


def test_product_of_many_tiles():
    g = gen(13, 89)
    for tokens, channels, inner in ((1, 70000, 64), (5, 30000, 512), (64, 30522, 256), (2049, 2500, 200), (4100, 8200, 128), (1030, 20011, 96),
                                    (20000, 300, 64)):
        check_product(tokens, channels, inner, g, torch.bfloat16)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shift,pad", [(0, 0), (0, 1), (1, 0), (1, 1), (2, 2), (0, 2), (3, 2), (8, 8), (5, 11)])
def test_product_of_many_tokens_to_rows_that_start_anywhere(shift, pad, dtype):
    g = gen(shift * 16 + pad, 91)
    for tokens, channels in ((300, 4100), (513, 3000 + pad), (1000, 2049)):
        x, w = eight(tokens, 150, g), eight(channels, 150, g)
        xs, ws = torch.rand(tokens, generator=g, device="cuda") + 0.01, torch.randn(channels, generator=g, device="cuda") * 0.01
        b = torch.randn(channels, generator=g, device="cuda")
        buf = torch.full((shift + tokens * (channels + pad) + 64,), math.nan, device="cuda").to(TYPES[dtype])
        out = torch.as_strided(buf, (tokens, channels), (channels + pad, 1), shift)
        for bias in (None, b):
            cd.matmul8(x, xs, w, ws, bias, out=out)
            assert torch.equal(out, product64(x, xs, w, ws, bias, TYPES[dtype]))
        assert buf.isfinite().sum() == tokens * channels      # and nothing around the rows


def test_product_of_the_largest_sums():
    for tokens in (1, 8, 9, 300):
        x = torch.full((tokens, 131072), -128, dtype=torch.int8, device="cuda")[:, :131071]
        w = torch.full((130, 131072), -128, dtype=torch.int8, device="cuda")[:, :131071]
        one, ones = torch.ones(tokens, device="cuda"), torch.ones(130, device="cuda")
        assert (cd.matmul8(x, one, w, ones, dtype=torch.float32) == 16384 * 131071).all()
        w[1::2] = 127
        assert (cd.matmul8(x, one, w, ones, dtype=torch.float32)[:, 1::2] == torch.tensor(-16256 * 131071.0)).all()


@pytest.mark.parametrize("tokens", [1, 8, 30, 300])
def test_product_scales_that_are_not_finite(tokens):
    g = gen(14, 97)
    x, w = eight(tokens, 200, g), eight(300, 200, g)
    xs, ws = torch.ones(tokens, device="cuda"), torch.ones(300, device="cuda")
    xs[0], ws[7], ws[8] = math.nan, 0.0, math.nan
    y = cd.matmul8(x, xs, w, ws, dtype=torch.float32)
    assert y[0].isnan().all() and y[:, 8].isnan().all() and not y[1:, 7].any() and y[1:, 9:].isfinite().all()


def test_product_without_tokens_or_channels():
    g = gen(15, 101)
    e = torch.empty(0, device="cuda")
    assert cd.matmul8(eight(0, 64, g), e, eight(5, 64, g), torch.ones(5, device="cuda")).shape == (0, 5)
    assert cd.matmul8(eight(5, 64, g), torch.ones(5, device="cuda"), eight(0, 64, g), e).shape == (5, 0)


# ---------------------------------------------------------------------------------------------
# all of them together
# ---------------------------------------------------------------------------------------------
def teacher_pass(x, r, w, head, head_scale):
    """A teacher's last layer: norm of the sum in 8 bits, logits, its list for a distillation."""
    q, scale, total, _ = cd.rms_norm8(x, w, r)
    logits = cd.matmul8(q, scale, head, head_scale)
    _, _, _, ids, top = cd.token_logprobs(logits, k=8)
    return total, logits, ids, top


def test_teacher_and_student_together():
    """A teacher's list by the 8-bit operators; a student's loss and gradient from a checkpoint, against 64 bits and
    what the list says."""
    g = gen(16, 103)
    rows, cols, vocab = 64, 256, 1000
    x, r = (torch.randn(rows, cols, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.rand(cols, generator=g, device="cuda") + 0.5
    head, head_scale = cd.quantize_rows(torch.randn(vocab, cols, generator=g, device="cuda") * 0.2)
    total, logits, ids, top = teacher_pass(x, r, w, head, head_scale)
    h = (x.float() + r.float()).bfloat16()
    q, _ = rows64(h.float() * w)
    scale = (h.float() * w).abs().amax(1).double() / 127 * (h.double().square().mean(1) + 1e-6).rsqrt()
    want = (q.double() @ head.double().T) * scale[:, None] * head_scale.double()
    close(logits, want, want.abs() * 2.0 ** -14 + round_tol(want, torch.bfloat16), "logits")
    assert torch.equal(total, h) and torch.equal(ids[:, 0], logits.float().argmax(1))
    # the student: its norm keeps a checkpoint, its loss goes back through it
    kept = cd.checkpoint8_like(x)
    y, _, rstd = cd.rms_norm(x, w, r, checkpoint=kept)
    W = (torch.randn(vocab, cols, generator=g, device="cuda") * 0.05).bfloat16()
    loss, dlogits = cd.distill(y @ W.T, ids, top, torch.full((rows,), 1.0 / rows, device="cuda"))
    dy = dlogits @ W
    dx, dw = cd.rms_norm_backward(dy, kept, w, rstd, dtotal=dy, groups=4)
    x64, s = restored64(*kept), rstd.double()[:, None]
    g64 = dy.double() * w.double()
    ref = s * (g64 - x64 * s * (g64 * x64 * s).mean(1, keepdim=True)) + dy.double()
    close(dx, ref, ref.abs().amax() * 2.0 ** -14 + round_tol(ref, torch.bfloat16), "dx")
    each = (dy.double() * x64 * s).view(4, -1, cols)
    close(dw, each.sum(1), each.abs().sum(1) * SUM + 1e-30, "dweight")


@pytest.mark.parametrize("tokens", [1, 2, 30, 300, 2100])
def test_captured_and_replayed(tokens):
    """One graph of the whole chain, replayed on other inputs in the same buffers."""
    g = gen(17, tokens)
    cols, vocab = 520, 1003
    head, head_scale = cd.quantize_rows(torch.randn(vocab, cols, generator=g, device="cuda"))
    w = torch.randn(cols, generator=g, device="cuda")
    x, r, dy = (torch.randn(tokens, cols, generator=g, device="cuda").bfloat16() for _ in range(3))

    def chain():
        kept = cd.checkpoint8_like(x)
        q, scale, total, rstd = cd.rms_norm8(x, w, r, checkpoint=kept)
        return (cd.matmul8(q, scale, head, head_scale), cd.checkpoint8_restore(*kept), cd.dequantize_rows(q, scale),
                *cd.rms_norm_backward(dy, kept, w, rstd, total))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain()
    for _ in range(3):
        for t in (x, r, dy):
            t.copy_(torch.randn(tokens, cols, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, chain()))


def test_streams():
    """On a stream given, after work queued there, and on the current one of another stream's context."""
    g = gen(18, 107)
    x = torch.randn(500, 1000, generator=g, device="cuda")
    head, head_scale = cd.quantize_rows(torch.randn(700, 1000, generator=g, device="cuda"))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late = x * 2
    q, scale, total, rstd = cd.rms_norm8(late, None, late, stream=side)
    y = cd.matmul8(q, scale, head, head_scale, stream=side)
    kept = cd.checkpoint8(late, stream=side)
    back = cd.checkpoint8_restore(*kept, stream=side)
    values = cd.dequantize_rows(q, scale, stream=side)
    dx, dw = cd.rms_norm_backward(late, kept, None, rstd, stream=side)
    side.synchronize()
    x2 = x * 2
    q2, scale2, total2, rstd2 = cd.rms_norm8(x2, None, x2)
    want = (cd.matmul8(q2, scale2, head, head_scale), cd.checkpoint8_restore(*cd.checkpoint8(x2)), cd.dequantize_rows(q2, scale2),
            *cd.rms_norm_backward(x2, cd.checkpoint8(x2), None, rstd2))
    for a, b in zip((y, back, values, dx, dw), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("tokens", [9, 100, 300, 3000])
def test_product_waits_that_run_out(tokens):
    g = gen(19, 109)
    x, w = eight(tokens, 2000, g), eight(1500, 2000, g)
    xs, ws = torch.ones(tokens, device="cuda"), torch.ones(1500, device="cuda")
    want = cd.matmul8(x, xs, w, ws).clone()
    try:
        cd.set_operator_wait_limit(0)
        got = cd.matmul8(x, xs, w, ws)
        torch.cuda.synchronize()
    finally:
        cd.set_operator_wait_limit(-1)
    assert got.isnan().all()
    assert torch.equal(cd.matmul8(x, xs, w, ws), want)


def test_calls_of_several_threads():
    """Sizes that differ in the shared memory their kernels take, from host threads with streams of their own."""
    import threading
    g = gen(21, 127)
    x, w = eight(400, 500, g), eight(9000, 500, g)
    xs, ws = torch.ones(400, device="cuda"), torch.ones(9000, device="cuda")
    a = [torch.randn(64, cols, generator=g, device="cuda") for cols in (100, 9000, 16000)]
    jobs = [lambda t=t: cd.matmul8(x[:t], xs[:t], w, ws) for t in (1, 20, 100, 400)]
    jobs += [lambda m=m: cd.rms_norm_backward(m, m, None, xs[:64])[1] for m in a]
    want = [j().clone() for j in jobs]
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(40):
                got = jobs[i]()
                torch.cuda.current_stream().synchronize()
                if not torch.equal(got, want[i]):
                    wrong.append(i)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_rows_far_apart():
    """Offsets beyond 2^32 bytes and elements."""
    stride = (1 << 31) - 64
    g = gen(20, 113)
    big = torch.empty(2 * stride + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (3, 1000), (stride, 1))
    x.copy_(torch.randn(3, 1000, generator=g, device="cuda"))
    near, w = x.clone(), torch.randn(1000, generator=g, device="cuda")
    y, _, rstd = cd.rms_norm(near, w)
    dx, dw = cd.rms_norm_backward(near, near, w, rstd)
    kept, exps = cd.checkpoint8(near)
    assert all(torch.equal(a, b) for a, b in zip(cd.checkpoint8(x), (kept, exps)))
    got = cd.rms_norm_backward(x, x, w, rstd)
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
    cd.rms_norm(x, w, out=(x, None, None))
    assert torch.equal(x, y)
    cd.checkpoint8_restore(kept, exps, out=x)
    assert torch.equal(x, cd.checkpoint8_restore(kept, exps, torch.bfloat16))
    head, head_scale = cd.quantize_rows(torch.randn(1000, 64, generator=g, device="cuda"))
    q, scale = cd.quantize_rows(torch.randn(3, 64, generator=g, device="cuda"))
    far = torch.as_strided(big.view(torch.int8), (3, 64), (stride // 16 * 16, 1))
    far.copy_(q)
    want = cd.matmul8(q, scale, head, head_scale)
    assert torch.equal(cd.matmul8(far, scale, head, head_scale), want)
    q20 = q.repeat(7, 1)[:20]
    cd.matmul8(far, scale, head, head_scale, out=torch.as_strided(big, (3, 1000), (stride, 1), 1024))
    assert torch.equal(torch.as_strided(big, (3, 1000), (stride, 1), 1024), want)
    far20 = torch.as_strided(big, (20, 1000), (stride // 10, 1), 0)
    cd.matmul8(q20, scale.repeat(7)[:20], head, head_scale, out=far20)
    assert torch.equal(far20, want.repeat(7, 1)[:20])
