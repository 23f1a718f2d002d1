"""The operators around a worker's loss against plain implementations in 64 bits.

Tolerances.  Outputs are rounded once to their type: a relative error of 2^-24 (binary32),
2^-8 (bfloat16) or 2^-11 (binary16; 2^-25 absolute among its subnormals).  Below that, every
bound comes from the sums: a sum of n positive binary32 terms that a thread adds one after the
other has a relative error of at most n 2^-24, an exponential of 2^-22, so a normaliser of up to
2^19 terms over at least 256 threads is off by at most 2^11 2^-24 + 2^-21 < 2^-12.9 and, with
rounding errors of random sign, by 2^-18; 2^-15 is what is allowed, which a lost or doubled
tile, list entry or tail exceeds in the tests' rows.  Indexes have to be equal.
"""
import math

import pytest
import torch

from paper_2111_00705_b200 import binding as cd

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}
SUM = 2.0 ** -15
INF = math.inf


def gen(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(hash(key) & 0x7FFFFFFF if not all(isinstance(k, int) for k in key) else sum(k * 7919 ** i for i, k in enumerate(key)))
    return g


def matrix(rows, cols, dtype, g, scale=1.0, pad=0, shift=0):
    """A rows x cols matrix with row stride cols + pad whose first element is `shift` elements
    behind a 256-byte boundary; what lies between and around the rows is NaN."""
    buf = torch.full((shift + rows * (cols + pad) + 16,), math.nan, device="cuda").to(dtype)
    m = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=g, device="cuda") * scale)
    return m


def close(got, want, tol, what=""):
    most = torch.finfo(got.dtype).max                           # what is beyond the type's range is rounded to infinity
    got, want = got.double(), want.double()
    want = torch.where(want > most, INF, torch.where(want < -most, -INF, want))
    same = (got == want) | (got.isnan() & want.isnan())
    fine = same | ((got - want).abs() <= tol)
    assert bool(fine.all()), "%s: worst excess %g at %s" % (
        what, float(torch.where(fine, 0.0, (got - want).abs() - tol).nan_to_num(INF).max()),
        (~fine).nonzero()[:3].tolist())


def round_tol(want, dtype):
    return want.abs() * UNIT[dtype] + TINY[dtype]


# ---------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------
def norm64(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    xh = (x - mean) * rstd
    return xh * (1.0 if w is None else w.double()) + (0.0 if b is None else b.double()), mean[:, 0], rstd[:, 0]


def check_norm(x, w, b, eps=1e-5, **kw):
    y, mean, rstd = cd.layer_norm(x, w, b, eps, **kw)
    torch.cuda.synchronize()
    ry, rm, rr = norm64(x, w, b, eps)
    big = x.double().abs().amax(1)
    close(mean, rm, SUM * 2.0 ** -4 * big + 1e-37, "mean")
    # the mean's rounding enters the deviations: |x| 2^-24 against their spread 1 / rstd
    close(rstd, rr, rr * (SUM + 2.0 ** -20 * (big * rr)), "rstd")
    xh = ((x.double() - rm[:, None]) * rr[:, None]).abs()
    inner = xh * SUM + 2.0 ** -20 * (big * rr)[:, None] * (1 + xh)
    wa = 1.0 if w is None else w.double().abs()
    ba = 0.0 if b is None else b.double().abs()
    close(y, ry, inner * wa + 2.0 ** -22 * (xh * wa + ba) + round_tol(ry, x.dtype), "y")
    return y, mean, rstd


COLS = [1, 2, 3, 5, 8, 31, 32, 33, 64, 100, 255, 256, 257, 511, 768, 1000, 1021, 1024, 1032, 2047, 2048, 2056, 4096, 4100, 8191,
        8192, 8200, 10001, 16384, 16392, 20000, 32768, 33000, 70001]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", COLS)
def test_norm_every_width(cols, dtype):
    g = gen(cols, len(dtype))
    for rows, pad, shift in ((1, 0, 0), (5, 0, 0), (3, 8, 0), (2, 3, 0), (7, 0, 1), (4, 1, 3)):
        x = matrix(rows, cols, TYPES[dtype], g, 2.0, pad, shift)
        w = torch.randn(cols + 8, generator=g, device="cuda")
        check_norm(x, w[8:], w[:cols] * 0.5)
        check_norm(x, w[1:cols + 1], w[3:cols + 3])


@pytest.mark.parametrize("wtype", list(TYPES))
@pytest.mark.parametrize("dtype", list(TYPES))
def test_norm_parameter_types_and_absent_parameters(dtype, wtype):
    g = gen(1, 2)
    for cols in (768, 1021, 5000):
        x = matrix(9, cols, TYPES[dtype], g)
        w, b = (torch.randn(cols, generator=g, device="cuda").to(TYPES[wtype]) for _ in range(2))
        check_norm(x, w, b)
        check_norm(x, w, None)
        check_norm(x, None, b)
        check_norm(x, None, None)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_norm_constant_rows_offsets_and_non_finite(dtype):
    dt = TYPES[dtype]
    g = gen(3, 4)
    x = matrix(6, 300, dt, g)
    x[0] = 1.0                                            # no spread: rstd = 1 / sqrt(eps)
    x[1] += 50.0                                          # a large common offset
    x[2] = 0.0
    x[3] *= 1e-3
    check_norm(x, None, None)
    x[4, 17], x[5, 3] = math.nan, INF
    y, mean, rstd = cd.layer_norm(x)
    assert y[4].isnan().all() and y[5].isnan().all() and not y[:4].isnan().any()


def test_norm_many_rows_of_every_shape():
    g = gen(5, 5)
    for rows, cols in ((70000, 8), (4097, 96), (2049, 768), (600, 4096), (149, 16384)):
        x = matrix(rows, cols, torch.bfloat16, g)
        check_norm(x, torch.randn(cols, generator=g, device="cuda"), torch.randn(cols, generator=g, device="cuda"))


def test_norm_in_place_broadcast_rows_and_selected_outputs():
    g = gen(6, 6)
    x = matrix(37, 1000, torch.float32, g)
    want = cd.layer_norm(x)[0].clone()
    y, mean, rstd = cd.layer_norm(x, out=(x, None, None))
    assert y is x and mean is None and rstd is None and torch.equal(x, want)
    row = matrix(1, 1000, torch.bfloat16, g)
    y = cd.layer_norm(row.expand(33, 1000))[0]
    assert torch.equal(y, cd.layer_norm(row)[0].expand(33, 1000))


def backward64(dy, x, w, mean, rstd, groups):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (x - mean) * rstd
    h = dy * (1.0 if w is None else w.double())
    dx = rstd * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    per = (groups, -1, x.shape[1])
    if x.shape[0] == 0:
        z = torch.zeros(groups, x.shape[1], device=x.device, dtype=torch.float64)
        return dx, z, z.clone(), z.clone(), z.clone(), dx
    scale = rstd * (h.abs() + h.abs().mean(1, keepdim=True) + xh.abs() * (h * xh).abs().mean(1, keepdim=True))
    return (dx, (dy * xh).view(per).sum(1), dy.view(per).sum(1), (dy * xh).abs().view(per).sum(1), dy.abs().view(per).sum(1),
            scale)


def check_backward(dy, x, w, groups=1, before=None, **kw):
    _, mean, rstd = cd.layer_norm(x)
    rdx, rdw, rdb, aw, ab, scale = backward64(dy, x, w, mean, rstd, groups)
    dx, dw, db = cd.layer_norm_backward(dy, x, w, mean, rstd, groups=groups, **kw)
    torch.cuda.synchronize()
    if before is not None:
        rdw, rdb, aw, ab = rdw + before[0], rdb + before[1], aw + before[0].abs(), ab + before[1].abs()
    if dx is not None:
        close(dx, rdx, scale * SUM + round_tol(rdx, x.dtype), "dx")
    if dw is not None:
        close(dw, rdw, aw * SUM + round_tol(rdw, dw.dtype), "dweight")
    if db is not None:
        close(db, rdb, ab * SUM + round_tol(rdb, db.dtype), "dbias")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols", COLS)
def test_norm_backward_every_width(cols, dtype):
    g = gen(cols, 31 + len(dtype))
    for rows, pad, shift, groups in ((1, 0, 0, 1), (6, 0, 0, 3), (35, 8, 0, 1), (4, 3, 0, 2), (7, 0, 1, 7)):
        x = matrix(rows, cols, TYPES[dtype], g, 1.5, pad, shift)
        dy = matrix(rows, cols, TYPES[dtype], g, 0.1, 0, 2 * shift)
        w = torch.randn(cols + 1, generator=g, device="cuda")
        check_backward(dy, x, w[1:], groups)


@pytest.mark.parametrize("cols", [2, 10, 66, 250, 258, 514, 766, 770, 1022, 2050, 4090, 4098, 5002, 6146, 8190, 8194])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_norm_rows_that_start_on_two_elements(cols, dtype):
    g = gen(cols, 5 + len(dtype))
    for rows, pad, shift, groups in ((1, 0, 0, 1), (6, 0, 2, 3), (35, 2, 0, 1), (300, 4, 2, 2), (7, 6, 4, 7), (4, 1, 0, 2)):
        x = matrix(rows, cols, TYPES[dtype], g, 1.5, pad, shift)
        dy = matrix(rows, cols, TYPES[dtype], g, 0.1, 2, shift)
        w = torch.randn(2 * cols, generator=g, device="cuda")
        check_norm(x, w[:cols], w[cols:])
        check_backward(dy, x, w[cols:], groups)


@pytest.mark.parametrize("rows,cols,groups", [(16384, 768, 8), (3001, 1021, 1), (5000, 64, 5), (70000, 8, 1), (1200, 4096, 4),
                                              (400, 10001, 2), (300, 16384, 1), (150, 33000, 3), (64, 3000, 64), (1999, 1, 1)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_norm_backward_many_rows_and_groups(rows, cols, groups, dtype):
    g = gen(rows, cols)
    x, dy = matrix(rows, cols, TYPES[dtype], g), matrix(rows, cols, TYPES[dtype], g, 0.05)
    check_backward(dy, x, torch.randn(cols, generator=g, device="cuda"), groups)
    check_backward(dy, x, None, groups)


@pytest.mark.parametrize("gtype", list(TYPES))
def test_norm_backward_into_strided_gradient_rows_and_accumulating(gtype):
    g = gen(8, 8)
    for cols, rows, groups in ((768, 96, 4), (1021, 33, 3), (5000, 16, 2)):
        x, dy = matrix(rows, cols, torch.bfloat16, g), matrix(rows, cols, torch.bfloat16, g, 0.1)
        w = torch.randn(cols, generator=g, device="cuda")
        buf = torch.full((groups, 3 * cols + 5), 7.0, device="cuda").to(TYPES[gtype])
        dw, db = buf[:, 1:cols + 1], buf[:, cols + 3:2 * cols + 3]
        out = (torch.empty_like(x), dw, db)
        check_backward(dy, x, w, groups, out=out)
        keep = (buf[:, :1], buf[:, cols + 1:cols + 3], buf[:, 2 * cols + 3:])
        assert all(bool((t == 7.0).all()) for t in keep)      # nothing beside the slices is touched
        before = (dw.double().clone(), db.double().clone())
        check_backward(dy, x, w, groups, before=before, out=out, accumulate=True)


def test_norm_backward_parts_alone_in_place_and_without_rows():
    g = gen(9, 9)
    for cols in (768, 1021, 20000):
        x, dy = matrix(40, cols, torch.float32, g), matrix(40, cols, torch.float32, g)
        w = torch.randn(cols, generator=g, device="cuda")
        _, mean, rstd = cd.layer_norm(x)
        dx, dw, db = cd.layer_norm_backward(dy, x, w, mean, rstd, groups=2)
        e = lambda: torch.full((2, cols), math.nan, device="cuda")
        a, b, c = (cd.layer_norm_backward(dy, x, w, mean, rstd, groups=2, out=o)
                   for o in ((torch.empty_like(x), None, None), (None, e(), None), (None, None, e())))
        assert torch.equal(a[0], dx) and torch.equal(b[1], dw) and torch.equal(c[2], db)
        dy2, x2 = dy.clone(), x.clone()
        got = cd.layer_norm_backward(dy2, x, w, mean, rstd, groups=2, out=(dy2, e(), e()))
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)
        got = cd.layer_norm_backward(dy, x2, w, mean, rstd, groups=2, out=(x2, e(), e()))
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)
        none = torch.empty(0, cols, device="cuda")
        got = cd.layer_norm_backward(none, none, w, mean[:0], rstd[:0], groups=3, out=(none, e().new_full((3, cols), 5.0),
                                                                                     e().new_full((3, cols), 5.0)))
        assert not got[1].any() and not got[2].any()


def test_norm_gradient_against_differences():
    """Along random directions; with f = sum(dy y), second differences bound the error by h^2 / 6
    times a third derivative of order one (h = 2^-7), rounding by 2^-20 |f| / h."""
    g = gen(10, 10)
    x, dy = matrix(8, 96, torch.float32, g), matrix(8, 96, torch.float32, g)
    w, b = torch.randn(96, generator=g, device="cuda"), torch.randn(96, generator=g, device="cuda")
    _, mean, rstd = cd.layer_norm(x, w, b)
    dx, dw, db = cd.layer_norm_backward(dy, x, w, mean, rstd)
    f = lambda x, w, b: (cd.layer_norm(x, w, b)[0].double() * dy.double()).sum(1)
    h = 2.0 ** -7
    v = torch.randn(8, 96, generator=g, device="cuda")
    num = (f(x + h * v, w, b) - f(x - h * v, w, b)) / (2 * h)
    close(num, (dx.double() * v).sum(1), 0.02, "dx")
    u = torch.randn(96, generator=g, device="cuda")
    for grad, lo, hi in ((dw, (w - h * u, b), (w + h * u, b)), (db, (w, b - h * u), (w, b + h * u))):
        num = ((f(x, *hi) - f(x, *lo)) / (2 * h)).sum()
        close(num, (grad[0].double() * u).sum(), 0.02, "parameters")


# ---------------------------------------------------------------------------------------------
# token log probabilities
# ---------------------------------------------------------------------------------------------
def logprobs64(z, tokens, k, temperature):
    z = z.double()
    bad = (z.isnan() | (z == INF)).any(1)
    y = z / temperature
    m = y.amax(1, keepdim=True)
    m = torch.where(m.isfinite(), m, 0.0)
    ls = torch.log(torch.exp(y - m).sum(1))
    lse = m[:, 0] + ls
    lp = (y - m) - ls[:, None]                                  # m may be the type's lowest value: not y - lse
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
    ent = torch.where(lse == -INF, 0.0, ent)
    lse = torch.where(bad, math.nan, lse)
    ent = torch.where(bad, math.nan, ent)
    lp = torch.where(y == -INF, -INF, lp)
    at = None
    if tokens is not None:
        t = tokens.long()
        at = lp.gather(1, t.clamp(0, z.shape[1] - 1)[:, None])[:, 0]
        at = torch.where(bad, math.nan, at)
        at = torch.where(t < 0, 0.0, torch.where(t >= z.shape[1], math.nan, at))
    order = torch.sort(z + 0.0, dim=1, descending=True, stable=True).indices[:, :k]
    top = lp.gather(1, order)
    ids = torch.where(bad[:, None] | (top == -INF), -1, order)
    top = torch.where(bad[:, None], math.nan, top)
    return at, ent, lse, ids, top


def check_logprobs(z, tokens, k, temperature=1.0, **kw):
    got = cd.token_logprobs(z, tokens, k=k, temperature=temperature, **kw)
    torch.cuda.synchronize()
    want = logprobs64(z, tokens, k, temperature)
    lp_tol = lambda w: SUM + w.abs().nan_to_num(posinf=0.0) * 2.0 ** -21
    for name, a, b in zip(("logprob", "entropy", "lse", "ids", "top"), got, want):
        if a is None:
            continue
        if name == "ids":
            assert torch.equal(a.long(), b), (name, (a.long() != b).nonzero()[:4].tolist())
        else:
            # the entropy's sum of p log p carries the terms' relative errors, up to log(vocab) each
            close(a, b, lp_tol(b) * (3.0 if name == "entropy" else 1.0), name)
    return got


VOCABS = [1, 2, 7, 8, 31, 33, 64, 100, 127, 128, 129, 500, 1000, 1023, 1024, 1025, 2000, 4097, 8192, 16384, 30522, 32771, 50021,
          65536, 100001, 131072]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_logprobs_every_width(vocab, dtype):
    g = gen(vocab, 77 + len(dtype))
    for rows, pad, shift, scale, k in ((1, 0, 0, 2.0, 1), (5, 0, 0, 3.0, 20), (3, 8, 0, 0.5, 64), (4, 5, 0, 1.0, 128),
                                       (2, 0, 1, 8.0, 5), (6, 1, 3, 0.0, 7)):
        z = matrix(rows, vocab, TYPES[dtype], g, scale, pad, shift)
        tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        check_logprobs(z, tokens, min(k, vocab), 1.0 if rows % 2 else 0.7)


def test_logprobs_longest_rows():
    g = gen(12, 12)
    for dtype in TYPES.values():
        z = matrix(3, cd.MAX_VOCAB, dtype, g, 2.0, 0, 1)
        check_logprobs(z, torch.tensor([0, cd.MAX_VOCAB - 1, 77777], device="cuda"), 128)


@pytest.mark.parametrize("rows,vocab,k", [(3000, 5, 3), (2000, 1000, 20), (700, 30522, 20), (300, 50021, 0), (200, 131072, 64)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_logprobs_many_rows(rows, vocab, k, dtype):
    g = gen(rows, vocab, 3)
    z = matrix(rows, vocab, TYPES[dtype], g, 3.0)
    z[::3, vocab // 2:vocab // 2 + vocab // 5] = -INF
    check_logprobs(z, torch.randint(0, vocab, (rows,), generator=g, device="cuda"), k, 2.0)


def hard_rows(vocab, dtype, g):
    """Rows where a selection or a normaliser can go wrong."""
    lowest = torch.finfo(dtype).min
    i = torch.arange(vocab, device="cuda", dtype=torch.float32)
    rows = [torch.full((vocab,), 0.25, device="cuda"),                       # all equal
            torch.full((vocab,), -INF, device="cuda"),                       # nothing left
            torch.full((vocab,), lowest, device="cuda"),                     # the type's lowest value everywhere
            i / vocab * 8, -i / vocab * 8]                                   # ascending, descending (with ties)
    r = torch.full((vocab,), -INF, device="cuda"); r[vocab // 3] = 1.5; rows.append(r)            # one token left
    r = torch.full((vocab,), lowest, device="cuda"); r[vocab - 1] = -3.0; r[0] = 2.0; rows.append(r)
    r = torch.randn(vocab, generator=g, device="cuda"); r[::2] = -INF; rows.append(r)
    r = torch.randn(vocab, generator=g, device="cuda"); r[1::3] = lowest; rows.append(r)
    r = torch.randn(vocab, generator=g, device="cuda"); r[:min(300, vocab)] += 20.0; rows.append(r)   # the top in one place
    r = torch.randn(vocab, generator=g, device="cuda"); r[(i % 4096) < 8] += 20.0; rows.append(r)     # ... of every few tiles
    r = torch.randn(vocab, generator=g, device="cuda"); r[vocab // 2:vocab // 2 + 3000] = 9.0; rows.append(r)   # 3000 ties on top
    r = torch.zeros(vocab, device="cuda"); r[::2] = -0.0; rows.append(r)                                # zeros of both signs
    r = torch.randn(vocab, generator=g, device="cuda") + 1000.0; rows.append(r)                        # a large offset
    r = torch.randn(vocab, generator=g, device="cuda"); r[vocab // 2] = math.nan; rows.append(r)
    r = torch.randn(vocab, generator=g, device="cuda"); r[vocab // 4] = INF; rows.append(r)
    r = torch.full((vocab,), math.nan, device="cuda"); rows.append(r)
    r = torch.full((vocab,), -INF, device="cuda"); r[0] = math.nan; rows.append(r)
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [1, 3, 40, 1000, 5003, 32768, 70001, 131072])
def test_logprobs_hard_rows(vocab, dtype):
    g = gen(vocab, 5)
    z = hard_rows(vocab, TYPES[dtype], g)
    tokens = torch.full((z.shape[0],), vocab // 3, device="cuda")
    for k in (0, 1, 17, 64, 128):
        check_logprobs(z, tokens, min(k, vocab))
    check_logprobs(z, tokens.int(), min(5, vocab), 0.3)


def test_logprobs_tokens_that_are_none_or_out_of_range_and_selected_outputs():
    g = gen(14, 14)
    z = matrix(6, 1000, torch.bfloat16, g)
    z[5] = math.nan
    tokens = torch.tensor([-100, -1, 1000, 1 << 40, 999, -1], device="cuda")
    got = check_logprobs(z, tokens, 4)
    assert got[0][0] == 0 and got[0][5] == 0 and got[0][2:4].isnan().all()
    full = cd.token_logprobs(z, tokens, k=4)
    n = torch.full((6,), 3.0, device="cuda")
    a = cd.token_logprobs(z, None, out=(None, n, None, None, None))
    assert torch.equal(a[1][:5], full[1][:5])
    b = cd.token_logprobs(z, k=4)
    assert b[0] is None and torch.equal(b[3], full[3]) and torch.equal(b[4][:5], full[4][:5])
    c = cd.token_logprobs(z, tokens.clamp(-5, 2000).int(), k=4)
    assert c[3].dtype == torch.int32 and torch.equal(c[3].long(), full[3])


def test_logprobs_offsets_beyond_32_bits_and_repeated_rows():
    g = gen(15, 15)
    stride = (1 << 30) + 16
    buf = torch.empty(2 * stride + 2000, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((3, 2000), (stride, 1))
    z.copy_(torch.randn(3, 2000, generator=g, device="cuda"))
    out = torch.empty(2 * stride + 2000, dtype=torch.bfloat16, device="cuda").as_strided((3, 2000), (stride, 1))
    tokens = torch.tensor([1, 2, 3], device="cuda")
    lp, ent, lse, ids, top = check_logprobs(z, tokens, 9)
    check_logprobs_backward(z, tokens, lse, ent, lp, ent, out=out)
    same = z[2:].expand(5, 2000)
    got = cd.token_logprobs(same, tokens[:1].expand(5).contiguous(), k=9)
    assert torch.equal(got[3], ids[2:].expand(5, 9)) and torch.equal(got[2], lse[2:].expand(5))


def backward_logprobs64(z, tokens, lse, ent, dlp, dent, temperature):
    z64 = z.double()
    lp = z64 / temperature - lse.double()[:, None]
    p = lp.exp()
    lp = torch.where(p > 0, lp, 0.0)
    rows, vocab = z.shape
    g = torch.zeros(rows, 1, device="cuda", dtype=torch.float64)
    one = torch.zeros_like(z64)
    if dlp is not None:
        t = tokens.long()
        ok = (t >= 0) & (t < vocab)
        g = torch.where(ok, dlp.double(), 0.0)[:, None]
        one.scatter_(1, t.clamp(0, vocab - 1)[:, None], ok.double()[:, None])
    u = torch.zeros_like(g) if dent is None else dent.double()[:, None]
    H = torch.zeros_like(g) if dent is None else ent.double()[:, None]
    d = (g * (one - p) - u * p * (lp + H)) / temperature
    size = (g.abs() * (one + p) + u.abs() * p * (lp.abs() + H.abs() + 1)) / temperature
    none = (z64 == -INF) | ((g == 0) & (u == 0)) | (lse.abs() >= 2.0 ** 24)[:, None]
    return torch.where(none, 0.0, d), torch.where(none, 0.0, size)


def check_logprobs_backward(z, tokens, lse, ent, dlp, dent, temperature=1.0, **kw):
    src = z.clone()
    got = cd.token_logprobs_backward(z, tokens, lse, ent, dlp, dent, temperature=temperature, **kw)
    torch.cuda.synchronize()
    want, size = backward_logprobs64(src, tokens, lse, ent, dlp, dent, temperature)
    # z / T and lse cancel: their products with log2(e) / T, rounded, are off by 2^-24 of |lse|
    reach = 2.0 ** -22 * (lse.double().abs() + (src.double() / temperature).abs().nan_to_num(posinf=0.0).amax(1))
    reach = torch.where(reach.isfinite(), reach, 0.0)[:, None]
    close(got, want, size * (SUM + reach) + round_tol(want, z.dtype), "dlogits")
    return got


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_logprobs_backward_every_width(vocab, dtype):
    g = gen(vocab, 99 + len(dtype))
    for rows, pad, shift, opad, oshift in ((1, 0, 0, 0, 0), (5, 0, 0, 0, 0), (3, 8, 0, 0, 0), (4, 5, 1, 5, 1), (2, 0, 1, 3, 2)):
        z = matrix(rows, vocab, TYPES[dtype], g, 2.0, pad, shift)
        if vocab > 4:
            z[0, 1:3] = -INF
        tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        lp, ent, lse, _, _ = cd.token_logprobs(z, tokens, temperature=0.7)
        dlp, dent = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
        buf = matrix(rows, vocab, TYPES[dtype], g, 0.0, opad, oshift)
        check_logprobs_backward(z, tokens, lse, ent, dlp, dent, 0.7, out=buf)
        check_logprobs_backward(z, tokens, lse, None, dlp, None, 0.7)
        check_logprobs_backward(z, None, lse, ent, None, dent, 0.7)
        around = buf.as_strided((rows * (vocab + opad) + 16,), (1,), oshift)
        mask = torch.ones(rows * (vocab + opad) + 16, dtype=torch.bool, device="cuda")
        mask.as_strided((rows, vocab), (vocab + opad, 1)).fill_(False)
        assert around[mask].isnan().all()                      # nothing beside the rows is written


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [3, 1000, 30522])
def test_logprobs_backward_hard_rows_in_place_and_ignored(vocab, dtype):
    g = gen(vocab, 6)
    z = hard_rows(vocab, TYPES[dtype], g)[:14]                 # the rows that have a distribution, or are empty
    n = z.shape[0]
    tokens = torch.full((n,), vocab // 3, device="cuda")
    tokens[2], tokens[4] = -100, vocab
    lp, ent, lse, _, _ = cd.token_logprobs(z, tokens)
    dlp, dent = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    a = check_logprobs_backward(z, tokens, lse, ent, dlp, dent)
    b = check_logprobs_backward(z, tokens, lse, ent, dlp, None)
    assert not b[2].any() and not b[4].any() and not a[1].any()
    zz = z.clone()
    assert torch.equal(cd.token_logprobs_backward(zz, tokens, lse, ent, dlp, dent, out=zz), a)
    bad = z.clone(); bad[2] = math.nan
    assert not cd.token_logprobs_backward(bad, tokens, lse, ent, dlp, None)[2].any()


def test_logprobs_gradient_against_differences():
    """h = 2^-6 along directions of largest component about 3: third derivatives of lse and
    entropy are of order 10, so h^2 / 6 of them is below 0.002; rounding adds 2^-19 / h."""
    g = gen(16, 16)
    z = matrix(6, 500, torch.float32, g, 2.0)
    tokens = torch.randint(0, 500, (6,), generator=g, device="cuda")
    dlp, dent = torch.randn(6, generator=g, device="cuda"), torch.randn(6, generator=g, device="cuda")
    _, ent, lse, _, _ = cd.token_logprobs(z, tokens, temperature=1.5)
    dz = cd.token_logprobs_backward(z, tokens, lse, ent, dlp, dent, temperature=1.5)

    def f(z):
        lp, ent, _, _, _ = cd.token_logprobs(z, tokens, temperature=1.5)
        return lp.double() * dlp + ent.double() * dent
    h = 2.0 ** -6
    v = torch.randn(6, 500, generator=g, device="cuda")
    close((f(z + h * v) - f(z - h * v)) / (2 * h), (dz.double() * v).sum(1), 0.005, "differences")


# ---------------------------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------------------------
def distill64(z, ids, teacher, dloss, temperature, rest):
    """Row by row, from the definition."""
    rows, vocab = z.shape
    losses, ltol, grads, gtol = [], [], [], []
    for i in range(rows):
        y = z[i].double() / temperature
        t, ix = teacher[i].double(), ids[i].long()
        used = (ix >= 0) & (ix < vocab)
        if not rest:
            used &= t != -INF
        ix, t = ix[used], t[used]
        q = (t.exp() if rest else torch.softmax(t, 0)) if len(ix) else t
        full = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, ix, q)
        inside = torch.zeros(vocab, dtype=torch.bool, device="cuda")
        inside[ix] = True
        r = 1.0 - float(q.sum()) if rest and int(inside.sum()) < vocab else 0.0
        r = max(r, 0.0) if r == r else r
        m = float(y.max()) if float(y.max()) > -INF else 0.0
        e = torch.exp(y - m)
        lse = m + float(e.sum().log())
        lp = torch.where(y == -INF, -INF, (y - m) - e.sum().log())
        p = torch.where(y == -INF, 0.0, lp.exp()) if lse > -INF else torch.zeros_like(y)
        qs, ls = full[inside], lp[inside]
        term = torch.where(qs == 0, 0.0, qs * (qs.log() - ls))
        size = torch.where(qs == 0, 0.0, qs * (qs.log().abs() + ls.abs() + 1)).nan_to_num(posinf=0.0).sum()
        loss = term.sum()
        # relative to m as well, which may be the type's lowest value
        log_rest = torch.logsumexp((y - m).masked_fill(inside, -INF), 0) - e.sum().log() if lse > -INF else torch.full_like(e.sum(), -INF)
        if r > 0:
            loss = loss + r * (math.log(r) - log_rest)
            size = size + r * (abs(math.log(r)) + log_rest.abs().nan_to_num(posinf=0.0) + 1)
            # the rest of the teacher's list is what its probabilities leave: off by their rounding
            size = size + (abs(math.log(r)) + log_rest.abs().nan_to_num(posinf=0.0)) * 2.0 ** -8
        bad = bool((y.isnan() | (y == INF)).any())
        if len(ix) == 0:
            loss = torch.zeros((), dtype=torch.float64, device="cuda")
        elif not bad and lse == -INF:
            loss = torch.full((), INF, dtype=torch.float64, device="cuda")
        if bad:
            loss = torch.full((), math.nan, dtype=torch.float64, device="cuda")
        losses.append(loss)
        ltol.append(size)
        if dloss is not None:
            g = float(dloss[i]) / temperature
            over = r * torch.exp(lp - log_rest) if r > 0 and float(log_rest) > -INF else torch.zeros_like(p)
            d = g * (p - full - torch.where(inside, 0.0, over))
            s = abs(g) * (p + full + torch.where(inside, 0.0, over + p * 2.0 ** -8))
            none = torch.full_like(inside, g == 0.0 or (len(ix) == 0 and not bad)) | (y == -INF)
            if bad:
                d = torch.full_like(d, math.nan)
            grads.append(torch.where(none, 0.0, d))
            gtol.append(torch.where(none, 0.0, s))
    return torch.stack(losses), torch.stack(ltol), (torch.stack(grads), torch.stack(gtol)) if dloss is not None else None


def check_distill(z, ids, teacher, dloss=None, temperature=1.0, rest=True, **kw):
    src = z.clone()
    loss, dz = cd.distill(z, ids, teacher, dloss=dloss, temperature=temperature, rest=rest, **kw)
    torch.cuda.synchronize()
    want, tol, grad = distill64(src, ids, teacher, dloss, temperature, rest)
    reach = (src.double() / temperature).abs().nan_to_num(posinf=0.0).amax(1) * 2.0 ** -22
    if loss is not None:
        close(loss, want, (SUM + reach) * tol + round_tol(want, torch.float32).nan_to_num(posinf=0.0), "loss")
    if dz is not None:
        close(dz, grad[0], grad[1] * (SUM + reach[:, None]) + round_tol(grad[0], z.dtype), "dlogits")
    return loss, dz


def teacher_list(rows, vocab, k, g, mass=0.9):
    ids = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:k] for _ in range(rows)])
    if k > vocab:                                              # more entries than tokens: the list ends with unused ones
        ids = torch.cat([ids, torch.full((rows, k - vocab), -1, device="cuda")], 1)
    lq = torch.log_softmax(torch.randn(rows, k, generator=g, device="cuda") * 2, 1) + math.log(mass)
    return ids, lq


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_distill_every_width(vocab, dtype):
    g = gen(vocab, 55 + len(dtype))
    for rows, pad, shift, opad, oshift, k, rest in ((1, 0, 0, 0, 0, 1, True), (3, 0, 0, 0, 0, 8, False), (2, 8, 0, 0, 0, 32, True),
                                                    (4, 5, 1, 5, 1, 128, True), (2, 0, 3, 3, 2, 100, False)):
        z = matrix(rows, vocab, TYPES[dtype], g, 2.0, pad, shift)
        ids, lq = teacher_list(rows, vocab, k, g)
        dloss = torch.randn(rows, generator=g, device="cuda") * (64.0 if dtype == "f16" else 1.0)
        buf = matrix(rows, vocab, TYPES[dtype], g, 0.0, opad, oshift)
        a, _ = check_distill(z, ids, lq, dloss, 0.7, rest, out=(torch.empty(rows, device="cuda"), buf))
        around = buf.as_strided((rows * (vocab + opad) + 16,), (1,), oshift)
        mask = torch.ones(rows * (vocab + opad) + 16, dtype=torch.bool, device="cuda")
        mask.as_strided((rows, vocab), (vocab + opad, 1)).fill_(False)
        assert around[mask].isnan().all()
        b, none = check_distill(z, ids.int(), lq, None, 0.7, rest)
        assert none is None and torch.equal(a, b)
        c = cd.distill(z, ids, lq, dloss, 0.7, rest, out=(None, torch.empty_like(z)))[1]
        assert torch.equal(c, buf)


def test_distill_longest_rows():
    g = gen(22, 22)
    for dtype in TYPES.values():
        z = matrix(2, cd.MAX_VOCAB, dtype, g, 2.0, 0, 1)
        ids, lq = teacher_list(2, cd.MAX_VOCAB, 128, g)
        for rest in (True, False):
            check_distill(z, ids, lq, torch.full((2,), 100.0, device="cuda"), 1.0, rest)


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [1, 3, 40, 1000, 5003, 32768, 70001])
def test_distill_hard_rows(vocab, dtype, rest):
    g = gen(vocab, 7)
    z = hard_rows(vocab, TYPES[dtype], g)
    n, k = z.shape[0], min(24, vocab)
    ids, lq = teacher_list(n, vocab, k, g)
    ids[5, 0] = vocab // 3                                      # the one token left in row 5
    dloss = torch.full((n,), 1.0, device="cuda")
    check_distill(z, ids, lq, dloss, 1.0, rest)
    dloss[::2] = 0.0
    _, dz = check_distill(z, ids, lq, dloss, 0.5, rest)
    assert not dz[::2].any()


@pytest.mark.parametrize("rest", [True, False])
def test_distill_lists_that_are_odd(rest):
    """Unused entries, repeated ids, zero probabilities, whole mass, no entry at all."""
    g = gen(23, 23)
    vocab, k = 600, 12
    z = matrix(9, vocab, torch.float32, g, 2.0)
    ids, lq = teacher_list(9, vocab, k, g)
    ids[0, 3], ids[0, 7] = -1, vocab + 5                        # unused
    ids[1] = -1                                                 # no entry
    ids[2, 4:8] = ids[2, 3]                                     # one token five times
    lq[3, 2:5] = -INF                                           # listed with probability 0
    lq[4] = -INF                                                # all of them
    lq[5] -= math.log(0.9)                                      # the list holds everything
    lq[6] -= 20.0                                               # hardly anything
    z[7, ids[7, :4]] = -INF                                     # the student excludes what the teacher wants
    z[8] -= 60.0                                                # the student is sure of the list: the rest is 1e-26
    z[8, ids[8]] += 60.0
    dloss = torch.linspace(0.5, 2.0, 9, device="cuda")
    loss, dz = check_distill(z, ids, lq, dloss, 1.0, rest)
    assert loss[1] == 0 and not dz[1].any() and loss[7] == INF
    zz = z.clone()
    got = cd.distill(zz, ids, lq, dloss, 1.0, rest, out=(torch.empty(9, device="cuda"), zz))
    assert torch.equal(got[1], dz) and torch.equal(got[0], loss)


def test_distill_of_a_whole_vocabulary_is_the_kl_divergence():
    g = gen(24, 24)
    z, t = matrix(5, 100, torch.float32, g, 2.0), matrix(5, 100, torch.float32, g, 2.0)
    lq = torch.log_softmax(t.double() / 1.5, 1)
    ids = torch.arange(100, device="cuda").expand(5, 100).contiguous()
    lp = torch.log_softmax(z.double() / 1.5, 1)
    kl = (lq.exp() * (lq - lp)).sum(1)
    for rest in (True, False):
        loss, dz = cd.distill(z, ids, lq.float(), torch.ones(5, device="cuda"), 1.5, rest)
        close(loss, kl, SUM * (1 + kl), "kl")
        close(dz, (lp.exp() - lq.exp()) / 1.5, torch.full_like(lp, 2 * SUM), "gradient")


@pytest.mark.parametrize("rest", [True, False])
def test_distill_gradient_against_differences(rest):
    """As above: truncation below 0.002, rounding 2^-19 / h."""
    g = gen(25, 25)
    z = matrix(6, 700, torch.float32, g, 2.0)
    ids, lq = teacher_list(6, 700, 16, g, 0.8)
    dloss = torch.randn(6, generator=g, device="cuda")
    _, dz = cd.distill(z, ids, lq, dloss, 1.5, rest)
    f = lambda z: cd.distill(z, ids, lq, None, 1.5, rest)[0].double() * dloss
    h = 2.0 ** -6
    v = torch.randn(6, 700, generator=g, device="cuda")
    close((f(z + h * v) - f(z - h * v)) / (2 * h), (dz.double() * v).sum(1), 0.005, "differences")


def test_distill_takes_what_token_logprobs_gives():
    g = gen(26, 26)
    t, z = matrix(20, 5000, torch.bfloat16, g, 3.0), matrix(20, 5000, torch.bfloat16, g, 3.0)
    t[3, 6:] = -INF                                             # fewer tokens than k: the list ends with -1
    _, _, _, ids, top = cd.token_logprobs(t, k=32, temperature=2.0)
    assert (ids[3, 6:] == -1).all()
    check_distill(z, ids, top, torch.ones(20, device="cuda"), 2.0, True)
    check_distill(z, ids, top, torch.ones(20, device="cuda"), 2.0, False)
    loss, _ = cd.distill(t, ids, top, None, 2.0, True)          # a student that is the teacher
    assert float(loss.abs().max()) < SUM * 10


# ---------------------------------------------------------------------------------------------
# how they run
# ---------------------------------------------------------------------------------------------
def every_operator(g, rows=33, vocab=2500, cols=1000, **kw):
    """All operators once on inputs made from g; the outputs."""
    z = matrix(rows, vocab, torch.bfloat16, g, 2.0)
    x = matrix(rows, cols, torch.bfloat16, g)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    ids, lq = teacher_list(rows, vocab, 16, g)
    one = torch.ones(rows, device="cuda")
    torch.cuda.synchronize()

    def call():
        y, mean, rstd = cd.layer_norm(x, **kw)
        back = cd.layer_norm_backward(y, x, None, mean, rstd, groups=3, **kw)
        lps = cd.token_logprobs(z, tokens, k=20, **kw)
        dz = cd.token_logprobs_backward(z, tokens, lps[2], lps[1], one, one, **kw)
        dis = cd.distill(z, ids, lq, one, **kw)
        return (y, mean, rstd, *back, *lps, dz, *dis)
    return call


def test_repeated_calls_give_the_same_bits():
    call = every_operator(gen(30, 30))
    first = [t.clone() for t in call()]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, call()))


def test_another_stream():
    side = torch.cuda.Stream()
    want = [t.clone() for t in every_operator(gen(31, 31))()]
    call = every_operator(gen(31, 31), stream=side)
    got = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    call = every_operator(gen(31, 31))
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_captured_in_a_graph():
    call = every_operator(gen(32, 32))
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_no_rows():
    z = torch.empty(0, 100, dtype=torch.bfloat16, device="cuda")
    assert [tuple(t.shape) for t in cd.token_logprobs(z, torch.empty(0, dtype=torch.int64, device="cuda"), k=3)] == [
        (0,), (0,), (0,), (0, 3), (0, 3)]
    assert cd.layer_norm(z)[0].shape == (0, 100)
    e = torch.empty(0, device="cuda")
    assert cd.token_logprobs_backward(z, torch.empty(0, dtype=torch.int64, device="cuda"), e, e, e, e).shape == (0, 100)
    assert cd.distill(z, torch.empty(0, 4, dtype=torch.int64, device="cuda"), torch.empty(0, 4, device="cuda"), e)[1].shape == (0, 100)
