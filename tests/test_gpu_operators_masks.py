"""Rows of logits with large finite values, as masks are often written (-1e10, -1e30, the type's
lowest value) and as a single logit can be, against 64 bits.

Tolerances.  Exponents are formed relative to the row's maximum in one rounding, from products
that are exact in 64 bits, so what a masked logit's size adds is a relative 2^-24 of outputs that
are themselves of that size (its log probability), and nothing to the others: a logit that adds to a
sum is within 200 of the maximum (times the temperature), where a rounding of its exponent is
below 200 log2(e) 2^-24 < 2^-15, and the scale's own rounding below 200 log2(e) 2^-25.  So every
term is good to SUM + 2^-14 whatever the mask, where the sums themselves are given SUM = 2^-15.
"""
import math

import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_operators import INF, SUM, TYPES, backward_logprobs64, check_logprobs, gen, hard_rows, round_tol, teacher_list

pytestmark = pytest.mark.gpu

TERM = SUM + 2.0 ** -14


def masks(dtype):
    return [-1e4, -65504.0] if dtype == torch.float16 else [-1e5, -1e8, -1e9, -1e10, -1e12, -1e20, -1e30, torch.finfo(dtype).min]


def masked_rows(vocab, dtype, g):
    i = torch.arange(vocab, device="cuda")
    rows = []
    for mask in masks(dtype):
        n = lambda: torch.randn(vocab, generator=g, device="cuda") * 2
        r = n(); r[vocab // 5:vocab - vocab // 5] = mask; rows.append(r)           # whole stretches, and threads, see nothing else
        r = torch.full((vocab,), mask, device="cuda"); r[vocab // 2] = 1.0; r[vocab - 1] = 0.5; rows.append(r)    # two tokens left
        r = n(); r[i % 7 != 3] = mask; rows.append(r)
        r = n(); r[:vocab // 2] = mask; r[::5] = -INF; rows.append(r)               # beside the other mask
        rows.append(torch.full((vocab,), mask, device="cuda"))                      # nothing else at all
        r = torch.full((vocab,), mask, device="cuda"); r[::3] = max(2 * mask, torch.finfo(dtype).min); rows.append(r)
        r = n(); r[vocab // 3] = -mask; rows.append(r)                              # one that is far above all others
    return torch.stack(rows).to(dtype)


VOCABS = [3, 40, 1000, 5003, 30522, 131072]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_log_probabilities_beside_large_finite_values(vocab, dtype):
    z = masked_rows(vocab, TYPES[dtype], gen(vocab, 41))
    tokens = torch.arange(z.shape[0], device="cuda") * 977 % vocab
    for temperature, k in ((1.0, 0), (0.5, min(20, vocab)), (3.0, min(64, vocab))):
        check_logprobs(z, tokens, k, temperature)
    check_logprobs(z.repeat(30, 1), tokens.repeat(30), min(5, vocab), 0.7)          # a block for every row


def softmax64(y):
    """(exp(y - max), its sum, max) of every row; 0 where everything is -inf."""
    m = y.amax(1, keepdim=True)
    m = torch.where(m == -INF, 0.0, m)
    e = torch.exp(y - m)
    return e, e.sum(1, keepdim=True), m


def distill64(z, ids, teacher, g, temperature, rest):
    """From the definition, valid ids, every row with something unmasked.  Differences of logits are
    formed before anything of ordinary size is added to them: 1e20 + log 16 is 1e20 in 64 bits too."""
    y = z.double() / temperature
    e, total, m = softmax64(y)
    p = e / total
    q = teacher.double().exp() if rest else torch.softmax(teacher.double(), 1)
    full = torch.zeros_like(y).scatter_add_(1, ids, q)                  # an index listed twice: one token with the sum
    inside = torch.zeros_like(y, dtype=torch.bool).scatter_(1, ids, True)
    r = (1.0 - q.sum(1, keepdim=True)).clamp(min=0.0) * (~inside).any(1, keepdim=True) if rest else torch.zeros_like(m)
    log_p = (y - m) - total.log()
    term = torch.where(full == 0, 0.0, full * (full.log() - log_p))
    size = torch.where(full == 0, 0.0, full * (full.log().abs() + log_p.abs() + 1))
    er, sum_r, mr = softmax64(y.masked_fill(inside, -INF))
    log_r = torch.where(sum_r == 0, -INF, (mr - m) + (sum_r.log() - total.log()))
    loss = term.sum(1) + torch.where(r > 0, r * (r.log() - log_r), 0.0)[:, 0]
    over = torch.where(sum_r > 0, r * er / sum_r, 0.0)
    grad = g * (p - full - torch.where(inside, 0.0, over)) / temperature
    gsize = g * (p + full + over + torch.where(inside, 0.0, p * 2.0 ** -8)) / temperature
    masked = y == -INF
    # r is what the teacher's probabilities leave, off by their rounding
    size = size.sum(1) + torch.where(r > 0, r + (r + 2.0 ** -8) * (r.log().abs() + log_r.abs()), 0.0)[:, 0]
    return loss, size, torch.where(masked, 0.0, grad), torch.where(masked, 0.0, gsize)


def near(got, want, tol, what):
    """|got - want| <= tol, where a value that may round beyond the type's range may be infinite."""
    most = torch.finfo(got.dtype).max
    got, want = got.double(), want.double()
    fine = (got == want) | ((got - want).abs() <= tol) | ((got.abs() == INF) & (want.abs() + tol > most) & (got * want > 0))
    assert bool(fine.all()), (what, (~fine).nonzero()[:4].tolist())


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_distillation_beside_large_finite_values(vocab, dtype, rest):
    g = gen(vocab, 43)
    z = masked_rows(vocab, TYPES[dtype], g)
    n, k = z.shape[0], min(24, vocab)
    ids, lq = teacher_list(n, vocab, k, g)
    ids[::2] = (torch.arange(k, device="cuda") + vocab // 2) % vocab                # among them the token that some masks leave
    for temperature in (1.0, 0.5, 3.0):
        dloss = torch.full((n,), 64.0, device="cuda")
        loss, dz = cd.distill(z, ids, lq, dloss, temperature, rest)
        torch.cuda.synchronize()
        want, size, grad, gsize = distill64(z, ids, lq, dloss[:, None], temperature, rest)
        near(loss, want, TERM * size.nan_to_num(posinf=0.0) + round_tol(want, torch.float32).nan_to_num(posinf=0.0), "loss")
        near(dz, grad, TERM * gsize + round_tol(grad, z.dtype), "dlogits")


@pytest.mark.parametrize("bad", [INF, -INF, math.nan])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [40, 1003, 30522, 131072])
def test_masked_logits_have_no_gradient_whatever_comes_in(vocab, dtype, bad):
    """A gradient coming in that is not finite (a loss scaled too far) reaches the row's unmasked logits only."""
    g = gen(vocab, 47)
    z = torch.randn(5, vocab, generator=g, device="cuda").to(TYPES[dtype])
    masked = torch.zeros(5, vocab, dtype=torch.bool, device="cuda")
    masked[:, vocab // 3:vocab // 2] = True
    masked[3, ::2] = True
    z[masked] = -INF
    tokens = torch.tensor([0, 1, 2, 3, vocab // 3], device="cuda")         # the last one is masked
    lp, ent, lse, _, _ = cd.token_logprobs(z, tokens)
    one, odd = torch.ones(5, device="cuda"), torch.tensor([1.0, bad, 1.0, bad, bad], device="cuda")
    hit = odd != 1.0
    good = cd.token_logprobs_backward(z, tokens, lse, ent, one, one)
    for dlp, dent in ((odd, None), (odd, one), (one, odd)):
        got = cd.token_logprobs_backward(z, tokens, lse, ent, dlp, dent)
        assert not got[masked].any() and not got[hit][~masked[hit]].isfinite().any()
        assert torch.equal(got[~hit], good[~hit]) or dent is None
    ids, lq = teacher_list(5, vocab, 8, g)
    ids[:, 0] = vocab // 3                                                  # listed and masked
    loss, good = cd.distill(z, ids, lq, one)
    got_loss, got = cd.distill(z, ids, lq, odd)
    assert torch.equal(loss, got_loss) and torch.equal(got[~hit], good[~hit])
    assert not got[masked].any() and not got[hit][~masked[hit]].isfinite().any()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_gradient_beside_large_finite_values(vocab, dtype):
    """Given lse and entropy.  A probability's exponent is off by 1.25 times 2^-23 of its own size, below
    126 where the probability is not 0: 2^-15 with everything else."""
    g = gen(vocab, 45)
    z = torch.cat([masked_rows(vocab, TYPES[dtype], g), hard_rows(vocab, TYPES[dtype], g)[:14]])
    n = z.shape[0]
    tokens = torch.arange(n, device="cuda") * 977 % vocab
    dlp, dent = torch.randn(2, n, generator=g, device="cuda").unbind(0)
    for temperature in (1.0, 0.5, 3.0):
        _, ent, lse, _, _ = cd.token_logprobs(z, tokens, temperature=temperature)
        for gl, ge in ((dlp, dent), (dlp, None)):
            got = cd.token_logprobs_backward(z, tokens, lse, ent, gl, ge, temperature)
            torch.cuda.synchronize()
            want, size = backward_logprobs64(z, tokens, lse, ent, gl, ge, temperature)
            near(got, want, 2.0 ** -15 * size + round_tol(want, z.dtype), "dlogits")


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [40, 1000, 5003, 32768, 70001])
def test_distillation_of_hard_rows(vocab, dtype, rest):
    """The hard rows again (without the one that is empty), where a logit at the type's lowest value allows nothing."""
    g = gen(vocab, 46)
    z = hard_rows(vocab, TYPES[dtype], g)[[0] + list(range(2, 14))]
    n, k = z.shape[0], 24
    ids, lq = teacher_list(n, vocab, k, g)
    ids[4, 0] = vocab // 3                                                  # the one token left in that row
    ids[5, :2] = torch.tensor([0, vocab - 1], device="cuda")                # the two that are not at the lowest value
    ids[5, 2:] = torch.arange(1, k - 1, device="cuda")
    dloss = torch.full((n,), 64.0, device="cuda")
    for temperature in (1.0, 0.5):
        loss, dz = cd.distill(z, ids, lq, dloss, temperature, rest)
        torch.cuda.synchronize()
        want, size, grad, gsize = distill64(z, ids, lq, dloss[:, None], temperature, rest)
        near(loss, want, TERM * size.nan_to_num(posinf=0.0) + round_tol(want, torch.float32).nan_to_num(posinf=0.0), "loss")
        near(dz, grad, TERM * gsize + round_tol(grad, z.dtype), "dlogits")
