"""Gradient of the log probabilities of rows with a large common offset, given lse, against 64 bits.

Tolerance.  The exponent t of a probability is off by at most 1.25 times 2^-23 |t| (one rounding of t, one
of the scale), whatever the offset; a probability of binary32 has |t| below 126, so p is good to
ln(2) 126 1.25 2^-23 < 2^-16, with the exponential's 2^-22 and a few products' 2^-24 below 2^-15.
"""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_operators import TYPES, backward_logprobs64, close, gen, round_tol

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("temperature", [1.0, 0.7, 3.0])
@pytest.mark.parametrize("offset", [0.0, 100.0, -1000.0, 8000.0, -3e4, 1e5, 3e6])
def test_gradient_of_rows_far_from_zero(offset, temperature, dtype):
    dt = TYPES[dtype]
    temperature = float(torch.tensor(temperature))            # as the entry point takes it, in binary32
    if dt == torch.float16 and offset > 6e4:
        offset /= 100.0
    g = gen(int(abs(offset)), 71)
    for vocab in (50, 1000, 30522):
        z = (torch.randn(6, vocab, generator=g, device="cuda") * 3 + offset).to(dt)
        tokens = torch.randint(0, vocab, (6,), generator=g, device="cuda")
        dlp, dent = torch.randn(2, 6, generator=g, device="cuda").unbind(0)
        lse = (z.double() / temperature).logsumexp(1).float()
        lp = z.double() / temperature - lse[:, None]
        ent = -(lp.exp() * lp).sum(1).float()
        for gl, ge in ((dlp, dent), (dlp, None), (None, dent)):
            got = cd.token_logprobs_backward(z, tokens, lse, ent, gl, ge, temperature)
            torch.cuda.synchronize()
            want, size = backward_logprobs64(z, tokens, lse, ent, gl, ge, temperature)
            close(got, want, size * 2.0 ** -15 + round_tol(want, dt), "dlogits")
