"""Log probabilities are at most 0 and entropies at least 0, for rows where they are all but 0 too."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from test_gpu_operators import TYPES, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [1, 2, 300, 5003, 131072])
def test_rows_that_are_sure(vocab, dtype):
    g = gen(vocab, 51)
    lift = torch.logspace(0, 7.5 if dtype != "f16" else 4.5, 200, device="cuda")
    for sign in (1.0, -1.0):
        z = torch.randn(200, vocab, generator=g, device="cuda")
        at = torch.randint(0, vocab, (200,), generator=g, device="cuda")
        if sign < 0:
            z -= 2.0 * lift[:, None]                                       # all of them far below 0, one half as far
        z[torch.arange(200, device="cuda"), at] = sign * lift
        z = z.to(TYPES[dtype]).clamp(min=torch.finfo(TYPES[dtype]).min)
        for temperature in (0.1, 0.7, 1.0, 3.0):
            lp, ent, lse, ids, top = cd.token_logprobs(z, at, k=1, temperature=temperature)
            assert bool((lp <= 0).all()) and bool((top <= 0).all()) and bool((ent >= 0).all())
