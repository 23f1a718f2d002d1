"""The example that runs the operators together with the optimizer: its gradients against
automatic differentiation in 64 bits, and its loss over a short training run."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from paper_2111_00705_b200 import example_distill as ex

pytestmark = pytest.mark.gpu


def test_gradients_against_automatic_differentiation():
    """Binary32 throughout; sums of up to 300 terms, a factor of two for the norm and the products:
    relative to the largest gradient of a segment errors stay below 2^-24 * 300 * 8 < 2^-12."""
    s = ex.Student(300, 72, 3, 10, k=12)
    g = torch.Generator(device="cuda").manual_seed(4)
    hidden = torch.randn(s.rows, s.cols, generator=g, device="cuda")
    teacher = torch.randn(s.d, generator=g, device="cuda") * 0.4
    tf32 = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        logits, _ = s.forward(hidden, teacher)
        _, _, _, ids, top = cd.token_logprobs(logits, k=s.k, temperature=s.temperature)
        loss = s.gradients(hidden, ids, top)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = tf32
    for i in range(3):
        rows = slice(10 * i, 10 * i + 10)
        p = s.params.double().requires_grad_()
        head, weight, bias = s.split(p)
        y = torch.nn.functional.layer_norm(hidden[rows].double(), (s.cols,), weight, bias, 1e-5)
        z = y @ head.T / s.temperature
        q, lp = top[rows].double().exp(), torch.log_softmax(z, 1)
        r = 1 - q.sum(1)
        rest = torch.logsumexp(lp.scatter(1, ids[rows], -torch.inf), 1)
        want = (q * (q.log() - lp.gather(1, ids[rows]))).sum(1) + r * (r.log() - rest)
        assert float((loss[rows] - want.detach()).abs().max()) < 1e-4
        (grad,) = torch.autograd.grad(want.mean(), p)
        for got, ref in zip(s.split(s.grads[i].double()), s.split(grad)):
            assert float((got - ref).abs().max()) <= 2.0 ** -12 * float(ref.abs().max())
    s.opt.close()


def test_the_loss_goes_down():
    losses = ex.train(steps=60)
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5]), losses


def test_every_worker_has_its_own_rows():
    """The gradient of a worker depends on its own rows alone."""
    s = ex.Student(100, 64, 2, 6)
    g = torch.Generator(device="cuda").manual_seed(5)
    hidden = torch.randn(s.rows, s.cols, generator=g, device="cuda").bfloat16()
    ids = torch.randint(0, 100, (s.rows, 5), generator=g, device="cuda")
    top = torch.full((s.rows, 5), -2.0, device="cuda")
    s.gradients(hidden, ids, top)
    first = s.grads.clone()
    hidden[6:] = 0.5
    s.gradients(hidden, ids, top)
    assert torch.equal(s.grads[0], first[0]) and not torch.equal(s.grads[1], first[1])
    s.opt.close()
