"""The example with its 8-bit parts: gradients against automatic differentiation in 64 bits at the activations that the
checkpoint stands for, and a run of it."""
import pytest
import torch

from paper_2111_00705_b200 import binding as cd
from paper_2111_00705_b200 import example_distill as ex

pytestmark = pytest.mark.gpu


def test_gradients_against_automatic_differentiation():
    """Binary32 throughout; sums of up to 300 terms, a factor of two for the norm and the products: relative to the
    largest gradient of a segment errors stay below 2^-24 * 300 * 8 < 2^-12.  The weight's gradient is that of
    sum dy xh w at the checkpoint's activations and the forward pass's rstd."""
    s = ex.Student8(300, 72, 3, 10, k=12)
    g = torch.Generator(device="cuda").manual_seed(4)
    x, stream = torch.randn(2, s.rows, s.cols, generator=g, device="cuda").unbind(0)
    teacher = s.teacher(torch.randn(s.d, generator=g, device="cuda") * 0.4)
    tf32 = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        ids, top = s.teacher_list((x, stream), teacher)
        loss = s.gradients((x, stream), ids, top)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = tf32
    total = x + stream
    held = cd.checkpoint8_restore(*cd.checkpoint8(total)).double()
    rstd = (total.double().square().mean(1, keepdim=True) + 1e-6).rsqrt()
    assert torch.equal(ids[:, 0], teacher_logits(s, total, rstd, teacher).argmax(1))
    for i in range(3):
        rows = slice(10 * i, 10 * i + 10)
        p = s.params.double().requires_grad_()
        head, weight = s.split(p)
        y = total[rows].double() * rstd[rows] * weight
        y.retain_grad()
        z = y @ head.T / s.temperature
        q, lp = top[rows].double().exp(), torch.log_softmax(z, 1)
        r = 1 - q.sum(1)
        rest = torch.logsumexp(lp.scatter(1, ids[rows], -torch.inf), 1)
        want = (q * (q.log() - lp.gather(1, ids[rows]))).sum(1) + r * (r.log() - rest)
        assert float((loss[rows] - want.detach()).abs().max()) < 1e-4
        want.mean().backward()
        dhead, dweight = s.split(s.grads[i].double())
        for got, ref in ((dhead, s.split(p.grad)[0]), (dweight, (y.grad * held[rows] * rstd[rows]).sum(0))):
            assert float((got - ref).abs().max()) <= 2.0 ** -12 * float(ref.abs().max())
    s.opt.close()


def teacher_logits(s, total, rstd, teacher):
    """The teacher's logits in 64 bits from its own 8-bit rows."""
    (head, head_scale), weight = teacher
    q, scale = cd.quantize_rows(total * weight)         # the rows that the norm's output has, without its factor
    return (q.double() @ head.double().T) * (scale.double()[:, None] * rstd) * head_scale.double()


def test_a_short_run():
    losses = ex.train(steps=4, workers=2, rows_per_worker=20, vocab=130, cols=40, eight_bits=True)
    assert len(losses) == 4 and all(0.0 < v < 100.0 for v in losses)
