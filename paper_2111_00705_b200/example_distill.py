"""Training with the operators around the loss: n workers distil a student from a teacher.

    python -m paper_2111_00705_b200.example_distill [--steps 60] [--workers 4]

Student and teacher are a layer norm and an output matrix on the same hidden states, the smallest
model that has all parts: the teacher's pass gives the k most probable tokens of every position
(token_logprobs), the student's loss and its gradient come from them (distill), the gradient goes
back through the matrix (two matrix products, torch) and the layer norm (layer_norm_backward, which
leaves every worker's sums over its own rows directly in that worker's row of the gradient buffer),
and one CDAdam step turns the n x d gradients into the next parameters.  The layer norm reads its
weight and bias as slices of the optimizer's parameter vector.
"""
import argparse

import torch

from . import binding as cd


class Student:
    """Parameters: the output matrix (vocab x cols), the layer norm's weight and bias, one vector
    of d floats owned by the optimizer; each of the three is a segment with its own scale."""

    def __init__(self, vocab, cols, workers, rows_per_worker, lr=5e-3, k=16, temperature=1.0, device="cuda", seed=0):
        self.vocab, self.cols, self.workers, self.k, self.temperature = vocab, cols, workers, k, temperature
        self.rows = workers * rows_per_worker
        self.head_end = vocab * cols
        self.d = self.head_end + 2 * cols
        g = torch.Generator(device=device).manual_seed(seed)
        x0 = torch.randn(self.d, generator=g, device=device) * cols ** -0.5
        x0[self.head_end:self.head_end + cols] = 1.0
        x0[self.head_end + cols:] = 0.0
        self.opt = cd.CDAdam(self.d, workers, cd.SIGN, offsets=[0, self.head_end, self.head_end + cols, self.d], x0=x0, lr=lr)
        self.params = self.opt.params()
        self.grads = torch.empty(workers, self.d, device=device)
        self.dloss = torch.full((self.rows,), 1.0 / rows_per_worker, device=device)

    def split(self, v):
        """(output matrix, weight, bias) of a parameter vector, or of rows of gradients."""
        h = self.head_end
        return v[..., :h].unflatten(-1, (self.vocab, self.cols)), v[..., h:h + self.cols], v[..., h + self.cols:]

    def forward(self, hidden, params):
        head, weight, bias = self.split(params)
        head = head.to(hidden.dtype)
        y, mean, rstd = cd.layer_norm(hidden, weight, bias)
        return y @ head.T, (head, y, mean, rstd)

    def gradients(self, hidden, teacher_ids, teacher_logprobs):
        """Fills the n x d gradient buffer; returns the loss of every row."""
        logits, (head, y, mean, rstd) = self.forward(hidden, self.params)
        loss, dlogits = cd.distill(logits, teacher_ids, teacher_logprobs, self.dloss, self.temperature)
        dhead, dweight, dbias = self.split(self.grads)
        n = self.workers
        dhead.copy_(torch.bmm(dlogits.view(n, -1, self.vocab).mT, y.view(n, -1, self.cols)))
        cd.layer_norm_backward(dlogits @ head, hidden, self.split(self.params)[1], mean, rstd, groups=n,
                               out=(None, dweight, dbias))
        return loss

    def step(self, hidden, teacher):
        logits, _ = self.forward(hidden, teacher)
        _, _, _, ids, top = cd.token_logprobs(logits, k=self.k, temperature=self.temperature)
        loss = self.gradients(hidden, ids, top)
        self.opt.step(self.grads)
        return loss.mean()


def train(steps=60, workers=4, rows_per_worker=128, vocab=1000, cols=64, dtype=torch.bfloat16, seed=0, **kw):
    """Trains on fresh hidden states every step; returns the mean loss of every step."""
    s = Student(vocab, cols, workers, rows_per_worker, seed=seed, **kw)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    teacher = torch.randn(s.d, generator=g, device="cuda") * 4 * cols ** -0.5
    losses = []
    for _ in range(steps):
        hidden = torch.randn(s.rows, cols, generator=g, device="cuda").to(dtype)
        losses.append(s.step(hidden, teacher))
    s.opt.device_status()
    s.opt.close()
    return torch.stack(losses).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    a = ap.parse_args()
    losses = train(a.steps, a.workers)
    for t in range(0, a.steps, max(1, a.steps // 10)):
        print("step %4d  loss %.4f" % (t + 1, losses[t]))
    print("last       loss %.4f" % losses[-1])


if __name__ == "__main__":
    main()
