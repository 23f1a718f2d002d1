"""Calls of one operator from several host threads, each on a stream of its own: what one call
sets up for its launch must not reach the others'."""
import threading

import pytest
import torch

from paper_2111_00705_b200 import binding as cd

pytestmark = pytest.mark.gpu


class Call:
    """One C call with all of its buffers; `outputs` are compared with what the call gave alone."""

    def __init__(self, fn, args, outputs, workspace=None):
        self.fn, self.args, self.outputs, self.workspace = fn, args, outputs, workspace
        self.stream = torch.cuda.Stream()

    def __call__(self):
        return self.fn(*self.args, self.stream.cuda_stream)


def forward(cols):
    x, y = torch.randn(64, cols, device="cuda").bfloat16(), torch.empty(64, cols, dtype=torch.bfloat16, device="cuda")
    mean, rstd = torch.empty(2, 64, device="cuda").unbind(0)
    p = [t.data_ptr() for t in (x, y, mean, rstd)]
    c = Call(cd.lib().cdadam_layer_norm, (p[0], cols, None, None, 64, cols, 1e-5, cd.BF16, cd.F32, p[1], cols, p[2], p[3]),
             (y, mean, rstd))
    c.keep = x
    return c


def backward(cols):
    rows = 640
    x, dy = torch.randn(rows, cols, device="cuda").bfloat16(), torch.randn(rows, cols, device="cuda").bfloat16()
    _, mean, rstd = cd.layer_norm(x)
    dx, dw, db = torch.empty_like(x), *torch.empty(2, 1, cols, device="cuda").unbind(0)
    ws = torch.full((cd.layer_norm_workspace(rows, cols) // 4,), 1e9, device="cuda")
    p = [t.data_ptr() for t in (dy, x, mean, rstd, dx, dw, db, ws)]
    c = Call(cd.lib().cdadam_layer_norm_backward,
             (p[0], cols, p[1], cols, None, p[2], p[3], rows, cols, 1, cd.BF16, cd.F32, cd.F32, p[4], cols, p[5], cols, p[6], cols,
              0, p[7], ws.numel() * 4), (dx, dw, db), ws)
    c.keep = (x, dy, mean, rstd)
    return c


def logprobs(vocab):
    z, tokens = torch.randn(3, vocab, device="cuda"), torch.tensor([0, 1, 2], device="cuda")
    out = (*torch.empty(3, 3, device="cuda").unbind(0), torch.empty(3, 64, dtype=torch.int64, device="cuda"),
           torch.empty(3, 64, device="cuda"))
    c = Call(cd.lib().cdadam_token_logprobs, (z.data_ptr(), vocab, tokens.data_ptr(), 3, vocab, cd.F32, 1, 1.0, 64,
                                              *(t.data_ptr() for t in out)), out)
    c.keep = (z, tokens)
    return c


def distill(vocab):
    z, dz, loss = torch.randn(2, vocab, device="cuda"), torch.empty(2, vocab, device="cuda"), torch.empty(2, device="cuda")
    ids, lq = torch.arange(16, device="cuda").repeat(2, 1), torch.full((2, 16), -3.0, device="cuda")
    one = torch.ones(2, device="cuda")
    c = Call(cd.lib().cdadam_distill, (z.data_ptr(), vocab, ids.data_ptr(), lq.data_ptr(), 2, vocab, 16, cd.F32, 1, 1.0, 1,
                                       one.data_ptr(), loss.data_ptr(), dz.data_ptr(), vocab), (loss, dz))
    c.keep = (z, ids, lq, one)
    return c


# sizes of one kernel that differ in the shared memory they take
SIZES = {"forward": (forward, (1280, 1792)), "backward": (backward, (1280, 1792)), "logprobs": (logprobs, (131072, 393216)),
         "distill": (distill, (131072, 393216))}


def prepared(which):
    make, sizes = SIZES[which]
    calls = [make(n) for n in sizes * 2]
    torch.cuda.synchronize()
    want = []
    for c in calls:
        assert c() == cd.OK
        torch.cuda.synchronize()
        want.append([t.clone() for t in c.outputs])
    return calls, want


def together(bodies):
    """Runs every body in a thread of its own; their results."""
    got = [None] * len(bodies)

    def run(i):
        torch.cuda.set_device(0)
        got[i] = bodies[i]()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(bodies))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return got


def test_a_refused_launch_leaves_the_sums_over_rows_alone():
    """A call that reports an error has not added up its workspace, which no kernel has written:
    1e9 everywhere.  (Calls of two sizes from four threads, where a launch was once refused now and then.)"""
    calls, want = prepared("backward")
    spaces = [torch.empty(100, c.workspace.numel(), device="cuda") for c in calls]

    def body(c, w, space):
        args = [c.args[:-2] + (s.data_ptr(), c.args[-1], c.stream.cuda_stream) for s in space]
        wrong = 0
        for a in args:
            if c.fn(*a) != cd.OK:
                c.stream.synchronize()
                wrong += not all(torch.equal(x, y) for x, y in zip(c.outputs, w))
        return wrong
    for _ in range(25):
        for s in spaces:
            s.fill_(1e9)
        torch.cuda.synchronize()
        assert together([lambda c=c, w=w, s=s: body(c, w, s) for c, w, s in zip(calls, want, spaces)]) == [0] * len(calls)


@pytest.mark.parametrize("which", list(SIZES))
def test_calls_of_two_sizes_from_four_threads(which):
    calls, want = prepared(which)
    for c in calls:
        for t in c.outputs:
            t.fill_(-7)
    torch.cuda.synchronize()
    codes = together([lambda c=c: [c() for _ in range(4000)] for c in calls])
    assert [sum(v != cd.OK for v in n) for n in codes] == [0] * len(calls), cd.last_error()
    for c, w in zip(calls, want):
        assert all(torch.equal(a, b) for a, b in zip(c.outputs, w))
