"""What a worker computes around its loss, as measurable cases.

Before a CD-Adam step every worker needs the gradient of its loss.  Three operators of that part
of a language model's training are measured here, in the forms a program calls them:

  layer norm            forward (rows of activations) and backward (dx, and for every worker the
                        sums over its rows that are the gradients of weight and bias)
  token log probability log softmax at given tokens, the entropy, and the k most probable tokens
                        (the teacher's pass); and the gradient with respect to the logits
  distillation          KL divergence from a teacher's k listed probabilities, with the rest of
                        the vocabulary as one further outcome or the list renormalised, and its
                        gradient with respect to the student's logits

`run` computes a case with elementary torch operations in binary32 (`own` false) or with the
package's entry points (`own` true).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


# --------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------
def _norm(name, rows, cols, dtype, backward=False, groups=1):
    return {"name": name, "op": "norm_backward" if backward else "norm", "rows": rows, "cols": cols, "dtype": dtype,
            "groups": groups}


def _logprob(name, rows, vocab, dtype, k=0, temperature=1.0, padding=0):
    return {"name": name, "op": "logprob", "rows": rows, "vocab": vocab, "dtype": dtype, "k": k,
            "temperature": temperature, "padding": padding}


def _logprob_backward(name, rows, vocab, dtype, entropy=True, temperature=1.0, padding=0):
    return {"name": name, "op": "logprob_backward", "rows": rows, "vocab": vocab, "dtype": dtype,
            "entropy": entropy, "temperature": temperature, "padding": padding}


def _distill(name, rows, vocab, dtype, k, temperature=1.0, rest=True, grad=True):
    return {"name": name, "op": "distill", "rows": rows, "vocab": vocab, "dtype": dtype, "k": k,
            "temperature": temperature, "rest": rest, "grad": grad}


def listed():
    return [
        # one decoding step of four sequences: a launch, hardly any data
        _norm("norm one token", 4, 768, "bf16"),
        # activations of 32 sequences of 512 tokens, kept in binary32
        _norm("norm f32", 16384, 768, "f32"),
        # the same batch in half precision going back: eight workers, 2048 rows each
        _norm("norm backward 8 workers", 16384, 768, "bf16", backward=True, groups=8),
        # an odd width and an odd number of rows: no row but the first is aligned
        _norm("norm backward odd", 3001, 1021, "f16", backward=True),
        # the widest batch: 32 sequences of 1024 tokens
        _norm("norm backward large", 32768, 4096, "bf16", backward=True),
        # sampling one token and reporting its 20 most probable alternatives
        _logprob("logprob one token", 1, 30522, "bf16", k=20, temperature=0.7),
        # evaluation of a few sequences in binary32, odd vocabulary, no alternatives
        _logprob("logprob odd f32", 509, 50021, "f32"),
        # the teacher's pass over a batch: 64 alternatives of each position, vocabulary padded
        _logprob("logprob teacher", 4096, 131072, "bf16", k=64, padding=96),
        # policy gradient with an entropy term on 8 sequences of 512 tokens
        _logprob_backward("logprob backward", 4096, 30522, "bf16"),
        # a small student's step, a short list
        _distill("distill small", 32, 30522, "f32", 8),
        # half precision, odd sizes, the list renormalised at temperature 2
        _distill("distill odd", 1023, 50021, "f16", 32, temperature=2.0, rest=False),
        # a batch of 8 sequences of 512 tokens, large vocabulary
        _distill("distill large", 4096, 131072, "bf16", 64),
    ]


def _log_uniform(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = min(max(v, lo), hi)
    return v if rng.random() < 0.5 or v < 64 else v // 16 * 16


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "logprob", "logprob_backward", "distill"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op.startswith("norm"):
        cols = _log_uniform(rng, 64, 8192)
        rows = _log_uniform(rng, 1, min(32768, (1 << 28) // (cols * SIZE[dtype])))
        groups = 1
        if op == "norm_backward":
            groups = rng.choice([1, 1, 2, 4, 8])
            rows = max(1, rows // groups) * groups
        c = _norm("", rows, cols, dtype, op == "norm_backward", groups)
    else:
        vocab = _log_uniform(rng, 1000, 131072)
        rows = _log_uniform(rng, 1, min(8192, (1 << 30) // (vocab * SIZE[dtype])))
        temperature = rng.choice([1.0, 1.0, 0.7, 2.0])
        if op == "logprob":
            c = _logprob("", rows, vocab, dtype, rng.choice([0, 1, 5, 20, 64]), temperature, rng.choice([0, 0, 37]))
        elif op == "logprob_backward":
            c = _logprob_backward("", rows, vocab, dtype, rng.random() < 0.5, temperature, rng.choice([0, 0, 37]))
        else:
            c = _distill("", rows, vocab, dtype, rng.choice([4, 16, 32, 64, 100]), temperature, rng.random() < 0.5,
                         rng.random() < 0.75)
    del c["name"]
    return c


def work(case):
    """Each input read once, each output written once; additions, multiplications and exponentials counted once each."""
    rows, size, op = case["rows"], SIZE[case["dtype"]], case["op"]
    if op.startswith("norm"):
        n, cols = rows * case["cols"], case["cols"]
        if op == "norm":                                   # x -> y; weight, bias; mean, rstd
            return {"bytes": 2 * n * size + 8 * cols + 8 * rows, "flops": 8 * n}
        return {"bytes": 3 * n * size + 4 * cols + 8 * cols * case["groups"] + 8 * rows, "flops": 14 * n}
    n = rows * case["vocab"]
    if op == "logprob":                                    # logits, tokens -> three scalars, k pairs
        return {"bytes": n * size + rows * (8 + 12 + 12 * case["k"]), "flops": 6 * n}
    if op == "logprob_backward":
        return {"bytes": 2 * n * size + rows * (8 + 16), "flops": 7 * n}
    return {"bytes": (2 if case["grad"] else 1) * n * size + rows * (12 * case["k"] + 8), "flops": (8 if case["grad"] else 4) * n}


# --------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------
def _logits(case, g, device):
    """Rows of logits of differing sharpness; the padding at the vocabulary's end is masked."""
    rows, vocab, dtype = case["rows"], case["vocab"], TYPES[case["dtype"]]
    sharp = 0.5 + 2.5 * torch.rand(rows, 1, generator=g, device=device)
    z = torch.empty(rows, vocab, dtype=dtype, device=device)
    step = max(1, (1 << 27) // vocab)
    for a in range(0, rows, step):
        part = z[a:a + step]
        part.copy_(torch.randn(part.shape, generator=g, device=device) * sharp[a:a + step])
    if case.get("padding"):
        z[:, vocab - case["padding"]:] = -math.inf
    return z


def _statistics(z, temperature):
    """Log normaliser and entropy of every row, as a forward pass saves them."""
    lse, ent = (torch.empty(z.shape[0], device=z.device) for _ in range(2))
    step = max(1, (1 << 26) // z.shape[1])
    for a in range(0, z.shape[0], step):
        part = z[a:a + step].double() / temperature
        l = torch.logsumexp(part, 1)
        lp = part - l[:, None]
        lse[a:a + step] = l
        ent[a:a + step] = -(lp.exp() * lp.clamp(min=-1e30)).sum(1)
    return lse, ent


def prepare(case, seed):
    device = "cuda"
    g = torch.Generator(device=device).manual_seed(int(seed))
    rows, op, dtype = case["rows"], case["op"], TYPES[case["dtype"]]
    s = {"case": dict(case)}
    if op.startswith("norm"):
        cols, groups = case["cols"], case["groups"]
        x = torch.randn(rows, cols, generator=g, device=device) * 1.5 + 0.3
        x[:, ::97] *= 8.0                                   # a few columns are much larger than the others
        s["x"] = x.to(dtype)
        # weight and bias are slices of the flat parameter vector that the optimizer holds
        params = torch.randn(4 * cols, generator=g, device=device) * 0.1
        s["weight"], s["bias"] = params[cols:2 * cols], params[2 * cols:3 * cols]
        s["weight"].add_(1.0)
        if op == "norm":
            s["out"] = (torch.empty(rows, cols, dtype=dtype, device=device), torch.empty(rows, device=device),
                        torch.empty(rows, device=device))
            return s
        xf = s["x"].float()
        s["mean"] = xf.mean(1)
        s["rstd"] = torch.rsqrt((xf - s["mean"][:, None]).square().mean(1) + EPS)
        s["dy"] = (torch.randn(rows, cols, generator=g, device=device) * 0.02).to(dtype)
        # and their gradients are slices of the workers' rows of the optimizer's gradient buffer
        grads = torch.zeros(groups, 4 * cols, device=device)
        s["out"] = (torch.empty(rows, cols, dtype=dtype, device=device), grads[:, cols:2 * cols], grads[:, 2 * cols:3 * cols])
        return s

    vocab = case["vocab"]
    s["logits"] = z = _logits(case, g, device)
    if op != "distill":
        real = vocab - case["padding"]
        s["tokens"] = torch.randint(0, real, (rows,), generator=g, device=device)
        if rows >= 16:
            s["tokens"][::16] = -100                        # positions that do not count
    if op == "logprob":
        k = case["k"]
        s["out"] = tuple(torch.empty(rows, device=device) for _ in range(3)) + (
            torch.empty(rows, k, dtype=torch.int64, device=device), torch.empty(rows, k, device=device))
    elif op == "logprob_backward":
        s["lse"], s["entropy"] = _statistics(z, case["temperature"])
        s["dlogprob"] = torch.randn(rows, generator=g, device=device)
        s["dentropy"] = torch.full((rows,), -0.01, device=device) if case["entropy"] else None
        s["out"] = torch.empty_like(z)
    else:
        k = case["k"]
        # k distinct tokens a row, and a student that already favours them
        start = torch.randint(0, vocab, (rows, 1), generator=g, device=device)
        step = torch.randint(1, vocab // k + 1, (rows, 1), generator=g, device=device)
        rank = torch.arange(k, device=device)
        s["ids"] = (start + step * rank) % vocab
        lift = (9.0 - 0.05 * rank).expand(rows, k) + torch.randn(rows, k, generator=g, device=device)
        z.scatter_(1, s["ids"], lift.to(dtype))
        listed_ = torch.log_softmax(3.0 * torch.rand(rows, k, generator=g, device=device) - 0.1 * rank, 1)
        mass = 0.6 + 0.39 * torch.rand(rows, 1, generator=g, device=device)
        s["teacher"] = listed_ + mass.log()
        scale = 1024.0 if case["dtype"] == "f16" else 1.0   # losses are scaled where gradients are in half precision
        s["dloss"] = torch.full((rows,), scale / rows, device=device) if case["grad"] else None
        s["out"] = (torch.empty(rows, device=device), torch.empty_like(z) if case["grad"] else None)
    return s


# --------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------
def run(state):
    return _call(state) if own else _plain(state)


def _call(s):
    from paper_2111_00705_b200 import binding as cd
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        return cd.layer_norm(s["x"], s["weight"], s["bias"], EPS, out=s["out"])
    if op == "norm_backward":
        return cd.layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], groups=c["groups"], out=s["out"])
    if op == "logprob":
        return cd.token_logprobs(s["logits"], s["tokens"], k=c["k"], temperature=c["temperature"], out=s["out"])
    if op == "logprob_backward":
        return cd.token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["entropy"], s["dlogprob"], s["dentropy"],
                                          temperature=c["temperature"], out=s["out"])
    return cd.distill(s["logits"], s["ids"], s["teacher"], dloss=s["dloss"], temperature=c["temperature"], rest=c["rest"],
                      out=s["out"])


def _plain(s):
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "logprob": _plain_logprob,
            "logprob_backward": _plain_logprob_backward, "distill": _plain_distill}[s["case"]["op"]](s)


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((xc * xc).mean(1) + EPS)
    y = xc * rstd[:, None] * s["weight"] + s["bias"]
    return y.to(s["x"].dtype), mean, rstd


def _plain_norm_backward(s):
    groups, cols = s["case"]["groups"], s["case"]["cols"]
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xhat = (s["x"].float() - s["mean"][:, None]) * rstd
    h = dy * s["weight"]
    dx = rstd * (h - h.mean(1, keepdim=True) - xhat * (h * xhat).mean(1, keepdim=True))
    dweight = (dy * xhat).view(groups, -1, cols).sum(1)
    dbias = dy.view(groups, -1, cols).sum(1)
    return dx.to(s["x"].dtype), dweight, dbias


def _plain_log_softmax(z, temperature):
    """(log softmax(z / T), log normaliser of z / T), of rows with at least one finite logit."""
    z = z.float() / temperature
    m = z.amax(1, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(1, keepdim=True))
    return z - lse, lse[:, 0]


def _plain_logprob(s):
    k, tokens = s["case"]["k"], s["tokens"]
    lp, lse = _plain_log_softmax(s["logits"], s["case"]["temperature"])
    p = torch.exp(lp)
    entropy = -(p * torch.where(p > 0, lp, 0.0)).sum(1)
    logprob = torch.where(tokens >= 0, lp.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    # descending by (value, lower index first): one 64-bit key of the value's bits and the index
    bits = (s["logits"].float() + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64) * (1 << 32) + (
        0xFFFFFFFF - torch.arange(lp.shape[1], device=lp.device))
    key = key.topk(k, 1).values
    ids = 0xFFFFFFFF - (key & 0xFFFFFFFF)
    top = lp.gather(1, ids)
    return logprob, entropy, lse, torch.where(top > -math.inf, ids, -1), top


def _plain_logprob_backward(s):
    z, t, tokens = s["logits"], s["case"]["temperature"], s["tokens"]
    lp = z.float() / t - s["lse"][:, None]
    p = torch.exp(lp)
    g = torch.where(tokens >= 0, s["dlogprob"], 0.0)[:, None]
    d = -g * p
    d.scatter_add_(1, tokens.clamp(min=0)[:, None], g)
    if s["dentropy"] is not None:
        d = d - s["dentropy"][:, None] * p * (torch.where(p > 0, lp, 0.0) + s["entropy"][:, None])
    return (d / t).to(z.dtype)


def _plain_distill(s):
    c, z, ids = s["case"], s["logits"], s["ids"]
    logq = s["teacher"]
    if not c["rest"]:
        logq, _ = _plain_log_softmax(logq, 1.0)
    q = torch.exp(logq)
    logp, _ = _plain_log_softmax(z, c["temperature"])
    listed_ = logp.gather(1, ids)
    loss = (q * (logq - listed_)).sum(1)
    p = torch.exp(logp)
    weight = 1.0
    if c["rest"]:
        r = (1.0 - q.sum(1)).clamp(min=0.0)
        rest = p.scatter(1, ids, 0.0).sum(1)
        loss = loss + torch.where(r > 0, r * (torch.log(r) - torch.log(rest)), 0.0)
        weight = (1.0 - r / rest)[:, None]
    if not c["grad"]:
        return loss, None
    d = (p * weight).scatter(1, ids, torch.exp(listed_) - q)
    return loss, (d * (s["dloss"] / c["temperature"])[:, None]).to(z.dtype)


# --------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# --------------------------------------------------------------------------------------------
def _parts(case, width):
    step = max(1, (1 << 24) // width)
    return [(a, min(a + step, case["rows"])) for a in range(0, case["rows"], step)]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("norm"):
        return _exact_norm(case, s)
    return {"logprob": _exact_logprob, "logprob_backward": _exact_logprob_backward, "distill": _exact_distill}[op](case, s)


def _exact_norm(case, s):
    rows, cols, groups = case["rows"], case["cols"], case["groups"]
    w, b = s["weight"].double(), s["bias"].double()
    if case["op"] == "norm":
        got = []
        for a, e in _parts(case, cols):
            x = s["x"][a:e].double()
            var, mean = torch.var_mean(x, 1, correction=0)
            got.append((torch.nn.functional.layer_norm(x, (cols,), w, b, EPS), mean, (var + EPS).pow(-0.5)))
        return tuple(torch.cat(v) for v in zip(*got))
    dx = []
    dw, db = (torch.zeros(groups, cols, dtype=torch.float64, device=w.device) for _ in range(2))
    per = rows // groups
    step = max(1, (1 << 24) // cols)
    for i in range(groups):
        for a in range(i * per, (i + 1) * per, step):
            e = min(a + step, (i + 1) * per)
            x, ww, bb = (t.detach().clone().requires_grad_() for t in (s["x"][a:e].double(), w, b))
            y = torch.nn.functional.layer_norm(x, (cols,), ww, bb, EPS)
            gx, gw, gb = torch.autograd.grad(y, (x, ww, bb), s["dy"][a:e].double())
            dx.append(gx)
            dw[i] += gw
            db[i] += gb
    return torch.cat(dx), dw, db


def _exact_logprob(case, s):
    k, got = case["k"], []
    for a, e in _parts(case, case["vocab"]):
        z, tok = s["logits"][a:e].double(), s["tokens"][a:e]
        lp = torch.log_softmax(z / case["temperature"], 1)
        at = torch.where(tok < 0, 0.0, lp[torch.arange(e - a, device=z.device), tok.clamp(min=0)])
        ent = -torch.special.xlogy(lp.exp(), lp.exp()).sum(1)
        top, ids = torch.sort(z, dim=1, descending=True, stable=True)
        top, ids = top[:, :k], ids[:, :k]
        got.append((at, ent, torch.logsumexp(z / case["temperature"], 1), ids.where(top > -math.inf, torch.full_like(ids, -1)),
                    lp.gather(1, ids)))
    return tuple(torch.cat(v) for v in zip(*got))


def _exact_logprob_backward(case, s):
    got = []
    for a, e in _parts(case, case["vocab"]):
        z, tok = s["logits"][a:e].double(), s["tokens"][a:e]
        masked = torch.isinf(z)
        z = z.masked_fill(masked, -1e300).requires_grad_()
        lp = torch.log_softmax(z / case["temperature"], 1)
        f = (lp.gather(1, tok.clamp(min=0)[:, None])[:, 0] * s["dlogprob"][a:e].double() * (tok >= 0)).sum()
        if s["dentropy"] is not None:
            f = f - ((lp.exp() * lp.masked_fill(masked, 0.0)).sum(1) * s["dentropy"][a:e].double()).sum()
        got.append(torch.autograd.grad(f, z)[0].masked_fill(masked, 0.0))
    return torch.cat(got)


def _exact_distill(case, s):
    loss, grad = [], []
    for a, e in _parts(case, case["vocab"]):
        z = s["logits"][a:e].double().requires_grad_()
        ids, t = s["ids"][a:e], s["teacher"][a:e].double()
        q = t.exp() if case["rest"] else torch.softmax(t, 1)
        y = z / case["temperature"]
        lse = torch.logsumexp(y, 1)
        f = torch.special.xlogy(q, q).sum(1) - (q * (y.gather(1, ids) - lse[:, None])).sum(1)
        if case["rest"]:
            r = 1.0 - q.sum(1)
            others = torch.logsumexp(y.scatter(1, ids, -math.inf), 1) - lse
            f = f + torch.special.xlogy(r, r) - r * others
        loss.append(f.detach())
        if case["grad"]:
            grad.append(torch.autograd.grad((f * s["dloss"][a:e].double()).sum(), z)[0])
    return torch.cat(loss), torch.cat(grad) if case["grad"] else None
