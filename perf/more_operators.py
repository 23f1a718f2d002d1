"""What a worker computes in 8 bits around its products, as measurable cases.

Four operators of a language model's training step, in the forms a program calls them:

  root-mean-square norm   with the residual's addition in front; its output in the activations' type,
                          or in 8-bit integers with one scale for each row (read back to compare)
  its backward pass       dx (with the gradient that comes along the residual) and for every worker
                          the sums over its rows that are the weight's gradient; the activations come
                          as they were, or from a checkpoint in 8 bits
  checkpoint              activations kept in 8 bits, a power of two for every 32 columns, and read back
  product                 8-bit activations (a scale for each token) with 8-bit weights (a scale for
                          each channel); the activations as the norm leaves them, or quantised first

`run` computes a case with elementary torch operations (`own` false) or with the package's entry
points (`own` true).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
BLOCK = 32          # columns of a checkpoint that share a power of two


# --------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------
def _norm(name, rows, cols, dtype, residual=True, eight=False):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "residual": residual, "eight": eight}


def _backward(name, rows, cols, dtype, groups=1, checkpoint=False, residual=True):
    return {"name": name, "op": "backward", "rows": rows, "cols": cols, "dtype": dtype, "groups": groups,
            "checkpoint": checkpoint, "residual": residual}


def _checkpoint(name, rows, cols, dtype):
    return {"name": name, "op": "checkpoint", "rows": rows, "cols": cols, "dtype": dtype}


def _product(name, tokens, channels, inner, dtype, quantise=False, bias=False):
    return {"name": name, "op": "product", "tokens": tokens, "channels": channels, "inner": inner, "dtype": dtype,
            "quantise": quantise, "bias": bias}


def listed():
    return [
        # one decoding step of four sequences: launches, hardly any data
        _norm("norm 8 bits one token", 4, 768, "bf16", eight=True),
        # an odd width in binary32, output in the activations' type
        _norm("norm odd f32", 3001, 1021, "f32"),
        # the teacher's pass over 32 sequences of 512 tokens, in front of an 8-bit product
        _norm("norm 8 bits large", 16384, 4096, "bf16", eight=True),
        # eight workers, 2048 rows each, activations as they were
        _backward("norm backward 8 workers", 16384, 768, "bf16", groups=8),
        # odd sizes in half precision, from a checkpoint
        _backward("norm backward odd", 3001, 1021, "f16", checkpoint=True),
        # the widest batch, 32 sequences of 1024 tokens, from a checkpoint
        _backward("norm backward large", 32768, 4096, "bf16", checkpoint=True),
        # activations of a few sequences in binary32, odd width
        _checkpoint("checkpoint odd f32", 1023, 5001, "f32"),
        # the widest batch's activations
        _checkpoint("checkpoint large", 32768, 4096, "bf16"),
        # one token's logits
        _product("product one token", 1, 30522, 768, "f32"),
        # 64 sequences decoded side by side
        _product("product 64 tokens", 64, 30522, 4096, "bf16", bias=True),
        # odd sizes, activations quantised on the way, logits in binary32
        _product("product odd", 509, 2003, 1021, "f32", quantise=True),
        # a teacher's logits of 8 sequences of 512 tokens, large vocabulary
        _product("product teacher", 4096, 131072, 4096, "bf16"),
    ]


def _log_uniform(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = min(max(v, lo), hi)
    return v if rng.random() < 0.5 or v < 64 else v // 16 * 16


def draw(rng):
    op = rng.choice(["norm", "norm", "backward", "backward", "checkpoint", "product", "product"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op == "product":
        inner = _log_uniform(rng, 64, 16384)
        channels = _log_uniform(rng, 64, min(131072, (1 << 29) // inner))
        tokens = _log_uniform(rng, 1, 4096)
        c = _product("", tokens, channels, inner, dtype, rng.random() < 0.4, rng.random() < 0.3)
    else:
        cols = _log_uniform(rng, 64, 16384)
        rows = _log_uniform(rng, 1, min(32768, (1 << 28) // (cols * SIZE[dtype])))
        if op == "norm":
            c = _norm("", rows, cols, dtype, rng.random() < 0.6, rng.random() < 0.6)
        elif op == "backward":
            groups = rng.choice([1, 1, 2, 4, 8])
            rows = max(1, rows // groups) * groups
            c = _backward("", rows, cols, dtype, groups, rng.random() < 0.6, rng.random() < 0.6)
        else:
            c = _checkpoint("", rows, cols, dtype)
    del c["name"]
    return c


def _kept(cols):
    """Bytes of a row of a checkpoint."""
    return cols + -(-cols // BLOCK)


def work(case):
    """Each input read once, each output written once; additions and multiplications counted once each."""
    op, size = case["op"], SIZE[case["dtype"]]
    if op == "product":
        t, n, k = case["tokens"], case["channels"], case["inner"]
        got = t * k + n * k + t * n * size + 4 * (t + n) + (4 * n if case["bias"] else 0)
        if case["quantise"]:
            got += t * k * (size + 1) + 4 * t
        return {"bytes": got, "flops": 2 * t * n * k}
    rows, cols = case["rows"], case["cols"]
    n = rows * cols
    if op == "norm":        # x, residual -> sum, rstd; y, or 8 bits and scales, which are read back to values
        got = n * size * (3 if case["residual"] else 1) + 4 * cols + 4 * rows
        got += n * (2 + size) + 8 * rows if case["eight"] else n * size
        return {"bytes": got, "flops": 6 * n}
    if op == "backward":    # dy, x or its checkpoint, dsum -> dx, dweight
        got = n * size * (3 if case["residual"] else 2) + 4 * cols * (1 + case["groups"]) + 4 * rows
        return {"bytes": got + (rows * _kept(cols) if case["checkpoint"] else n * size), "flops": 11 * n}
    return {"bytes": 2 * n * size + 2 * rows * _kept(cols), "flops": 3 * n}


# --------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------
def _bytes(rows, cols):
    """8-bit rows that start on 16 bytes, as the package's quantising calls lay them out."""
    return torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device="cuda")[:, :cols]


def _activations(rows, cols, dtype, g):
    """Rows of differing size with a few columns that are much larger than the others."""
    x = torch.randn(rows, cols, generator=g, device="cuda") * (0.5 + torch.rand(rows, 1, generator=g, device="cuda"))
    x[:, ::97] *= 8.0
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, dtype = case["op"], TYPES[case["dtype"]]
    s = {"case": dict(case)}
    if op == "product":
        t, n, k = case["tokens"], case["channels"], case["inner"]
        s["w8"] = _bytes(n, k)
        step = max(1, (1 << 27) // k)
        for a in range(0, n, step):                             # weights of a trained matrix: its rows' largest is 127
            part = torch.randn(min(step, n - a), k, generator=g, device="cuda")
            s["w8"][a:a + step] = (part * (127.0 / part.abs().amax(1, keepdim=True))).round()
        s["w_scale"] = (1.0 + torch.rand(n, generator=g, device="cuda")) * (0.02 / 127.0)
        s["bias"] = torch.randn(n, generator=g, device="cuda") * 0.1 if case["bias"] else None
        x = _activations(t, k, dtype, g)
        if case["quantise"]:
            s["x"] = x
            s["eight"] = (_bytes(t, k), torch.empty(t, device="cuda"))
        else:
            top = x.float().abs().amax(1, keepdim=True)
            s["x8"] = _bytes(t, k)
            s["x8"].copy_((x.float() * (127.0 / top)).round())
            s["x_scale"] = top[:, 0] / 127.0
        s["out"] = torch.empty(t, n, dtype=dtype, device="cuda")
        return s
    rows, cols = case["rows"], case["cols"]
    x = _activations(rows, cols, dtype, g)
    if op == "checkpoint":
        s["x"] = x
        s["kept"] = (_bytes(rows, cols), torch.empty(rows, -(-cols // BLOCK), dtype=torch.uint8, device="cuda"))
        s["out"] = torch.empty(rows, cols, dtype=dtype, device="cuda")
        return s
    # the weight is a slice of the flat parameter vector that the optimizer holds
    params = torch.randn(4 * cols, generator=g, device="cuda") * 0.1
    s["weight"] = params[cols:2 * cols]
    s["weight"].add_(1.0)
    if op == "norm":
        s["x"] = x
        s["residual"] = torch.randn(rows, cols, generator=g, device="cuda").to(dtype) if case["residual"] else None
        s["total"] = torch.empty(rows, cols, dtype=dtype, device="cuda") if case["residual"] else None
        s["rstd"] = torch.empty(rows, device="cuda")
        if case["eight"]:
            s["eight"] = (_bytes(rows, cols), torch.empty(rows, device="cuda"))
        s["y"] = torch.empty(rows, cols, dtype=dtype, device="cuda")
        return s
    # backward: what the forward pass kept
    s["rstd"] = torch.rsqrt(x.float().square().mean(1) + EPS)
    if case["checkpoint"]:
        q, e = _keep(x)
        s["x"] = (_bytes(rows, cols), e)
        s["x"][0].copy_(q)
    else:
        s["x"] = x
    s["dy"] = (torch.randn(rows, cols, generator=g, device="cuda") * 0.02).to(dtype)
    s["dtotal"] = (torch.randn(rows, cols, generator=g, device="cuda") * 0.02).to(dtype) if case["residual"] else None
    # its gradient is a slice of the workers' rows of the optimizer's gradient buffer
    grads = torch.zeros(case["groups"], 4 * cols, device="cuda")
    s["out"] = (torch.empty(rows, cols, dtype=dtype, device="cuda"), grads[:, cols:2 * cols])
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
        if not c["eight"]:
            return cd.rms_norm(s["x"], s["weight"], s["residual"], EPS, out=(s["y"], s["total"], s["rstd"]))
        q, scale, total, rstd = cd.rms_norm8(s["x"], s["weight"], s["residual"], EPS, out=s["eight"] + (s["total"], s["rstd"]))
        return cd.dequantize_rows(q, scale, out=s["y"]), total, rstd, scale
    if op == "backward":
        return cd.rms_norm_backward(s["dy"], s["x"], s["weight"], s["rstd"], s["dtotal"], groups=c["groups"], out=s["out"])
    if op == "checkpoint":
        q, e = cd.checkpoint8(s["x"], out=s["kept"])
        return cd.checkpoint8_restore(q, e, out=s["out"]), e
    x8, x_scale = cd.quantize_rows(s["x"], out=s["eight"]) if c["quantise"] else (s["x8"], s["x_scale"])
    return cd.matmul8(x8, x_scale, s["w8"], s["w_scale"], s["bias"], out=s["out"])


def _plain(s):
    return {"norm": _plain_norm, "backward": _plain_backward, "checkpoint": _plain_checkpoint,
            "product": _plain_product}[s["case"]["op"]](s)


def _whole(p):
    """(the whole numbers nearest to 127 p / max |p|, max |p| / 127) of binary32 rows; the quotients in 64 bits, for
    those that are next to a half."""
    top = p.abs().amax(1)
    most = torch.where(top > 0, top, 1.0)
    return (127.0 * p.double() / most.double()[:, None]).round().float(), top / 127.0


def _plain_norm(s):
    c, x = s["case"], s["x"]
    total = None
    if c["residual"]:
        x = total = (x.float() + s["residual"].float()).to(x.dtype)
    h = x.float()
    rstd = 1.0 / torch.sqrt((h * h).mean(1) + EPS)
    p = h * s["weight"]
    if not c["eight"]:
        return (p * rstd[:, None]).to(x.dtype), total, rstd
    q, scale = _whole(p)
    scale = scale * rstd
    return (q * scale[:, None]).to(x.dtype), total, rstd, scale


def _keep(x):
    """(whole numbers of up to 127 in magnitude, biased exponents): blocks of 32 columns, the largest from 64 up."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    e = (v.abs().amax(2).view(torch.int32) >> 23) - 6
    e = e.clamp(min=1)
    q = (v * _power(254 - e)[:, :, None]).round().clamp(-127, 127)
    return q.view(rows, -1)[:, :cols], e.to(torch.uint8)


def _power(biased):
    """2^(biased - 127)."""
    return (biased.to(torch.int32) << 23).view(torch.float32)


def _values(q, e):
    return q.float() * _power(e).repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _plain_backward(s):
    c, dy, rstd = s["case"], s["dy"].float(), s["rstd"][:, None]
    x = _values(*s["x"]) if c["checkpoint"] else s["x"].float()
    xhat = x * rstd
    h = dy * s["weight"]
    dx = rstd * (h - xhat * (h * xhat).mean(1, keepdim=True))
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].float()
    return dx.to(s["dy"].dtype), (dy * xhat).view(c["groups"], -1, c["cols"]).sum(1)


def _plain_checkpoint(s):
    q, e = _keep(s["x"])
    return _values(q, e).to(s["x"].dtype), e


def _plain_product(s):
    if s["case"]["quantise"]:
        x8, x_scale = _whole(s["x"].float())
    else:
        x8, x_scale = s["x8"], s["x_scale"]
    # sums of whole numbers beyond 2^24: in 64 bits
    y = (x8.double() @ s["w8"].double().T).float() * x_scale[:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["out"].dtype)


# --------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# --------------------------------------------------------------------------------------------
def _parts(rows, width):
    step = max(1, (1 << 25) // width)
    return [slice(a, min(a + step, rows)) for a in range(0, rows, step)]


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "backward": _exact_backward, "checkpoint": _exact_checkpoint,
            "product": _exact_product}[case["op"]](case, s)


def _two_to(e):
    """2^e, whole numbers e of a normal binary64 power."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_whole(p):
    """Of binary32 rows p: the q nearest to 127 p / max |p| (even ones at a half), and the value of one step."""
    p = p.double()
    top = p.abs().max(1, keepdim=True).values
    t = torch.where(top > 0, 127.0 * p / top, 0.0)
    low = torch.floor(t)
    up = (t - low > 0.5) | ((t - low == 0.5) & (torch.remainder(low, 2.0) == 1.0))
    return low + up, top[:, 0] / 127.0


def _exact_norm(case, s):
    got = []
    for a in _parts(case["rows"], case["cols"]):
        x = s["x"][a]
        if case["residual"]:
            x = torch.add(x.double(), s["residual"][a].double()).to(x.dtype)    # the sum is kept in the activations' type
        rstd = (x.double().pow(2).sum(1) / case["cols"] + EPS).pow(-0.5)
        if case["eight"]:
            # the products that are quantised are binary32's
            q, step = _exact_whole((x.double() * s["weight"].double()).float())
            y, more = q * (step * rstd)[:, None], (step * rstd,)
        else:
            y, more = torch.einsum("rc,c,r->rc", x.double(), s["weight"].double(), rstd), ()
        got.append((y, x.double() if case["residual"] else None, rstd) + more)
    return tuple(None if v[0] is None else torch.cat(v) for v in zip(*got))


def _exact_backward(case, s):
    cols, groups = case["cols"], case["groups"]
    w = s["weight"].double()
    dx, dw = [], torch.zeros(groups, cols, dtype=torch.float64, device=w.device)
    per = case["rows"] // groups
    for i in range(groups):
        for part in _parts(per, cols):
            a = slice(i * per + part.start, i * per + part.stop)
            if case["checkpoint"]:
                q, e = (v[a].double() for v in s["x"])
                x = q * _two_to(e.repeat_interleave(BLOCK, 1)[:, :cols] - 127.0)
            else:
                x = s["x"][a].double()
            r, dy = s["rstd"][a].double(), s["dy"][a].double()
            dw[i] += torch.einsum("rc,rc,r->c", dy, x, r)
            d = torch.einsum("rc,c,r->rc", dy, w, r) - x * (torch.einsum("rc,rc,c->r", dy, x, w) * r ** 3 / cols)[:, None]
            dx.append(d if s["dtotal"] is None else d + s["dtotal"][a].double())
    return torch.cat(dx), dw


def _exact_checkpoint(case, s):
    rows, cols = s["x"].shape
    got = []
    for a in _parts(rows, cols):
        v = torch.nn.functional.pad(s["x"][a].double(), (0, -cols % BLOCK)).unflatten(1, (-1, BLOCK))
        top = v.abs().amax(2, keepdim=True)
        e = torch.where(top > 0, torch.frexp(top).exponent - 7, -126).clamp(min=-126)      # the largest is 64 to 128 steps
        t = v * _two_to(-e)
        low = torch.floor(t)
        q = low + ((t - low > 0.5) | ((t - low == 0.5) & (torch.remainder(low, 2.0) == 1.0)))
        got.append((q.clamp(-127, 127) * _two_to(e)).flatten(1)[:, :cols])
    return torch.cat(got), None


def _exact_product(case, s):
    t, n = case["tokens"], case["channels"]
    if case["quantise"]:
        x8, x_scale = _exact_whole(s["x"].float())
    else:
        x8, x_scale = s["x8"].double(), s["x_scale"].double()
    y = torch.empty(t, n, dtype=torch.float64, device=x8.device)
    step = max(1, (1 << 27) // case["inner"])
    for a in range(0, n, step):
        part = torch.einsum("tk,nk->tn", x8, s["w8"][a:a + step].double())
        y[:, a:a + step] = part * torch.outer(x_scale, s["w_scale"][a:a + step].double())
    return y if s["bias"] is None else y.add_(s["bias"].double())
