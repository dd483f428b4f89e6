"""What stands around the sparse products in a training step, as cases that can be timed.

A program that trains a language model with N:M transposable masks, or recovers a pruned one from its dense teacher,
normalises and activates between the products with the compressed operands, forward and backward, and takes its loss from the
teacher's top logits.  Each operator appears from a few rows, where the latency of a call counts, to whole training batches.

A case is a dict of plain values:
  op    "norm"       layer norm of x + residual: result, sum, mean and reciprocal deviation of each row
        "norm_grad"  its gradients: input (with what reaches the residual stream by its other way), weight, bias
        "gelu"       GELU of x + bias
        "gelu_grad"  its gradients: input and bias
        "distill"    distillation from the teacher's top logits: loss and statistics of each row, and (grad) the gradient
        "distill_grad"  the gradient alone, from the statistics of an earlier call
  rows, cols (cols: the vocabulary of the losses), dt, pad (elements between the end of a row of x, or of the logits, and the next row)
  param (type of weight and bias), residual, tanh (form of GELU)
  k (teacher's logits of a row), temperature, index (bits), ragged (rows have fewer than k entries, down to none, and some rows
  do not count)
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def norm_case(rows, cols, dt, param="f32", residual=True, pad=0):
    return {"op": "norm", "rows": rows, "cols": cols, "dt": dt, "param": param, "residual": residual, "pad": pad}


def norm_grad_case(rows, cols, dt, param="f32", residual=True, pad=0):
    return dict(norm_case(rows, cols, dt, param, residual, pad), op="norm_grad")


def gelu_case(rows, cols, dt, param="f32", tanh=False, pad=0):
    return {"op": "gelu", "rows": rows, "cols": cols, "dt": dt, "param": param, "tanh": tanh, "pad": pad}


def gelu_grad_case(rows, cols, dt, param="f32", tanh=False, pad=0):
    return dict(gelu_case(rows, cols, dt, param, tanh, pad), op="gelu_grad")


def distill_case(rows, cols, k, dt, temperature, grad=True, index=32, ragged=False, pad=0):
    return {"op": "distill", "rows": rows, "cols": cols, "k": k, "dt": dt, "temperature": temperature, "grad": grad,
            "index": index, "ragged": ragged, "pad": pad}


def distill_grad_case(rows, cols, k, dt, temperature, index=32, ragged=False, pad=0):
    return dict(distill_case(rows, cols, k, dt, temperature, True, index, ragged, pad), op="distill_grad")


def listed():
    return [
        # one token through the model while it answers: the time of a call is all there is
        {"name": "norm_1x1024_bf16", **norm_case(1, 1024, "bf16", "bf16")},
        # the norm behind a block of an encoder layer, over a training batch of 8192 tokens
        {"name": "norm_8192x1024_bf16", **norm_case(8192, 1024, "bf16")},
        # its way back, weights kept in fp32
        {"name": "norm_grad_8192x1024_bf16", **norm_grad_case(8192, 1024, "bf16")},
        # a short, odd batch of an odd width in fp32
        {"name": "norm_grad_1003x2051_f32", **norm_grad_case(1003, 2051, "f32", residual=False)},
        # the feed-forward block's activation while a few sequences are decoded
        {"name": "gelu_16x4096_bf16", **gelu_case(16, 4096, "bf16", "bf16")},
        # and over a training batch
        {"name": "gelu_8192x4096_bf16", **gelu_case(8192, 4096, "bf16")},
        {"name": "gelu_grad_8192x4096_bf16", **gelu_grad_case(8192, 4096, "bf16")},
        # an odd layer in fp32 with the other form of GELU
        {"name": "gelu_grad_1003x1001_f32", **gelu_grad_case(1003, 1001, "f32", tanh=True)},
        # a classifier's evaluation against its teacher: the loss alone
        {"name": "distill_64x1000_f32", **distill_case(64, 1000, 16, "f32", 2.0, grad=False, index=64)},
        # a training step of a language model: loss and gradient of 4096 tokens
        {"name": "distill_4096x32000_bf16", **distill_case(4096, 32000, 64, "bf16", 1.0)},
        # a few long sequences' ends: few rows, a large vocabulary, long lists, padding among the tokens
        {"name": "distill_48x131072_f32", **distill_case(48, 131072, 256, "f32", 1.5, index=64, ragged=True)},
        # the gradient when its weights are known only after the loss; a vocabulary without a round size
        {"name": "distill_grad_1003x50021_bf16", **distill_grad_case(1003, 50021, 32, "bf16", 2.0, ragged=True)},
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def _width(rng, lo, hi, least):
    """Odd in two cases of five, else a multiple of 64."""
    cols = _log_uniform(rng, lo, hi)
    cols = cols if rng.random() < 0.4 else max(least, cols // 64 * 64)
    return cols + 64 if cols == 3 << 10 else cols


def draw(rng):
    most = work(distill_case(4096, 32000, 64, "bf16", 1.0))["bytes"]
    op = rng.choice(["norm", "norm_grad", "gelu", "gelu_grad", "distill", "distill", "distill_grad"])
    dt = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([8, 24, 5]) if rng.random() < 0.2 else 0
    if op.startswith("distill"):
        rows, cols = _log_uniform(rng, 1, 8192), _width(rng, 500, 200000, 512)
        k = min(_log_uniform(rng, 1, 256), cols // 2)
        more = {"index": rng.choice([32, 64]), "ragged": rng.random() < 0.4, "pad": pad}
        temperature = rng.choice([1.0, 1.0, 1.5, 2.0, 4.0])
        grad = op == "distill" and rng.random() < 0.7
        make = lambda r: distill_case(r, cols, k, dt, temperature, grad, **more) if op == "distill" else distill_grad_case(r, cols, k, dt, temperature, **more)  # noqa: E731
    else:
        rows, cols = _log_uniform(rng, 1, 32768), _width(rng, 64, 16384, 64)
        param = rng.choice(["f32", dt])
        flag = rng.random() < 0.5
        make = lambda r: {"norm": norm_case, "norm_grad": norm_grad_case, "gelu": gelu_case, "gelu_grad": gelu_grad_case}[op](r, cols, dt, param, flag, pad)  # noqa: E731
    while rows > 1 and work(make(rows))["bytes"] > most:
        rows = rows * 2 // 3
    return make(rows)


def _size(dt):
    return 4 if dt == "f32" else 2


def work(case):
    op, rows, cols = case["op"], case["rows"], case["cols"]
    whole = rows * cols * _size(case["dt"])                       # one tensor of the call
    if op.startswith("distill"):
        lists = rows * case["k"] * (_size(case["dt"]) + case["index"] // 8)
        row = 4 * rows * (3 if op == "distill" else 2) + (4 * rows if case["grad"] else 0)
        return {"bytes": whole * (2 if case["grad"] else 1) + lists + row, "flops": rows * cols * (8 if case["grad"] else 4)}
    vector = cols * _size(case["param"])
    if op == "norm":
        return {"bytes": whole * (4 if case["residual"] else 2) + 2 * vector + 8 * rows, "flops": 8 * rows * cols}
    if op == "norm_grad":
        return {"bytes": whole * (4 if case["residual"] else 3) + 3 * vector + 8 * rows, "flops": 14 * rows * cols}
    if op == "gelu":
        return {"bytes": 2 * whole + vector, "flops": 12 * rows * cols}
    return {"bytes": 3 * whole + 2 * vector, "flops": 20 * rows * cols}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, rows, cols, dt = case["op"], case["rows"], case["cols"], TYPES[case["dt"]]

    def normal(shape, scale=1.0, shift=0.0, to=dt):
        return (torch.randn(shape, device="cuda", generator=gen) * scale + shift).to(to)

    def wide(scale=1.0):                        # rows x cols inside rows of cols + pad elements
        return normal((rows, cols + case["pad"]), scale)[:, :cols]

    def out(dtype=dt, *shape):
        return torch.empty(shape or (rows, cols), dtype=dtype, device="cuda")

    s = {"case": case}
    if op.startswith("distill"):
        k = case["k"]
        s["logits"] = wide(2.0)
        # a list's entries are distinct, in no order and anywhere in the vocabulary
        base = torch.randperm(cols, device="cuda", generator=gen)[:k]
        shift = torch.randint(0, cols, (rows, 1), device="cuda", generator=gen)
        at = (base[None, :] + shift) % cols
        # the student half knows its teacher: high logits where the teacher has them, with errors
        top = torch.randn((rows, k), device="cuda", generator=gen).abs() * 3.0 + 4.0
        s["logits"].scatter_(1, at, (top + torch.randn((rows, k), device="cuda", generator=gen)).to(dt))
        s["teacher"] = top.to(dt)
        if case["ragged"]:
            have = torch.randint(0, k + 1, (rows, 1), device="cuda", generator=gen)
            have[0] = k                                         # one row at least has something to learn
            at = torch.where(torch.arange(k, device="cuda")[None, :] < have, at, -1)
        s["index"] = at.to(torch.int32 if case["index"] == 32 else torch.int64)
        counts = torch.rand(rows, device="cuda", generator=gen) < (0.8 if case["ragged"] else 1.0)
        counts[0] = True
        s["row_weight"] = counts.float() / rows if case["grad"] else None
        s["row_max"], s["row_sum"] = out(torch.float32, rows), out(torch.float32, rows)
        if op == "distill_grad":                # as the loss's call has left them
            z = s["logits"].double()
            top_z = z.amax(1)
            s["row_max"].copy_(top_z)
            s["row_sum"].copy_(((z - top_z[:, None]) / case["temperature"]).exp().sum(1))
        s["loss"] = out(torch.float32, rows)
        s["dlogits"] = out() if case["grad"] else None
        return s
    param = TYPES[case["param"]]
    s["bias"] = normal((cols,), 0.1, 0.0, param)
    if op.startswith("norm"):
        s["weight"] = normal((cols,), 0.1, 1.0, param)
        s["x"] = wide()
        s["residual"] = normal((rows, cols), 2.0, 0.1) if op == "norm" and case["residual"] else None
        s["mean"], s["rstd"] = out(torch.float32, rows), out(torch.float32, rows)
        if op == "norm":
            s["y"], s["total"] = out(), out() if case["residual"] else None
        else:
            x = s["x"].double()
            s["mean"].copy_(x.mean(1))
            s["rstd"].copy_((x.var(1, correction=0) + EPS).rsqrt())
            s["dy"] = normal((rows, cols), 0.1)
            s["dtotal"] = normal((rows, cols), 0.1) if case["residual"] else None
            s["dx"], s["dweight"], s["dbias"] = out(), out(param, cols), out(param, cols)
        return s
    s["x"], s["y"] = wide(1.5), out()
    if op == "gelu_grad":
        s["dy"], s["dx"], s["dbias"] = normal((rows, cols), 0.1), s.pop("y"), out(param, cols)
    return s


def _workspace(s, alloc, of):
    """A program allocates it once and keeps it from call to call."""
    if "workspace" not in s:
        s["workspace"] = alloc(of)
    return s["workspace"]


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2102_08124_amd import binding as tm

    case = s["case"]
    op = case["op"]
    if op == "norm":
        tm.tmask_layer_norm(s["x"], s["y"], s["weight"], s["bias"], residual=s["residual"], total=s["total"], mean=s["mean"],
                            rstd=s["rstd"], eps=EPS)
        return {"y": s["y"], "total": s["total"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "norm_grad":
        tm.tmask_layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["dx"], s["weight"], dweight=s["dweight"],
                                     dbias=s["dbias"], dtotal=s["dtotal"], workspace=_workspace(s, tm.alloc_layer_norm_workspace, s["x"]))
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    if op == "gelu":
        tm.tmask_bias_gelu(s["x"], s["y"], s["bias"], tanh=case["tanh"])
        return {"y": s["y"]}
    if op == "gelu_grad":
        tm.tmask_bias_gelu_backward(s["dy"], s["x"], s["dx"], s["bias"], dbias=s["dbias"], tanh=case["tanh"],
                                    workspace=_workspace(s, tm.alloc_bias_gelu_workspace, s["x"]))
        return {"dx": s["dx"], "dbias": s["dbias"]}
    if op == "distill":
        tm.tmask_distill(s["logits"], s["teacher"], s["index"], case["temperature"], s["loss"], row_max=s["row_max"],
                         row_sum=s["row_sum"], dlogits=s["dlogits"], row_weight=s["row_weight"],
                         workspace=_workspace(s, tm.alloc_distill_workspace, s["logits"]))
        return {"loss": s["loss"], "row_max": s["row_max"], "row_sum": s["row_sum"], "dlogits": s["dlogits"]}
    tm.tmask_distill_backward(s["logits"], s["teacher"], s["index"], case["temperature"], s["row_max"], s["row_sum"], s["dlogits"],
                              row_weight=s["row_weight"])
    return {"dlogits": s["dlogits"]}


# The plain forms: elementary operations in 32 bits, rounded once at the end.

def _run_plain(s):
    case = s["case"]
    op, dt = case["op"], TYPES[case["dt"]]
    if op == "norm":
        t = s["x"].float()
        if s["residual"] is not None:
            t = t + s["residual"].float()
        mean = t.mean(1)
        away = t - mean[:, None]
        rstd = ((away * away).mean(1) + EPS).rsqrt()
        y = away * rstd[:, None] * s["weight"].float() + s["bias"].float()
        return {"y": y.to(dt), "total": t.to(dt) if s["residual"] is not None else None, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        dy = s["dy"].float()
        xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        dxh = dy * s["weight"].float()
        dx = s["rstd"][:, None] * (dxh - dxh.mean(1, keepdim=True) - xh * (dxh * xh).mean(1, keepdim=True))
        if s["dtotal"] is not None:
            dx = dx + s["dtotal"].float()
        param = TYPES[case["param"]]
        return {"dx": dx.to(dt), "dweight": (dy * xh).sum(0).to(param), "dbias": dy.sum(0).to(param)}
    if op.startswith("gelu"):
        u = s["x"].float() + s["bias"].float()
        if case["tanh"]:
            c = math.sqrt(2.0 / math.pi)
            th = torch.tanh(c * (u + 0.044715 * u * u * u))
            share, slope = 0.5 * (1.0 + th), 0.5 * (1.0 - th * th) * c * (1.0 + 0.134145 * u * u)
        else:
            share, slope = 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5))), torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
        if op == "gelu":
            return {"y": (u * share).to(dt)}
        dx = s["dy"].float() * (share + u * slope)
        return {"dx": dx.to(dt), "dbias": dx.sum(0).to(TYPES[case["param"]])}
    T = case["temperature"]
    z = s["logits"].float()
    there = s["index"] >= 0
    at = s["index"].long().clamp(min=0)
    t = torch.where(there, s["teacher"].float() / T, -math.inf)
    some = there.any(1, keepdim=True)
    t = torch.where(some, t, 0.0)                                # a row without an entry has no distribution: its p are made 0 below
    t_away = t - t.amax(1, keepdim=True)
    t_exp = t_away.exp()
    t_sum = t_exp.sum(1, keepdim=True)
    p = torch.where(there, t_exp / t_sum, 0.0)
    row_max = z.amax(1) if op == "distill" else s["row_max"]
    away = (z - row_max[:, None]) / T
    e = away.exp()
    row_sum = e.sum(1) if op == "distill" else s["row_sum"]
    got = {}
    if op == "distill":
        log_q = away.gather(1, at) - row_sum.log()[:, None]
        log_p = torch.where(there, t_away, 0.0) - t_sum.log()
        got = {"loss": T * T * (p * (log_p - log_q)).sum(1), "row_max": row_max, "row_sum": row_sum, "dlogits": None}
    if case["grad"]:
        w = T * s["row_weight"][:, None]
        dz = torch.where(some, w * e / row_sum[:, None], 0.0)
        dz.scatter_add_(1, at, -w * p)
        got["dlogits"] = dz.to(dt)
    return got


# The definitions in 64 bits; gradients by differentiating the forward formula.

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    wide = lambda key: s[key].double() if s.get(key) is not None else None  # noqa: E731
    if op == "norm":
        t = wide("x") if s["residual"] is None else wide("x") + wide("residual")
        var, mean = torch.var_mean(t, 1, correction=0, keepdim=True)
        y = (t - mean) / torch.sqrt(var + EPS) * wide("weight") + wide("bias")
        return {"y": y, "total": None if s["residual"] is None else t, "mean": mean[:, 0], "rstd": 1.0 / torch.sqrt(var[:, 0] + EPS)}
    if op == "norm_grad":
        t, weight, bias = (wide(key).requires_grad_() for key in ("x", "weight", "bias"))
        var, mean = torch.var_mean(t, 1, correction=0, keepdim=True)
        y = (t - mean) / torch.sqrt(var + EPS) * weight + bias
        aim = (y * wide("dy")).sum() + (0.0 if s["dtotal"] is None else (t * wide("dtotal")).sum())
        dx, dweight, dbias = torch.autograd.grad(aim, (t, weight, bias))
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if op.startswith("gelu"):
        x, bias = wide("x").requires_grad_(), wide("bias").requires_grad_()
        u = x + bias
        if case["tanh"]:
            y = u / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (u + 0.044715 * u ** 3)))
        else:
            y = 0.5 * u * torch.special.erfc(-u / math.sqrt(2.0))
        if op == "gelu":
            return {"y": y.detach()}
        dx, dbias = torch.autograd.grad((y * wide("dy")).sum(), (x, bias))
        return {"dx": dx, "dbias": dbias}
    T = case["temperature"]
    got = {"loss": [], "row_max": [], "row_sum": [], "dlogits": []}
    step = max(1, (1 << 26) // case["cols"])                     # rows at a time
    for r in range(0, case["rows"], step):
        z = s["logits"][r:r + step].double().requires_grad_()
        index, teacher = s["index"][r:r + step].long(), s["teacher"][r:r + step].double()
        away = z / T
        lse = torch.logsumexp(away, 1, keepdim=True)
        score = torch.where(index >= 0, teacher / T, torch.full_like(teacher, -1e300))
        log_p = torch.log_softmax(score, 1)
        p = torch.where(index >= 0, log_p.exp(), 0.0)
        log_q = away.gather(1, index.clamp(min=0)) - lse
        loss = T * T * (torch.where(p > 0, p * (log_p - log_q), 0.0)).sum(1)
        if case["grad"]:
            aim = (loss * s["row_weight"][r:r + step].double()).sum()
            got["dlogits"].append(torch.autograd.grad(aim, z)[0])
        z_max = z.detach().amax(1)
        got["loss"].append(loss.detach())
        got["row_max"].append(z_max)
        got["row_sum"].append((lse.detach()[:, 0] - z_max / T).exp())
    got = {key: torch.cat(parts) if parts else None for key, parts in got.items()}
    return got if op == "distill" else {"dlogits": got["dlogits"]}
