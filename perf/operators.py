"""The training-step operators, as work that can be timed: layer norm, the cross entropy of a projection on a large
vocabulary, and the orthogonalised update, each in plain torch operations (own = False) and through
paper_2108_03645_b200.train (own = True).

All arithmetic of the plain form is in 32 bits, whatever the type of the inputs, and is rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LN_EPS = 1e-5
NS_EPS = 1e-7
NS_STEPS = 5
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315  # coefficients of the quintic that the Muon optimiser iterates


def listed():
    return [
        # Layer norm. rows = tokens of the step, cols = the model's width; "pad" = further columns between two rows
        # (the input is a slice of a wider buffer).
        # a handful of tokens at a narrow model: only latency counts
        {"name": "norm-few-rows", "op": "norm", "rows": 7, "cols": 512, "dtype": "f32", "wdtype": "f32", "pad": 0, "train": False},
        # evaluation of one ordinary batch
        {"name": "norm-forward", "op": "norm", "rows": 8192, "cols": 2048, "dtype": "bf16", "wdtype": "bf16", "pad": 0, "train": False},
        # a training step on a ragged batch, odd width, rows that start on no 16-byte boundary
        {"name": "norm-train-odd", "op": "norm", "rows": 4099, "cols": 1001, "dtype": "f16", "wdtype": "f32", "pad": 6, "train": True},
        # a training step on the largest batch of a wide model
        {"name": "norm-train-wide", "op": "norm", "rows": 32768, "cols": 4096, "dtype": "bf16", "wdtype": "f32", "pad": 0, "train": True},
        # Cross entropy. rows = tokens, vocab x cols = the output projection; ignored = share of tokens without a target.
        # scoring a few tokens: the projection is read once, for next to nothing
        {"name": "loss-few-tokens", "op": "loss", "rows": 5, "cols": 1024, "vocab": 32000, "dtype": "bf16", "ignored": 0.0, "pad": 0, "train": False},
        # evaluation of an ordinary batch
        {"name": "loss-forward", "op": "loss", "rows": 4096, "cols": 1024, "vocab": 50000, "dtype": "bf16", "ignored": 0.1, "pad": 0, "train": False},
        # a training step on a ragged batch: odd number of tokens, of columns and of vocabulary entries, scaled loss in fp16
        {"name": "loss-train-odd", "op": "loss", "rows": 1023, "cols": 777, "vocab": 32001, "dtype": "f16", "ignored": 0.3, "pad": 7, "train": True},
        # a training step on the largest batch of a wide model with a large vocabulary
        {"name": "loss-train-large", "op": "loss", "rows": 8192, "cols": 2048, "vocab": 128000, "dtype": "bf16", "ignored": 0.1, "pad": 0, "train": True},
        # Orthogonalised update of `count` matrices of one shape.
        # one small matrix: five steps of three short products, latency counts
        {"name": "update-small", "op": "update", "count": 1, "m": 128, "n": 256, "dtype": "f32"},
        # the matrices of twelve layers of a small model at once
        {"name": "update-layers", "op": "update", "count": 12, "m": 768, "n": 768, "dtype": "bf16"},
        # odd sizes, more rows than columns
        {"name": "update-odd", "op": "update", "count": 3, "m": 1999, "n": 1001, "dtype": "f32"},
        # one feed-forward matrix of a wide model
        {"name": "update-wide", "op": "update", "count": 1, "m": 4096, "n": 8192, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _most(op):
    return max(_cost(c) for c in listed() if c["op"] == op)


def _cost(case):
    w = work(case)
    return w["bytes"] + w["flops"] / 200


def draw(rng):
    op = rng.choice(["norm", "loss", "update"])
    while True:
        if op == "norm":
            case = {"op": op, "rows": _log(rng, 1, 32768), "cols": _log(rng, 64, 16384), "dtype": rng.choice(["f32", "bf16", "f16"]),
                    "pad": rng.choice([0, 0, 8, 3]), "train": rng.random() < 0.7}
            case["wdtype"] = rng.choice(["f32", case["dtype"]])
        elif op == "loss":
            case = {"op": op, "rows": _log(rng, 1, 16384), "cols": _log(rng, 64, 4096), "vocab": _log(rng, 100, 150000),
                    "dtype": rng.choice(["bf16", "bf16", "f16"]), "ignored": rng.choice([0.0, 0.1, 0.5]),
                    "pad": rng.choice([0, 0, 8, 3]), "train": rng.random() < 0.7}
            if rng.random() < 0.6:  # widths of models are round, as a rule
                case["cols"] = max(64, case["cols"] // 64 * 64)
        else:
            case = {"op": op, "count": _log(rng, 1, 16), "m": _log(rng, 32, 8192), "n": _log(rng, 32, 8192),
                    "dtype": rng.choice(["f32", "bf16"])}
            if rng.random() < 0.6:
                case["m"], case["n"] = max(32, case["m"] // 32 * 32), max(32, case["n"] // 32 * 32)
        if _cost(case) <= _most(op):
            return case


def _wide(t, pad):
    """The values of t as a slice of a buffer that has `pad` more columns."""
    if not pad:
        return t
    wide = torch.empty(t.shape[0], t.shape[1] + pad, dtype=t.dtype, device=t.device)
    wide.fill_(float("nan"))  # nobody reads what lies between two rows
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = {"case": dict(case)}
    if case["op"] == "norm":
        n, d, wt = case["rows"], case["cols"], DTYPES[case["wdtype"]]
        # activations of a residual stream: an offset and a scale of its own for each row, a few large columns
        x = randn(n, d) * (0.5 + torch.rand(n, 1, generator=g, device="cuda") * 2) + randn(n, 1) + 0.5
        x[:, ::97] *= 6
        s["x"] = _wide(x.to(dt), case["pad"])
        s["w"] = (1 + 0.2 * randn(d)).to(wt)
        s["b"] = (0.1 * randn(d)).to(wt)
        if case["train"]:
            s["dy"] = _wide((randn(n, d) * 0.02).to(dt), case["pad"])
    elif case["op"] == "loss":
        n, d, v = case["rows"], case["cols"], case["vocab"]
        # a model that has learnt something: a token's hidden vector leans towards its target's row
        w = (randn(v, d) * (2 / math.sqrt(d))).to(dt)
        t = torch.randint(0, v, (n,), generator=g, device="cuda")
        h = randn(n, d) + w.index_select(0, t).float() * (4 * torch.rand(n, 1, generator=g, device="cuda"))
        t[torch.rand(n, generator=g, device="cuda") < case["ignored"]] = -100
        s["h"], s["w"], s["t"] = _wide(h.to(dt), case["pad"]), _wide(w, case["pad"]), t
        if case["train"]:
            # the mean over the tokens that have a target; fp16 training scales its loss
            scale = 4096.0 if case["dtype"] == "f16" else 1.0
            s["dloss"] = torch.full((n,), scale / max(1, n), device="cuda")
    else:
        c, m, n = case["count"], case["m"], case["n"]
        # a momentum buffer: a part of low rank, and noise
        r = max(1, min(m, n) // 4)
        u = torch.bmm(randn(c, m, r), randn(c, r, n)) / math.sqrt(r) + 0.5 * randn(c, m, n)
        s["g"] = (u * 1e-3).to(dt)
    return s


def _norm_plain(s):
    x = s["x"].float()
    w, b = s["w"].float(), s["b"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = torch.rsqrt((xc * xc).mean(1) + LN_EPS)
    xh = xc * rstd[:, None]
    out = {"y": (xh * w + b).to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if s["case"]["train"]:
        dy = s["dy"].float()
        gr = dy * w
        dx = rstd[:, None] * (gr - gr.mean(1, keepdim=True) - xh * (gr * xh).mean(1, keepdim=True))
        out["dx"] = dx.to(s["x"].dtype)
        out["dweight"] = (dy * xh).sum(0).to(s["w"].dtype)
        out["dbias"] = dy.sum(0).to(s["w"].dtype)
    return out


def _loss_plain(s):
    h, w, t = s["h"].float(), s["w"].float(), s["t"]
    v = w.shape[0]
    live = (t >= 0) & (t < v)
    at = torch.where(live, t, torch.zeros_like(t))[:, None]
    logits = h @ w.t()
    lt = logits.gather(1, at)[:, 0]
    top = logits.amax(1, keepdim=True)
    e = logits.sub_(top).exp_()
    z = e.sum(1, keepdim=True)
    lse = (z.log() + top)[:, 0]
    out = {"loss": torch.where(live, lse - lt, torch.zeros_like(lt)), "lse": lse}
    if s["case"]["train"]:
        gn = torch.where(live, s["dloss"], torch.zeros_like(lt))[:, None]
        p = e.mul_(gn / z)
        p.scatter_add_(1, at, -gn)
        out["dhidden"] = (p @ w).to(s["h"].dtype)
        out["dweight"] = (p.t() @ h).to(s["w"].dtype)
    return out


def _update_plain(s):
    x = s["g"].float()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    flip = x.shape[1] > x.shape[2]
    if flip:
        x = x.transpose(1, 2)
    for _ in range(NS_STEPS):
        a = x @ x.transpose(1, 2)
        x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
    if flip:
        x = x.transpose(1, 2)
    return {"update": x.to(torch.bfloat16).contiguous()}


def run(s):
    op = s["case"]["op"]
    if not own:
        return _norm_plain(s) if op == "norm" else _loss_plain(s) if op == "loss" else _update_plain(s)
    from paper_2108_03645_b200 import train

    if op == "norm":
        y, mean, rstd = train.layer_norm(s["x"], s["w"], s["b"], eps=LN_EPS)
        out = {"y": y, "mean": mean, "rstd": rstd}
        if s["case"]["train"]:
            out["dx"], out["dweight"], out["dbias"] = train.layer_norm_backward(s["dy"], s["x"], mean, rstd, s["w"])
        return out
    if op == "loss":
        loss, lse = train.linear_cross_entropy(s["h"], s["w"], s["t"])
        out = {"loss": loss, "lse": lse}
        if s["case"]["train"]:
            out["dhidden"], out["dweight"] = train.linear_cross_entropy_backward(s["dloss"], s["h"], s["w"], s["t"], lse)
        return out
    return {"update": train.orthogonalize(s["g"], steps=NS_STEPS, coefficients=(NS_A, NS_B, NS_C), eps=NS_EPS)}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        n, d = case["rows"], case["cols"]
        wsize = 4 if case["wdtype"] == "f32" else 2
        # forward: x in, y out; backward: dy in, dx out (x is read once for both)
        return {"bytes": (4 if case["train"] else 2) * n * d * size + 8 * n + (4 if case["train"] else 2) * d * wsize,
                "flops": (20 if case["train"] else 8) * n * d}
    if case["op"] == "loss":
        n, d, v = case["rows"], case["cols"], case["vocab"]
        times = 2 if case["train"] else 1  # the gradients are as large as the inputs
        # the logits once, and their gradient against each factor
        return {"bytes": times * (n + v) * d * size + 8 * n + (12 if case["train"] else 8) * n,
                "flops": (6 if case["train"] else 2) * n * d * v}
    c, m, n = case["count"], min(case["m"], case["n"]), max(case["m"], case["n"])
    # a step: X X^T and A A, both symmetric (one half has to be computed), and the product with X
    return {"bytes": c * m * n * (size + 2), "flops": c * NS_STEPS * (m * m * n + m * m * m + 2 * m * m * n)}


def _norm_exact(s):
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0)
    rstd = 1 / (var + LN_EPS).sqrt()
    xh = (x - mean[:, None]) / (var + LN_EPS).sqrt()[:, None]
    out = {"y": torch.addcmul(b, xh, w), "mean": mean, "rstd": rstd}
    if s["case"]["train"]:
        dy = s["dy"].double()
        d = x.shape[1]
        gr = dy * w
        # the derivative of (x - mean) / sigma, column by column: subtract the parts along 1 and along xh
        out["dx"] = (gr - gr.sum(1, keepdim=True) / d - xh * (torch.einsum("nd,nd->n", gr, xh)[:, None] / d)) * rstd[:, None]
        out["dweight"] = torch.einsum("nd,nd->d", dy, xh)
        out["dbias"] = dy.sum(0)
    return out


def _loss_exact(s):
    h, w, t = s["h"].double(), s["w"].double(), s["t"]
    n, v = h.shape[0], w.shape[0]
    loss, lses, dh = [], [], []
    dw = torch.zeros_like(w)
    step = max(1, (1 << 28) // v)
    for r in range(0, n, step):  # whole rows, a block at a time
        hb, tb = h[r:r + step], t[r:r + step]
        live = (tb >= 0) & (tb < v)
        l = torch.einsum("nd,vd->nv", hb, w)
        lse = torch.logsumexp(l, 1)
        rows = torch.nonzero(live)[:, 0]
        lb = torch.zeros_like(lse)
        lb[rows] = lse[rows] - l[rows, tb[rows]]
        loss.append(lb)
        lses.append(lse)
        if s["case"]["train"]:
            p = torch.softmax(l, 1)
            p[rows, tb[rows]] -= 1
            p *= (s["dloss"][r:r + step].double() * live)[:, None]
            dh.append(p @ w)
            dw += p.t() @ hb
    out = {"loss": torch.cat(loss), "lse": torch.cat(lses)}
    if s["case"]["train"]:
        out["dhidden"], out["dweight"] = torch.cat(dh), dw
    return out


def _update_exact(s):
    out = []
    for g in s["g"].double():
        x = g / (torch.linalg.vector_norm(g) + NS_EPS)
        for _ in range(NS_STEPS):
            # odd polynomial of the matrix, from the other side than the plain form where the shape allows
            if x.shape[0] <= x.shape[1]:
                a = x @ x.T
                x = NS_A * x + NS_B * (a @ x) + NS_C * (a @ (a @ x))
            else:
                a = x.T @ x
                x = NS_A * x + NS_B * (x @ a) + NS_C * ((x @ a) @ a)
        out.append(x)
    return {"update": torch.stack(out)}


def exact(case, seed):
    s = prepare(case, seed)
    if work(case)["flops"] > 2e13:  # more than about 20 seconds in 64 bits
        return None
    return _norm_exact(s) if case["op"] == "norm" else _loss_exact(s) if case["op"] == "loss" else _update_exact(s)
