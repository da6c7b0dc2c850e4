"""The operators of an attention layer's training step, as work that can be timed: norms of queries and keys with the
rotation of their positions, causal attention over packed sequences with grouped heads, and the norm and the clipping of all
gradients, each in plain torch operations (own = False) and through paper_2108_03645_b200.train (own = True).

The plain form computes in 32 bits, whatever the type of the inputs, and rounds once at the end; angles of positions and the
sum over all gradients are in 64 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NORM_EPS = 1e-6
CLIP_EPS = 1e-6
ROTARY_BASE = 10000.0


def listed():
    return [
        # Norm and rotation. heads, kv = query and key heads; rotary = rotated values of a head's dim; "first" = the position of
        # the first token; "packed" = queries and keys are slices of one product's output.
        # a handful of tokens of a narrow model in 32 bits: only latency counts
        {"name": "rotate-few-tokens", "op": "rotate", "tokens": 5, "heads": 8, "kv": 2, "dim": 64, "rotary": 64, "dtype": "f32",
         "wdtype": "f32", "interleaved": False, "packed": False, "first": 0, "train": False},
        # evaluation of an ordinary batch, in place of a slice of the fused projection
        {"name": "rotate-forward", "op": "rotate", "tokens": 8192, "heads": 16, "kv": 4, "dim": 128, "rotary": 128, "dtype": "bf16",
         "wdtype": "bf16", "interleaved": False, "packed": True, "first": 0, "train": False},
        # a training step at far positions: neighbouring pairs, a part of an odd head rotated, ragged batch
        {"name": "rotate-train-odd", "op": "rotate", "tokens": 4099, "heads": 12, "kv": 3, "dim": 81, "rotary": 40, "dtype": "f16",
         "wdtype": "f32", "interleaved": True, "packed": True, "first": 1000003, "train": True},
        # a training step on the largest batch
        {"name": "rotate-train-large", "op": "rotate", "tokens": 65536, "heads": 32, "kv": 8, "dim": 128, "rotary": 128, "dtype": "bf16",
         "wdtype": "f32", "interleaved": False, "packed": True, "first": 0, "train": True},
        # Attention. `sequences` lengths between `shortest` and `longest` (spread over their logarithm, made from `lengths`);
        # tail = tokens behind the last sequence, which belong to none.
        # scoring a few short prompts: only latency counts
        {"name": "attend-short", "op": "attend", "sequences": 9, "shortest": 1, "longest": 40, "lengths": 1, "tail": 0, "heads": 8, "kv": 2,
         "dim": 64, "dtype": "bf16", "packed": True, "train": False},
        # evaluation of an ordinary batch of ragged documents
        {"name": "attend-forward", "op": "attend", "sequences": 12, "shortest": 64, "longest": 4096, "lengths": 2, "tail": 0, "heads": 16,
         "kv": 4, "dim": 128, "dtype": "bf16", "packed": True, "train": False},
        # a training step of many short samples, a key for every query head
        {"name": "attend-train-samples", "op": "attend", "sequences": 128, "shortest": 256, "longest": 256, "lengths": 3, "tail": 0, "heads": 16,
         "kv": 16, "dim": 64, "dtype": "bf16", "packed": False, "train": True},
        # a training step in fp16 with odd heads, ragged lengths from one token on, and a padded end
        {"name": "attend-train-odd", "op": "attend", "sequences": 40, "shortest": 1, "longest": 3001, "lengths": 4, "tail": 77, "heads": 15,
         "kv": 3, "dim": 77, "dtype": "f16", "packed": False, "train": True},
        # a training step on one long context
        {"name": "attend-train-long", "op": "attend", "sequences": 1, "shortest": 16384, "longest": 16384, "lengths": 5, "tail": 0, "heads": 16,
         "kv": 4, "dim": 128, "dtype": "bf16", "packed": True, "train": True},
        # Norm and clipping of all gradients of a model: `layers` blocks of `width` and an embedding of `vocab` rows; "limit" = the
        # largest norm allowed, as a share of about the present one; clip False: the norm alone.
        # one small block: only latency counts
        {"name": "clip-small", "op": "clip", "layers": 1, "width": 200, "vocab": 101, "dtype": "f32", "limit": 0.5, "clip": True},
        # the norm of a small model's gradients, as a step logs it
        {"name": "clip-norm", "op": "clip", "layers": 12, "width": 1024, "vocab": 32000, "dtype": "bf16", "limit": 1.0, "clip": False},
        # a step of a large model
        {"name": "clip-large", "op": "clip", "layers": 24, "width": 2048, "vocab": 128001, "dtype": "bf16", "limit": 0.1, "clip": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] + w["flops"] / 200


def _most(op):
    return max(_cost(c) for c in listed() if c["op"] == op)


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8])
    return kv * rng.choice([1, 1, 2, 3, 4, 5, 8]), kv


def draw(rng):
    op = rng.choice(["rotate", "attend", "attend", "clip"])
    while True:
        if op == "rotate":
            heads, kv = _heads(rng)
            dim = rng.choice([32, 64, 64, 128, 128, 96, 80, 2 * rng.randint(16, 64), rng.randint(33, 128)])
            case = {"op": op, "tokens": _log(rng, 1, 65536), "heads": heads, "kv": kv, "dim": dim,
                    "rotary": dim // 2 * 2 if rng.random() < 0.7 else 2 * rng.randint(1, dim // 2), "dtype": rng.choice(["f32", "bf16", "f16"]),
                    "interleaved": rng.random() < 0.3, "packed": rng.random() < 0.6, "first": rng.choice([0, 0, 31, _log(rng, 1, 4000000)]),
                    "train": rng.random() < 0.7}
            case["wdtype"] = rng.choice(["f32", case["dtype"]])
        elif op == "attend":
            heads, kv = _heads(rng)
            shortest = _log(rng, 1, 4096)
            case = {"op": op, "sequences": _log(rng, 1, 200), "shortest": shortest, "longest": _log(rng, shortest, 16384),
                    "lengths": rng.randrange(1 << 30), "tail": rng.choice([0, 0, 0, 5, 300]), "heads": heads, "kv": kv,
                    "dim": rng.choice([64, 64, 128, 128, 128, 32, 96, 80, rng.randint(33, 128)]), "dtype": rng.choice(["bf16", "bf16", "f16"]),
                    "packed": rng.random() < 0.5, "train": rng.random() < 0.7}
        else:
            case = {"op": op, "layers": _log(rng, 1, 24), "width": _log(rng, 64, 2048), "vocab": _log(rng, 100, 130000),
                    "dtype": rng.choice(["f32", "bf16", "f16"]), "limit": rng.choice([0.1, 0.5, 2.0]), "clip": rng.random() < 0.7}
        if _cost(case) <= _most(op):
            return case


def _lengths(case):
    rng = random.Random(case["lengths"])
    return [_log(rng, case["shortest"], case["longest"]) for _ in range(case["sequences"])]


def _shapes(case):
    """(shape, is a vector of 32 bits) of every parameter of the model."""
    d = case["width"]
    out = [((case["vocab"], d), False)]
    for _ in range(case["layers"]):
        out += [((d, d), False), ((d // 4, d), False), ((d // 4, d), False), ((d, d), False), ((4 * d, d), False), ((d, 4 * d), False)]
        out += [((d,), True), ((d,), True), ((d,), True), ((64,), True), ((64,), True)]
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    def split(parts, packed):
        """Tensors [tokens][heads][dim], as they come from one product (slices of a row) or each by itself."""
        if not packed:
            return [p.to(dt) for p in parts]
        row = torch.cat([p.to(dt) for p in parts], 1)
        return list(row.split([p.shape[1] for p in parts], 1))

    s = {"case": dict(case)}
    if case["op"] == "rotate":
        n, h, kv, d, wt = case["tokens"], case["heads"], case["kv"], case["dim"], DTYPES[case["wdtype"]]
        # projections of a residual stream: every head with a scale of its own, a few large columns
        x = randn(n, h + kv, d) * (0.3 + 2 * rand(1, h + kv, 1))
        x[:, :, ::29] *= 5
        s["q"], s["k"] = split([x[:, :h], x[:, h:]], case["packed"])
        s["qw"], s["kw"] = (1 + 0.2 * randn(d)).to(wt), (1 + 0.2 * randn(d)).to(wt)
        s["positions"] = case["first"] + torch.arange(n, device="cuda")
        r = case["rotary"]
        s["frequencies"] = ROTARY_BASE ** (torch.arange(r // 2, device="cuda", dtype=torch.float64) * (-2.0 / r))
        if case["train"]:
            s["dq"], s["dk"] = (randn(n, h, d) * 0.02).to(dt), (randn(n, kv, d) * 0.02).to(dt)
    elif case["op"] == "attend":
        lengths = _lengths(case)
        n, h, kv, d = sum(lengths) + case["tail"], case["heads"], case["kv"], case["dim"]
        ends = torch.tensor([0] + lengths).cumsum(0)
        # normed queries and keys; a share of each key is common to all tokens, so that some are looked at by many
        q = randn(n, h, d) + randn(1, h, d)
        k = randn(n, kv, d) + rand(n, kv, 1) * randn(1, kv, d)
        v = randn(n, kv, d)
        for t in (q, k, v):
            t[n - case["tail"]:] = float("nan")  # whatever was in the buffer
        s["q"], s["k"], s["v"] = split([q, k, v], case["packed"])
        s["offsets"] = ends.cuda()
        s["lengths"] = lengths
        if case["train"]:
            # fp16 training scales its loss
            s["dout"] = (randn(n, h, d) * (1e-2 if case["dtype"] == "f16" else 1e-5)).to(dt)
    else:
        count = sum(math.prod(shape) for shape, _ in _shapes(case))
        scale = 1 / math.sqrt(count)
        s["gradients"] = [(randn(*shape) * (scale * 10 ** (i % 5 / 4 - 0.5))).to(torch.float32 if vector else dt)
                          for i, (shape, vector) in enumerate(_shapes(case))]
        s["limit"] = case["limit"]
        if case["clip"]:
            # the clipped gradients go into two flat buffers, as an optimiser keeps them: the matrices' and the vectors'
            s["flat"] = [torch.empty(sum(t.numel() for t, (_, v) in zip(s["gradients"], _shapes(case)) if v == vector), device="cuda",
                                     dtype=torch.float32 if vector else dt) for vector in (False, True)]
            s["out"], at = [], [0, 0]
            for t, (shape, vector) in zip(s["gradients"], _shapes(case)):
                s["out"].append(s["flat"][vector][at[vector]:at[vector] + t.numel()].view(shape))
                at[vector] += t.numel()
    return s


def _angles(s):
    a = s["positions"].double()[:, None] * s["frequencies"]
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _turn(x, cos, sin, interleaved):
    """x [tokens][heads][dim] with its first values turned by the angles."""
    half = cos.shape[-1]
    out = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        out[..., :half], out[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    return out


def _rotate_plain(s):
    cos, sin = _angles(s)
    turned = s["case"]["interleaved"]
    out = {}
    for name in ("q", "k"):
        x, w = s[name].float(), s[name + "w"].float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + NORM_EPS)
        xr = x * r
        out[name] = _turn(xr * w, cos, sin, turned).to(s[name].dtype)
        if s["case"]["train"]:
            g = _turn(s["d" + name].float(), cos, -sin, turned)
            gw = g * w
            out["d" + name] = (r * (gw - xr * (gw * xr).mean(-1, keepdim=True))).to(s[name].dtype)
            out["d" + name + "w"] = (g * xr).sum((0, 1)).to(s[name + "w"].dtype)
    return out


def _blocks(s):
    """(first token of the sequence, first and last + 1 row of a block of its queries)"""
    at = 0
    for length in s["lengths"]:
        step = max(1, (1 << 28) // (s["case"]["heads"] * length))
        for r in range(0, length, step):
            yield at, r, min(r + step, length)
        at += length


def _attend_plain(s):
    case = s["case"]
    h, kv, scale = case["heads"], case["kv"], 1 / math.sqrt(case["dim"])
    times = h // kv
    q, k, v = (s[x].float() for x in ("q", "k", "v"))
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[0], h, device=q.device)
    if case["train"]:
        do = s["dout"].float()
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for at, r0, r1 in _blocks(s):
        qb = q[at + r0:at + r1].transpose(0, 1)
        kb = k[at:at + r1].repeat_interleave(times, 1).transpose(0, 1)
        vb = v[at:at + r1].repeat_interleave(times, 1).transpose(0, 1)
        hidden = torch.arange(r1, device=q.device)[None, :] > torch.arange(r0, r1, device=q.device)[:, None]
        p = torch.bmm(qb, kb.transpose(1, 2)).mul_(scale).masked_fill_(hidden, float("-inf"))
        top = p.amax(2, keepdim=True)
        p = p.sub_(top).exp_()
        z = p.sum(2, keepdim=True)
        p = p.div_(z)
        o = torch.bmm(p, vb)
        out[at + r0:at + r1] = o.transpose(0, 1)
        lse[at + r0:at + r1] = (z.log() + top)[..., 0].t()
        if case["train"]:
            dob = do[at + r0:at + r1].transpose(0, 1)
            dv[at:at + r1] += torch.bmm(p.transpose(1, 2), dob).view(kv, times, r1, -1).sum(1).transpose(0, 1)
            ds = p.mul_(torch.bmm(dob, vb.transpose(1, 2)).sub_((dob * o).sum(2, keepdim=True))).mul_(scale)
            dq[at + r0:at + r1] = torch.bmm(ds, kb).transpose(0, 1)
            dk[at:at + r1] += torch.bmm(ds.transpose(1, 2), qb).view(kv, times, r1, -1).sum(1).transpose(0, 1)
    res = {"out": out.to(s["q"].dtype), "lse": lse}
    if case["train"]:
        res["dq"], res["dk"], res["dv"] = (x.to(s["q"].dtype) for x in (dq, dk, dv))
    return res


def _clip_plain(s):
    total = sum(g.float().square().sum(dtype=torch.float64) for g in s["gradients"])
    norm = total.sqrt()
    res = {"norm": norm.float()}
    if s["case"]["clip"]:
        factor = (s["limit"] / (norm + CLIP_EPS)).clamp(max=1.0).float()
        for o, g in zip(s["out"], s["gradients"]):
            o.copy_(g.float() * factor)
        res["matrices"], res["vectors"] = s["flat"]
    return res


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return _rotate_plain(s) if op == "rotate" else _attend_plain(s) if op == "attend" else _clip_plain(s)
    from paper_2108_03645_b200 import train

    if op == "rotate":
        args = (s["q"], s["k"], s["positions"], s["frequencies"], s["qw"], s["kw"])
        out = dict(zip(("q", "k"), train.qk_norm(*args, eps=NORM_EPS, interleaved=case["interleaved"])))
        if case["train"]:
            grads = train.qk_norm_backward(s["dq"], s["dk"], *args, eps=NORM_EPS, interleaved=case["interleaved"])
            dq, dk, dqw, dkw = grads
            out.update(dq=dq, dqw=dqw, dk=dk, dkw=dkw)
            out = {k: out[k] for k in ("q", "dq", "dqw", "k", "dk", "dkw")}
        return out
    if op == "attend":
        out, lse = train.attention(s["q"], s["k"], s["v"], s["offsets"])
        res = {"out": out, "lse": lse}
        if case["train"]:
            res["dq"], res["dk"], res["dv"] = train.attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, s["offsets"])
        return res
    if not case["clip"]:
        return {"norm": train.gradient_norm(s["gradients"])}
    norm = train.clip_gradients(s["gradients"], s["limit"], out=s["out"], eps=CLIP_EPS)
    return {"norm": norm, "matrices": s["flat"][0], "vectors": s["flat"][1]}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotate":
        n, h, d = case["tokens"], case["heads"] + case["kv"], case["dim"]
        # forward: x in, y out; backward: dy in, dx out (x is read once for both)
        return {"bytes": (4 if case["train"] else 2) * n * h * d * size + 8 * n + 4 * case["rotary"],
                "flops": (24 if case["train"] else 9) * n * h * d}
    if case["op"] == "attend":
        lengths = _lengths(case)
        n, h, kv, d = sum(lengths) + case["tail"], case["heads"], case["kv"], case["dim"]
        pairs = sum(x * (x + 1) // 2 for x in lengths)
        # q, k, v in, out and lse out; dout in, three gradients out; two products forward, five backward
        times = 2 if case["train"] else 1
        return {"bytes": times * 2 * n * (h + kv) * d * size + 4 * n * h + 8 * len(lengths), "flops": (14 if case["train"] else 4) * h * d * pairs}
    count = sum(math.prod(shape) * (4 if vector else size) for shape, vector in _shapes(case))
    return {"bytes": count * (2 if case["clip"] else 1), "flops": count // size * (3 if case["clip"] else 2)}


def _rotate_exact(s):
    # a pair of values as a complex number, turned by a unit one; gradients from a graph
    angle = s["positions"].double()[:, None] * s["frequencies"]
    unit = torch.polar(torch.ones_like(angle), angle)[:, None]
    half, out = angle.shape[1], {}
    for name in ("q", "k"):
        x, w = (t.double().detach().requires_grad_() for t in (s[name], s[name + "w"]))
        y = w * x / (torch.linalg.vector_norm(x, dim=-1, keepdim=True).square() / x.shape[-1] + NORM_EPS).sqrt()
        front, rest = y[..., :2 * half], y[..., 2 * half:]
        pairs = front.unflatten(-1, (half, 2)) if s["case"]["interleaved"] else front.unflatten(-1, (2, half)).transpose(-1, -2)
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit)
        turned = turned if s["case"]["interleaved"] else turned.transpose(-1, -2)
        y = torch.cat([turned.flatten(-2), rest], -1)
        out[name] = y.detach()
        if s["case"]["train"]:
            out["d" + name], out["d" + name + "w"] = torch.autograd.grad(y, (x, w), s["d" + name].double())
    return out


def _attend_exact(s):
    case, names = s["case"], ("q", "k", "v")
    h, kv, d = case["heads"], case["kv"], case["dim"]
    x = [s[name].double() for name in names]
    out, lse = torch.zeros_like(x[0]), torch.zeros(x[0].shape[0], h, dtype=torch.float64, device="cuda")
    grads = [torch.zeros_like(t) for t in x]
    at = 0
    for length in s["lengths"]:
        rows = slice(at, at + length)
        at += length
        allowed = torch.ones(length, length, dtype=torch.bool, device="cuda").tril()
        for head in range(h):  # one head of one sequence as one graph
            part = [x[0][rows, head], x[1][rows, head // (h // kv)], x[2][rows, head // (h // kv)]]
            part = [t.detach().requires_grad_(case["train"]) for t in part]
            score = torch.where(allowed, part[0] @ part[1].T / d ** 0.5, -torch.inf)
            o = torch.softmax(score, 1) @ part[2]
            out[rows, head], lse[rows, head] = o.detach(), torch.logsumexp(score.detach(), 1)
            if case["train"]:
                for i, t in enumerate(torch.autograd.grad(o, part, s["dout"][rows, head].double())):
                    grads[i][rows, head if i == 0 else head // (h // kv)] += t
    res = {"out": out, "lse": lse}
    if case["train"]:
        res["dq"], res["dk"], res["dv"] = grads
    return res


def _clip_exact(s):
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double()) for g in s["gradients"]]))
    res = {"norm": norm}
    if s["case"]["clip"]:
        factor = min(1.0, s["limit"] / (float(norm) + CLIP_EPS))
        for name, vector in (("matrices", False), ("vectors", True)):
            res[name] = torch.cat([g.double().flatten() * factor for g, (_, v) in zip(s["gradients"], _shapes(s["case"])) if v == vector])
    return res


def exact(case, seed):
    w = work(case)
    if w["flops"] > 2e13 or (case["op"] == "attend" and case["sequences"] * case["heads"] > 8000):  # more than about 20 seconds in 64 bits
        return None
    s = prepare(case, seed)
    return _rotate_exact(s) if case["op"] == "rotate" else _attend_exact(s) if case["op"] == "attend" else _clip_exact(s)
