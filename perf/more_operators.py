"""Timed cases of the operators around a layer of experts and of 8-bit activation checkpoints, through the Python API.

A case names an `op`, its sizes and its types:

* ``route``: T tokens' logits over E experts to the k experts of each, their weights and the slots' order by expert;
  `score` "softmax" or "sigmoid", `bias` for balance, the best `top_groups` of `groups`, weights renormalised or not,
  `padded` tokens at the end that are not routed; `grad`: the logits' gradient of the weights' instead;
* ``checkpoint``: T rows of n activations to 8 bits with a scale for each `group` of columns, and back;
* ``linear_grad_q8``: gradient of a linear layer whose input and pre-activations were kept in 8 bits;
* ``expert_linear``: act(x W_e^T + b_e) of every slot of a routed batch, E experts with n inputs and m outputs; from
  the tokens' rows, or (`combine`) from the slots' rows with the outputs weighted and summed for each token;
* ``expert_grad``: its gradient (inputs, weights, biases, the pre-activation gradients that the tokens of an estimate
  hold, with `combine` the routing weights' too); `q8`: input and pre-activations were kept in 8 bits.

The listed cases run from one token to prompts and training batches; `draw` gives others of the same ranges, odd sizes
among them.  With `own` false, `run` computes the plain form: scores in 64 bits (an expert's rank may hang on the last
bit), everything else in 32, rounded once at the end.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 128   # columns that share a scale in the checkpoints of layers


def listed():
    return [
        # serving: one token's way to 8 of 128 experts
        dict(name="route_1x128", op="route", T=1, E=128, k=8, dtype="bf16", score="softmax", bias=False, groups=1,
             top_groups=1, renorm=True, padded=False, grad=False),
        # training: a batch with padding over many experts in groups, balanced by a bias
        dict(name="route_16384x256", op="route", T=16384, E=256, k=8, dtype="f32", score="sigmoid", bias=True, groups=8,
             top_groups=4, renorm=True, padded=True, grad=False),
        # training: the router's gradient over a number of experts that nothing divides
        dict(name="route_grad_8191x61", op="route", T=8191, E=61, k=4, dtype="f32", score="softmax", bias=True, groups=1,
             top_groups=1, renorm=False, padded=False, grad=True),
        # training: what a small fp32 layer keeps, at a width that no group divides
        dict(name="checkpoint_777x1001_f32", op="checkpoint", T=777, n=1001, group=64, dtype="f32"),
        # training: what a layer of the widest model keeps of a batch
        dict(name="checkpoint_8192x8192", op="checkpoint", T=8192, n=8192, group=128, dtype="bf16"),
        # training: the gradient of a small layer at odd widths
        dict(name="linear_grad_q8_1021x1000x777", op="linear_grad_q8", T=1021, n=1000, m=777, act="silu", bias=True),
        # training: the gradient of an MLP up projection
        dict(name="linear_grad_q8_4096x4096x11008", op="linear_grad_q8", T=4096, n=4096, m=11008, act="gelu", bias=True),
        # serving: one token through the up projections of its experts
        dict(name="expert_linear_1x4096x2048", op="expert_linear", T=1, E=64, k=8, n=4096, m=2048, act="silu", bias=False,
             combine=False, padded=False),
        # serving: 37 sequences' tokens through odd down projections, summed
        dict(name="expert_linear_37x1000x777", op="expert_linear", T=37, E=12, k=3, n=1000, m=777, act="none", bias=True,
             combine=True, padded=True),
        # serving: a prompt through the up projections
        dict(name="expert_linear_4096x4096x2048", op="expert_linear", T=4096, E=64, k=4, n=4096, m=2048, act="gelu",
             bias=True, combine=False, padded=False),
        # training: the gradient of down projections of a few experts at odd widths, the routing's with it
        dict(name="expert_grad_1021x500x333", op="expert_grad", T=1021, E=7, k=2, n=500, m=333, act="none", bias=True,
             combine=True, q8=False, padded=True),
        # training: the gradient of the up projections, their activations kept in 8 bits
        dict(name="expert_grad_4096x4096x2048", op="expert_grad", T=4096, E=64, k=4, n=4096, m=2048, act="gelu", bias=True,
             combine=False, q8=True, padded=False),
    ]


def _size(rng, lo, hi):
    """Log-uniform in [lo, hi]; every other one a multiple of 64 (where that is not 0)."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 64:
        v = v // 64 * 64
    return v


def draw(rng):
    op = rng.choice(["route", "route", "checkpoint", "linear_grad_q8", "expert_linear", "expert_linear", "expert_grad", "expert_grad"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * _size(rng, max(4, 8 // groups), 256 // groups)
        top = rng.randint(1, groups)
        return dict(op=op, T=_size(rng, 1, 16384), E=E, k=rng.randint(1, min(8, top * (E // groups))),
                    dtype=rng.choice(["bf16", "f32"]), score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                    groups=groups, top_groups=top, renorm=rng.random() < 0.7, padded=rng.random() < 0.3,
                    grad=rng.random() < 0.4)
    if op == "checkpoint":
        n = _size(rng, 64, 16384)
        return dict(op=op, T=_size(rng, 1, min(16384, (1 << 26) // n)), n=n, group=rng.choice([32, 64, 128, 256]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    act, bias = rng.choice(["none", "relu", "gelu", "silu"]), rng.random() < 0.5
    if op == "linear_grad_q8":
        n, m = _size(rng, 128, 11008), _size(rng, 128, 11008)
        T = max(1, min(_size(rng, 16, 4096), (1 << 36) // (n * m)))
        return dict(op=op, T=T, n=n, m=m, act=act, bias=bias)
    n, m, E = _size(rng, 128, 4096), _size(rng, 128, 4096), _size(rng, 4, 128)
    E = max(4, min(E, (1 << 29) // (n * m)))
    k = rng.randint(1, min(8, E))
    T = max(1, min(_size(rng, 1, 4096), (1 << 36) // (n * m * k)))
    c = dict(op=op, T=T, E=E, k=k, n=n, m=m, act=act, bias=bias, combine=rng.random() < 0.4, padded=rng.random() < 0.3)
    if op == "expert_grad":
        c["q8"] = rng.random() < 0.5
    return c


# ------------------------------------------------------------------ inputs
def _to_q8(x, group):
    """Codes and scales of rows: what a program that kept them in 8 bits has in hand."""
    T, n = x.shape
    cols = (n + group - 1) // group
    f = torch.nn.functional.pad(x.double(), (0, cols * group - n)).view(T, cols, group)
    big = f.abs().amax(dim=2, keepdim=True)
    q = torch.round(127 * f / big).view(T, cols * group)[:, :n].to(torch.int8).contiguous()
    return q, (big[:, :, 0].float() / 127).contiguous()


def _routed(T, E, k, valid, randn):
    """A routing of T tokens, `valid` of them: weights, experts, slots by expert, where each expert's start, their places."""
    logits = randn(T, E, dtype=torch.float32) + 0.7 * randn(E, dtype=torch.float32)   # some experts are liked more
    p = torch.softmax(logits, dim=1)
    w, e = torch.topk(p, k, dim=1)
    w = w / w.sum(dim=1, keepdim=True)
    w[valid:], e[valid:] = 0, -1
    flat = e.reshape(-1)
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=DEV)
    place = torch.where(flat < 0, -1, place).view(T, k)
    order = torch.where(torch.arange(T * k, device=DEV) < valid * k, order, -1)
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    offsets[1:] = torch.cumsum((key[:, None] == torch.arange(E, device=DEV)).sum(dim=0), dim=0)
    return dict(weights=w, experts=e.int(), order=order.int(), offsets=offsets.int(), place=place.int())


def _valid(case):
    return max(1, case["T"] - case["T"] // 8) if case["padded"] else case["T"]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 29)

    def randn(*shape, dtype=torch.bfloat16, scale=1.0, shift=0.0):
        return torch.randn(shape, device=DEV, generator=g).mul_(scale).add_(shift).to(dtype)

    op, s = case["op"], dict(case)
    if op == "route":
        T, E = case["T"], case["E"]
        s["logits"] = (1.5 * randn(T, E, dtype=torch.float32) + 0.7 * randn(E, dtype=torch.float32)).to(TYPES[case["dtype"]])
        s["b"] = randn(E, dtype=torch.float32, scale=0.05) if case["bias"] else None
        s["mask"] = torch.arange(T, device=DEV) < _valid(case) if case["padded"] else None
        if case["grad"]:   # of experts that the forward pass chose
            s["experts"] = _choose(s["logits"], s)[1].int()
            s["dw"] = randn(T, case["k"], dtype=torch.float32)
        return s
    if op == "checkpoint":
        # activations with a few large channels, as residual streams have
        loud = torch.exp(0.7 * torch.randn(case["n"], device=DEV, generator=g))
        s["x"] = (torch.randn((case["T"], case["n"]), device=DEV, generator=g) * loud).to(TYPES[case["dtype"]])
        return s
    T, n, m = case["T"], case["n"], case["m"]
    rows, lead = T, ()
    if op != "linear_grad_q8":
        valid = _valid(case)
        s["r"] = _routed(T, case["E"], case["k"], valid, randn)
        rows, lead = T * case["k"], (case["E"],)
    s["W"] = randn(*lead, m, n, scale=1 / math.sqrt(n))
    s["b"] = randn(*lead, m, scale=0.1) if case["bias"] else None
    x = randn(rows if case.get("combine") else T, n)
    if op == "expert_linear":
        s["x"] = x
        return s
    z = randn(rows, m) if case["act"] != "none" else None
    if case.get("combine"):
        s["dout"], s["y"] = randn(T, m), randn(rows, m)
        s["y"][valid * case["k"]:] = 0
    else:
        s["dy"] = randn(rows, m)
    if op == "linear_grad_q8" or case["q8"]:
        s["x"], s["z"] = _to_q8(x, GROUP), None if z is None else _to_q8(z, GROUP)
    else:
        s["x"], s["z"] = x, z
    return s


# ------------------------------------------------------------- plain forms
def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":   # the tanh form: z sigmoid(2 c (z + 0.044715 z^3)), c = sqrt(2 / pi)
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    k = 2 * math.sqrt(2 / math.pi)
    p = 1 / (1 + torch.exp(-k * (z + 0.044715 * z * z * z)))
    return p + z * p * (1 - p) * k * (1 + 3 * 0.044715 * z * z)


def _scores(logits, score):
    v = logits.double()
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-v))
    e = torch.exp(v - v.amax(dim=1, keepdim=True))
    return e / e.sum(dim=1, keepdim=True)


def _best(c, count):
    """The `count` largest of each row in their order, the lowest index first among equals: one after the other."""
    c, picks = c.clone(), []
    for _ in range(count):
        picks.append(torch.argmax(c, dim=1, keepdim=True))
        c.scatter_(1, picks[-1], -math.inf)
    return torch.cat(picks, dim=1)


def _choose(logits, s):
    score, k, groups = _scores(logits, s["score"]), s["k"], s["groups"]
    c = score if s["b"] is None else score + s["b"].double()
    if groups > 1:
        size = s["E"] // groups
        of = torch.arange(s["E"], device=DEV) // size
        parts = c.view(-1, groups, size)
        rank = parts.amax(dim=2)
        if size > 1:   # the two best of a group speak for it
            first = torch.argmax(parts, dim=2, keepdim=True)
            rank = rank + parts.scatter(2, first, -math.inf).amax(dim=2)
        kept = (_best(rank, s["top_groups"])[:, :, None] == of).any(dim=1)
        c = torch.where(kept, c, -math.inf)
    e = _best(c, k)
    w = torch.gather(score, 1, e)
    if s["renorm"]:
        w = w / w.sum(dim=1, keepdim=True)
    if s["mask"] is not None:
        w, e = torch.where(s["mask"][:, None], w, 0), torch.where(s["mask"][:, None], e, -1)
    return w, e


def _plain_route(s):
    T, E, k = s["T"], s["E"], s["k"]
    if s["grad"]:
        p = _scores(s["logits"], s["score"])
        e = s["experts"].long()
        live = e >= 0
        e = torch.clamp(e, min=0)
        w, dw = torch.where(live, torch.gather(p, 1, e), 0), torch.where(live, s["dw"].double(), 0)
        if s["renorm"]:
            total = torch.where(live[:, :1], w.sum(dim=1, keepdim=True), 1)
            dw = (dw - (dw * w).sum(dim=1, keepdim=True) / total) / total
        dp = torch.zeros_like(p).scatter_add_(1, e, torch.where(live, dw, 0))
        if s["score"] == "sigmoid":
            out = dp * p * (1 - p)
        else:
            out = p * (dp - (p * dp).sum(dim=1, keepdim=True))
        return out.to(s["logits"].dtype)
    w, e = _choose(s["logits"], s)
    flat = e.reshape(-1)
    key = torch.where(flat < 0, E, flat)
    order = torch.argsort(key, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=DEV)
    offsets = (key[:, None] <= torch.arange(-1, E, device=DEV)).sum(dim=0)
    order = torch.where(torch.arange(T * k, device=DEV) < offsets[-1], order, -1)
    return w.float(), e.int(), order.int(), offsets.int(), torch.where(flat < 0, -1, place).view(T, k).int()


def _plain_from_q8(kept, group):
    q, scale = kept
    return q.float() * torch.repeat_interleave(scale, group, dim=1)[:, :q.shape[1]]


def _plain_rows(v):
    if v is None:
        return None
    return _plain_from_q8(v, GROUP) if isinstance(v, tuple) else v.float()


def _plain_expert_linear(s):
    r, k = s["r"], s["k"]
    P, ends = s["T"] * k, s["r"]["offsets"].tolist()
    y = torch.zeros((P, s["m"]), device=DEV)
    tokens = torch.div(r["order"].long(), k, rounding_mode="floor")
    for e in range(s["E"]):
        a, b = ends[e], ends[e + 1]
        if a == b:
            continue
        z = (s["x"][a:b] if s["combine"] else s["x"][tokens[a:b]]).float() @ s["W"][e].float().T
        y[a:b] = _act(z if s["b"] is None else z + s["b"][e].float(), s["act"])
    if not s["combine"]:
        return y.to(torch.bfloat16)
    live = r["place"] >= 0
    rows = y[torch.clamp(r["place"].long(), min=0)]
    return (torch.where(live, r["weights"], 0)[:, :, None] * rows).sum(dim=1).to(torch.bfloat16)


def _plain_expert_grad(s):
    r, T, k, n, m = s["r"], s["T"], s["k"], s["n"], s["m"]
    bf16, P, ends = torch.bfloat16, s["T"] * s["k"], s["r"]["offsets"].tolist()
    count = ends[-1]
    slots = torch.clamp(r["order"].long(), min=0)
    tokens = torch.div(slots, k, rounding_mode="floor")
    live = (torch.arange(P, device=DEV) < count)[:, None]
    x = _plain_rows(s["x"])
    dweights = None
    if s["combine"]:
        d = s["dout"].float()[tokens]
        g = d * r["weights"].reshape(-1)[slots][:, None]
        dots = (d * s["y"].float()).sum(dim=1)
        dweights = torch.where(r["place"] >= 0, dots[torch.clamp(r["place"].long(), min=0)], 0)
    else:
        g = s["dy"].float()
        x = x[tokens]
    if s["z"] is not None:
        g = g * _act_grad(_plain_rows(s["z"]), s["act"])
    g = torch.where(live, g, 0)
    dx, dw = torch.zeros((P, n), device=DEV), torch.zeros((s["E"], m, n), dtype=bf16, device=DEV)
    db = torch.zeros((s["E"], m), device=DEV)
    for e in range(s["E"]):
        a, b = ends[e], ends[e + 1]
        if a == b:
            continue
        dx[a:b] = g[a:b] @ s["W"][e].float()
        dw[e] = (g[a:b].T @ x[a:b]).to(bf16)
        db[e] = g[a:b].sum(dim=0)
    if not s["combine"]:
        rows = dx[torch.clamp(r["place"].long(), min=0)]
        dx = torch.where((r["place"] >= 0)[:, :, None], rows, 0).sum(dim=1)
    out = [dx.to(bf16), dw, g.to(bf16)]
    out += [db.to(bf16)] if s["b"] is not None else []
    return out + ([dweights] if s["combine"] else [])


def _plain(s):
    op = s["op"]
    if op == "route":
        return _plain_route(s)
    if op == "expert_linear":
        return _plain_expert_linear(s)
    if op == "expert_grad":
        return _plain_expert_grad(s)
    if op == "checkpoint":
        x, T, n, group = s["x"], s["T"], s["n"], s["group"]
        cols = (n + group - 1) // group
        f = torch.zeros((T, cols * group), dtype=torch.float64, device=DEV)   # codes hang on halves
        f[:, :n] = x
        f = f.view(T, cols, group)
        big = f.abs().amax(dim=2, keepdim=True)
        scale = big.float() / 127
        back = (torch.round(127 * f / big).float() * scale).view(T, -1)[:, :n]
        return back.to(x.dtype), scale[:, :, 0]
    x, W, g = _plain_rows(s["x"]), s["W"].float(), s["dy"].float()
    if s["z"] is not None:
        g = g * _act_grad(_plain_rows(s["z"]), s["act"])
    out = [(g @ W).to(torch.bfloat16), (g.T @ x).to(torch.bfloat16), g.to(torch.bfloat16)]
    return out + [g.sum(dim=0).to(torch.bfloat16)] if s["b"] is not None else out


# ------------------------------------------------------------------ a pass
def run(s):
    if not own:
        return _plain(s)
    import paper_2609_14706_amd as ffe
    op = s["op"]
    if op == "route":
        if s["grad"]:
            return ffe.route_backward(s["dw"], s["logits"], s["experts"], score=s["score"], renormalise=s["renorm"])
        return tuple(ffe.route(s["logits"], s["k"], score=s["score"], bias=s["b"], groups=s["groups"],
                               top_groups=s["top_groups"], renormalise=s["renorm"], mask=s["mask"]))
    if op == "checkpoint":
        kept = ffe.checkpoint_q8(s["x"], group=s["group"])
        return ffe.checkpoint_restore(kept, dtype=s["x"].dtype), kept.scale

    def rows(v):
        return ffe.Checkpoint(v[0], v[1], GROUP) if isinstance(v, tuple) else v

    if op == "linear_grad_q8":
        dx, dw, g, db = ffe.linear_backward(s["dy"], rows(s["x"]), s["W"], preact=rows(s["z"]), activation=s["act"],
                                            need_bias=s["b"] is not None)
        return [dx, dw, g] + ([db] if db is not None else [])
    r = ffe.Routing(**s["r"])
    if op == "expert_linear":
        y, _ = ffe.expert_linear(s["x"], s["W"], r, bias=s["b"], activation=s["act"], by_slot=s["combine"])
        return ffe.expert_combine(y, r) if s["combine"] else y
    dy, dweights = ffe.expert_combine_backward(s["dout"], s["y"], r) if s["combine"] else (s["dy"], None)
    dx, dw, g, db = ffe.expert_linear_backward(dy, rows(s["x"]), s["W"], r, preact=rows(s["z"]), activation=s["act"],
                                               by_slot=s["combine"], need_bias=s["b"] is not None)
    return [dx, dw, g] + ([db] if db is not None else []) + ([dweights] if dweights is not None else [])


def work(case):
    op, T = case["op"], case["T"]
    if op == "route":
        E, k, e = case["E"], case["k"], 4 if case["dtype"] == "f32" else 2
        if case["grad"]:   # logits, weights' gradient, experts in, logits' gradient out
            return {"bytes": 2 * T * E * e + 8 * T * k, "flops": 8 * T * E}
        # logits, bias, mask in; weights, experts, order, places, offsets out
        more = (4 * E if case["bias"] else 0) + (T if case["padded"] else 0)
        return {"bytes": T * E * e + 16 * T * k + 4 * (E + 1) + more, "flops": (4 + k) * T * E}
    if op == "checkpoint":   # rows in, codes and scales out; in again, rows out
        n, e = case["n"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * T * (n * (e + 1) + 4 * ((n + case["group"] - 1) // case["group"])), "flops": 4 * T * n}
    n, m = case["n"], case["m"]

    def kept(rows, cols):   # a checkpoint
        return rows * (cols + 4 * ((cols + GROUP - 1) // GROUP))

    acts = case["act"] != "none"
    if op == "linear_grad_q8":   # x, W, dy, z in; dx, dW, g, db out
        b = 2 * m if case["bias"] else 0
        return {"bytes": kept(T, n) + (kept(T, m) if acts else 0) + 2 * (2 * m * n + 2 * T * m + T * n) + b,
                "flops": 4 * T * m * n}
    E, k, valid = case["E"], case["k"], _valid(case)
    P, used = valid * k, min(E, valid * k)
    xin = P if case["combine"] else valid
    if op == "expert_linear":
        b = 2 * used * m if case["bias"] else 0
        out = T if case["combine"] else T * k
        return {"bytes": 2 * (used * m * n + xin * n + out * m) + b + 4 * (T * k + E + 1), "flops": 2 * P * m * n}
    b = 2 * E * m if case["bias"] else 0
    moved = 2 * (used * m * n + E * m * n) + 4 * (2 * T * k + E + 1) + b
    moved += kept(xin, n) if case["q8"] else 2 * xin * n
    moved += (kept(P, m) if case["q8"] else 2 * P * m) if acts else 0
    moved += 2 * (T * k if case["combine"] else T) * n + 2 * T * k * m                 # dx, g
    moved += 2 * (valid * m + P * m) + 8 * T * k if case["combine"] else 2 * P * m     # dout, y, weights and theirs; dy
    return {"bytes": moved, "flops": 4 * P * m * n}


# ------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "route":
        return _exact_route(s)
    if op == "checkpoint":
        x, cols = s["x"].double(), []
        scales = []
        for part in torch.split(x, s["group"], dim=1):
            big = part.abs().max(dim=1, keepdim=True).values
            step = big / 127
            cols.append((part * 127 / big).round() * step)
            scales.append(step)
        return torch.cat(cols, dim=1), torch.cat(scales, dim=1)
    f = {key: v.double() if isinstance(v, torch.Tensor) else v for key, v in s.items()}
    for key in ("x", "z"):
        if isinstance(f.get(key), tuple):
            q, scale = f[key]
            f[key] = torch.cat([c * scale[:, j:j + 1].double() for j, c in enumerate(torch.split(q.double(), GROUP, dim=1))], dim=1)
    if op == "linear_grad_q8":
        g = f["dy"] if f["z"] is None else f["dy"] * _exact_slope(f["z"], s["act"])
        out = [torch.matmul(g, f["W"]), torch.matmul(f["x"].T, g).T, g]
        return out + [g.sum(0)] if s["b"] is not None else out
    T, E, k, n, m = s["T"], s["E"], s["k"], s["n"], s["m"]
    experts, place = s["r"]["experts"].long(), s["r"]["place"].long()
    w = s["r"]["weights"].double()
    f64 = dict(dtype=torch.float64, device=DEV)
    if op == "expert_linear":
        y = torch.zeros((T * k, m), **f64)
        for e in range(E):
            t, j = torch.nonzero(experts == e, as_tuple=True)
            p = place[t, j]
            z = torch.matmul(f["W"][e], f["x"][p if s["combine"] else t].T).T
            if s["b"] is not None:
                z = z + f["b"][e]
            if s["act"] == "relu":
                z = torch.where(z > 0, z, torch.zeros_like(z))
            elif s["act"] == "silu":
                z = z * torch.sigmoid(z)
            elif s["act"] == "gelu":
                z = 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
            y[p] = z
        if not s["combine"]:
            return y
        out = torch.zeros((T, m), **f64)
        for j in range(k):
            t = torch.nonzero(experts[:, j] >= 0)[:, 0]
            out[t] += w[t, j, None] * y[place[t, j]]
        return out
    dx = torch.zeros((T * k if s["combine"] else T, n), **f64)
    dw, db, g = torch.zeros((E, m, n), **f64), torch.zeros((E, m), **f64), torch.zeros((T * k, m), **f64)
    dweights = torch.zeros((T, k), **f64)
    for e in range(E):
        t, j = torch.nonzero(experts == e, as_tuple=True)
        p = place[t, j]
        if s["combine"]:
            dweights[t, j] = torch.einsum("tm,tm->t", f["dout"][t], f["y"][p])
            ge, xe = f["dout"][t] * w[t, j, None], f["x"][p]
        else:
            ge, xe = f["dy"][p], f["x"][t]
        if f["z"] is not None:
            ge = ge * _exact_slope(f["z"][p], s["act"])
        dxe = torch.matmul(f["W"][e].T, ge.T).T
        if s["combine"]:
            dx[p] = dxe
        else:
            dx.index_add_(0, t, dxe)
        dw[e], db[e], g[p] = torch.matmul(xe.T, ge).T, ge.sum(0), ge
    out = [dx, dw, g] + ([db] if s["b"] is not None else [])
    return out + ([dweights] if s["combine"] else [])


def _exact_route(s):
    v, E, k, T = s["logits"].double(), s["E"], s["k"], s["T"]
    p = torch.sigmoid(v) if s["score"] == "sigmoid" else torch.softmax(v, dim=1)
    if s["grad"]:
        out = torch.zeros_like(v)
        e = s["experts"].long()
        t = torch.nonzero(e[:, 0] >= 0)[:, 0]
        e, p, dw = e[t], p[t], s["dw"].double()[t]
        rows, chosen = torch.arange(len(t), device=DEV)[:, None], torch.gather(p, 1, e)
        # how each weight hangs on each score, then each score on each logit
        if s["renorm"]:
            total = chosen.sum(1, keepdim=True)
            dchosen = dw / total - (dw * chosen).sum(1, keepdim=True) / total ** 2
        else:
            dchosen = dw
        if s["score"] == "sigmoid":
            d = torch.zeros_like(p)
            d[rows, e] = dchosen * chosen * torch.sigmoid(-torch.gather(v[t], 1, e))
        else:
            d = -p * (dchosen * chosen).sum(1, keepdim=True)
            d[rows, e] += dchosen * chosen
        out[t] = d
        return out
    c = p if s["b"] is None else p + s["b"].double()
    if s["groups"] > 1:
        parts = c.view(T, s["groups"], -1)
        rank = torch.topk(parts, min(2, parts.shape[2]), dim=2).values.sum(2)
        last = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, s["top_groups"]:]
        c = parts.scatter(1, last[:, :, None].expand(-1, -1, parts.shape[2]), -math.inf).reshape(T, E)
    e = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k]
    w = p.gather(1, e)
    w = w / w.sum(1, keepdim=True) if s["renorm"] else w
    live = torch.ones(T, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"]
    w, e = w * live[:, None], torch.where(live[:, None], e, -1)
    order, place, offsets = [], torch.full((T * k,), -1, device=DEV), [0]
    flat, slots = e.reshape(-1), torch.arange(T * k, device=DEV)
    for x in range(E):
        mine = slots[flat == x]
        place[mine] = torch.arange(len(mine), device=DEV) + offsets[-1]
        order.append(mine)
        offsets.append(offsets[-1] + len(mine))
    order.append(torch.full((T * k - offsets[-1],), -1, device=DEV))
    return w, e.int(), torch.cat(order).int(), torch.tensor(offsets, device=DEV).int(), place.view(T, k).int()


def _exact_slope(z, act):
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if act == "silu":
        e = torch.exp(-z)
        return 1 / (1 + e) + z * e / (1 + e).square()
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t.square()) * c * (1 + 3 * 0.044715 * z.square())
