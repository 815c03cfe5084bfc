"""Cases of the operators around an expert sublayer: what is timed, on which inputs, and what the answer has to be.

They are what N workers' tokens pass on their way through such a sublayer and back: a root-mean-square norm of the
residual sum, the router's choice of experts, the tokens' way into the order of their (worker, expert) groups and back,
and the (gated) activation between the experts' two products, whose input is kept in 8 bits for the backward pass.

8-bit rows: blocks of 32 columns share a power of two, the smallest 2^e, e in [-127, 127], with which no finite value of
the block passes 448 * 2^e; an element is its value over 2^e rounded to e4m3.  The two halves of a gated activation's input
are blocked each on its own.

Routing: scores s = softmax or sigmoid of the logits; experts are chosen by c = s + bias: first the groups_kept groups with
the largest sums of their group_top largest c, then the k largest c within them, in descending order; ties go to the
lower index.  The weights are the chosen s, over their sum if renormalised, times `scale`.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


# ---- cases -------------------------------------------------------------------------------------------------------
def _route(name, op, tokens, experts, k, dtype, scores, bias, groups, kept, top, renormalise, scale):
    return {"name": name, "op": op, "tokens": tokens, "experts": experts, "k": k, "dtype": dtype, "scores": scores, "bias": bias,
            "groups": groups, "kept": kept, "top": top, "renormalise": renormalise, "scale": scale}


def _move(name, op, tokens, workers, experts, k, cols, dtype, packed, skew):
    """packed: the tokens are 8-bit rows; skew: how unevenly they fall on the experts."""
    return {"name": name, "op": op, "tokens": tokens, "workers": workers, "experts": experts, "k": k, "cols": cols, "dtype": dtype,
            "packed": packed, "skew": skew}


def _activation(name, op, rows, cols, kind, gated, dtype):
    """cols: of the output; the input has twice as many if gated."""
    return {"name": name, "op": op, "rows": rows, "cols": cols, "kind": kind, "gated": gated, "dtype": dtype}


def _norm(name, op, rows, cols, dtype, stream, packed, workers):
    """stream: the type of the residual stream, or "" for a norm alone; packed: an output in 8 bits too."""
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "stream": stream, "packed": packed, "workers": workers}


def listed():
    return [
        # a short step of one worker: sixteen tokens, two of eight experts each, where the call itself is what counts
        _route("route 16", "route", 16, 8, 2, "bf16", "softmax", False, 1, 1, 1, True, 1.0),
        # a long step over many small experts: sigmoid scores, a bias that balances the load, groups
        _route("route 32768 groups", "route", 32768, 256, 8, "f32", "sigmoid", True, 8, 4, 2, True, 2.5),
        # the gradient to the logits where the weights are plain softmax scores, an odd number of tokens and experts
        _route("route gradient 5003", "route_grad", 5003, 60, 4, "bf16", "softmax", False, 1, 1, 1, False, 1.0),
        # two workers' tokens, kept as 8-bit rows by the norm, sorted again for the weight gradients of a backward pass
        _move("dispatch 1000 packed", "dispatch", 1000, 2, 6, 3, 1032, "bf16", True, 1.0),
        # eight workers' long step: sort by (worker, expert) and spread to four experts each
        _move("dispatch 16384", "dispatch", 16384, 8, 16, 4, 2048, "bf16", False, 0.3),
        # and the experts' outputs back to the tokens, weighted and added to the residual stream
        _move("combine 16384", "combine", 16384, 8, 16, 4, 2048, "bf16", False, 0.3),
        # the gradient of that, on an odd width (a pruned model)
        _move("combine gradient odd f16", "combine_grad", 5003, 2, 6, 2, 777, "f16", False, 1.0),
        # one training pass through a gated activation, its input kept in 8 bits: a short step ...
        _activation("activation 128", "activation", 128, 1024, "silu", True, "bf16"),
        # ... and a long one
        _activation("activation 32768", "activation", 32768, 2304, "silu", True, "bf16"),
        # the backward pass alone from the kept rows, for an ungated activation of an odd width
        _activation("activation gradient odd", "activation_grad", 6007, 2303, "gelu", False, "f16"),
        # eight workers' long batches, the residual stream in binary32, the output in bf16 and in 8 bits for the backward pass
        _norm("norm 32768 packed", "norm", 32768, 1024, "bf16", "f32", True, 8),
        # the gradient on wide rows, weight gradients by worker
        _norm("norm gradient 8192", "norm_grad", 8192, 4096, "bf16", "bf16", False, 8),
    ]


def _log(rng, lo, hi):
    """A whole number, its logarithm spread evenly over [lo, hi]; half of the time a multiple of 8."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and n >= 16:
        n = n // 8 * 8
    return min(hi, max(lo, n))


def draw(rng):
    op = rng.choice(["route", "route", "route_grad", "dispatch", "combine", "combine_grad", "activation", "activation", "activation_grad",
                     "norm", "norm", "norm_grad"])
    while True:
        if op in ("route", "route_grad"):
            groups = rng.choice([1, 1, 2, 4, 8])
            experts, k = groups * _log(rng, 2, 512 // groups), _log(rng, 1, 16)
            kept = rng.randint(1, groups)
            case = _route("", op, _log(rng, 1, 32768), experts, k, rng.choice(list(TYPES)), rng.choice(["softmax", "sigmoid"]),
                          rng.random() < 0.5, groups, kept, rng.choice([1, 2]), rng.random() < 0.5, rng.choice([1.0, 2.5]))
            ok = k <= kept * (experts // groups) and case["tokens"] * experts <= 32768 * 256 and case["tokens"] * k <= 32768 * 8
        elif op in ("dispatch", "combine", "combine_grad"):
            case = _move("", op, _log(rng, 1, 32768), _log(rng, 1, 8), _log(rng, 2, 64), _log(rng, 1, 8), _log(rng, 32, 8192),
                         rng.choice(list(TYPES)), op == "dispatch" and rng.random() < 0.5, round(rng.uniform(0.0, 1.5), 2))
            ok = case["k"] <= case["experts"] and case["tokens"] * case["k"] * case["cols"] <= (32 if case["dtype"] == "f32" else 64) << 20
        elif op in ("activation", "activation_grad"):
            case = _activation("", op, _log(rng, 1, 32768), _log(rng, 16, 16384), rng.choice(["silu", "gelu", "gelu_tanh"]),
                               rng.random() < 0.6, rng.choice(list(TYPES)))
            ok = case["rows"] * case["cols"] <= 1 << 25
        else:
            dtype = rng.choice(list(TYPES))
            case = _norm("", op, _log(rng, 1, 32768), _log(rng, 16, 8192), dtype, rng.choice(["", dtype, "f32"]),
                         op == "norm" and rng.random() < 0.5, _log(rng, 1, 16))
            ok = case["rows"] * case["cols"] <= 1 << 25
        if ok:
            del case["name"]
            return case


# ---- inputs ------------------------------------------------------------------------------------------------------
def _worker_offsets(tokens, workers, host):
    cuts = sorted(host.randint(0, tokens) for _ in range(workers - 1)) if host.random() < 0.3 else \
        [tokens * n // workers for n in range(1, workers)]
    return torch.tensor([0, *cuts, tokens], dtype=torch.int64, device="cuda")


def _pack(x, halves=1):
    """The 8-bit rows of a float tensor: (values e4m3 [rows, cols], scales e8m0 [rows, halves * blocks])."""
    rows, cols = x.shape[0], x.shape[1] // halves
    blocks = (cols + 31) // 32
    f = torch.zeros(rows, halves, blocks * 32, device="cuda")
    f[:, :, :cols] = x.float().view(rows, halves, cols)
    f = f.view(rows, halves, blocks, 32)
    mantissa, exponent = torch.frexp(f.abs().amax(-1))  # largest = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = torch.where(mantissa > 0.875, exponent - 8, exponent - 9).clamp(min=-127)
    e = torch.where(mantissa == 0, -127, e)
    inverse = ((127 - e) << 23).to(torch.int32).view(torch.float32)  # 2^-e by its bits
    q = (f * inverse.unsqueeze(-1)).to(torch.float8_e4m3fn)
    q = q.view(rows, halves, blocks * 32)[:, :, :cols].reshape(rows, halves * cols)
    return q, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu).view(rows, halves * blocks)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    host = random.Random(seed)
    s = dict(case)
    s["T"] = T = TYPES[case["dtype"]]
    op = case["op"]
    if op in ("route", "route_grad"):
        t, e, k = case["tokens"], case["experts"], case["k"]
        s["logits"] = (1.5 * normal(t, e) + 0.5 * normal(e)).to(T)  # some experts are liked better
        s["bias"] = 0.1 * normal(e) if case["bias"] else None
        if op == "route_grad":
            s["chosen"] = torch.argsort(normal(t, e), dim=1)[:, :k].to(torch.int32).contiguous()
            s["dweights"] = 1e-2 * normal(t, k)
    elif op in ("dispatch", "combine", "combine_grad"):
        t, n, e, k, c = (case[i] for i in ("tokens", "workers", "experts", "k", "cols"))
        taste = normal(t, e) + case["skew"] * normal(e)
        chosen = torch.argsort(taste, dim=1, descending=True)[:, :k].to(torch.int32)
        chosen[torch.rand(t, generator=gen, device="cuda") < 0.02] = -1  # padding
        s["chosen"], s["at"] = chosen.contiguous(), _worker_offsets(t, n, host)
        if op == "dispatch":
            x = normal(t, c) * torch.exp(0.5 * normal(c))
            s["x"] = _pack(x) if case["packed"] else x.to(T)
        else:
            s["offsets"], s["place"] = _sort(s["chosen"], e, s["at"])
            s["weights"] = torch.rand(t, k, generator=gen, device="cuda") + 0.1
            s["weights"] /= s["weights"].sum(1, keepdim=True)
            s["rows"] = normal(t * k, c).to(T)
            if op == "combine":
                s["residual"] = 2 * normal(t, c)
            else:
                s["dout"] = (1e-2 * normal(t, c)).to(T)
    elif op in ("activation", "activation_grad"):
        rows, cols, halves = case["rows"], case["cols"], 2 if case["gated"] else 1
        a = (normal(rows, halves * cols) * torch.exp(0.5 * normal(halves * cols))).to(T)
        s["dy"] = (1e-2 * normal(rows, cols)).to(T)
        if op == "activation":
            s["a"] = a
        else:
            s["kept"] = _pack(a, halves)
    else:
        rows, cols = case["rows"], case["cols"]
        s["stream"] = TYPES[case["stream"]] if case["stream"] else None
        s["weight"] = 1 + 0.1 * normal(cols)
        x = normal(rows, cols) * torch.exp(0.5 * normal(cols))  # some channels carry more than others
        if op == "norm":
            s["x"] = x.to(T)
            if s["stream"] is not None:
                s["residual"] = (2 * normal(rows, cols)).to(s["stream"])
        else:  # what the forward pass left
            h = x.to(s["stream"] or T)
            s["h"], s["rstd"] = h, torch.rsqrt(h.float().square().mean(-1) + EPS)
            s["dy"] = (1e-2 * normal(rows, cols)).to(T)
            if s["stream"] is not None:
                s["dh"] = (1e-2 * normal(rows, cols)).to(s["stream"])
            s["offsets"] = _worker_offsets(rows, case["workers"], host)
    return s


# ---- the plain form: elementary torch operations in 32 bits ------------------------------------------------------
def _scores(logits, kind):
    if kind == "sigmoid":
        return 1 / (1 + torch.exp(-logits))
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _best(v, n):
    """Indices of the n largest values of each row, in descending order; of equal ones the lower index first."""
    return torch.sort(v, dim=1, descending=True, stable=True).indices[:, :n]


def _choose(s):
    """Which experts are chosen, by scores in 64 bits: in 32 the order of neighbours is lost."""
    c = _scores(s["logits"].double(), s["scores"])
    if s["bias"] is not None:
        c = c + s["bias"].double()
    t, e = c.shape
    if s["groups"] > 1:
        parts = c.view(t, s["groups"], -1)
        strength = parts.sort(dim=2, descending=True).values[:, :, :s["top"]].sum(2)
        keep = torch.zeros_like(strength).scatter_(1, _best(strength, s["kept"]), 1.0)
        c = torch.where(keep.bool().unsqueeze(2), parts, -math.inf).reshape(t, e)
    return _best(c, s["k"])


def _weights(s, scores, chosen):
    w = scores.gather(1, chosen.long())
    return (w / w.sum(1, keepdim=True) if s["renormalise"] else w) * s["scale"]


def _sort(chosen, experts, at):
    """(offsets, place): the stable order of (token, slot) pairs by (worker, expert); -1 where there is no expert or worker."""
    t, k = chosen.shape
    token = torch.arange(t, device="cuda").unsqueeze(1)
    worker = (token >= at[1:]).sum(1, keepdim=True)
    groups = (at.numel() - 1) * experts
    lost = (chosen < 0) | (chosen >= experts) | (token < at[0]) | (token >= at[-1])
    key = torch.where(lost, groups, worker * experts + chosen).flatten()
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order).scatter_(0, order, torch.arange(t * k, device="cuda"))
    counts = torch.zeros(groups + 1, dtype=torch.int64, device="cuda").scatter_add_(0, key, torch.ones_like(key))
    offsets = torch.zeros(groups + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = counts[:groups].cumsum(0)
    return offsets, torch.where(lost, -1, place.view(t, k)).to(torch.int32)


def _unpack(rows8, halves=1):
    q, scales = rows8
    rows, cols = q.shape[0], q.shape[1] // halves
    scale = scales.float().view(rows, halves, -1).repeat_interleave(32, dim=2)[:, :, :cols]
    return (q.float().view(rows, halves, cols) * scale).view(rows, halves * cols)


def _to_places(values, place, rows):
    """Rows of zeros with values[t, j] in row place[t, j]; a row behind the last takes what has no place."""
    out = torch.zeros(rows + 1, values.shape[2], device="cuda")
    out[torch.where(place < 0, rows, place).flatten().long()] = values.reshape(-1, values.shape[2])
    return out[:rows]


def _slope(x, kind):
    """(f(x), f'(x))"""
    if kind == "silu":
        p = 1 / (1 + torch.exp(-x))
        return x * p, p * (1 + x * (1 - p))
    if kind == "gelu":
        p = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
        return x * p, p + x * torch.exp(-0.5 * x * x) * math.sqrt(0.5 / math.pi)
    c = math.sqrt(2 / math.pi)
    p = 1 / (1 + torch.exp(-2 * c * (x + 0.044715 * x * x * x)))  # (1 + tanh(z)) / 2 = 1 / (1 + exp(-2z))
    return x * p, p + x * p * (1 - p) * 2 * c * (1 + 3 * 0.044715 * x * x)


def _through(a, s):
    f, slope = _slope(a[:, :s["cols"]], s["kind"])
    return (f * a[:, s["cols"]:] if s["gated"] else f), f, slope


def _plain(s):
    T, op = s["T"], s["op"]
    if op == "route":
        chosen = _choose(s)
        return [chosen.to(torch.int32), _weights(s, _scores(s["logits"].float(), s["scores"]), chosen)]
    if op == "route_grad":
        scores, chosen = _scores(s["logits"].float(), s["scores"]), s["chosen"].long()
        w, dw = _weights(s, scores, chosen), s["dweights"]
        if s["renormalise"]:
            total = scores.gather(1, chosen).sum(1, keepdim=True)
            dw = (dw - (dw * w).sum(1, keepdim=True) / s["scale"]) / total
        ds = torch.zeros_like(scores).scatter_(1, chosen, s["scale"] * dw)
        if s["scores"] == "sigmoid":
            return (ds * scores * (1 - scores)).to(T)
        return (scores * (ds - (ds * scores).sum(1, keepdim=True))).to(T)
    if op == "dispatch":
        offsets, place = _sort(s["chosen"], s["experts"], s["at"])
        x = _unpack(s["x"]) if s["packed"] else s["x"].float()
        return [offsets, place, _to_places(x.unsqueeze(1).expand(-1, s["k"], -1), place, place.numel()).to(T)]
    if op in ("combine", "combine_grad"):
        place = s["place"]
        w = torch.where(place < 0, 0.0, s["weights"])
        there = s["rows"].float()[place.clamp(min=0).long()]
        if op == "combine":
            return s["residual"] + (there * w.unsqueeze(2)).sum(1)
        dout = s["dout"].float().unsqueeze(1)
        return [_to_places(dout * w.unsqueeze(2), place, place.numel()).to(T), torch.where(place < 0, 0.0, (there * dout).sum(2))]
    if op in ("activation", "activation_grad"):
        halves, dy = 2 if s["gated"] else 1, s["dy"].float()
        kept = _unpack(s["kept"] if op == "activation_grad" else _pack(s["a"], halves), halves)
        again, f, slope = _through(kept, s)
        da = torch.cat([dy * slope * kept[:, s["cols"]:], dy * f], 1) if s["gated"] else dy * slope
        return ([] if op == "activation_grad" else [_through(s["a"].float(), s)[0].to(T)]) + [da.to(T), again.to(T)]
    if op == "norm":
        h = s["x"].float()
        if s["stream"] is not None:
            h = h + s["residual"].float()
        rstd = torch.rsqrt(h.square().mean(-1) + EPS)
        y = h * rstd[:, None] * s["weight"]
        return [y.to(T), rstd] + ([h.to(s["stream"])] if s["stream"] is not None else []) + \
            ([_unpack(_pack(y)).to(torch.bfloat16)] if s["packed"] else [])
    dy, rstd, at = s["dy"].float(), s["rstd"][:, None], s["offsets"]
    unit = s["h"].float() * rstd
    g = dy * s["weight"]
    dh = (g - unit * (g * unit).mean(-1, keepdim=True)) * rstd
    if s["stream"] is not None:
        dh = dh + s["dh"].float()
    token = torch.arange(dy.shape[0], device="cuda")
    member = ((token >= at[:-1, None]) & (token < at[1:, None])).double()
    dw = (member @ (dy * unit).double()).float()  # long sums
    return [dh.to(T), dw] + ([dh.to(s["stream"])] if s["stream"] is not None else [])


# ---- the framework's calls ---------------------------------------------------------------------------------------
def _framework(s):
    import paper_2501_05633_b200 as rt
    T, op = s["T"], s["op"]
    if op == "route":
        return list(rt.route(s["logits"], s["k"], scores=s["scores"], bias=s["bias"], groups=s["groups"], groups_kept=s["kept"],
                             group_top=s["top"], renormalise=s["renormalise"], scale=s["scale"]))
    if op == "route_grad":
        return rt.route_backward(s["dweights"], s["logits"], s["chosen"], scores=s["scores"], renormalise=s["renormalise"], scale=s["scale"])
    if op == "dispatch":
        offsets, place = rt.sort_tokens(s["chosen"], s["experts"], s["at"])
        return [offsets, place, rt.spread_tokens(rt.Rows8(*s["x"]) if s["packed"] else s["x"], place, offsets, dtype=T)]
    if op == "combine":
        return rt.join_tokens(s["rows"], s["place"], s["weights"], residual=s["residual"])
    if op == "combine_grad":
        return list(rt.join_tokens_backward(s["dout"], s["rows"], s["place"], s["weights"], s["offsets"]))
    if op == "activation":
        y, kept = rt.activation(s["a"], s["kind"], gated=s["gated"], keep8=True)
        return [y, *rt.activation_backward(s["dy"], kept, s["kind"], gated=s["gated"], want_y=True)]
    if op == "activation_grad":
        return list(rt.activation_backward(s["dy"], rt.Rows8(*s["kept"]), s["kind"], gated=s["gated"], want_y=True))
    if op == "norm":
        y, y8, h, rstd = rt.rms_norm(s["x"], s["weight"], eps=EPS, residual=s.get("residual"), want_y8=s["packed"])
        return [y, rstd] + ([h] if s["stream"] is not None else []) + ([rt.unpack8(y8)] if s["packed"] else [])
    dx, dresidual, dw = rt.rms_norm_backward(s["dy"], s["h"], s["rstd"], s["weight"], dh=s.get("dh"), offsets=s["offsets"])
    return [dx, dw] + ([dresidual] if s["stream"] is not None else [])


def run(state):
    return _framework(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    T, op = size[case["dtype"]], case["op"]
    if op in ("route", "route_grad"):
        t, e, k = case["tokens"], case["experts"], case["k"]
        logits = t * k if op == "route_grad" and (case["renormalise"] or case["scores"] == "sigmoid") else t * e
        return {"bytes": logits * T + 8 * t * k + (t * e * T if op == "route_grad" else 4 * e * case["bias"]), "flops": 8 * t * e}
    if op in ("dispatch", "combine", "combine_grad"):
        t, k, c = case["tokens"], case["k"], case["cols"]
        if op == "dispatch":
            one = t * (c + (c + 31) // 32) if case["packed"] else t * c * T
            return {"bytes": one + t * k * c * T + 8 * t * k + 8 * case["workers"] * case["experts"], "flops": t * k * c}
        if op == "combine":
            return {"bytes": t * k * c * T + 8 * t * c + 8 * t * k, "flops": 2 * t * k * c}
        return {"bytes": 2 * t * k * c * T + t * c * T + 12 * t * k, "flops": 3 * t * k * c}
    if op in ("activation", "activation_grad"):
        n, halves = case["rows"] * case["cols"], 2 if case["gated"] else 1
        kept = halves * case["rows"] * (case["cols"] + (case["cols"] + 31) // 32)
        back = n * T + kept + n * T * halves + n * T  # dy and the kept rows; the gradient, the output again
        return {"bytes": back + (n * T * (halves + 1) + kept if op == "activation" else 0), "flops": 30 * n}
    n, S = case["rows"] * case["cols"], size.get(case["stream"], 0)
    if op == "norm":  # x, y and the residual in and out; the values that the 8 bits stand for
        return {"bytes": n * (2 * T + 2 * S) + 4 * case["rows"] + 4 * case["cols"] + 2 * n * case["packed"], "flops": 6 * n}
    return {"bytes": n * (2 * T + (3 * S or T)) + 4 * case["rows"] + 4 * case["cols"] * (1 + case["workers"]), "flops": 10 * n}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------
def _exact_scores(logits, kind):
    if kind == "sigmoid":
        return torch.special.expit(logits)
    return torch.exp(logits - torch.logsumexp(logits, 1, keepdim=True))


def _exact_choice(c, case):
    """Token by token on the host."""
    c, size = c.cpu().numpy(), case["experts"] // case["groups"]
    chosen = np.empty((case["tokens"], case["k"]), np.int32)
    for t, row in enumerate(c):
        groups = [row[g * size:(g + 1) * size] for g in range(case["groups"])]
        strength = np.array([np.partition(g, size - min(size, case["top"]))[size - min(size, case["top"]):].sum() for g in groups])
        kept = set(np.lexsort((np.arange(len(groups)), -strength))[:case["kept"]].tolist())
        there = np.array([i for i in range(case["experts"]) if i // size in kept])
        chosen[t] = there[np.lexsort((there, -row[there]))[:case["k"]]]
    return torch.from_numpy(chosen).cuda()


def _exact_order(chosen, experts, at):
    chosen, at = chosen.cpu().numpy(), at.tolist()
    place, offsets, n = np.full(chosen.shape, -1, np.int32), [0], 0
    for lo, hi in zip(at, at[1:]):
        for e in range(experts):
            token, slot = np.nonzero(chosen[lo:hi] == e)
            place[lo + token, slot] = n + np.arange(len(token))
            n += len(token)
            offsets.append(n)
    return torch.tensor(offsets, device="cuda"), torch.from_numpy(place).cuda()


def _exact_unpacked(q, scales, cols):
    """Values of the rows whose blocks of 32 begin anew every `cols` columns."""
    column = torch.arange(q.shape[1], device="cuda")
    block = column // cols * ((cols + 31) // 32) + column % cols // 32
    return q.double() * torch.exp2(scales.view(torch.uint8).double() - 127)[:, block]


def _exact_rounded(x, cols):
    """x as its 8-bit rows hold it, in float64."""
    out = torch.empty_like(x, dtype=torch.float64)
    for c0 in range(0, x.shape[1], cols):
        for lo in range(c0, c0 + cols, 32):
            part = x[:, lo:min(lo + 32, c0 + cols)].double()
            most = part.abs().amax(1, keepdim=True)
            mantissa, e = torch.frexp(most / 448)
            e = torch.where(most > 0, (e - (mantissa == 0.5).int()).double(), -127.0).clamp(-127, 127)
            unit = part / torch.exp2(e)
            step = torch.exp2(torch.floor(torch.log2(unit.abs().clamp(min=2.0 ** -6))) - 3)
            out[:, lo:lo + part.shape[1]] = torch.round(unit / step) * step * torch.exp2(e)
    return out


def _exact_activation(a, dy, case):
    a = a.detach().requires_grad_()
    x = a[:, :case["cols"]]
    if case["kind"] == "silu":
        f = x * torch.special.expit(x)
    elif case["kind"] == "gelu":
        f = x * torch.special.ndtr(x)
    else:
        f = 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    y = f * a[:, case["cols"]:] if case["gated"] else f
    return y.detach(), torch.autograd.grad(y, a, dy)[0]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "route":
        scores = _exact_scores(s["logits"].double(), case["scores"])
        chosen = _exact_choice(scores if s["bias"] is None else scores + s["bias"].double(), case)
        w = torch.take_along_dim(scores, chosen.long(), 1)
        return [chosen, case["scale"] * (w / w.sum(1, keepdim=True) if case["renormalise"] else w)]
    if op == "route_grad":
        logits = s["logits"].double().requires_grad_()
        w = torch.take_along_dim(_exact_scores(logits, case["scores"]), s["chosen"].long(), 1)
        w = case["scale"] * (w / w.sum(1, keepdim=True) if case["renormalise"] else w)
        return torch.autograd.grad(w, logits, s["dweights"].double())[0]
    if op in ("dispatch", "combine", "combine_grad"):
        offsets, place = _exact_order(s["chosen"], case["experts"], s["at"])
        token, slot = torch.nonzero(place >= 0, as_tuple=True)
        to = place[token, slot].long()
        if op == "dispatch":
            x = _exact_unpacked(*s["x"], case["cols"]) if case["packed"] else s["x"].double()
            rows = torch.zeros(place.numel(), case["cols"], dtype=torch.float64, device="cuda")
            rows[to] = x[token]
            return [offsets, place, rows]
        w = s["weights"].double()[token, slot]
        if op == "combine":
            return s["residual"].double().index_add_(0, token, s["rows"][to].double() * w[:, None])
        dout, drows = s["dout"].double(), torch.zeros(s["rows"].shape, dtype=torch.float64, device="cuda")
        drows[to] = w[:, None] * dout[token]
        dw = torch.zeros(place.shape, dtype=torch.float64, device="cuda")
        dw[token, slot] = torch.einsum("rc,rc->r", dout[token], s["rows"][to].double())
        return [drows, dw]
    if op in ("activation", "activation_grad"):
        dy = s["dy"].double()
        if op == "activation_grad":
            again, da = _exact_activation(_exact_unpacked(*s["kept"], case["cols"]), dy, case)
            return [da, again]
        again, da = _exact_activation(_exact_rounded(s["a"], case["cols"]), dy, case)
        return [_exact_activation(s["a"].double(), dy, case)[0], da, again]
    if op == "norm":
        h = s["x"].double() + (s["residual"].double() if s["stream"] is not None else 0.0)
        n = h.shape[1]
        rstd = 1 / (torch.einsum("rc,rc->r", h, h) / n + EPS).sqrt()
        y = torch.einsum("rc,r,c->rc", h, rstd, s["weight"].double())
        return [y, rstd] + ([h] if s["stream"] is not None else []) + ([_exact_rounded(y, n)] if case["packed"] else [])
    h = s["h"].double()
    rstd, n = s["rstd"].double(), h.shape[1]
    g = s["dy"].double() * s["weight"].double()
    dh = rstd[:, None] * g - (rstd ** 3 * torch.einsum("rc,rc->r", g, h) / n)[:, None] * h
    if s["stream"] is not None:
        dh += s["dh"].double()
    at = s["offsets"].tolist()
    dw = torch.stack([torch.einsum("rc,rc,r->c", s["dy"][lo:hi].double(), h[lo:hi], rstd[lo:hi]) for lo, hi in zip(at, at[1:])])
    return [dh, dw] + ([dh] if s["stream"] is not None else [])
