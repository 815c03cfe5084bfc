"""The training operators' cases: what is timed, on which inputs, and what the answer has to be.

The operators are those with which a model's backward pass fills the sparsifier's accumulator rows for all N workers
of one GPU: dropout from a counter-based generator, layer norm (alone, or with the dropout and the residual sum before
it) with its gradient, and the products of tokens with their experts' matrices with their gradients.  The tokens of
all workers lie in one array, sorted by worker (by worker and expert for the products); `offsets` says where each
group begins.  Weight gradients are formed per worker, in binary32.

Dropout keeps the element in column c of row r where the 16-bit number that Philox4x32-10 (Salmon, Moraes, Dror and
Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) gives it is at least t = round(65536 p), and scales it by
65536 / (65536 - t).  Counter: (c // 8, r mod 2^32, r // 2^32, subsequence); key: the 64-bit seed, low word first.
Of the four output words, number (c % 8) // 2 is the element's, its low half for even c and its high half for odd c.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5


# ---- cases -------------------------------------------------------------------------------------------------------
def _dropout(name, rows, cols, dtype, p):
    return {"name": name, "op": "dropout", "rows": rows, "cols": cols, "dtype": dtype, "p": p}


def _norm(name, op, rows, cols, dtype, stream, p, workers):
    """stream: the type of the residual stream, or "" for a layer norm alone.  workers: groups of rows."""
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "stream": stream, "p": p, "workers": workers}


def _product(name, op, tokens, workers, experts, width, out, dtype, skew):
    """width: columns of a token; out: rows of an expert's [out, width] matrix; skew: how unevenly the tokens fall."""
    return {"name": name, "op": op, "tokens": tokens, "workers": workers, "experts": experts, "width": width, "out": out,
            "dtype": dtype, "skew": skew}


def listed():
    return [
        # a short step of one worker: sixteen tokens of GPT-2 small's width, where the call itself is what counts
        _dropout("dropout 16", 16, 768, "bf16", 0.1),
        # attention and feed-forward dropout of a long step in full precision
        _dropout("dropout 16384 f32", 16384, 2048, "f32", 0.2),
        # the sublayer's end for eight workers with sixteen tokens each: dropout, residual sum, layer norm
        _norm("norm 128", "norm", 128, 768, "bf16", "bf16", 0.1, 8),
        # a layer norm alone on an odd width (a pruned or probed model), full precision
        _norm("norm alone odd f32", "norm", 6007, 1023, "f32", "", 0.0, 4),
        # eight workers' long batches, the residual stream held in binary32 beside bf16 activations
        _norm("norm 32768", "norm", 32768, 1024, "bf16", "f32", 0.1, 8),
        # the gradients of the two fused cases
        _norm("norm gradient 128", "norm_grad", 128, 768, "bf16", "bf16", 0.1, 8),
        _norm("norm gradient 32768", "norm_grad", 32768, 1024, "bf16", "bf16", 0.1, 8),
        # a few tokens for each of eight experts: the experts' weights are all there is to read
        _product("experts 96", "product", 96, 1, 8, 768, 1024, "bf16", 0.5),
        # a long step of four workers over sixteen experts
        _product("experts 32768", "product", 32768, 4, 16, 2048, 2304, "bf16", 0.3),
        # the gradient to the tokens, odd sizes that no 16-byte row divides
        _product("experts dx odd f16", "product_dx", 5003, 2, 6, 777, 1030, "f16", 1.0),
        # weight gradients into the rows of eight workers: a short, skewed step and a long one
        _product("experts dw 1000", "product_dw", 1000, 4, 4, 768, 768, "bf16", 1.5),
        _product("experts dw 32768", "product_dw", 32768, 8, 4, 1024, 2304, "bf16", 0.3),
    ]


def _log(rng, lo, hi):
    """A whole number, its logarithm spread evenly over [lo, hi]; half of the time a multiple of 8."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and n >= 16:
        n = n // 8 * 8
    return min(hi, max(lo, n))


def draw(rng):
    op = rng.choice(["dropout", "norm", "norm", "norm_grad", "norm_grad", "product", "product_dx", "product_dw"])
    while True:
        if op == "dropout":
            case = _dropout("", _log(rng, 1, 16384), _log(rng, 1, 8192), rng.choice(list(TYPES)), rng.choice([0.05, 0.1, 0.2, 0.5]))
            ok = 64 <= case["rows"] * case["cols"] <= 1 << 25
        elif op in ("norm", "norm_grad"):
            dtype = rng.choice(list(TYPES))
            stream = rng.choice(["", dtype, "f32"])
            case = _norm("", op, _log(rng, 1, 32768), _log(rng, 16, 8192), dtype, stream,
                         rng.choice([0.0, 0.1, 0.3]) if stream else 0.0, _log(rng, 1, 16))
            ok = case["rows"] * case["cols"] <= 1 << 24
        else:
            case = _product("", op, _log(rng, 1, 32768), _log(rng, 1, 8), _log(rng, 1, 16), _log(rng, 32, 4096), _log(rng, 32, 4096),
                            rng.choice(["bf16", "f16"]), round(rng.uniform(0.0, 1.5), 2))
            pairs = case["workers"] * case["experts"] if op == "product_dw" else case["experts"]
            ok = (case["tokens"] * case["width"] * case["out"] <= 32768 * 1024 * 2304
                  and pairs * case["width"] * case["out"] <= 1 << 26)
        if ok:
            del case["name"]
            return case


# ---- inputs ------------------------------------------------------------------------------------------------------
def _group_sizes(total, groups, skew, seed):
    """Ragged group sizes that sum to `total`: every row falls into group g with a probability of its own."""
    r = np.random.default_rng(seed)
    share = np.exp(skew * r.standard_normal(groups))
    return [int(n) for n in r.multinomial(total, share / share.sum())]


def _offsets(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int64, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    host = random.Random(seed)
    s = {"op": case["op"], "dtype": TYPES[case["dtype"]], "p": case.get("p", 0.0), "seed": host.getrandbits(64),
         "subsequence": host.getrandbits(32)}
    if case["op"] == "dropout":
        s["x"] = normal(case["rows"], case["cols"]).to(s["dtype"])
    elif case["op"] in ("norm", "norm_grad"):
        rows, cols, T = case["rows"], case["cols"], s["dtype"]
        s["stream"] = TYPES[case["stream"]] if case["stream"] else None
        s["weight"], s["bias"] = 1 + 0.1 * normal(cols), 0.1 * normal(cols)
        spread = torch.exp(0.5 * normal(cols))  # some channels carry more than others, and the mean is not zero
        x = normal(rows, cols) * spread + 0.2
        if case["op"] == "norm":
            s["x"] = x.to(T)
            if s["stream"] is not None:
                s["residual"] = (2 * normal(rows, cols) * spread).to(s["stream"])
        else:  # what the forward pass left: its sum, mean and 1 / sqrt(variance + eps)
            h = x.to(s["stream"] or T)
            f = h.float()
            s["h"], s["mean"] = h, f.mean(-1)
            s["rstd"] = torch.rsqrt((f - s["mean"][:, None]).square().mean(-1) + EPS)
            s["dy"] = (1e-2 * normal(rows, cols)).to(T)
            if s["stream"] is not None:
                s["dh"] = (1e-2 * normal(rows, cols)).to(s["stream"])
            s["sizes"] = _group_sizes(rows, case["workers"], 0.3, seed)
            s["offsets"] = _offsets(s["sizes"])
    else:
        n, e, k, m, T = case["workers"], case["experts"], case["width"], case["out"], s["dtype"]
        s["sizes"] = _group_sizes(case["tokens"], n * e, case["skew"], seed)
        s["offsets"] = _offsets(s["sizes"])
        s["n"], s["e"] = n, e
        if case["op"] != "product_dx":
            s["x"] = normal(case["tokens"], k).to(T)
        if case["op"] != "product":
            s["dy"] = (1e-2 * normal(case["tokens"], m)).to(T)
        if case["op"] != "product_dw":
            s["w"] = (normal(e, m, k) / math.sqrt(k)).to(T)
        else:  # the workers' rows of the flat gradient, this layer's matrices behind a norm's two vectors
            rows = torch.zeros(n, 2 * k + e * m * k, device="cuda")
            s["out"] = rows[:, 2 * k:].view(n, e, m, k)
    return s


# ---- the plain form: elementary torch operations in 32 bits ------------------------------------------------------
def _philox_words(rows, groups, seed, subsequence):
    """Philox4x32-10's four output words for every (row, group of eight columns), as int64 in [0, 2^32)."""
    mask = 0xFFFFFFFF
    row = torch.arange(rows, device="cuda").unsqueeze(1)
    c0 = torch.arange(groups, device="cuda").unsqueeze(0).expand(rows, groups)
    c1, c2, c3 = row & mask, row >> 32, subsequence
    k0, k1 = seed & mask, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # modulo 2^64: the low 64 bits are the product's
        c0, c1, c2, c3 = ((b >> 32) & mask) ^ c1 ^ k0, b & mask, ((a >> 32) & mask) ^ c3 ^ k1, a & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return torch.stack([c0, c1, c2, c3], -1)


def _drop(x, p, seed, subsequence):
    """Dropout of a float32 [rows, cols] tensor."""
    t = int(round(65536 * p))
    if t == 0:
        return x
    rows, cols = x.shape
    words = _philox_words(rows, (cols + 7) // 8, seed, subsequence)
    number = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(rows, -1)[:, :cols]
    return torch.where(number >= t, x * (65536 / (65536 - t)), 0.0)


def _plain(s):
    T = s["dtype"]
    if s["op"] == "dropout":
        return _drop(s["x"].float(), s["p"], s["seed"], s["subsequence"]).to(T)
    if s["op"] == "norm":
        h = _drop(s["x"].float(), s["p"], s["seed"], s["subsequence"])
        if s["stream"] is not None:
            h = h + s["residual"].float()
        mean = h.mean(-1)
        centred = h - mean[:, None]
        rstd = torch.rsqrt(centred.square().mean(-1) + EPS)
        y = centred * rstd[:, None] * s["weight"] + s["bias"]
        return [y.to(T), mean, rstd] + ([h.to(s["stream"])] if s["stream"] is not None else [])
    if s["op"] == "norm_grad":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        unit = (s["h"].float() - s["mean"][:, None]) * rstd
        g = dy * s["weight"]
        dh = (g - g.mean(-1, keepdim=True) - unit * (g * unit).mean(-1, keepdim=True)) * rstd
        if s["stream"] is not None:
            dh = dh + s["dh"].float()
        dw = torch.stack([part.sum(0) for part in (dy * unit).split(s["sizes"])])
        db = torch.stack([part.sum(0) for part in dy.split(s["sizes"])])
        dx = _drop(dh, s["p"], s["seed"], s["subsequence"]).to(T)
        return [dx, dw, db] + ([dh.to(s["stream"])] if s["stream"] is not None else [])
    if s["op"] == "product_dw":
        pairs = zip(s["dy"].float().split(s["sizes"]), s["x"].float().split(s["sizes"]))
        return torch.stack([dy.T @ x for dy, x in pairs]).view(s["out"].shape)
    w = s["w"].float()
    if s["op"] == "product":
        return torch.cat([x @ w[g % s["e"]].T for g, x in enumerate(s["x"].float().split(s["sizes"]))]).to(T)
    return torch.cat([dy @ w[g % s["e"]] for g, dy in enumerate(s["dy"].float().split(s["sizes"]))]).to(T)


# ---- the framework's calls ---------------------------------------------------------------------------------------
def _framework(s):
    import paper_2501_05633_b200 as rt
    if s["op"] == "dropout":
        return rt.dropout(s["x"], s["p"], s["seed"], s["subsequence"])
    if s["op"] == "norm":
        y, h, mean, rstd = rt.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, residual=s.get("residual"), p=s["p"],
                                         seed=s["seed"], subsequence=s["subsequence"])
        return [y, mean, rstd] + ([h] if s["stream"] is not None else [])
    if s["op"] == "norm_grad":
        dx, dresidual, dw, db = rt.layer_norm_backward(s["dy"], s["h"], s["mean"], s["rstd"], s["weight"], offsets=s["offsets"],
                                                       dh=s.get("dh"), p=s["p"], seed=s["seed"], subsequence=s["subsequence"])
        return [dx, dw, db] + ([dresidual] if s["stream"] is not None else [])
    if s["op"] == "product_dw":
        return rt.grouped_matmul_dw(s["dy"], s["x"], s["offsets"], out=s["out"])
    if s["op"] == "product":
        return rt.grouped_matmul(s["x"], s["w"], s["offsets"])
    return rt.grouped_matmul(s["dy"], s["w"].transpose(1, 2), s["offsets"])


def run(state):
    return _framework(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * size[case["dtype"]], "flops": n}
    if case["op"] in ("norm", "norm_grad"):
        n, T, S = case["rows"] * case["cols"], size[case["dtype"]], size.get(case["stream"], 0)
        if case["op"] == "norm":  # x and y, the residual and the sum; two statistics a row, two vectors
            return {"bytes": n * (2 * T + 2 * S) + 8 * case["rows"] + 8 * case["cols"], "flops": 8 * n}
        # dy and dx, the sum (of x's type where there is no stream), its gradient in and out; statistics, weight, gradients
        return {"bytes": n * (2 * T + (3 * S or T)) + 8 * case["rows"] + 4 * case["cols"] * (1 + 2 * case["workers"]), "flops": 14 * n}
    t, k, m, e = case["tokens"], case["width"], case["out"], case["experts"]
    if case["op"] == "product_dw":
        return {"bytes": 2 * t * (k + m) + 4 * case["workers"] * e * m * k, "flops": 2 * t * m * k}
    return {"bytes": 2 * t * (k + m) + 2 * e * m * k, "flops": 2 * t * m * k}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------
def _mul_hi_lo(a, constant):
    """High and low 32 bits of a * constant by 16-bit halves."""
    a1, a0, b1, b0 = a >> 16, a & 0xFFFF, constant >> 16, constant & 0xFFFF
    low = a0 * b0
    mid1, mid2 = a1 * b0, a0 * b1
    carry = ((low >> 16) + (mid1 & 0xFFFF) + (mid2 & 0xFFFF)) >> 16
    return a1 * b1 + (mid1 >> 16) + (mid2 >> 16) + carry, (low + ((mid1 & 0xFFFF) << 16) + ((mid2 & 0xFFFF) << 16)) & 0xFFFFFFFF


def _exact_factor(rows, cols, s):
    """What dropout multiplies each element by, as float64 [rows, cols]."""
    t = int(round(65536 * s["p"]))
    if t == 0:
        return torch.ones(rows, cols, dtype=torch.float64, device="cuda")
    groups = (cols + 7) // 8
    index = torch.arange(rows * groups, device="cuda")
    r = index // groups
    x = [index % groups, r % 2**32, r // 2**32, torch.full_like(index, s["subsequence"])]
    for i in range(10):
        key = [(s["seed"] % 2**32 + i * 0x9E3779B9) % 2**32, (s["seed"] // 2**32 + i * 0xBB67AE85) % 2**32]
        h0, l0 = _mul_hi_lo(x[0], 0xD2511F53)
        h1, l1 = _mul_hi_lo(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
    factor = torch.empty(rows * groups, 8, dtype=torch.float64, device="cuda")
    for j in range(8):
        number = (x[j // 2] >> (16 * (j % 2))) % 65536
        factor[:, j] = (number >= t).double() * (65536.0 / (65536 - t))
    return factor.view(rows, 8 * groups)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "dropout":
        return s["x"].double() * _exact_factor(*s["x"].shape, s)
    if s["op"] == "norm":
        h = s["x"].double() * _exact_factor(*s["x"].shape, s)
        if s["stream"] is not None:
            h += s["residual"].double()
        n = h.shape[1]
        mean = h.sum(1) / n
        var = (h * h).sum(1) / n - mean * mean
        rstd = 1 / (var + EPS).sqrt()
        y = torch.addcmul(s["bias"].double(), (h - mean[:, None]) * rstd[:, None], s["weight"].double())
        return [y, mean, rstd] + ([h] if s["stream"] is not None else [])
    if s["op"] == "norm_grad":
        dy, rstd, n = s["dy"].double(), s["rstd"].double()[:, None], s["dy"].shape[1]
        unit = (s["h"].double() - s["mean"].double()[:, None]) * rstd
        g = dy * s["weight"].double()
        a, b = g.sum(1, keepdim=True), torch.einsum("rc,rc->r", g, unit)[:, None]
        dh = rstd * (n * g - a - unit * b) / n
        if s["stream"] is not None:
            dh += s["dh"].double()
        dw = torch.zeros(case["workers"], n, dtype=torch.float64, device="cuda")
        worker = torch.repeat_interleave(torch.arange(case["workers"], device="cuda"), torch.tensor(s["sizes"], device="cuda"))
        db = dw.clone().index_add_(0, worker, dy)
        dw.index_add_(0, worker, dy * unit)
        return [dh * _exact_factor(*dh.shape, s), dw, db] + ([dh] if s["stream"] is not None else [])
    at = s["offsets"].tolist()
    if s["op"] == "product_dw":
        out = torch.zeros(s["n"] * s["e"], case["out"], case["width"], dtype=torch.float64, device="cuda")
        for g, (lo, hi) in enumerate(zip(at, at[1:])):
            out[g] = torch.einsum("tm,tk->mk", s["dy"][lo:hi].double(), s["x"][lo:hi].double())
        return out.view(s["out"].shape)
    w, a = s["w"].double(), s["x" if s["op"] == "product" else "dy"]
    out = torch.zeros(a.shape[0], case["out"] if s["op"] == "product" else case["width"], dtype=torch.float64, device="cuda")
    for g, (lo, hi) in enumerate(zip(at, at[1:])):
        out[lo:hi] = torch.einsum("tk,mk->tm" if s["op"] == "product" else "tm,mk->tk", a[lo:hi].double(), w[g % s["e"]])
    return out
