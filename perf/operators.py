"""Cases of the operators that train a language model's replicas beside the delayed averaging.

Everything lives where the local step wants it: K replicas are the rows of ``[K, ld]`` arrays, a weight
matrix or an embedding table is a contiguous slice of every row.

``ortho``   momentum, then five Newton-Schulz steps on every matrix of every replica: the direction a
            local step subtracts (gradient array in, direction out, momentum array updated in place).
``lookup``  embedding rows of a token batch, scaled.
``gradient`` the embedding table's gradient from the activations' gradient, in the gradient array.

A token below zero (padding) selects nothing: a zero row forwards, no contribution backwards.
"""
import math

import torch

own = False

BF16, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF16, "f32": F32}
STEPS, COEF, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
#: the dearest case that draw() may give, in operations and in bytes: the largest listed ones
MOST_FLOPS, MOST_BYTES = 1.1e13, 1.6e9


def listed():
    return [
        # the smallest call: one adapter-sized matrix of a single replica; latency counts
        {"name": "ortho 64x96 f32", "op": "ortho", "K": 1, "matrices": "64x96", "dtype": "f32", "gap": 0, "mu": 0.95, "nesterov": True},
        # odd sizes, both orientations, slices that start on odd elements (a head and a projection of a small model)
        {"name": "ortho odd bf16", "op": "ortho", "K": 3, "matrices": "333x1000 1001x77 129x129", "dtype": "bf16", "gap": 5, "mu": 0.9, "nesterov": False},
        # one transformer block of width 1024 (four projections, a feed-forward pair) in four replicas, bfloat16 gradients
        {"name": "ortho block bf16", "op": "ortho", "K": 4, "matrices": "1024x1024 1024x1024 1024x1024 1024x1024 4096x1024 1024x4096",
         "dtype": "bf16", "gap": 1024, "mu": 0.95, "nesterov": True},
        # the same block in two replicas with float32 gradients and directions
        {"name": "ortho block f32", "op": "ortho", "K": 2, "matrices": "1024x1024 1024x1024 1024x1024 1024x1024 4096x1024 1024x4096",
         "dtype": "f32", "gap": 1024, "mu": 0.95, "nesterov": True},
        # a layer of the 4096-wide network in all eight replicas: the largest products
        {"name": "ortho 4096 bf16", "op": "ortho", "K": 8, "matrices": "4096x4096", "dtype": "bf16", "gap": 0, "mu": 0.95, "nesterov": True},
        # one new token for each of eight replicas, from the bfloat16 copy of the weights
        {"name": "lookup one token", "op": "lookup", "K": 8, "T": 1, "V": 32000, "D": 1024, "wt": "bf16", "ot": "bf16", "it": "i64", "pad": 0.0, "gap": 0},
        # odd width, odd offset, float32 masters, padded sequences
        {"name": "lookup odd f32", "op": "lookup", "K": 2, "T": 3001, "V": 5003, "D": 333, "wt": "f32", "ot": "f32", "it": "i64", "pad": 0.1, "gap": 7},
        # a training batch of 64 sequences of 512 in each of four replicas of width 1024
        {"name": "lookup batch bf16", "op": "lookup", "K": 4, "T": 32768, "V": 32000, "D": 1024, "wt": "bf16", "ot": "bf16", "it": "i64", "pad": 0.05, "gap": 0},
        # the same odd table's gradient: most of the work is finding the rows
        {"name": "gradient odd f32", "op": "gradient", "K": 2, "T": 3001, "V": 5003, "D": 333, "at": "f32", "gt": "f32", "it": "i64", "pad": 0.1,
         "zipf": 1.1, "acc": False, "gap": 7},
        # the gradient of the training batch, into the bfloat16 gradient array
        {"name": "gradient batch bf16", "op": "gradient", "K": 4, "T": 32768, "V": 32000, "D": 1024, "at": "bf16", "gt": "bf16", "it": "i64",
         "pad": 0.05, "zipf": 1.1, "acc": False, "gap": 0},
        # a table tied to the output layer: added to the float32 gradient that is there already
        {"name": "gradient tied f32", "op": "gradient", "K": 8, "T": 8192, "V": 50000, "D": 1024, "at": "bf16", "gt": "f32", "it": "i32", "pad": 0.0,
         "zipf": 1.1, "acc": True, "gap": 64},
        # small vocabulary (bytes, or a corpus with one dominant token): long runs of the same row
        {"name": "gradient hot bf16", "op": "gradient", "K": 4, "T": 65536, "V": 259, "D": 512, "at": "bf16", "gt": "f32", "it": "i64", "pad": 0.0,
         "zipf": 2.0, "acc": False, "gap": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["ortho", "ortho", "lookup", "gradient", "gradient"])
        if op == "ortho":
            shapes = [(_log(rng, 32, 4096), _log(rng, 32, 4096)) for _ in range(rng.randint(1, 4))]
            c = {"op": op, "K": rng.randint(1, 8), "matrices": " ".join("%dx%d" % s for s in shapes), "dtype": rng.choice(["bf16", "f32"]),
                 "gap": rng.choice([0, 1, 8, 1024]), "mu": rng.choice([0.0, 0.9, 0.95]), "nesterov": rng.random() < 0.5}
        else:
            c = {"op": op, "K": rng.randint(1, 8), "T": _log(rng, 1, 65536), "V": _log(rng, 2, 128000), "D": rng.choice([_log(rng, 8, 4096), 64 * rng.randint(1, 32)]),
                 "it": rng.choice(["i32", "i64"]), "pad": rng.choice([0.0, 0.1, 0.5]), "gap": rng.choice([0, 3, 64])}
            if op == "lookup":
                c.update(wt=rng.choice(["bf16", "f32"]), ot=rng.choice(["bf16", "f32"]))
            else:
                c.update(at=rng.choice(["bf16", "f32"]), gt=rng.choice(["bf16", "f32"]), zipf=rng.choice([0.0, 1.1, 1.6]), acc=rng.random() < 0.4)
        w = work(c)
        whole = c["K"] * (c["V"] * c["D"] * 4 + c["T"] * c["D"] * 6) if op != "ortho" else 0  # the table itself has to fit as well
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and whole <= 6e9:
            return c


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["matrices"].split()]


def _layout(case):
    """Where each matrix starts in a row, and the row's length: `gap` elements before, between and after them."""
    at, places = case["gap"], []
    for r, c in _shapes(case):
        places.append((at, r, c))
        at += r * c + case["gap"]
    return places, at


def _scale(r, c):
    return max(1.0, r / c) ** 0.5


def _like_gradient(gen, K, r, c, size):
    """A gradient of a linear layer: a sum over fewer examples than the matrix has rows, and noise on top."""
    q = max(1, min(r, c) // 8)
    u = torch.randn(K, r, q, generator=gen, device="cuda") * (torch.arange(1, q + 1, device="cuda") ** -0.5)
    x = u @ torch.randn(K, q, c, generator=gen, device="cuda")
    return size * (x / x.square().mean().sqrt() + 0.3 * torch.randn(K, r, c, generator=gen, device="cuda"))


def _tokens(gen, case, zipf):
    K, T, V = case["K"], case["T"], case["V"]
    p = (torch.arange(V, device="cuda", dtype=torch.float64) + 2.7) ** -zipf
    cdf = (p / p.sum()).cumsum(0)
    rank = torch.searchsorted(cdf, torch.rand(K, T, generator=gen, device="cuda", dtype=torch.float64)).clamp_(max=V - 1)
    tok = torch.randperm(V, generator=gen, device="cuda")[rank]
    tok = torch.where(torch.rand(K, T, generator=gen, device="cuda") < case["pad"], -1, tok)
    return tok.to(torch.int32 if case["it"] == "i32" else torch.int64)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "ortho":
        places, ld = _layout(case)
        K = case["K"]
        g, m = torch.zeros(K, ld, device="cuda"), torch.zeros(K, ld, device="cuda")
        for at, r, c in places:
            g[:, at:at + r * c] = _like_gradient(gen, K, r, c, 1e-3).view(K, -1)
            m[:, at:at + r * c] = _like_gradient(gen, K, r, c, 5e-3).view(K, -1)
        s.update(g=g.to(DT[case["dtype"]]), m=m if case["mu"] else None, places=places)
        s["out"] = torch.zeros_like(s["g"])
        if own:
            from paper_2006_00441_b200 import binding as B
            s["op"] = B.Ortho(K, ld, [(at, r, c, _scale(r, c)) for at, r, c in places], dtype=B.DASGD_F32 if case["dtype"] == "f32" else B.DASGD_BF16_MASTER_F32,
                              momentum=case["mu"], nesterov=case["nesterov"], steps=STEPS, coefficients=COEF, eps=EPS)
        return s
    K, T, V, D = (case[k] for k in "KTVD")
    ld, s["scale"] = V * D + 2 * case["gap"], D ** 0.5
    s["tokens"] = _tokens(gen, case, case.get("zipf", 1.1))
    if case["op"] == "lookup":
        s["w"] = (0.02 * torch.randn(K, ld, generator=gen, device="cuda")).to(DT[case["wt"]])
    else:
        s["dy"] = (1e-3 * torch.randn(K, T, D, generator=gen, device="cuda")).to(DT[case["at"]])
        # with `acc` what the output layer left there; every pass adds to it once more
        s["g"] = (1e-3 * torch.randn(K, ld, generator=gen, device="cuda") if case["acc"] else torch.zeros(K, ld, device="cuda")).to(DT[case["gt"]])
    if own:
        from paper_2006_00441_b200 import binding as B
        s["op"] = B.Embedding(K, ld, case["gap"], V, D, scale=s["scale"], max_tokens=T)
    return s


def run(s):
    case = s["case"]
    if case["op"] == "ortho":
        if own:
            s["op"].step(s["g"], s["m"], out=s["out"])
        else:
            _plain_ortho(s)
        return {"direction": s["out"], "momentum": s["m"]} if s["m"] is not None else {"direction": s["out"]}
    if case["op"] == "lookup":
        return s["op"].lookup(s["w"], s["tokens"], out_dtype=DT[case["ot"]]) if own else _plain_lookup(s)
    if own:
        s["op"].gradient(s["dy"], s["tokens"], s["g"], accumulate=case["acc"])
    else:
        _plain_gradient(s)
    return s["g"]


def _plain_ortho(s):
    case = s["case"]
    K, mu, (a, b, c) = case["K"], case["mu"], COEF
    for at, rows, cols in s["places"]:
        here = slice(at, at + rows * cols)
        u = s["g"][:, here].float()
        if mu:
            g, u = u, torch.add(u, s["m"][:, here], alpha=mu)
            s["m"][:, here] = u
            if case["nesterov"]:
                u = torch.add(g, u, alpha=mu)
        x = u.view(K, rows, cols)
        x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
        for _ in range(STEPS):
            if rows <= cols:
                p = x @ x.mT
                x = a * x + (b * p + c * (p @ p)) @ x
            else:
                p = x.mT @ x
                x = a * x + x @ (b * p + c * (p @ p))
        s["out"][:, here] = (_scale(rows, cols) * x).reshape(K, -1).to(s["out"].dtype)


def _plain_lookup(s):
    case, tok = s["case"], s["tokens"].long()
    K, V, D, gap = (case[k] for k in ("K", "V", "D", "gap"))
    table = s["w"][:, gap:gap + V * D].view(K, V, D)
    rows = table[torch.arange(K, device=tok.device)[:, None], tok.clamp(min=0)].float()
    return (s["scale"] * rows * (tok >= 0)[..., None]).to(DT[case["ot"]])


def _plain_gradient(s):
    case, tok = s["case"], s["tokens"].long()
    K, V, D, gap = (case[k] for k in ("K", "V", "D", "gap"))
    rows = (tok.clamp(min=0) + V * torch.arange(K, device=tok.device)[:, None]).view(-1)
    dy = (s["dy"].float() * (tok >= 0)[..., None]).view(-1, D)
    total = torch.zeros(K * V, D, device=tok.device).index_add_(0, rows, dy).mul_(s["scale"]).view(K, V * D)
    here = s["g"][:, gap:gap + V * D]
    here.copy_(here.float() + total if case["acc"] else total)


def _size(t):
    return {"bf16": 2, "f32": 4, "i32": 4, "i64": 8}[t]


def work(case):
    K = case["K"]
    if case["op"] == "ortho":
        el, fl = 0, 0.0
        for r, c in _shapes(case):
            n, w = min(r, c), max(r, c)
            el += r * c
            fl += STEPS * (2.0 * n * n * w + n * n * w + 1.0 * n ** 3)  # X X^T and its square are symmetric: half of each
        return {"bytes": K * el * (2 * _size(case["dtype"]) + (8 if case["mu"] else 0)), "flops": K * fl}
    T, V, D = case["T"], case["V"], case["D"]
    toks = K * T * _size(case["it"])
    kept = T * (1 - case["pad"])
    p = (torch.arange(V, dtype=torch.float64) + 2.7) ** -case.get("zipf", 1.1)
    distinct = float((1 - (1 - p / p.sum()) ** kept).sum())  # the rows that a batch meets, on average
    if case["op"] == "lookup":
        return {"bytes": int(toks + K * D * (distinct * _size(case["wt"]) + T * _size(case["ot"]))), "flops": int(K * T * D)}
    table = 2 * distinct if case["acc"] else V  # added to: the rows met are read and written; else: the whole table is written
    return {"bytes": int(toks + K * D * (kept * _size(case["at"]) + table * _size(case["gt"]))), "flops": int(K * D * kept)}


def exact(case, seed):
    """The definitions in 64 bits, replica by replica."""
    s = prepare(case, seed)
    K = case["K"]
    if case["op"] == "ortho":
        a, b, c = COEF
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        mom = None if s["m"] is None else s["m"].double()
        for k in range(K):
            for at, rows, cols in s["places"]:
                here = slice(at, at + rows * cols)
                d = s["g"][k, here].double()
                if mom is not None:
                    mom[k, here] = case["mu"] * mom[k, here] + d
                    d = d + case["mu"] * mom[k, here] if case["nesterov"] else mom[k, here]
                x = d.reshape(rows, cols)
                tall = rows > cols
                x = (x.T if tall else x) / (torch.linalg.vector_norm(x) + EPS)
                eye = torch.eye(x.shape[0], dtype=torch.float64, device="cuda")
                for _ in range(STEPS):
                    p = x @ x.T
                    x = (a * eye + p @ (b * eye + c * p)) @ x
                out[k, here] = (_scale(rows, cols) * (x.T if tall else x)).reshape(-1)
        return {"direction": out, "momentum": mom} if mom is not None else {"direction": out}
    V, D, gap = case["V"], case["D"], case["gap"]
    res = []
    for k in range(K):
        keep = s["tokens"][k] >= 0
        tok = s["tokens"][k][keep].long()
        if case["op"] == "lookup":
            y = torch.zeros(case["T"], D, dtype=torch.float64, device="cuda")
            y[keep] = s["w"][k, gap:gap + V * D].view(V, D).double()[tok] * s["scale"]
        else:
            order = torch.argsort(tok, stable=True)
            sums = torch.zeros(V, D, dtype=torch.float64, device="cuda").index_put_((tok[order],), s["dy"][k][keep][order].double(), accumulate=True)
            y = s["g"][k].double()
            y[gap:gap + V * D] += sums.view(-1) * s["scale"]
        res.append(y)
    return torch.stack(res)
