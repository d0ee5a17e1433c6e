"""Workloads of the stand-alone operators: orthogonalisation, layer norm and expert routing.

Each case is one call pattern of a training or serving program. ``run`` computes it either with
the library's kernels (``own``) or in plain elementary torch operations in 32 bits; ``exact``
computes it in 64 bits by a route of its own. Sizes are those of the workloads in
``paper_2607_20548_gb300/workloads.py`` (hidden 2048, experts of width 768, 64 experts, FFN 8192)
with odd and ragged ones beside them.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
QUINTIC = (15 / 8, -10 / 8, 3 / 8)  # the optimizer's default Newton-Schulz polynomial
NS_EPS, LN_EPS, COEF = 1e-7, 1e-5, 0.01


def listed():
    return [
        # the router's 2048 x 64 momentum: one small tall matrix, where the number of launches counts
        dict(name="orth_router_2048x64_bf16", op="orth", batch=1, m=2048, n=64, dtype="bf16", steps=16, view=False),
        # one projection of a layer's 64 experts, gathered as a batch of bf16 momenta
        dict(name="orth_experts_64x768x2048_bf16", op="orth", batch=64, m=768, n=2048, dtype="bf16", steps=16,
             view=False),
        # gate, up and down of a dense block, gathered in one orientation and passed as a transposed
        # view: the largest bf16 work
        dict(name="orth_ffn_3x8192x2048_bf16", op="orth", batch=3, m=8192, n=2048, dtype="bf16", steps=16, view=True),
        # the four attention projections with their momenta in fp32, the optimizer's own type
        dict(name="orth_attn_4x2048x2048_fp32", op="orth", batch=4, m=2048, n=2048, dtype="fp32", steps=16,
             view=False),
        # ragged shards of a tensor-parallel weight: odd sides, fp16
        dict(name="orth_odd_5x1365x777_fp16", op="orth", batch=5, m=1365, n=777, dtype="fp16", steps=8, view=True),
        # a single token's norm while serving
        dict(name="norm_1x2048_bf16_fwd", op="norm", rows=1, width=2048, dtype="bf16", wdtype="bf16", train=False),
        # a training micro-batch at the model's width, fp32 weights
        dict(name="norm_8192x2048_bf16_train", op="norm", rows=8192, width=2048, dtype="bf16", wdtype="fp32",
             train=True),
        # odd rows and an odd width in fp32
        dict(name="norm_1023x4099_fp32_train", op="norm", rows=1023, width=4099, dtype="fp32", wdtype="fp32",
             train=True),
        # the widest layer and a long batch: bound by memory
        dict(name="norm_32768x8192_bf16_train", op="norm", rows=32768, width=8192, dtype="bf16", wdtype="fp32",
             train=True),
        # one token of a serving step through the router
        dict(name="route_1x64_k8_fp32_fwd", op="route", tokens=1, experts=64, k=8, dtype="fp32", normalize=True,
             masked=False, train=False),
        # a training micro-batch, packed sequences with padding masked out, two experts unavailable
        dict(name="route_65536x64_k8_bf16_train", op="route", tokens=65536, experts=64, k=8, dtype="bf16",
             normalize=True, masked=True, train=True),
        # a whole accumulation step's tokens over an odd number of experts, fp32 logits
        dict(name="route_500009x127_k6_fp32_train", op="route", tokens=500009, experts=127, k=6, dtype="fp32",
             normalize=False, masked=True, train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["orth", "norm", "route"])
    if op == "orth":
        while True:
            c = dict(op="orth", batch=_log(rng, 1, 64), m=_log(rng, 24, 8192), n=_log(rng, 24, 8192),
                     dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), steps=rng.randint(5, 16),
                     view=rng.random() < 0.5)
            cost = work(c)["flops"] * (3 if c["dtype"] == "fp32" else 1)
            if 3072 not in (c["m"], c["n"]) and min(c["m"], c["n"]) <= 2600 and cost <= 5e12:
                return c
    if op == "norm":
        while True:
            c = dict(op="norm", rows=_log(rng, 1, 60000), width=_log(rng, 48, 16384),
                     dtype=rng.choice(["bf16", "fp16", "fp32"]), wdtype="fp32", train=rng.random() < 0.75)
            c["wdtype"] = rng.choice(["fp32", c["dtype"]])
            if c["width"] != 3072 and c["rows"] * c["width"] <= 1 << 27:
                return c
    while True:
        c = dict(op="route", tokens=_log(rng, 1, 500000), experts=_log(rng, 8, 512), k=rng.randint(1, 8),
                 dtype=rng.choice(["bf16", "fp32"]), normalize=rng.random() < 0.5, masked=rng.random() < 0.5,
                 train=rng.random() < 0.75)
        if c["tokens"] * c["experts"] <= 1 << 25:
            return c


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    c = dict(case)
    if c["op"] == "orth":
        # a gradient's momentum: a few strong directions over a noise floor
        b, m, n = c["batch"], c["m"], c["n"]
        q = min(8, m, n)
        M = rand(b, m, q) @ rand(b, q, n) * (0.5 / math.sqrt(q)) + rand(b, m, n)
        M = (M * 1e-3).to(DTYPES[c["dtype"]])
        # a view: the weight is held transposed, and the operator gets its strides
        c["M"] = M.transpose(1, 2).contiguous().transpose(1, 2) if c["view"] else M
        return c
    dt = DTYPES[c["dtype"]]
    if c["op"] == "norm":
        r, w = c["rows"], c["width"]
        c["x"] = (rand(r, w) * (0.5 + 2 * torch.rand(r, 1, generator=g, device=DEV)) + 0.3 * rand(r, 1)).to(dt)
        c["weight"] = (1 + 0.1 * rand(w)).to(DTYPES[c["wdtype"]])
        c["bias"] = (0.1 * rand(w)).to(DTYPES[c["wdtype"]])
        if c["train"]:
            c["dy"] = (rand(r, w) * 0.01).to(dt)
        return c
    t, e = c["tokens"], c["experts"]
    # uneven experts: each token's logits over a preference that all tokens share
    z = rand(t, e) + 0.7 * rand(e)
    if c["masked"]:
        if e - c["k"] >= 2:
            z[:, 1] = z[:, e - 1] = -math.inf  # experts that take no tokens
        c["mask"] = torch.rand(t, generator=g, device=DEV) < 0.9
        z = torch.where(c["mask"][:, None], z, torch.full_like(z, math.nan))  # padding holds anything
    else:
        c["mask"] = None
    c["logits"] = z.to(dt)
    if c["train"]:
        c["dgates"] = rand(t, c["k"]) * (1e-2 / t)
    return c


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2607_20548_gb300 as lib
    if s["op"] == "orth":
        return lib.muon_orthogonalize(s["M"], ns_steps=s["steps"], eps=NS_EPS)
    if s["op"] == "norm":
        y, mean, rstd = lib.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=LN_EPS)
        if not s["train"]:
            return y
        return (y,) + tuple(lib.layer_norm_backward(s["dy"], s["x"], mean, rstd, s["weight"]))
    r = lib.route_forward(s["logits"], s["k"], mask=s["mask"], normalize=s["normalize"], coef=COEF)
    out = (r.indices, r.gates, r.counts, r.loss)
    if not s["train"]:
        return out
    return out + (lib.route_backward(s["logits"], r, dgates=s["dgates"]),)


def _plain(s):
    if s["op"] == "orth":
        return _plain_orth(s)
    return _plain_norm(s) if s["op"] == "norm" else _plain_route(s)


def _plain_orth(s):
    X = s["M"].float()
    X = X / X.square().sum((1, 2), keepdim=True).sqrt().clamp_min(NS_EPS)
    tall = X.shape[1] > X.shape[2]
    X = X.mT if tall else X
    a, b, c = QUINTIC
    for _ in range(s["steps"]):
        S = X @ X.mT
        X = a * X + (b * S + c * (S @ S)) @ X
    return (X.mT if tall else X).to(s["M"].dtype).contiguous()


def _plain_norm(s):
    x, w = s["x"].float(), s["weight"].float()
    xc = x - x.mean(1, keepdim=True)
    rstd = (xc.square().mean(1, keepdim=True) + LN_EPS).rsqrt()
    xh = xc * rstd
    y = (xh * w + s["bias"].float()).to(s["x"].dtype)
    if not s["train"]:
        return y
    dy = s["dy"].float()
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return y, dx.to(s["x"].dtype), (dy * xh).sum(0), dy.sum(0)


def _plain_route(s):
    z, k, e = s["logits"].float(), s["k"], s["experts"]
    live = torch.ones_like(z[:, 0], dtype=torch.bool) if s["mask"] is None else s["mask"]
    z = torch.where(live[:, None], z, torch.zeros_like(z))
    p = (z - z.amax(1, keepdim=True)).exp()
    p = p / p.sum(1, keepdim=True) * live[:, None]
    top, idx = torch.sort(z, dim=1, descending=True, stable=True)
    top, idx = top[:, :k], idx[:, :k]
    chosen = live[:, None] & (top > -math.inf)
    gates = p.gather(1, idx) * chosen
    total = gates.sum(1, keepdim=True).clamp_min(1e-38)
    if s["normalize"]:
        gates = gates / total
    hot = torch.zeros_like(z).scatter_(1, idx, chosen.float())
    counts, n = hot.sum(0), live.sum().clamp_min(1).float()
    load = COEF * e / (k * n) * counts
    loss = (load * p.sum(0)).sum() / n
    out = (torch.where(chosen, idx, torch.full_like(idx, -1)).int(), gates, counts.int(), loss)
    if not s["train"]:
        return out
    d = s["dgates"] * chosen
    if s["normalize"]:
        d = (d - (d * gates).sum(1, keepdim=True)) / total * chosen
    u = torch.zeros_like(z).scatter_(1, idx, d) + load / n
    return out + ((p * (u - (p * u).sum(1, keepdim=True))).to(s["logits"].dtype),)


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "orth":
        # in the space of the smaller side's Gram matrix: every step is a polynomial in it, so the
        # result is one accumulated polynomial times M
        M = s["M"].double()
        M = M.mT if M.shape[1] > M.shape[2] else M
        M = M / torch.linalg.matrix_norm(M, keepdim=True).clamp_min(NS_EPS)
        out = torch.empty_like(M)
        eye = torch.eye(M.shape[1], dtype=torch.float64, device=DEV)
        a, b, c = QUINTIC
        for i in range(M.shape[0]):
            G, Q = M[i] @ M[i].T, eye
            for _ in range(s["steps"]):
                W = a * eye + G @ (b * eye + c * G)
                G, Q = W @ G @ W, W @ Q
            out[i] = Q @ M[i]
        return (out.mT if s["m"] > s["n"] else out).contiguous()
    if s["op"] == "norm":
        x = s["x"].double()
        w = s["weight"].double()
        var, mu = torch.var_mean(x, 1, correction=0, keepdim=True)
        sd = (var + LN_EPS).sqrt()
        y = (x - mu) / sd * w + s["bias"].double()
        if not s["train"]:
            return y
        # the gradient by the chain rule through the mean and the variance
        dy = s["dy"].double()
        g, n = dy * w, x.shape[1]
        dvar = -0.5 * (g * (x - mu)).sum(1, keepdim=True) / sd ** 3
        dmu = -g.sum(1, keepdim=True) / sd
        dx = g / sd + dvar * 2 * (x - mu) / n + dmu / n
        return y, dx, torch.einsum("rw,rw->w", dy, (x - mu) / sd), dy.sum(0)
    z, k, e = s["logits"].double(), s["k"], s["experts"]
    t = z.shape[0]
    live = torch.ones(t, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"]
    z[~live] = 0.0
    p = torch.softmax(z, 1)
    p[~live] = 0.0
    rest, idx, val = z.clone(), [], []
    for _ in range(k):  # the first of the largest ones left, k times
        i = rest.argmax(1, keepdim=True)
        ok = live[:, None] & (rest.gather(1, i) > -math.inf)
        idx.append(torch.where(ok, i, torch.full_like(i, -1)))
        val.append(torch.where(ok, p.gather(1, i), torch.zeros_like(p[:, :1])))
        rest.scatter_(1, i, -math.inf)
    idx, val = torch.cat(idx, 1), torch.cat(val, 1)
    total = val.sum(1, keepdim=True)
    gates = val / torch.where(total > 0, total, torch.ones_like(total)) if s["normalize"] else val
    counts = torch.bincount(idx[idx >= 0], minlength=e).double()
    n = max(1, int(live.sum()))
    loss = COEF * e / (k * n) * (counts @ p.sum(0)) / n
    out = (idx.int(), gates, counts.int(), loss)
    if not s["train"]:
        return out
    # the gradient through the chosen probabilities' Jacobian, one choice at a time
    up = (COEF * e / (k * n * n) * counts)[None, :].expand(t, e)
    dz = p * (up - (p * up).sum(1, keepdim=True))
    d = torch.where(idx >= 0, s["dgates"].double(), torch.zeros_like(val))
    if s["normalize"]:
        d = torch.where(idx >= 0, (d - (d * gates).sum(1, keepdim=True)) / total, torch.zeros_like(d))
    dz -= p * (d * val).sum(1, keepdim=True)
    dz.scatter_add_(1, idx.clamp_min(0).long(), d * val)
    return out + (dz,)


def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if case["op"] == "orth":
        # the Gram matrix and its square are symmetric: half of each
        b, r, k = case["batch"], min(case["m"], case["n"]), max(case["m"], case["n"])
        return {"bytes": 2 * b * r * k * size,
                "flops": case["steps"] * b * (r * (r + 1) * k + r * (r + 1) * r + 2 * r * r * k)}
    if case["op"] == "norm":
        n, w = case["rows"] * case["width"], case["width"]
        ws = 4 if case["wdtype"] == "fp32" else 2
        # a training pass is two calls: x is read by both
        return {"bytes": n * size * (5 if case["train"] else 2) + w * (2 * ws + (ws + 8 if case["train"] else 0)),
                "flops": n * (20 if case["train"] else 8)}
    t, e, k = case["tokens"], case["experts"], case["k"]
    fwd = t * e * size + t * (8 * k + int(case["masked"])) + 4 * e
    bwd = 2 * t * e * size + t * (12 * k + int(case["masked"])) if case["train"] else 0
    return {"bytes": fwd + bwd, "flops": t * e * (12 if case["train"] else 6)}
