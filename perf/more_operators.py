"""Workloads of the operators of a transformer block: the gated feed-forward, dense and over experts, and the
norms of queries and keys with the position rotation.

Each case is one call pattern of a training or serving program. ``run`` computes it either with the
library's kernels (``own``) or in plain elementary torch operations in 32 bits; ``exact`` computes it in
64 bits by a route of its own. Sizes are those of the workloads in ``paper_2607_20548_gb300/workloads.py``
(hidden 2048, FFN 8192, 64 experts of width 768; projections of 2048 as 16 heads of 128) with odd and ragged
ones beside them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS, BASE = 1e-6, 10000.0


def listed():
    return [
        # one token through a dense block while serving: bound by the weights' bytes
        dict(name="ffn_1x2048x8192_bf16_fwd", op="ffn", rows=1, dropped=0, groups=0, hidden=2048, width=8192,
             dtype="bf16", act="silu", columns=False, train=False),
        # a decode batch of two dozen requests
        dict(name="ffn_24x2048x8192_bf16_fwd", op="ffn", rows=24, dropped=0, groups=0, hidden=2048, width=8192,
             dtype="bf16", act="silu", columns=False, train=False),
        # the same batch size through a layer's 64 experts, 8 for each token, sorted by expert
        dict(name="ffn_experts_192x64x2048x768_bf16_fwd", op="ffn", rows=192, dropped=0, groups=64, hidden=2048,
             width=768, dtype="bf16", act="silu", columns=False, train=False),
        # a training micro-batch through the dense block: the largest products
        dict(name="ffn_8192x2048x8192_bf16_train", op="ffn", rows=8192, dropped=0, groups=0, hidden=2048, width=8192,
             dtype="bf16", act="silu", columns=False, train=True),
        # 4096 tokens and 8 experts for each, padded tokens' rows behind the last expert's
        dict(name="ffn_experts_32768x64x2048x768_bf16_train", op="ffn", rows=32768, dropped=1500, groups=64,
             hidden=2048, width=768, dtype="bf16", act="silu", columns=False, train=True),
        # ragged shards of a tensor-parallel block, weights held transposed, odd sides
        dict(name="ffn_odd_1023x777x1365_fp16_train", op="ffn", rows=1023, dropped=0, groups=0, hidden=777,
             width=1365, dtype="fp16", act="gelu", columns=True, train=True),
        # a few experts in fp32, the optimizer's own type
        dict(name="ffn_experts_2000x5x2048x768_fp32_train", op="ffn", rows=2000, dropped=0, groups=5, hidden=2048,
             width=768, dtype="fp32", act="silu", columns=False, train=True),
        # one token's queries and keys while serving
        dict(name="qk_1x16x4x128_bf16_fwd", op="qk", tokens=1, heads=16, kv_heads=4, dim=128, rotary=128,
             interleaved=False, dtype="bf16", wdtype="bf16", fused=True, train=False),
        # a training micro-batch, slices of the fused projection's rows
        dict(name="qk_8192x16x4x128_bf16_train", op="qk", tokens=8192, heads=16, kv_heads=4, dim=128, rotary=128,
             interleaved=False, dtype="bf16", wdtype="fp32", fused=True, train=True),
        # odd heads in fp32, rotated in part and by neighbouring pairs
        dict(name="qk_3001x7x3x80_fp32_train", op="qk", tokens=3001, heads=7, kv_heads=3, dim=80, rotary=40,
             interleaved=True, dtype="fp32", wdtype="fp32", fused=False, train=True),
        # a long prompt's prefill, and a whole accumulation step's tokens: bound by memory
        dict(name="qk_65536x16x16x128_fp16_fwd", op="qk", tokens=65536, heads=16, kv_heads=16, dim=128, rotary=128,
             interleaved=False, dtype="fp16", wdtype="fp16", fused=True, train=False),
        dict(name="qk_131072x16x4x128_bf16_train", op="qk", tokens=131072, heads=16, kv_heads=4, dim=128, rotary=128,
             interleaved=False, dtype="bf16", wdtype="fp32", fused=False, train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.55:
        while True:
            groups = rng.choice([0, 0, _log(rng, 2, 64)])
            rows = _log(rng, 1, 32768)
            c = dict(op="ffn", rows=rows, dropped=rng.randint(0, rows // 8) if groups else 0, groups=groups,
                     hidden=_log(rng, 64, 4096), width=_log(rng, 64, 8192),
                     dtype=rng.choice(["bf16", "bf16", "bf16", "fp16", "fp32"]), act=rng.choice(["silu", "silu", "gelu"]),
                     columns=rng.random() < 0.3, train=rng.random() < 0.6)
            if rng.random() < 0.6:  # most models' sides are multiples of 64
                c["hidden"], c["width"] = -(-c["hidden"] // 64) * 64, -(-c["width"] // 64) * 64
            most = 2.4e12 if c["dtype"] != "fp32" else 1e11
            if work(c)["flops"] <= most and max(groups, 1) * c["hidden"] * c["width"] <= 64 * 2048 * 768:
                return c
    while True:
        dim = rng.choice([32, 64, 64, 96, 128, 128, 192, 256, 2 * rng.randint(16, 128)])
        heads = _log(rng, 1, 32)
        c = dict(op="qk", tokens=_log(rng, 1, 131072), heads=heads, kv_heads=rng.randint(1, heads), dim=dim,
                 rotary=rng.choice([dim, dim, 2 * rng.randint(1, dim // 2)]), interleaved=rng.random() < 0.4,
                 dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), wdtype="fp32", fused=rng.random() < 0.5,
                 train=rng.random() < 0.6)
        c["wdtype"] = rng.choice(["fp32", c["dtype"]])
        if c["tokens"] * (c["heads"] + c["kv_heads"]) * dim <= 1 << 28:
            return c


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    c, dt = dict(case), DTYPES[case["dtype"]]
    if c["op"] == "ffn":
        rows, k, n = c["rows"], c["hidden"], c["width"]
        lead = (c["groups"],) if c["groups"] else ()

        def weight(m, n):
            w = (rand(*lead, m, n) / math.sqrt(m)).to(dt)
            return w.mT.contiguous().mT if c["columns"] else w  # held as [out, in]
        c["w_gate"], c["w_up"], c["w_down"] = weight(k, n), weight(k, n), weight(n, k)
        c["x"], c["dy"] = rand(rows, k).to(dt), (0.02 * rand(rows, k)).to(dt) if c["train"] else None
        c["offsets"], c["lengths"] = None, [rows]
        if lead:
            # uneven experts, about as a balance loss leaves them; rows behind the last one's hold anything
            host = np.random.default_rng(seed)
            share = np.exp(0.3 * host.standard_normal(c["groups"]))
            lengths = host.multinomial(rows - c["dropped"], share / share.sum())
            c["lengths"] = [int(v) for v in lengths]
            c["offsets"] = torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32, device=DEV)
            c["x"][rows - c["dropped"]:] = math.nan
            if c["train"]:
                c["dy"][rows - c["dropped"]:] = math.nan
        return c
    t, h, kv, d, r = c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["rotary"]
    if c["fused"]:  # slices of a projection to queries, keys and values
        qkv = rand(t, (h + 2 * kv) * d).to(dt).view(t, h + 2 * kv, d)
        c["q"], c["k"] = qkv[:, :h], qkv[:, h:h + kv]
    else:
        c["q"], c["k"] = rand(t, h, d).to(dt), rand(t, kv, d).to(dt)
    c["q_weight"], c["k_weight"] = ((1 + 0.1 * rand(d)).to(DTYPES[c["wdtype"]]) for _ in range(2))
    # the table of the model's longest context, and packed sequences: positions begin again at each one
    places = max(4096, min(t, 32768))
    angle = torch.arange(places, dtype=torch.float64, device=DEV)[:, None] * BASE ** (
        -torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r)
    c["cos"], c["sin"] = angle.cos().float(), angle.sin().float()
    start = int(torch.randint(0, places, (1,), generator=g, device=DEV))
    c["positions"] = (torch.arange(t, device=DEV) + start) % places
    if c["train"]:
        c["dq"], c["dk"] = (0.02 * rand(t, h, d)).to(dt), (0.02 * rand(t, kv, d)).to(dt)
    return c


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2607_20548_gb300 as lib
    if s["op"] == "ffn":
        w = (s["w_gate"], s["w_up"], s["w_down"])
        y, pre = lib.ffn_forward(s["x"], *w, offsets=s["offsets"], act=s["act"], keep=s["train"])
        if not s["train"]:
            return y
        return (y,) + tuple(lib.ffn_backward(s["dy"], s["x"], pre, *w, offsets=s["offsets"], act=s["act"]))
    how = dict(positions=s["positions"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
               interleaved=s["interleaved"])
    out = tuple(lib.qk_rotary_forward(s["q"], s["k"], s["cos"], s["sin"], **how))
    if not s["train"]:
        return out
    return out + tuple(lib.qk_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["cos"], s["sin"], **how))


def _plain(s):
    return _plain_ffn(s) if s["op"] == "ffn" else _plain_qk(s)


def _plain_ffn(s):
    dt, rows, groups = s["x"].dtype, s["rows"], s["groups"]
    wg, wu, wd = s["w_gate"].float(), s["w_up"].float(), s["w_down"].float()
    if groups:  # a batch of matrices as high as the longest group; the place of each row in it
        high, off = max(max(s["lengths"]), 1), s["offsets"].long()
        at = torch.arange(rows, device=DEV)
        group = (at[:, None] >= off[None, 1:]).sum(1)
        live = at < off[-1]
        group = group.clamp_max(groups - 1)
        place = torch.where(live, group * high + at - off[group], groups * high)

        def spread(t):
            out = torch.zeros(groups * high + 1, t.shape[1], device=DEV)
            out[place] = torch.where(live[:, None], t.float(), torch.zeros((), device=DEV))
            return out[:-1].view(groups, high, t.shape[1])

        def gather(t):
            t = t.reshape(groups * high, t.shape[2])
            return torch.cat([t, torch.zeros_like(t[:1])])[place]
    else:
        spread, gather = (lambda t: t.float()), (lambda t: t)
    x = spread(s["x"])
    g, u = x @ wg, x @ wu
    if s["act"] == "silu":
        gate = 1 / (1 + (-g).exp())
        a, da = g * gate, gate * (1 + g * (1 - gate))
    else:
        normal = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        a, da = g * normal, normal + g * (-0.5 * g * g).exp() / math.sqrt(2 * math.pi)
    h = a * u
    y = gather(h @ wd).to(dt)
    if not s["train"]:
        return y
    dy = spread(s["dy"])
    dh = dy @ wd.mT
    dg, du = dh * u * da, dh * a
    dx = gather(dg @ wg.mT + du @ wu.mT).to(dt)
    return y, dx, (x.mT @ dg).to(dt), (x.mT @ du).to(dt), (h.mT @ dy).to(dt)


def _turn(s, m, c, sn):
    """The first ``rotary`` elements turned by the angles of cosine c and sine sn."""
    r = s["rotary"]
    if s["interleaved"]:
        a, b = m[..., 0:r:2], m[..., 1:r:2]
        turned = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    else:
        a, b = m[..., :r // 2], m[..., r // 2:r]
        turned = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    return torch.cat([turned, m[..., r:]], -1)


def _plain_qk(s):
    dt = s["q"].dtype
    c, sn = s["cos"][s["positions"]][:, None], s["sin"][s["positions"]][:, None]

    def forward(x, w):
        n = x.float() * (x.float().square().mean(-1, keepdim=True) + EPS).rsqrt()
        return _turn(s, n * w.float(), c, sn).to(dt)

    def backward(dy, x, w):
        r = (x.float().square().mean(-1, keepdim=True) + EPS).rsqrt()
        n, dm = x.float() * r, _turn(s, dy.float(), c, -sn)
        g = dm * w.float()
        return (r * (g - n * (g * n).mean(-1, keepdim=True))).to(dt), (dm * n).sum((0, 1))
    out = forward(s["q"], s["q_weight"]), forward(s["k"], s["k_weight"])
    if not s["train"]:
        return out
    dq, dwq = backward(s["dq"], s["q"], s["q_weight"])
    dk, dwk = backward(s["dk"], s["k"], s["k_weight"])
    return out + (dq, dk, dwq, dwk)


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "ffn":
        x, k, train = s["x"], s["hidden"], s["train"]
        lead = s["groups"] or 1
        w = [s[n].reshape(lead, *s[n].shape[-2:]) for n in ("w_gate", "w_up", "w_down")]
        y = torch.zeros(s["rows"], k, dtype=torch.float64, device=DEV)
        dx = torch.zeros_like(y)
        dw = [torch.zeros(v.shape, dtype=torch.float64, device=DEV) for v in w] if train else []
        at = 0
        for i, length in enumerate(s["lengths"]):  # one group after another, the gradients by reverse differentiation
            if length:
                own_rows = slice(at, at + length)
                leaves = [t.double().requires_grad_(train) for t in (x[own_rows], w[0][i], w[1][i], w[2][i])]
                g = leaves[0] @ leaves[1]
                a = g * torch.sigmoid(g) if s["act"] == "silu" else g * torch.special.ndtr(g)
                out = (a * (leaves[0] @ leaves[2])) @ leaves[3]
                y[own_rows] = out.detach()
                if train:
                    grads = torch.autograd.grad(out, leaves, s["dy"][own_rows].double())
                    dx[own_rows] = grads[0]
                    for v, grad in zip(dw, grads[1:]):
                        v[i] = grad
            at += length
        if not train:
            return y
        return (y, dx) + tuple(v.reshape(s[n].shape) for v, n in zip(dw, ("w_gate", "w_up", "w_down")))
    r = s["rotary"]
    # each pair as a complex number, turned by a product
    turn = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"]][:, None]

    def form(x, w):
        m = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w
        head = m[..., :r]
        z = torch.view_as_complex(head.unflatten(-1, (r // 2, 2)).contiguous()) if s["interleaved"] else \
            torch.complex(head[..., :r // 2], head[..., r // 2:])
        z = torch.view_as_real(z * turn)
        head = z.flatten(-2) if s["interleaved"] else torch.cat([z[..., 0], z[..., 1]], -1)
        return torch.cat([head, m[..., r:]], -1)
    out, grads, sums = [], [], []
    for n in ("q", "k"):
        leaves = [t.double().requires_grad_(s["train"]) for t in (s[n], s[n + "_weight"])]
        o = form(*leaves)
        out.append(o.detach())
        if s["train"]:
            dx, dw = torch.autograd.grad(o, leaves, s["d" + n].double())
            grads.append(dx)
            sums.append(dw)
        del o, leaves
    return tuple(out + grads + sums)


def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if case["op"] == "ffn":
        rows, k, n = case["rows"] - case["dropped"], case["hidden"], case["width"]
        weights = 3 * k * n * size * max(1, min(case["groups"], rows))
        # training: a forward and a backward call, each of which reads x and the weights; g and u in 32 bits
        # are the forward call's output and the backward call's input
        moved = 2 * rows * k * size + weights
        if case["train"]:
            moved += 3 * rows * k * size + 2 * weights + 2 * rows * 2 * n * 4
        return {"bytes": moved, "flops": (18 if case["train"] else 6) * rows * k * n}
    n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
    table = case["tokens"] * 8 + 8 * (case["rotary"] // 2) * max(1, min(case["tokens"], 32768))
    return {"bytes": n * size * (5 if case["train"] else 2) + table * (2 if case["train"] else 1),
            "flops": n * (26 if case["train"] else 8)}
