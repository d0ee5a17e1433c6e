"""The operators of a transformer block together and at their edges: a block's norms, rotation, routing and experts in
one run with its backward pass, calls in CUDA graphs, waits that run out, sizes whose offsets pass 32 bits, sums longer
than one accumulator takes, and what lies behind a workspace."""
import pytest
import torch

from paper_2607_20548_gb300 import (ffn_backward, ffn_forward, layer_norm_backward, layer_norm_forward,
                                    qk_rotary_backward, qk_rotary_forward, route_backward, route_forward)
from paper_2607_20548_gb300 import soap as S
from tests.test_gpu_ffn import _check, _operands, _run

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def _experts(cuda, t, tokens, hidden, width, experts, seed=0):
    g = torch.Generator(device=cuda).manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=cuda, generator=g)  # noqa: E731
    return dict(x=r(tokens, hidden).to(t), gain=(1 + 0.1 * r(hidden)), shift=0.1 * r(hidden),
                router=(r(hidden, experts) / hidden ** 0.5).float(), dy=(0.1 * r(tokens, hidden)).to(t),
                w=[(r(experts, hidden, width) / hidden ** 0.5).to(t), (r(experts, hidden, width) / hidden ** 0.5).to(t),
                   (r(experts, width, hidden) / width ** 0.5).to(t)])


def _moe(s, k):
    """Layer norm, a router's choice, the experts' feed-forward over the sorted choices, their sum with the gates; and
    the gradients of all of it."""
    n, mean, rstd = layer_norm_forward(s["x"], s["gain"], s["shift"])
    logits = n.float() @ s["router"]
    r = route_forward(logits, k, coef=0.02)
    flat = r.indices.flatten()
    order = torch.argsort(flat, stable=True)
    token = order // k
    offsets = torch.cat([torch.zeros(1, dtype=torch.int32, device=flat.device), r.counts.cumsum(0, dtype=torch.int32)])
    rows = n[token]
    y, pre = ffn_forward(rows, *s["w"], offsets=offsets, keep=True)
    gates = r.gates.flatten()[order]
    out = torch.zeros(s["x"].shape, device=flat.device).index_add_(0, token, y.float() * gates[:, None])
    # back
    dy = s["dy"].float()[token]
    dgates = torch.empty_like(gates)
    dgates[order] = (dy * y.float()).sum(-1)
    dz = route_backward(logits, r, dgates.view(r.gates.shape))
    dys = (dy * gates[:, None]).to(y.dtype)
    drows, *dw = ffn_backward(dys, rows, pre, *s["w"], offsets=offsets)
    dn = (dz @ s["router"].mT).index_add_(0, token, drows.float()).to(n.dtype)
    dx, dgain, dshift = layer_norm_backward(dn, s["x"], mean, rstd, s["gain"])
    return out, dx, dgain, dshift, n.float().mT @ dz, dw, r


def test_experts_layer_against_fp64(cuda):
    tokens, hidden, width, experts, k = 300, 96, 64, 6, 2
    s = _experts(cuda, F32, tokens, hidden, width, experts)
    out, dx, dgain, dshift, drouter, dw, r = _moe(s, k)
    leaf = {n: s[n].double().requires_grad_() for n in ("x", "gain", "shift", "router")}
    w = [m.double().requires_grad_() for m in s["w"]]
    n = torch.nn.functional.layer_norm(leaf["x"], (hidden,), leaf["gain"], leaf["shift"], 1e-5)
    p = (n @ leaf["router"]).softmax(-1)
    top = p.gather(-1, r.indices.long())
    gates = top / top.sum(-1, keepdim=True)
    want = torch.zeros_like(n)
    for e in range(experts):
        h = torch.nn.functional.silu(n @ w[0][e]) * (n @ w[1][e]) @ w[2][e]
        want = want + h * (gates * (r.indices == e)).sum(-1, keepdim=True)
    loss = 0.02 * experts / (k * tokens) * (r.counts.double() * p.mean(0)).sum()
    grads = torch.autograd.grad((want * s["dy"].double()).sum() + loss, [leaf[n] for n in ("x", "gain", "shift", "router")] + w)
    # every step is fp32 to a few dozen roundings of its terms' magnitudes; 1e-4 of a result's largest value is 1700 of
    # them, for sums of up to 96 x 64 terms of mixed signs
    for got, exact in zip([out, dx, dgain, dshift, drouter, *dw], [want.detach(), *grads]):
        assert float((got.double() - exact).abs().max()) <= 1e-4 * float(exact.abs().max())


def test_attention_inputs_against_fp64(cuda):
    tokens, hidden, heads, kv, dim = 70, 128, 4, 2, 32
    g = torch.Generator(device=cuda).manual_seed(1)
    r = lambda *s: torch.randn(*s, device=cuda, generator=g)  # noqa: E731
    x, wqkv = r(tokens, hidden), r(hidden, (heads + 2 * kv) * dim) / hidden ** 0.5
    gain, shift, wq, wk = 1 + 0.1 * r(hidden), 0.1 * r(hidden), 1 + 0.1 * r(dim), 1 + 0.1 * r(dim)
    angle = torch.arange(tokens, device=cuda, dtype=torch.float64)[:, None] / 100 ** (torch.arange(16, device=cuda) / 16)
    cos, sin = angle.cos().float(), angle.sin().float()
    n, mean, rstd = layer_norm_forward(x, gain, shift)
    qkv = (n @ wqkv).view(tokens, heads + 2 * kv, dim)
    q, k = qkv[:, :heads], qkv[:, heads:heads + kv]
    oq, ok = qk_rotary_forward(q, k, cos, sin, None, wq, wk)
    dq, dk = r(*q.shape), r(*k.shape)
    gq, gk, gwq, gwk = qk_rotary_backward(dq, dk, q, k, cos, sin, None, wq, wk)
    dqkv = torch.cat([gq, gk, torch.zeros_like(gk)], 1).view(tokens, -1)
    dx, dgain, _ = layer_norm_backward(dqkv @ wqkv.mT, x, mean, rstd, gain)
    xs, gs, ws, qs, ks = (v.double().requires_grad_() for v in (x, gain, wqkv, wq, wk))
    ref = (torch.nn.functional.layer_norm(xs, (hidden,), gs, shift.double(), 1e-5) @ ws).view(tokens, -1, dim)

    def turn(v, w):
        m = v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
        z = torch.complex(m[..., :16], m[..., 16:]) * torch.complex(cos.double(), sin.double())[:, None]
        return torch.cat([z.real, z.imag], -1)
    want = turn(ref[:, :heads], qs), turn(ref[:, heads:heads + kv], ks)
    grads = torch.autograd.grad((want[0] * dq.double()).sum() + (want[1] * dk.double()).sum(), [xs, gs, qs, ks])
    # as above (the plain products between the operators may round to tf32 nowhere: torch's default)
    for got, exact in zip([oq, ok, dx, dgain, gwq, gwk], [*(v.detach() for v in want), *grads]):
        assert float((got.double() - exact).abs().max()) <= 1e-4 * float(exact.abs().max())


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("rows,hidden,width,groups", [(5, 64, 96, 1), (40, 128, 200, 4), (600, 200, 136, 2), (90, 77, 51, 1)])
def test_replay(cuda, t, rows, hidden, width, groups):
    """Captured calls replay on new inputs, other offsets among them, with the bits that direct calls give."""
    def inputs(seed):
        g = torch.Generator(device=cuda).manual_seed(seed)
        cuts = torch.randint(0, rows + 1, (groups - 1,), device=cuda, generator=g).sort()[0]
        off = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), rows)]).int()
        x, dy, w, _ = _operands(cuda, [rows // groups] * groups, hidden, width, t, seed=seed)
        x, dy = (torch.randn(rows, hidden, device=cuda, generator=g).to(t) for _ in range(2))
        q, k = (torch.randn(rows, n, 64, device=cuda, generator=g).to(t) for n in (3, 1))
        pos = torch.randint(0, 50, (rows,), device=cuda, generator=g)
        return [x, dy, *w, off, q, k, pos]

    cos, sin = torch.randn(50, 16, device=cuda), torch.randn(50, 16, device=cuda)

    def step(x, dy, a, b, c, off, q, k, pos):
        y, pre = ffn_forward(x, a, b, c, offsets=off, keep=True)
        out = qk_rotary_forward(q, k, cos, sin, pos)
        return [y, *ffn_backward(dy, x, pre, a, b, c, offsets=off), *out, *qk_rotary_backward(*out, q, k, cos, sin, pos)]

    held = inputs(0)
    side = torch.cuda.Stream(cuda)
    side.wait_stream(torch.cuda.current_stream(cuda))
    with torch.cuda.stream(side):
        step(*held)
    torch.cuda.current_stream(cuda).wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*held)
    for seed in (1, 2):
        fresh = inputs(seed)
        for a, b in zip(held, fresh):
            a.copy_(b)
        graph.replay()
        graph.replay()
        for got, want in zip(out, step(*fresh)):
            assert torch.equal(got, want)


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("lengths", [[3], [300], [200, 0, 150], [1, 2, 3]])
def test_ffn_wait_runs_out(cuda, t, lengths):
    """While the flag is unset no unit is taken, the waits run out (20 ms) and all results are NaN."""
    x, dy, w, off = _operands(cuda, lengths, 64, 96, t)
    y, pre = ffn_forward(x, *w, offsets=off, keep=True)
    want = [y, *ffn_backward(dy, x, pre, *w, offsets=off)]

    def both(*status):
        a, b = status or (None, None)
        return [ffn_forward(x, *w, offsets=off, status=a)[0], *ffn_backward(dy, x, pre, *w, offsets=off, status=b)]
    status = [torch.zeros(1, dtype=torch.int32, device=cuda) for _ in range(2)]
    hold = torch.zeros(1, dtype=torch.int32, device=cuda)
    torch.cuda.synchronize()
    try:
        S.soap_wait_limit(20_000_000, hold)
        got = both(*status)
        torch.cuda.synchronize()
        hold.fill_(1)
        free = both()
        torch.cuda.synchronize()
    finally:
        S.soap_wait_limit(0, None)
    assert [int(s) for s in status] == [S.STATUS_TIMEOUT] * 2
    assert all(bool(v.isnan().all()) for v in got)
    clean = [torch.zeros(1, dtype=torch.int32, device=cuda) for _ in range(2)]
    again = both(*clean)
    assert [int(s) for s in clean] == [0, 0]
    for a, b, c in zip(want, free, again):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("t", [BF, F32])
def test_qk_wait_runs_out(cuda, t):
    q, k = torch.randn(4000, 8, 128, device=cuda).to(t), torch.randn(4000, 2, 128, device=cuda).to(t)
    want = [*qk_rotary_forward(q, k), *qk_rotary_backward(q, k, q, k)]
    status = [torch.zeros(1, dtype=torch.int32, device=cuda) for _ in range(2)]
    hold = torch.zeros(1, dtype=torch.int32, device=cuda)
    torch.cuda.synchronize()
    try:
        S.soap_wait_limit(20_000_000, hold)
        got = [*qk_rotary_forward(q, k, status=status[0]), *qk_rotary_backward(q, k, q, k, status=status[1])]
        torch.cuda.synchronize()
    finally:
        S.soap_wait_limit(0, None)
    assert [int(s) for s in status] == [S.STATUS_TIMEOUT] * 2
    assert all(bool(v.isnan().all()) for v in got)
    again = [*qk_rotary_forward(q, k), *qk_rotary_backward(q, k, q, k)]
    assert all(torch.equal(a, b) for a, b in zip(want, again))


@pytest.mark.parametrize("t", [BF, HF])
@pytest.mark.parametrize("lengths,hidden,width", [([140000], 64, 72), ([3, 70000, 0, 66000], 72, 64)])
def test_sums_longer_than_an_accumulator(cuda, t, lengths, hidden, width):
    _run(cuda, lengths, hidden, width, t)


def test_many_groups(cuda):
    g = torch.Generator().manual_seed(4)
    lengths = [int(v) if v < 40 else 0 for v in torch.randint(0, 60, (1024,), generator=g)]
    _run(cuda, lengths, 40, 24, BF, before=1, behind=7)
    lengths[500] = 3000
    _run(cuda, lengths[:700], 40, 24, HF)


def test_rows_past_32_bits(cuda):
    """x, y and their gradients of more than 2^31 elements, g and u of more than 2^29 bytes, each part as it should be
    (its bits may differ from a call of its own, whose sums may go in parts)."""
    rows, hidden, width = 1_100_000, 2048, 64
    g = torch.Generator(device=cuda).manual_seed(5)
    x = torch.empty(rows, hidden, dtype=BF, device=cuda)
    for part in x.split(100_000):
        part.copy_(torch.randn(part.shape, device=cuda, generator=g, dtype=BF))
    w = [torch.randn(a, b, device=cuda, generator=g).to(BF) / a ** 0.5 for a, b in ((hidden, width), (hidden, width), (width, hidden))]
    y, pre = ffn_forward(x, *w, keep=True)
    dx = ffn_backward(x, x, pre, *w, params=False)[0]
    for at in (0, 1 << 20, rows - 300):
        part = slice(at, at + 300)
        _check(x[part], w, "silu", y[part], x[part], (dx[part], None, None, None))


def test_heads_past_32_bits(cuda):
    tokens = 1_100_000
    q = torch.randn(tokens, 16, 128, device=cuda, dtype=HF)
    k = q[:, :2]
    angle = torch.arange(tokens, device=cuda)[:, None] * torch.logspace(0, -4, 64, device=cuda)
    cos, sin = angle.cos(), angle.sin()
    out = qk_rotary_forward(q, k, cos, sin)
    grads = qk_rotary_backward(q, k, q, k, cos, sin, params=False)
    for at in (0, tokens - 5000):
        part = slice(at, at + 5000)
        pos = torch.arange(at, at + 5000, device=cuda)
        a = qk_rotary_forward(q[part], k[part], cos, sin, pos)
        b = qk_rotary_backward(q[part], k[part], q[part], k[part], cos, sin, pos, params=False)
        assert torch.equal(out[0][part], a[0]) and torch.equal(out[1][part], a[1])
        assert torch.equal(grads[0][part], b[0]) and torch.equal(grads[1][part], b[1])


@pytest.mark.parametrize("rows,hidden,width,groups", [(1, 64, 64, 1), (60, 128, 1000, 1), (64, 64, 2100, 2), (65, 2048, 64, 1),
                                                      (300, 1600, 72, 3), (700, 256, 2048, 1), (129, 65, 33, 5)])
@pytest.mark.parametrize("t", [BF, F32])
def test_nothing_behind_the_workspace(cuda, t, rows, hidden, width, groups):
    """Calls get a workspace of just the size that is asked for, and leave what lies behind it alone."""
    lib, dt = S.load_library(), S.DTYPES[t]
    off = torch.tensor([rows * i // groups for i in range(groups + 1)], dtype=torch.int32, device=cuda)
    x, w, d = (torch.randn(*s, device=cuda).to(t) for s in ((rows, hidden), (groups, hidden, width), (groups, width, hidden)))
    y, grads = torch.empty_like(x), [torch.empty_like(m) for m in (w, w, d)]
    mat = lambda m: S.layer_matrix(m.data_ptr(), m.shape[-1], m.shape[-1] * m.shape[-2], 0)  # noqa: E731
    pre = torch.empty(lib.layer_ffn_pre_elems(rows, width, groups) + 64, device=cuda)
    pre.fill_(7.0)
    mats, stream = (mat(w), mat(w), mat(d)), torch.cuda.current_stream(cuda).cuda_stream
    for back in (0, 1):
        size = lib.layer_ffn_workspace_bytes(rows, hidden, width, groups, dt, hidden % 8 == width % 8 == 0, back)
        ws = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device=cuda)
        head = (rows, hidden, width, groups, off.data_ptr())
        tail = (None, ws.data_ptr(), size, stream)
        if back:
            code = lib.layer_ffn_backward(*head, x.data_ptr(), hidden, x.data_ptr(), hidden, dt, *mats, 0, pre.data_ptr(),
                                          y.data_ptr(), hidden, *(mat(m) for m in grads), *tail)
        else:
            code = lib.layer_ffn_forward(*head, x.data_ptr(), hidden, dt, *mats, 0, y.data_ptr(), hidden, pre.data_ptr(), *tail)
        assert code == 0
        assert bool((ws[size:] == 0xA5).all()) and bool((pre[-64:] == 7.0).all())


def test_operands_off_their_units(cuda):
    """Operands that begin inside a 16-byte unit are copied; results of a leading dimension of their own."""
    x, dy, w, _ = _operands(cuda, [50], 64, 80, BF, dense=True, seed=3)
    move = lambda t: torch.cat([t.new_zeros(3), t.flatten()])[3:].view(t.shape)  # noqa: E731
    y, pre = ffn_forward(x, *w, keep=True)
    grads = ffn_backward(dy, x, pre, *w)
    ms = [move(m) for m in w]
    y2, pre2 = ffn_forward(move(x), *ms, keep=True)
    assert torch.equal(y, y2)
    assert all(torch.equal(a, b) for a, b in zip(grads, ffn_backward(move(dy), move(x), pre2, *ms)))
    _check(x, w, "silu", y, dy, grads)


@pytest.mark.parametrize("tokens,dim", [(3, 64), (4000, 128), (900, 50)])
@pytest.mark.parametrize("t", [BF, F32])
def test_heads_in_place(cuda, t, tokens, dim):
    """Results over their operands (C interface): the bits of results of their own."""
    lib, dt = S.load_library(), S.DTYPES[t]
    q, k = torch.randn(tokens, 6, dim, device=cuda).to(t), torch.randn(tokens, 2, dim, device=cuda).to(t)
    dq, dk = torch.randn(q.shape, device=cuda).to(t), torch.randn(k.shape, device=cuda).to(t)
    w = 1 + 0.1 * torch.randn(dim, device=cuda)
    cos, sin = torch.randn(tokens, dim // 2, device=cuda), torch.randn(tokens, dim // 2, device=cuda)
    want = qk_rotary_forward(q, k, cos, sin, None, w, w)
    back = qk_rotary_backward(dq, dk, q, k, cos, sin, None, w, w)
    h = lambda v: S.layer_heads(v.data_ptr(), 0, v.stride(0), v.stride(1))  # noqa: E731
    sizes = (1, tokens, 6, 2, dim, dim, 0)
    how = (dt, w.data_ptr(), w.data_ptr(), 0, 1e-6, cos.data_ptr(), sin.data_ptr(), tokens, None, 0)
    stream = torch.cuda.current_stream(cuda).cuda_stream
    a, b = q.clone(), k.clone()
    assert lib.layer_qk_forward(*sizes, h(a), h(b), *how, h(a), h(b), None, stream) == 0
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    size = lib.layer_qk_workspace_bytes(1, tokens, 6, 2, dim)
    ws, dw = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device=cuda), torch.empty(2, dim, device=cuda)
    for over_q in (False, True):
        a, b, c, d = dq.clone(), dk.clone(), q.clone(), k.clone()
        to = (c, d) if over_q else (a, b)
        assert lib.layer_qk_backward(*sizes, h(a), h(b), h(c), h(d), *how, h(to[0]), h(to[1]), dw[0].data_ptr(),
                                     dw[1].data_ptr(), None, ws.data_ptr(), size, stream) == 0
        assert torch.equal(to[0], back[0]) and torch.equal(to[1], back[1])
        assert torch.equal(dw[0], back[2]) and torch.equal(dw[1], back[3])
    assert bool((ws[size:] == 0xA5).all())
