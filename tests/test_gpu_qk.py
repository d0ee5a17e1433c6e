"""Queries' and keys' norms with the rotation by position (include/layer.h, layer_qk_*) against fp64.

Tolerance (from the arithmetic): with u = 2^-24, a lane adds 16 squares in order and up to 32 lanes' sums pairwise:
the sum is within 22 u of itself, r within 11 u, the two roundings of the mean and of eps's addition, half of which reach it, and the root's 4 u; n and m add one each and the rotation two of its own terms: within 24 u of the terms' magnitudes, and one
rounding to the type. The gradients' terms in the same way: dm within 2 u of its terms, sums of products with it
within 26 u of the sum of magnitudes. dweight adds up a warp's heads (at most 2 + tokens heads / 2400 of them
in order), then at most 5 + 8 + 40 + 16 partial sums.
"""
import pytest
import torch

from paper_2607_20548_gb300 import qk_rotary_backward, qk_rotary_forward
from paper_2607_20548_gb300 import soap as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
ROUND = {t: torch.finfo(t).eps / 2 for t in (F32, BF, HF)}
TINY = {F32: 1e-37, BF: 1e-37, HF: 2.0 ** -25}  # half a subnormal step


def _turn(m, c, s, inter):
    r = 2 * c.shape[-1]
    if inter:
        a, b = m[..., 0:r:2], m[..., 1:r:2]
        t = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = m[..., :r // 2], m[..., r // 2:r]
        t = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([t, m[..., r:]], -1)


def _terms(m, c, s, inter):
    """The sum of the magnitudes of the rotation's terms: |a c| + |b s|, |b c| + |a s|."""
    r = 2 * c.shape[-1]
    m, c, s = m.abs(), c.abs(), s.abs()
    if inter:
        a, b = m[..., 0:r:2], m[..., 1:r:2]
        t = torch.stack([a * c + b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = m[..., :r // 2], m[..., r // 2:r]
        t = torch.cat([a * c + b * s, b * c + a * s], -1)
    return torch.cat([t, m[..., r:]], -1)


def _close(got, want, slack):
    assert got.shape == want.shape
    bound = ROUND[got.dtype] * want.abs() * 1.001 + slack + TINY[got.dtype]
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())


def _table(cuda, places, rotary):
    at = torch.arange(places, device=cuda, dtype=torch.float64)[:, None] * 100.0 ** (
        -torch.arange(0, rotary, 2, device=cuda, dtype=torch.float64) / max(rotary, 1))
    return at.cos().float(), at.sin().float()


def _check(q, k, cos, sin, pos, wq, wk, eps, inter, dq=None, dk=None, out=None, grads=None):
    lead = q.shape[:-2]
    if cos is None:
        cos = sin = torch.zeros(1, 0, device=q.device)
        at = torch.zeros(lead, dtype=torch.int64, device=q.device)
    else:
        at = (torch.arange(lead[-1] if lead else 1, device=q.device) if pos is None else pos).expand(lead).long()
    c, s = cos.double()[at][..., None, :], sin.double()[at][..., None, :]
    for i, (x, w, d) in enumerate(((q, wq, dq), (k, wk, dk))):
        x = x.double()
        w = torch.ones(x.shape[-1], device=x.device, dtype=torch.float64) if w is None else w.double()
        r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
        n = x * r
        if out is not None:
            _close(out[i], _turn(n * w, c, s, inter), 24 * U * _terms(n * w, c, s, inter))
        if grads is None:
            continue
        dm, big = _turn(d.double(), c, -s, inter), _terms(d.double(), c, s, inter)
        g = dm * w
        mean = (g * n).mean(-1, keepdim=True)
        slack = 24 * U * r * (big * w.abs() + n.abs() * mean.abs()) \
            + 64 * U * r * n.abs() * (big * w.abs() * n.abs()).mean(-1, keepdim=True)
        _close(grads[i], r * (g - n * mean), slack)
        if grads[2 + i] is not None:
            many = x.numel() // x.shape[-1]
            dims = tuple(range(x.dim() - 1))
            err = (grads[2 + i].double() - (dm * n).sum(dims)).abs()
            assert bool((err <= (100 + many / 2400) * U * (big * n.abs()).sum(dims) + 1e-37).all())


def _run(cuda, lead, heads, kv, dim, rotary, inter, t, wt, seed=0, pos_t=torch.int64, make=None, places=97):
    g = torch.Generator(device=cuda).manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=cuda, generator=g)  # noqa: E731
    make = make or (lambda n: (r(*lead, n, dim) * (0.2 + r(*lead, n, 1).abs())).to(t))
    q, k = make(heads), make(kv)
    wq, wk = ((1 + 0.2 * r(dim)).to(wt) if wt else None for _ in range(2))
    dq, dk = (0.1 * r(*q.shape)).to(t), (0.1 * r(*k.shape)).to(t)
    cos, sin = _table(cuda, places, rotary) if rotary else (None, None)
    pos = torch.randint(0, places, lead, device=cuda, generator=g).to(pos_t) if rotary else None
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    how = dict(cos=cos, sin=sin, positions=pos, q_weight=wq, k_weight=wk, eps=1e-5, interleaved=inter, status=status)
    out = qk_rotary_forward(q, k, **how)
    grads = qk_rotary_backward(dq, dk, q, k, **how)
    assert all(a.dtype == t for a in out + grads[:2]) and grads[2].dtype == grads[3].dtype == F32
    _check(q, k, cos, sin, pos, wq, wk, 1e-5, inter, dq, dk, out, grads)
    assert int(status) == 0


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("t,wt", [(BF, F32), (BF, BF), (HF, HF), (F32, F32), (HF, None)])
@pytest.mark.parametrize("lead,heads,kv,dim,rotary", [
    ((1,), 16, 4, 128, 128), ((37,), 7, 3, 80, 40), ((3, 5), 2, 1, 2, 2), ((9,), 5, 5, 50, 14), ((4,), 33, 1, 64, 0),
    ((2, 11), 3, 3, 512, 512), ((13,), 1, 1, 96, 96), ((6,), 4, 2, 256, 128), ((5,), 3, 2, 510, 510), ((5,), 9, 2, 66, 66),
    ((700,), 20, 3, 32, 16), ((8,), 2, 2, 192, 190), ((), 3, 1, 36, 20)])
def test_against_fp64(cuda, lead, heads, kv, dim, rotary, t, wt, inter):
    _run(cuda, lead, heads, kv, dim, rotary, inter, t, wt)


@pytest.mark.parametrize("t", [BF, F32])
def test_many_tokens(cuda, t):
    _run(cuda, (20011,), 6, 2, 128, 64, False, t, F32, pos_t=torch.int32)
    _run(cuda, (3, 3001), 5, 1, 70, 70, True, t, F32)


@pytest.mark.parametrize("name", ["fused", "heads_first", "odd_start", "apart", "expanded"])
def test_layouts(cuda, name):
    lead, dim = (3, 10), 64
    g = torch.Generator(device=cuda).manual_seed(5)

    def make(n):
        r = lambda *s: torch.randn(*s, device=cuda, generator=g).bfloat16()  # noqa: E731
        if name == "fused":
            return r(3, 10, 9, dim)[:, :, 9 - n:]
        if name == "heads_first":
            return r(3, n, 10, dim).transpose(1, 2)
        if name == "odd_start":
            return r(3, 10, n, dim + 3)[..., 3:]
        if name == "apart":
            return r(3, 10, n, 2 * dim)[..., ::2]
        return r(1, 10, 1, dim).expand(3, 10, n, dim)
    _run(cuda, lead, 4, 2, dim, dim, False, BF, BF, make=make)


def test_positions_default_and_of_a_sequence(cuda):
    q, k = torch.randn(2, 12, 3, 32, device=cuda), torch.randn(2, 12, 1, 32, device=cuda)
    cos, sin = _table(cuda, 12, 32)
    a = qk_rotary_forward(q, k, cos, sin)
    _check(q, k, cos, sin, None, None, None, 1e-6, False, out=a)
    for pos in (torch.arange(12, device=cuda), torch.arange(12, device=cuda).expand(2, 12)):
        b = qk_rotary_forward(q, k, cos, sin, pos)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_positions_out_of_range(cuda):
    q, k, w = torch.randn(5, 2, 16, device=cuda), torch.randn(5, 1, 16, device=cuda), torch.ones(16, device=cuda)
    cos, sin = _table(cuda, 8, 16)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    pos = torch.tensor([0, 8, -1, 1 << 40, 7], device=cuda)
    out = qk_rotary_forward(q, k, cos, sin, pos, w, w, status=status)
    assert int(status) == S.STATUS_RANGE
    good = torch.tensor([0, 4], device=cuda)
    for o in out:
        assert bool(o[1:4].isnan().all()) and bool(o[good].isfinite().all())
    status.zero_()
    grads = qk_rotary_backward(q, k, q, k, cos, sin, pos, w, w, status=status)
    assert int(status) == S.STATUS_RANGE
    for o in grads[:2]:
        assert bool(o[1:4].isnan().all()) and bool(o[good].isfinite().all())
    assert bool(grads[2].isnan().all()) and bool(grads[3].isnan().all())


def test_bad_heads_stay_to_themselves(cuda):
    q, k = torch.randn(6, 4, 64, device=cuda).bfloat16(), torch.randn(6, 2, 64, device=cuda).bfloat16()
    cos, sin = _table(cuda, 6, 64)
    want = qk_rotary_forward(q, k, cos, sin)
    q[2, 1, 5], q[3, 0, 0], q[4, 3] = float("inf"), float("nan"), 0.0
    got = qk_rotary_forward(q, k, cos, sin)
    assert bool((got[0][4, 3] == 0).all()) and torch.equal(got[1], want[1])
    same = torch.ones(6, 4, dtype=torch.bool, device=cuda)
    same[2, 1] = same[3, 0] = same[4, 3] = False
    assert torch.equal(got[0][same], want[0][same])
    assert bool(got[0][3, 0].isnan().all()) and not bool(got[0][2, 1].isfinite().all())


def test_nothing_to_do_and_without_params(cuda):
    cos, sin = _table(cuda, 4, 8)
    q, k = torch.randn(0, 2, 8, device=cuda), torch.randn(0, 1, 8, device=cuda)
    assert qk_rotary_forward(q, k, cos, sin)[0].shape == q.shape
    grads = qk_rotary_backward(q, k, q, k, cos, sin)
    assert bool((grads[2] == 0).all()) and bool((grads[3] == 0).all())
    q, k = torch.randn(3, 2, 8, device=cuda), torch.randn(3, 0, 8, device=cuda)
    full = qk_rotary_backward(q, k, q, k, cos, sin)
    part = qk_rotary_backward(q, k, q, k, cos, sin, params=False)
    assert part[2] is part[3] is None and torch.equal(part[0], full[0]) and bool((full[3] == 0).all())


def test_other_stream_and_repeatable(cuda):
    q, k = torch.randn(500, 8, 128, device=cuda).bfloat16(), torch.randn(500, 2, 128, device=cuda).bfloat16()
    cos, sin = _table(cuda, 500, 128)
    a = qk_rotary_forward(q, k, cos, sin) + qk_rotary_backward(q, k, q, k, cos, sin)
    side = torch.cuda.Stream(cuda)
    side.wait_stream(torch.cuda.current_stream(cuda))
    b = qk_rotary_forward(q, k, cos, sin, stream=side) + qk_rotary_backward(q, k, q, k, cos, sin, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_gradients_against_differences(cuda):
    g = torch.Generator(device=cuda).manual_seed(3)
    q, k = (torch.randn(2, n, 12, device=cuda, generator=g) for n in (2, 1))
    wq, wk = (1 + 0.1 * torch.randn(12, device=cuda, generator=g) for _ in range(2))
    dq, dk = torch.randn(q.shape, device=cuda, generator=g), torch.randn(k.shape, device=cuda, generator=g)
    cos, sin = _table(cuda, 2, 8)

    def value(q, k, wq, wk):
        a, b = qk_rotary_forward(q, k, cos, sin, None, wq, wk)
        return float((a.double() * dq).sum() + (b.double() * dk).sum())
    grads = qk_rotary_backward(dq, dk, q, k, cos, sin, None, wq, wk)
    # central differences of step h: the third derivative's h^2 (of order one here, times 40 terms) and the values'
    # rounding, 40 terms of 24 u each of order one, over h
    h = 2.0 ** -7
    tol = 40 * h * h + 40 * 24 * U / h
    for i, (t, grad) in enumerate(zip((q, k, wq, wk), grads)):
        for e in range(0, t.numel(), 5):
            ends = []
            for sign in (1, -1):
                args = [x.clone() for x in (q, k, wq, wk)]
                args[i].view(-1)[e] += sign * h
                ends.append((value(*args), float(args[i].view(-1)[e])))
            slope = (ends[0][0] - ends[1][0]) / (ends[0][1] - ends[1][1])
            assert abs(slope - float(grad.view(-1)[e])) <= tol


def test_binding_refusals(cuda):
    q, k = torch.randn(4, 2, 8, device=cuda), torch.randn(4, 1, 8, device=cuda)
    cos, sin = _table(cuda, 4, 8)
    w = torch.ones(8, device=cuda)
    for args, kw in (((q, k[:3], cos, sin), {}), ((q, k[..., :6], cos, sin), {}), ((q, k, cos, None), {}),
                     ((q, k, cos[:, :2], sin), {}), ((q[..., :6], k[..., :6], cos, sin), {}),
                     ((q, k, cos, sin, torch.arange(3, device=cuda)), {}), ((q, k, cos, sin), dict(q_weight=w[:4])),
                     ((q[..., :7], k[..., :7]), {}), ((q[0, 0], k, cos, sin), {})):
        with pytest.raises(ValueError):
            qk_rotary_forward(*args, **kw)
    for args in ((q, k.half(), cos, sin), (q, k, cos.double(), sin), (q, k, cos, sin, torch.ones(4, device=cuda)),
                 (q.cpu(), k, cos, sin), (q.double(), k.double(), cos, sin)):
        with pytest.raises(TypeError):
            qk_rotary_forward(*args)
    with pytest.raises(ValueError):
        qk_rotary_backward(q[:3], k, q, k, cos, sin)
    with pytest.raises(S.SoapError):
        qk_rotary_forward(q, k, cos, sin, eps=-1.0)
