"""Expert routing and its gradient (include/layer.h) against fp64.

Choices and counts are compared exactly: both sides order the logits themselves, which are the same
numbers in both, ties by the lower index. Tolerance of the rest (from the arithmetic, u = 2^-24):
exp's argument z - max is exact to |z - max| u and the exponential to a few units more, so a
probability's relative error is within (32 + 4 |z - max|) u, here |z - max| < 30; sums over a row
and over tokens keep within 100 u + tokens / 600 u of their magnitudes; gradients are products and
differences of such terms, rounded once to the logits' type.
"""
import pytest
import torch

from paper_2607_20548_gb300 import route_backward, route_forward
from paper_2607_20548_gb300 import soap as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
REL = 152 * U
OUT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}  # one rounding
INF = float("inf")


def _ref(z, k, mask, normalize, coef, dgates=None, dloss=1.0):
    z = z.double().cpu()
    t, e = z.shape
    live = torch.ones(t, dtype=torch.bool) if mask is None else mask.cpu().clone()
    live &= (z > -INF).any(1) | z.isnan().any(1)
    z = torch.where(live[:, None], z, torch.zeros_like(z))
    p = torch.softmax(z, 1) * live[:, None]
    order = torch.sort(z, dim=1, descending=True, stable=True)
    idx, top = order.indices[:, :k], order.values[:, :k]
    ok = live[:, None] & (top > -INF)
    pc = p.gather(1, idx) * ok
    total = pc.sum(1, keepdim=True)
    gates = torch.where(ok, pc / total, pc) if normalize else pc
    hot = torch.zeros(t, e, dtype=torch.float64).scatter_(1, idx, ok.double())
    counts, n = hot.sum(0), int(live.sum())
    mean = p.sum(0) / max(n, 1)
    loss = coef * e / (k * max(n, 1)) * float((counts * mean).sum())
    out = dict(indices=torch.where(ok, idx, torch.full_like(idx, -1)), gates=gates, counts=counts, mean=mean, loss=loss,
               n=n, p=p)
    up = coef * dloss * e / (k * max(n, 1) ** 2) * counts[None, :].expand(t, e)
    d = torch.zeros(t, k, dtype=torch.float64) if dgates is None else dgates.double().cpu() * ok
    if normalize:
        d = torch.where(ok, (d - (d * gates).sum(1, keepdim=True)) / total, d)
    u = up.clone().scatter_add_(1, idx, d)
    out["dz"] = p * (u - (p * u).sum(1, keepdim=True))
    # magnitudes of the gradient's terms (the gates' gradient is itself a difference)
    dm = torch.zeros(t, k, dtype=torch.float64) if dgates is None else dgates.double().cpu().abs() * ok
    if normalize:
        dm = torch.where(ok, (dm + (dm * gates).sum(1, keepdim=True)) / total, dm)
    um = up.abs().clone().scatter_add_(1, idx, dm)
    out["mag"] = p * (um + (p * um).sum(1, keepdim=True))
    return out


def _check(cuda, z, k, mask=None, normalize=True, coef=0.02, dloss=1.5, grads=True, seed=1):
    g = torch.Generator(device=cuda).manual_seed(seed)
    dg = torch.randn(z.shape[0], k, device=cuda, generator=g) if grads else None
    want = _ref(z, k, mask, normalize, coef, dg, dloss)
    r = route_forward(z, k, mask=mask, normalize=normalize, coef=coef)
    assert r.indices.dtype == r.counts.dtype == torch.int32 and r.gates.dtype == torch.float32
    assert torch.equal(r.indices.cpu().long(), want["indices"])
    assert torch.equal(r.counts.cpu().double(), want["counts"]) and int(r.live) == want["n"]
    assert bool(((r.gates.cpu().double() - want["gates"]).abs() <= REL * 2 * want["gates"]).all())
    rel = REL + z.shape[0] / 600 * U
    assert bool(((r.mean_probs.cpu().double() - want["mean"]).abs() <= rel * want["mean"] + 1e-30).all())
    assert abs(float(r.loss) - want["loss"]) <= rel * want["loss"]
    dz = route_backward(z, r, dgates=dg, dloss=dloss)
    assert dz.dtype == z.dtype and dz.shape == z.shape
    err = (dz.cpu().double() - want["dz"]).abs()
    tiny = 2.0 ** -25 if z.dtype == torch.float16 else 1e-37
    bound = OUT[z.dtype] * want["dz"].abs() * 1.001 + 4 * REL * want["mag"] + tiny
    assert bool((err <= bound).all()), float((err / bound).max())
    return r


def _logits(cuda, t, e, dtype, seed=0):
    g = torch.Generator(device=cuda).manual_seed(seed)
    return (torch.randn(t, e, device=cuda, generator=g) + torch.randn(e, device=cuda, generator=g)).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t,e,k", [(1, 1, 1), (1, 64, 8), (2, 8, 8), (5, 3, 2), (37, 7, 1), (64, 16, 4), (100, 17, 5),
                                   (33, 32, 32), (1000, 33, 3), (513, 64, 6), (129, 127, 6), (70, 128, 8), (65, 200, 9),
                                   (40, 256, 8), (31, 500, 10), (17, 1024, 32)])
@pytest.mark.parametrize("normalize", [True, False])
def test_sizes(cuda, t, e, k, dtype, normalize):
    _check(cuda, _logits(cuda, t, e, dtype, seed=t + e), k, normalize=normalize)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_tokens_and_same_bits(cuda, dtype):
    z = _logits(cuda, 30011, 60, dtype)
    g = torch.Generator(device=cuda).manual_seed(2)
    mask = torch.rand(30011, device=cuda, generator=g) < 0.7
    r = _check(cuda, z, 4, mask=mask)
    again = route_forward(z, 4, mask=mask, coef=0.02)
    for a, b in zip(r[:6], again[:6]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("e,k", [(1, 1), (8, 2), (31, 3), (33, 8), (64, 8), (127, 6), (190, 4), (193, 7), (384, 5), (61, 9)])
@pytest.mark.parametrize("normalize", [True, False])
def test_many_tokens_sizes(cuda, e, k, dtype, normalize):
    """Enough tokens for a thread each, around the sizes where the layout of a row changes, with padding,
    an unavailable expert, ties and rows that cannot fill their choice."""
    t = 15000 + e
    z = _logits(cuda, t, e, dtype, seed=e)
    z[100:200] = z[100:200].round()
    if e > 2 * k:
        z[:, e // 2] = -INF
        z[300, k - 1:] = -INF
    if e > 1:
        z[301] = -INF
    g = torch.Generator(device=cuda).manual_seed(e)
    mask = torch.rand(t, device=cuda, generator=g) < 0.9
    z[~mask] = float("nan")
    _check(cuda, z, k, mask=mask, normalize=normalize)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("e,k", [(64, 8), (127, 6)])
def test_many_tokens_layouts_and_nonfinite(cuda, e, k, dtype):
    """A thread per token: the same bits for any alignment and leading dimension; rows with NaN (of either
    sign) or +inf; the gradient written over the logits."""
    z = _logits(cuda, 20000, e, dtype, seed=3)
    want = route_forward(z, k)
    dwant = route_backward(z, want, dgates=torch.ones_like(want.gates))
    for pad, off in ((8, 8), (1, 1), (2, 0), (4, 2)):
        big = torch.full((20000, e + pad), float("nan"), device=cuda, dtype=dtype)
        v = big[:, off:off + e]
        v.copy_(z)
        got = route_forward(v, k)
        assert all(torch.equal(a, b) for a, b in zip(want[:6], got[:6]))
        assert torch.equal(route_backward(v, got, dgates=torch.ones_like(got.gates)), dwant)
    z[7, 3], z[8, 0], z[9, 1] = float("nan"), INF, -float("nan")
    z[10] = -INF
    z[10, 2] = -float("nan")
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    r = route_forward(z, k, status=status)
    assert int(status) == S.STATUS_NONFINITE and r.loss.isnan()
    bad = torch.zeros(20000, dtype=torch.bool, device=cuda)
    bad[7:11] = True
    assert (r.indices[bad] == -1).all() and r.gates[bad].isnan().all() and r.gates[~bad].isfinite().all()
    assert torch.equal(r.indices[~bad], want.indices[~bad]) and int(r.live) == 20000
    dz = route_backward(z, r, dgates=torch.ones_like(r.gates))
    assert dz[bad].isnan().all() and dz[~bad].isfinite().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("e,k", [(6, 3), (64, 8), (100, 5), (300, 7)])
def test_ties_go_to_the_lower_index(cuda, e, k, dtype):
    g = torch.Generator(device=cuda).manual_seed(e)
    z = torch.randint(-1, 2, (200, e), device=cuda, generator=g).to(dtype)
    z[0] = 0
    z[1, ::2] = -0.0  # equal to +0
    z[1, 1::2] = 0.0
    _check(cuda, z, k)


@pytest.mark.parametrize("e,k", [(8, 2), (64, 8), (127, 6)])
@pytest.mark.parametrize("normalize", [True, False])
def test_masked_rows_and_unavailable_experts(cuda, e, k, normalize):
    """Masked rows hold anything; -inf logits are never chosen, down to rows with fewer than k left and rows
    with none, which are not counted; a type's lowest value is a logit like others."""
    z = _logits(cuda, 96, e, torch.float32)
    mask = torch.ones(96, dtype=torch.bool, device=cuda)
    for i, v in enumerate((float("nan"), INF, -INF, 3e38)):
        z[i], mask[i] = v, False
    z[:, 1] = -INF
    z[10, :] = -INF
    z[11, 1:] = -INF
    z[12, 2:] = torch.finfo(torch.float32).min
    z[13] = torch.finfo(torch.float32).min
    z[14, k - 1:] = -INF
    r = _check(cuda, z, k, mask=mask, normalize=normalize)
    # expert 1 is left in row 13 alone, where all logits are equal: its first k are chosen
    assert int(r.counts[1]) == 1 and int(r.live) == 91
    assert (r.indices[10] == -1).all() and not r.gates[10].any()
    assert int(r.indices[11, 0]) == 0 and (r.indices[11, 1:] == -1).all()


def test_nothing_left(cuda):
    z = _logits(cuda, 50, 64, torch.bfloat16)
    mask = torch.zeros(50, dtype=torch.bool, device=cuda)
    r = route_forward(z, 8, mask=mask)
    assert float(r.loss) == 0.0 and int(r.live) == 0 and not r.counts.any() and not r.mean_probs.any()
    assert (r.indices == -1).all() and not r.gates.any()
    assert not route_backward(z, r, dgates=torch.ones_like(r.gates)).any()
    empty = z[:0]
    r = route_forward(empty, 8)
    assert r.indices.shape == (0, 8) and float(r.loss) == 0.0 and not r.counts.any() and int(r.live) == 0
    assert route_backward(empty, r).shape == (0, 64)


@pytest.mark.parametrize("e", [8, 64, 300])
def test_nonfinite(cuda, e):
    z = _logits(cuda, 40, e, torch.float32)
    z[3, 2], z[7, 5] = -float("nan"), INF
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    r = route_forward(z, 4, status=status)
    assert int(status) == S.STATUS_NONFINITE
    bad = torch.zeros(40, dtype=torch.bool, device=cuda)
    bad[3] = bad[7] = True
    assert (r.indices[bad] == -1).all() and r.gates[bad].isnan().all() and r.gates[~bad].isfinite().all()
    assert r.loss.isnan() and int(r.counts.sum()) == 38 * 4
    dz = route_backward(z, r, dgates=torch.ones_like(r.gates))
    assert dz[bad].isnan().all() and dz[~bad].isfinite().all()


def test_balanced_choice_and_layouts(cuda):
    # every expert the same number of times, even probabilities: the loss is coef
    z = torch.zeros(64, 64, device=cuda)
    z[torch.arange(64), torch.arange(64)] = 1e-3
    assert abs(float(route_forward(z, 1, coef=0.5).loss) - 0.5) <= 0.5 * REL
    z = _logits(cuda, 30, 64, torch.bfloat16)
    want = route_forward(z, 8)
    for pad, off in ((8, 8), (1, 1), (2, 0)):
        big = torch.full((30, 64 + pad), float("nan"), device=cuda, dtype=torch.bfloat16)
        v = big[:, off:off + 64]
        v.copy_(z)
        got = route_forward(v, 8)
        assert all(torch.equal(a, b) for a, b in zip(want[:6], got[:6]))
        assert torch.equal(route_backward(v, got), route_backward(z, want))
    z3 = z.view(2, 15, 64)
    got = route_forward(z3, 8, mask=torch.ones(2, 15, dtype=torch.bool, device=cuda))
    assert got.indices.shape == (2, 15, 8) and torch.equal(got.gates.view(30, 8), want.gates)
    assert route_backward(z3, got).shape == z3.shape


@pytest.mark.parametrize("normalize", [True, False])
def test_against_differences(cuda, normalize):
    """<dz, d> against central differences of loss + sum(c gates), with the counts' part held constant by
    taking the loss's derivative at fixed counts: sum_e counts_e mean_probs_e. 1e-3 of the terms covers the
    truncation and fp32 rounding over the step."""
    z = _logits(cuda, 40, 24, torch.float32, seed=4)
    g = torch.Generator(device=cuda).manual_seed(8)
    c = torch.randn(40, 3, device=cuda, generator=g) / 40
    r = route_forward(z, 3, normalize=normalize, coef=0.7)
    dz = route_backward(z, r, dgates=c, dloss=2.0)
    h = 2.0 ** -9
    counts = r.counts.double()
    for seed in range(4):
        d = torch.randn(z.shape, device=cuda, generator=g)
        ends = []
        for s in (h, -h):
            q = route_forward(z + s * d, 24, normalize=False)  # every expert's probability
            p = torch.zeros(40, 24, device=cuda).scatter_(1, q.indices.long(), q.gates).double()
            pc = p.gather(1, r.indices.long())
            gates = pc / pc.sum(1, keepdim=True) if normalize else pc
            ends.append(float(2.0 * 0.7 * 24 / (3 * 40) * (counts * p.sum(0)).sum() / 40 + (c.double() * gates).sum()))
        diff = (ends[0] - ends[1]) / (2 * h)
        terms = float((dz.double() * d.double()).abs().sum())
        assert abs(diff - float((dz.double() * d.double()).sum())) <= 1e-3 * terms


def test_other_stream(cuda):
    z = _logits(cuda, 5000, 64, torch.bfloat16)
    want = route_forward(z, 8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = route_forward(z, 8, stream=s)
    dz = route_backward(z, got, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want[:6], got[:6])) and torch.equal(dz, route_backward(z, want))


def test_refusals(cuda):
    z = _logits(cuda, 8, 16, torch.float32)
    r = route_forward(z, 2)
    with pytest.raises(TypeError):
        route_forward(z.cpu(), 2)
    with pytest.raises(TypeError):
        route_forward(z.double(), 2)
    for k in (0, 17, -1):
        with pytest.raises(ValueError):
            route_forward(z, k)
    with pytest.raises(ValueError):
        route_forward(torch.zeros(2, 1025, device=cuda), 2)
    with pytest.raises(ValueError):
        route_forward(torch.zeros(2, 64, device=cuda), 33)
    with pytest.raises(ValueError):
        route_forward(z, 2, mask=torch.ones(7, dtype=torch.bool, device=cuda))
    with pytest.raises(TypeError):
        route_forward(z, 2, mask=torch.ones(8, device=cuda))
    with pytest.raises(S.SoapError):
        route_forward(z, 2, coef=float("inf"))
    with pytest.raises(ValueError):
        route_backward(z[:4], r)
    with pytest.raises(ValueError):
        route_backward(z, r, dgates=torch.zeros(8, 3, device=cuda))
    with pytest.raises(TypeError):
        route_backward(z, r, dgates=torch.zeros(8, 2, device=cuda, dtype=torch.bfloat16))
