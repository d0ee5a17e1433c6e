"""The gated feed-forward block and its backward pass (include/layer.h, layer_ffn_*) against fp64.

Tolerance (from the arithmetic). u is an fp32 rounding, t a rounding to the operands' type. A sum of K products in
fp32, added up in runs whose partial sums are added in turn, is within e(K) = (64 + K / 64) 2^-24 of the sum of the
products' magnitudes (the tensor cores add 16 products at a time and cut: K / 16 steps of at most 2^-23 of the
sum so far, half of it on average). fp32 operands are used to 2^-24 of themselves.
  g, u:  e(hidden) of |x| |Wg|, |x| |Wu|
  h:     what g's and u's errors move (|act'| <= 1.13), a few u, and t of h
  y:     |h's error| |Wd|, e(width) of |h| |Wd|, and t of y
and in the same way for the gradients, whose dg, du and h are rounded to t. h's and dg's roundings are independent of
one another, so that their sums are far inside these bounds, which add up magnitudes.
"""
import pytest
import torch

from paper_2607_20548_gb300 import ffn_backward, ffn_forward
from paper_2607_20548_gb300 import soap as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
HALF = {t: torch.finfo(t).eps / 2 for t in (F32, BF, HF)}
TINY = {F32: 1e-37, BF: 1e-37, HF: 2.0 ** -25}


def _e(k):
    return (64 + k / 64) * U


def _act(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    p = torch.special.ndtr(g)
    return g * p, p + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5


def _near(name, got, want, slack):
    assert got.shape == want.shape, name
    bound = 1.001 * HALF[got.dtype] * want.abs() + slack + TINY[got.dtype]
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), (name, float((err / bound).max()))


def _check(x, w, act, y, dy=None, grads=None):
    """One group's results: its rows' x, y, dy, its weights and their gradients."""
    t, (rows, hidden), width = x.dtype, x.shape, w[0].shape[-1]
    half, tiny = HALF[t] * 1.001, TINY[t]
    x, (wg, wu, wd) = x.double(), (m.double() for m in w)
    g, u = x @ wg, x @ wu
    eg, eu = (_e(hidden) * (x.abs() @ m.abs()) for m in (wg, wu))
    a, da = _act(g, act)
    h = a * u
    ea = 1.13 * eg + 16 * U * (a.abs() + g.abs())
    eh = ea * u.abs() + a.abs() * eu + ea * eu + (half + 4 * U) * h.abs() + tiny
    _near("y", y, h @ wd, eh @ wd.abs() + _e(width) * (h.abs() @ wd.abs()))
    if dy is None:
        return
    dy = dy.double()
    dh, edh = dy @ wd.mT, _e(hidden) * (dy.abs() @ wd.mT.abs())
    # act' moves by |act''| <= 0.8 per error of g
    eda = 0.8 * eg + 16 * U * (1 + g.abs())
    dg, du = dh * u * da, dh * a
    edg = edh * (u * da).abs() + (dh.abs() + edh) * (eu * da.abs() + u.abs() * eda + eu * eda) \
        + (half + 4 * U) * dg.abs() + tiny
    edu = edh * a.abs() + (dh.abs() + edh) * ea + (half + 4 * U) * du.abs() + tiny
    dx, dwg, dwu, dwd = grads
    _near("dx", dx, dg @ wg.mT + du @ wu.mT, edg @ wg.mT.abs() + edu @ wu.mT.abs()
          + _e(2 * width) * (dg.abs() @ wg.mT.abs() + du.abs() @ wu.mT.abs()))
    if dwg is None:
        return
    xa = x.mT.abs()
    _near("dwg", dwg, x.mT @ dg, xa @ edg + _e(rows) * (xa @ dg.abs()))
    _near("dwu", dwu, x.mT @ du, xa @ edu + _e(rows) * (xa @ du.abs()))
    _near("dwd", dwd, h.mT @ dy, eh.mT @ dy.abs() + _e(rows) * (h.mT.abs() @ dy.abs()))


def _operands(cuda, lengths, hidden, width, t, columns=(False, False), before=0, behind=0, dense=False, seed=0, pad=0):
    """x, dy, weights, offsets; rows of no group hold NaN. pad: elements between a matrix's rows (or columns)."""
    g = torch.Generator(device=cuda).manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=cuda, generator=g)  # noqa: E731
    rows = before + sum(lengths) + behind

    def mat(m, n, scale, transposed):
        lead = () if dense else (len(lengths),)
        if transposed:
            return ((r(*lead, n, m + pad) * scale).to(t)[..., :m]).mT
        return (r(*lead, m, n + pad) * scale).to(t)[..., :n]
    w = [mat(hidden, width, hidden ** -0.5, columns[0]), mat(hidden, width, hidden ** -0.5, columns[0]),
         mat(width, hidden, width ** -0.5, columns[1])]
    x, dy = r(rows, hidden + pad).to(t)[:, :hidden], (0.1 * r(rows, hidden + pad)).to(t)[:, :hidden]
    off = None
    if not dense:
        ends = before + torch.tensor([0] + lengths).cumsum(0)
        off = ends.to(torch.int32).to(cuda)
        for v in (x, dy):
            v[:before] = float("nan")
            v[before + sum(lengths):] = float("nan")
    return x, dy, w, off


def _run(cuda, lengths, hidden, width, t, act="silu", train=True, **kw):
    x, dy, w, off = _operands(cuda, lengths, hidden, width, t, **kw)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    y, pre = ffn_forward(x, *w, offsets=off, act=act, keep=train, status=status)
    assert y.dtype == t and y.shape == x.shape and (pre is not None) == train
    grads = ffn_backward(dy, x, pre, *w, offsets=off, act=act, status=status) if train else None
    torch.cuda.synchronize()
    assert int(status) == 0
    if train:
        assert [a.shape for a in grads] == [x.shape] + [m.shape for m in w] and all(a.dtype == t for a in grads)
        for a, m in zip(grads[1:], w):  # the weights' order
            assert (a.stride(-2) == 1 or a.shape[-2] == 1) if m.stride(-2) == 1 and m.stride(-1) != 1 \
                else a.stride(-1) == 1 or a.shape[-1] == 1
    at = kw.get("before", 0)
    for i, n in enumerate(lengths):
        rows = slice(at, at + n)
        pick = (lambda m: m) if off is None else (lambda m: m[i])
        _check(x[rows], [pick(m) for m in w], act, y[rows], dy[rows] if train else None,
               [grads[0][rows]] + [pick(m) for m in grads[1:]] if train else None)
        if train and n == 0:
            assert not any(bool(pick(m).any()) for m in grads[1:])
        at += n
    for out in [y] + ([grads[0]] if train else []):
        assert not bool(out[:kw.get("before", 0)].any()) and not bool(out[at:].any())


@pytest.mark.parametrize("columns", [(False, False), (True, True), (True, False)])
@pytest.mark.parametrize("t", [BF, HF, F32])
@pytest.mark.parametrize("rows,hidden,width", [(1, 64, 128), (3, 1, 1), (37, 72, 200), (256, 256, 512), (300, 520, 264),
                                               (1, 1, 300), (130, 100, 7), (257, 129, 131)])
def test_dense(cuda, rows, hidden, width, t, columns):
    _run(cuda, [rows], hidden, width, t, columns=columns, dense=True, act="gelu" if width % 3 == 0 else "silu")


@pytest.mark.parametrize("columns", [(False, False), (True, True)])
@pytest.mark.parametrize("t", [BF, HF, F32])
@pytest.mark.parametrize("lengths,hidden,width,before,behind", [
    ([5], 64, 64, 0, 0), ([0, 3, 0, 260, 1], 136, 72, 0, 0), ([256, 255, 257], 64, 320, 3, 5), ([0, 0], 40, 24, 2, 1),
    ([1] * 70, 32, 48, 0, 9), ([33, 0, 31], 77, 51, 1, 0), ([700, 2], 260, 136, 0, 130)])
def test_groups(cuda, lengths, hidden, width, before, behind, t, columns):
    _run(cuda, lengths, hidden, width, t, columns=columns, before=before, behind=behind)


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("pad", [8, 3])
def test_slices(cuda, t, pad):
    _run(cuda, [140], 72, 136, t, pad=pad, dense=True)
    _run(cuda, [70, 0, 40], 72, 136, t, pad=pad, columns=(True, False))


@pytest.mark.parametrize("t,rows,hidden,width", [(BF, 24, 1024, 2048), (BF, 2000, 512, 1024), (F32, 600, 512, 768),
                                                 (HF, 5000, 128, 64), (BF, 1, 4096, 64), (F32, 3000, 64, 64), (HF, 60, 128, 1000),
                                                 (BF, 64, 64, 2100), (BF, 20, 2100, 100), (BF, 65, 100, 4000),
                                                 (HF, 17, 1600, 1600)])
def test_larger(cuda, t, rows, hidden, width):
    _run(cuda, [rows], hidden, width, t, dense=True)


@pytest.mark.parametrize("t", [BF, F32])
def test_serving(cuda, t):
    _run(cuda, [1], 512, 1536, t, dense=True, train=False)
    _run(cuda, [2, 0, 1, 7], 256, 192, t, train=False, behind=2)


@pytest.mark.parametrize("rows,hidden,width", [(1, 512, 512), (13, 300, 200), (1, 4096, 70), (64, 64, 1000),
                                               (200, 64, 500), (1500, 8, 300)])
@pytest.mark.parametrize("t", [BF, HF])
def test_few_results_round_once(cuda, t, rows, hidden, width):
    """h, dg and du are kept to twice the type's bits: the results' own rounding is all that is left of 16 bits."""
    x, dy, w, _ = _operands(cuda, [rows], hidden, width, t, dense=True)
    y, pre = ffn_forward(x, *w, keep=True)
    got = [y, *ffn_backward(dy, x, pre, *w)]
    leaves = [v.double().requires_grad_() for v in (x, *w)]
    g = leaves[0] @ leaves[1]
    out = (g * torch.sigmoid(g) * (leaves[0] @ leaves[2])) @ leaves[3]
    want = [out.detach(), *torch.autograd.grad(out, leaves, dy.double())]
    for a, b in zip(got, want):
        # a rounding's error is spread evenly over a step of 2^-m to 2^(1-m) of the value, at most 0.58 of half the
        # step's largest part in root mean square; fp16's smallest steps do not count here
        err = float((a.double() - b).norm() / b.norm())
        assert err <= 0.6 * HALF[t] + 1e-5, err


def test_leading_dimensions_and_without_params(cuda):
    x, dy, w, _ = _operands(cuda, [24], 64, 96, BF, dense=True)
    y, pre = ffn_forward(x, *w, keep=True)
    y3, pre3 = ffn_forward(x.view(2, 3, 4, 64), *w, keep=True)
    assert torch.equal(y3.view(24, 64), y)
    full = ffn_backward(dy, x, pre, *w)
    part = ffn_backward(dy.view(2, 3, 4, 64), x.view(2, 3, 4, 64), pre3, *w, params=False)
    assert torch.equal(part[0].view(24, 64), full[0]) and part[1] is part[2] is part[3] is None


def test_no_rows(cuda):
    w = [torch.randn(8, 16, device=cuda), torch.randn(8, 16, device=cuda), torch.randn(16, 8, device=cuda)]
    x = torch.randn(0, 8, device=cuda)
    y, pre = ffn_forward(x, *w, keep=True)
    assert y.shape == (0, 8)
    grads = ffn_backward(y, x, pre, *w)
    assert grads[0].shape == (0, 8) and not any(bool(g.any()) for g in grads[1:])


def test_bad_offsets(cuda):
    """Offsets that fall or pass the rows: raised to the largest before, cut at the rows, and told."""
    x, dy, w, _ = _operands(cuda, [4, 5, 6], 32, 40, BF)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    for bad, good in (([0, 9, 4, 15], [0, 9, 9, 15]), ([-3, 4, 8, 1 << 30], [0, 4, 8, 15]), ([20, 1, 2, 3], [15] * 4)):
        status.zero_()
        off = [torch.tensor(v, dtype=torch.int32, device=cuda) for v in (bad, good)]
        got, pre = ffn_forward(x, *w, offsets=off[0], keep=True, status=status)
        assert int(status) == S.STATUS_RANGE
        want, pre2 = ffn_forward(x, *w, offsets=off[1], keep=True)
        assert torch.equal(got, want)
        for a, b in zip(ffn_backward(dy, x, pre, *w, offsets=off[0]), ffn_backward(dy, x, pre2, *w, offsets=off[1])):
            assert torch.equal(a, b)


@pytest.mark.parametrize("t", [BF, F32])
def test_bad_rows_stay_to_themselves(cuda, t):
    x, dy, w, off = _operands(cuda, [100, 90, 70], 64, 80, t)
    y, pre = ffn_forward(x, *w, offsets=off, keep=True)
    grads = ffn_backward(dy, x, pre, *w, offsets=off)
    x[130, 5], dy[131, 7] = float("inf"), float("nan")
    y2, pre2 = ffn_forward(x, *w, offsets=off, keep=True)
    grads2 = ffn_backward(dy, x, pre2, *w, offsets=off)
    same = torch.ones(260, dtype=torch.bool, device=cuda)
    same[130] = False
    assert torch.equal(y2[same], y[same]) and not bool(y2[130].isfinite().any())
    same[131] = False
    assert torch.equal(grads2[0][same], grads[0][same]) and bool(grads2[0][131].isnan().all())
    for a, b in zip(grads2[1:], grads[1:]):
        assert torch.equal(a[[0, 2]], b[[0, 2]]) and not torch.equal(a[1], b[1])


def test_other_stream_and_repeatable(cuda):
    x, dy, w, off = _operands(cuda, [300, 0, 500], 256, 320, BF)
    y, pre = ffn_forward(x, *w, offsets=off, keep=True)
    a = [y, *ffn_backward(dy, x, pre, *w, offsets=off)]
    side = torch.cuda.Stream(cuda)
    side.wait_stream(torch.cuda.current_stream(cuda))
    y, pre = ffn_forward(x, *w, offsets=off, keep=True, stream=side)
    b = [y, *ffn_backward(dy, x, pre, *w, offsets=off, stream=side)]
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_two_calls_at_once(cuda):
    x, dy, w, off = _operands(cuda, [300, 40, 500], 256, 320, BF)
    want = ffn_forward(x, *w, offsets=off)[0]
    sides = [torch.cuda.Stream(cuda) for _ in range(3)]
    for s in sides:
        s.wait_stream(torch.cuda.current_stream(cuda))
    outs = [ffn_forward(x, *w, offsets=off, stream=s)[0] for _ in range(4) for s in sides]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_gradients_against_differences(cuda):
    x, dy, w, off = _operands(cuda, [3, 4], 6, 5, F32, seed=2)
    dy = dy * 10

    def value(x, *w):
        return float((ffn_forward(x, *w, offsets=off)[0].double() * dy).sum())
    _, pre = ffn_forward(x, *w, offsets=off, keep=True)
    grads = ffn_backward(dy, x, pre, *w, offsets=off)
    # central differences of step h: h^2 times a third derivative of order ten, and the value's rounding over h (42
    # terms of order one, each within 100 u)
    h = 2.0 ** -8
    tol = 10 * h * h + 42 * 100 * U / h
    for i, (t, grad) in enumerate(zip((x, *w), grads)):
        for e in range(0, t.numel(), 7):
            ends = []
            for sign in (1, -1):
                args = [v.clone() for v in (x, *w)]
                args[i].view(-1)[e] += sign * h
                ends.append((value(*args), float(args[i].view(-1)[e])))
            slope = (ends[0][0] - ends[1][0]) / (ends[0][1] - ends[1][1])
            assert abs(slope - float(grad.reshape(-1)[e])) <= tol


def test_binding_refusals(cuda):
    x, dy, w, off = _operands(cuda, [4, 5], 16, 24, BF)
    d = [m[0] for m in w]
    for args, kw in (((x, *w), {}), ((x, *d), dict(offsets=off)), ((x[:, :8], *d), {}), ((x, d[0], d[1][:, :8], d[2]), {}),
                     ((x, *d), dict(act="relu")), ((x, *w), dict(offsets=off[:2])), ((x, *w), dict(offsets=off[:1])),
                     ((x, d[0], d[1], d[0]), {})):
        with pytest.raises(ValueError):
            ffn_forward(*args, **kw)
    for args, kw in (((x, d[0].half(), d[1], d[2]), {}), ((x, *w), dict(offsets=off.long())), ((x.cpu(), *d), {}),
                     ((x.double(), *(m.double() for m in d)), {})):
        with pytest.raises(TypeError):
            ffn_forward(*args, **kw)
    _, pre = ffn_forward(x, *d, keep=True)
    with pytest.raises(ValueError):
        ffn_backward(dy[:5], x, pre, *d)
    with pytest.raises(ValueError):
        ffn_backward(dy, x, pre[:-8], *d)
