"""Layer norm and its backward pass (include/layer.h) against fp64.

Tolerance (from the arithmetic): with u = 2^-24, the row statistics are sums of `width` fp32 terms
formed in runs of at most 16 and then pairwise, so their relative error is within 32 u of the sum of
the terms' magnitudes; x - mu carries |mu| times that. y adds a few roundings of its own terms and
one rounding to the type. dx is three such terms; dweight and dbias sum over rows in runs of
rows / 152 and then in order: within (rows / 152 + 200) u of the sum of magnitudes.
"""
import pytest
import torch

from paper_2607_20548_gb300 import layer_norm_backward, layer_norm_forward
from paper_2607_20548_gb300 import soap as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
OUT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}  # one rounding
TINY = {torch.float32: 1e-38, torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}  # half a subnormal step
SHAPES = [(1, 1), (1, 2048), (3, 7), (5, 31), (4, 64), (33, 100), (257, 255), (16, 1000), (9, 4099), (300, 512),
          (7, 8192), (2, 16384), (1000, 96), (2, 16385), (3, 20000)]
TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
         (torch.float16, torch.float32), (torch.float16, torch.float16)]


def _ref(x, w, b, eps, dy=None):
    x = x.double()
    mu = x.mean(-1, keepdim=True)
    rstd = 1 / (x.sub(mu).square().mean(-1, keepdim=True) + eps).sqrt()
    xh = (x - mu) * rstd
    wd = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    y = xh * wd + (0 if b is None else b.double())
    if dy is None:
        return y, mu, rstd, xh
    dy = dy.double()
    g = dy * wd
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), xh, rstd, g


def _near(got, want, dtype, slack):
    err = (got.double() - want).abs()
    bound = OUT[dtype] * want.abs() * 1.001 + slack + TINY[dtype]
    assert bool((err <= bound).all()), float((err / bound).max())


def _inputs(cuda, rows, width, dtype, wdtype, seed=0, offset=0.5):
    g = torch.Generator(device=cuda).manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=cuda, generator=g)  # noqa: E731
    x = (r(rows, width) * (0.5 + r(rows, 1).abs()) + offset * r(rows, 1)).to(dtype)
    return x, (1 + 0.2 * r(width)).to(wdtype), (0.2 * r(width)).to(wdtype), (0.1 * r(rows, width)).to(dtype)


def _check_forward(x, w, b, eps, y, mean, rstd):
    ry, mu, rs, xh = _ref(x, w, b, eps)
    assert y.dtype == x.dtype and mean.dtype == rstd.dtype == torch.float32
    e_mu = 32 * U * x.double().abs().mean(-1, keepdim=True)
    # the error of the mean moves every x - mu; the variance's relative error is the centred ones'
    e_xh = e_mu * rs + (64 * U + 2 * (e_mu * rs) ** 2) * xh.abs()
    assert bool(((mean.double().unsqueeze(-1) - mu).abs() <= e_mu + 1e-38).all())
    assert bool(((rstd.double().unsqueeze(-1) / rs - 1).abs() <= 64 * U + 2 * (e_mu * rs) ** 2).all())
    wd = 1.0 if w is None else w.double().abs()
    _near(y, ry, x.dtype, e_xh * wd + 4 * U * ry.abs() + 4 * U * (xh * wd).abs())


def _check_backward(x, w, eps, dy, dx, dw, db):
    rx, rw, rb, xh, rs, g = _ref(x, w, None, eps, dy)
    e_mu = 32 * U * x.double().abs().mean(-1, keepdim=True)
    e_xh = e_mu * rs + (64 * U + 2 * (e_mu * rs) ** 2) * xh.abs()
    m2 = (g * xh).abs().mean(-1, keepdim=True)
    # the slack of each of dx's terms: sums within 32 u, xh's own error in the third one and in its mean
    slack = rs * (80 * U * (g.abs() + g.abs().mean(-1, keepdim=True) + xh.abs() * m2) + e_xh * m2
                  + xh.abs() * (g.abs() * e_xh).mean(-1, keepdim=True))
    _near(dx, rx, x.dtype, slack)
    rows = x.shape[0]
    k = (rows / 152 + 200) * U
    d = dy.double().abs()
    if dw is not None:
        assert dw.dtype == db.dtype == torch.float32
        assert bool(((dw.double() - rw).abs() <= k * (d * xh.abs()).sum(0) + (d * e_xh).sum(0) + 1e-38).all())
        assert bool(((db.double() - rb).abs() <= k * d.sum(0) + 1e-38).all())


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_forward_and_backward(cuda, rows, width, dtype, wdtype):
    x, w, b, dy = _inputs(cuda, rows, width, dtype, wdtype, seed=rows + width)
    y, mean, rstd = layer_norm_forward(x, w, b, eps=1e-5)
    _check_forward(x, w, b, 1e-5, y, mean, rstd)
    dx, dw, db = layer_norm_backward(dy, x, mean, rstd, w)
    _check_backward(x, w, 1e-5, dy, dx, dw, db)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_optional_parts(cuda, dtype):
    x, w, b, dy = _inputs(cuda, 20, 136, dtype, torch.float32)
    for ww, bb in ((None, None), (w, None), (None, b)):
        y, mean, rstd = layer_norm_forward(x, ww, bb)
        _check_forward(x, ww, bb, 1e-5, y, mean, rstd)
        dx, dw, db = layer_norm_backward(dy, x, mean, rstd, ww, params=False)
        assert dw is None and db is None
        _check_backward(x, ww, 1e-5, dy, dx, None, None)


@pytest.mark.parametrize("rows", [2000, 40000])
def test_many_rows(cuda, rows):
    x, w, b, dy = _inputs(cuda, rows, 264, torch.bfloat16, torch.float32, seed=rows)
    y, mean, rstd = layer_norm_forward(x, w, b)
    _check_forward(x, w, b, 1e-5, y, mean, rstd)
    got = layer_norm_backward(dy, x, mean, rstd, w)
    _check_backward(x, w, 1e-5, dy, *got)
    for a, c in zip(got, layer_norm_backward(dy, x, mean, rstd, w)):
        assert torch.equal(a, c)


def test_large_offset_and_constant_rows(cuda):
    """A mean far above the spread (where E[x^2] - mu^2 would cancel), and rows without any spread."""
    x, w, b, dy = _inputs(cuda, 40, 768, torch.float32, torch.float32, offset=300.0)
    x[3] = 0.25
    x[4] = 0.0
    y, mean, rstd = layer_norm_forward(x, w, b)
    _check_forward(x, w, b, 1e-5, y, mean, rstd)
    assert torch.equal(y[3], b) and torch.equal(y[4], b)
    _check_backward(x, w, 1e-5, dy, *layer_norm_backward(dy, x, mean, rstd, w))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_strides_and_leading_dimensions(cuda, dtype):
    x, w, b, dy = _inputs(cuda, 24, 200, dtype, torch.float32)
    y, mean, rstd = layer_norm_forward(x, w, b)
    want = (y,) + layer_norm_backward(dy, x, mean, rstd, w)
    for pad, off in ((8, 0), (8, 8), (1, 0), (3, 1), (5, 5)):
        bx, bg = (torch.full((24, 200 + pad), float("nan"), device=cuda, dtype=dtype) for _ in range(2))
        vx, vg = bx[:, off:off + 200], bg[:, off:off + 200]
        vx.copy_(x)
        vg.copy_(dy)
        yy, m2, r2 = layer_norm_forward(vx, w, b)
        _check_forward(x, w, b, 1e-5, yy, m2, r2)
        _check_backward(x, w, 1e-5, dy, *layer_norm_backward(vg, vx, m2, r2, w))
    x4 = x.view(2, 3, 4, 200)
    y4, m4, r4 = layer_norm_forward(x4, w, b)
    assert y4.shape == x4.shape and m4.shape == (2, 3, 4) and torch.equal(y4.view(24, 200), want[0])
    got = layer_norm_backward(dy.view(2, 3, 4, 200), x4, m4, r4, w)
    assert torch.equal(got[0].view(24, 200), want[1]) and torch.equal(got[1], want[2])
    xt = x.t().contiguous().t()  # column-major: copied
    assert torch.equal(layer_norm_forward(xt, w, b)[0], want[0])


def test_empty_and_nonfinite(cuda):
    w = torch.ones(64, device=cuda)
    x = torch.empty(0, 64, device=cuda)
    y, mean, rstd = layer_norm_forward(x, w, w)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, dw, db = layer_norm_backward(x, x, mean, rstd, w)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    x = torch.randn(6, 64, device=cuda)
    x[2, 5], x[4, 63] = float("nan"), float("inf")
    y, mean, rstd = layer_norm_forward(x, w, w)
    bad = torch.tensor([False, False, True, False, True, False], device=cuda)
    assert y[bad].isnan().all() and y[~bad].isfinite().all()
    dx, _, _ = layer_norm_backward(torch.ones_like(x), x, mean, rstd, w)
    assert dx[bad].isnan().all() and dx[~bad].isfinite().all()


def test_against_differences(cuda):
    """<dx, d>, <dw, d> and <db, d> against central differences of sum(c y): the step's truncation, and fp32
    rounding of y over the step, are both within 1e-3 of the terms."""
    x, w, b, c = _inputs(cuda, 12, 96, torch.float32, torch.float32, seed=5)
    y, mean, rstd = layer_norm_forward(x, w, b)
    grads = layer_norm_backward(c, x, mean, rstd, w)
    g = torch.Generator(device=cuda).manual_seed(9)
    h = 2.0 ** -8
    for i, p in enumerate((x, w, b)):
        d = torch.randn(p.shape, device=cuda, generator=g)
        ends = []
        for s in (h, -h):
            args = [x, w, b]
            args[i] = p + s * d
            ends.append(float((c.double() * layer_norm_forward(*args)[0].double()).sum()))
        diff = (ends[0] - ends[1]) / (2 * h)
        terms = float((grads[i].double() * d.double()).abs().sum())
        assert abs(diff - float((grads[i].double() * d.double()).sum())) <= 1e-3 * terms


def test_other_stream(cuda):
    x, w, b, dy = _inputs(cuda, 500, 512, torch.bfloat16, torch.float32)
    y, mean, rstd = layer_norm_forward(x, w, b)
    want = layer_norm_backward(dy, x, mean, rstd, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y2, m2, r2 = layer_norm_forward(x, w, b, stream=s)
    got = layer_norm_backward(dy, x, m2, r2, w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, y2) and all(torch.equal(a, c) for a, c in zip(want, got))


def test_refusals(cuda):
    x, w, b, dy = _inputs(cuda, 4, 64, torch.bfloat16, torch.float32)
    y, mean, rstd = layer_norm_forward(x, w, b)
    with pytest.raises(TypeError):
        layer_norm_forward(x.cpu())
    with pytest.raises(TypeError):
        layer_norm_forward(x.double())
    with pytest.raises(TypeError):
        layer_norm_forward(x, w, b.to(torch.bfloat16))
    with pytest.raises(TypeError):
        layer_norm_forward(x, w.half())
    with pytest.raises(ValueError):
        layer_norm_forward(x, w[:32])
    with pytest.raises(ValueError):
        layer_norm_forward(torch.empty(3, 0, device=cuda))
    with pytest.raises(S.SoapError):
        layer_norm_forward(x, w, b, eps=-1.0)
    with pytest.raises(S.SoapError):
        layer_norm_forward(x, w, b, eps=float("nan"))
    with pytest.raises(TypeError):
        layer_norm_backward(dy.float(), x, mean, rstd, w)
    with pytest.raises(ValueError):
        layer_norm_backward(dy[:2], x, mean, rstd, w)
    with pytest.raises(ValueError):
        layer_norm_backward(dy, x, mean[:2], rstd, w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,width,pad,off", [(1, 301, 3, 1), (2, 511, 1, 0), (1, 4099, 9, 5), (700, 1537, 7, 3),
                                                (2500, 511, 5, 2), (2500, 2051, 1, 1), (3, 8191, 2, 1), (2, 9001, 3, 2)])
def test_rows_between_other_data(cuda, dtype, rows, width, pad, off):
    """Rows that begin and end inside 16-byte units, NaN on both sides of each: nothing of the neighbours counts."""
    x, w, b, dy = _inputs(cuda, rows, width, dtype, torch.float32, seed=width)
    bx, bg = (torch.full((rows, width + pad), float("nan"), device=cuda, dtype=dtype) for _ in range(2))
    vx, vg = bx[:, off:off + width], bg[:, pad - off:pad - off + width]
    vx.copy_(x)
    vg.copy_(dy)
    y, mean, rstd = layer_norm_forward(vx, w, b)
    _check_forward(x, w, b, 1e-5, y, mean, rstd)
    _check_backward(x, w, 1e-5, dy, *layer_norm_backward(vg, vx, mean, rstd, w))
