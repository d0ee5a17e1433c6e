"""The stand-alone operators where one part of a kernel hands data to another: lanes of a row, warps of a
CTA, CTAs of a pair."""
import math

import pytest
import torch

from paper_2607_20548_gb300 import (layer_norm_backward, layer_norm_forward, muon_orthogonalize, route_backward,
                                    route_forward)
from paper_2607_20548_gb300 import soap as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


# ---- routing -------------------------------------------------------------------------------

@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("e,k", [(64, 8), (127, 6), (190, 8)])
def test_choices_in_the_other_lanes_half(cuda, e, k, shift):
    """Many tokens' fp32 rows: two lanes share a row, four logits in turn, and choice q is the business of
    lane q % 2. Here every choice lies among the other lane's logits (shifted: some of them), whose
    probabilities that lane has written just before. Tolerance: as for the gradient in test_gpu_route.py, 152 u of
    a probability and 4 such terms in a row's products."""
    t = 16000
    g = torch.Generator(device=cuda).manual_seed(e + shift)
    z = torch.randn(t, e, device=cuda, generator=g)
    rows = torch.arange(t, device=cuda)
    want = []
    for q in range(k):  # the q-th largest at a place of unit 2 j (lane 0's) for odd q, 2 j + 1 for even ones
        unit = 2 * q + (1 - q % 2)
        at = (4 * unit + (rows + q + shift) % 4 + 4 * (shift // 2)) % (e - 2)
        z[rows, at] = 20.0 - q
        want.append(at)
    r = route_forward(z, k)
    assert torch.equal(r.indices.long(), torch.stack(want, 1))
    dg = torch.randn(t, k, device=cuda, generator=g)
    dz = route_backward(z, r, dgates=dg)
    p = torch.softmax(z.double(), 1)
    up = (0.01 * e / (k * t ** 2) * r.counts.double())[None].expand(t, e).clone()
    pc = p.gather(1, r.indices.long())
    total = pc.sum(1, keepdim=True)
    gates = pc / total
    d = (dg.double() - (dg.double() * gates).sum(1, keepdim=True)) / total
    dm = (dg.double().abs() + (dg.double().abs() * gates).sum(1, keepdim=True)) / total
    um = up.clone().scatter_add_(1, r.indices.long(), dm)
    up.scatter_add_(1, r.indices.long(), d)
    ref = p * (up - (p * up).sum(1, keepdim=True))
    mag = p * (um + (p * um).sum(1, keepdim=True))
    bound = U * ref.abs() + 4 * 152 * U * mag + 1e-37
    assert bool(((dz.double() - ref).abs() <= bound).all())
    assert torch.equal(dz, route_backward(z, r, dgates=dg))


# ---- orthogonalisation ---------------------------------------------------------------------

QUINTIC = (15 / 8, -10 / 8, 3 / 8)


def _ortho_ref(M, steps, eps=1e-7):
    X = M.double()
    X = X / torch.linalg.matrix_norm(X, keepdim=True).clamp_min(eps)
    tall = X.shape[-2] > X.shape[-1]
    X = X.mT if tall else X
    a, b, c = QUINTIC
    for _ in range(steps):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.mT if tall else X


def _ortho_tol(dtype, steps, m, n):
    """As in test_gpu_ortho.py: 3 stored results a step of 11 or 22 bits, a gain of 2, one unit of the
    accumulator per 16 products, one rounding to the type."""
    b = 11 if dtype == torch.bfloat16 else 22
    return torch.finfo(dtype).eps / 2 + 2 * math.sqrt(3 * steps) * 2.0 ** -b + math.ceil(max(m, n) / 16) * 2.0 ** -23


def _momentum(cuda, shape, dtype, seed=0, scale=1e-3):
    g = torch.Generator(device=cuda).manual_seed(seed)
    *lead, m, n = shape
    q = min(4, m, n)
    low = torch.randn(*lead, m, q, device=cuda, generator=g) @ torch.randn(*lead, q, n, device=cuda, generator=g)
    return ((low * (0.5 / math.sqrt(q)) + torch.randn(*lead, m, n, device=cuda, generator=g)) * scale).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(700, 150, 190), (700, 190, 150), (400, 256, 256), (300, 129, 600), (150, 256, 260)])
def test_long_runs_of_diagonal_tiles(cuda, shape, dtype):
    """Sides of 129 to 256: every tile of S and B lies on the diagonal, where one of a CTA's two loading
    threads has nothing to load; a large batch gives a pair of CTAs long runs of them."""
    M = _momentum(cuda, shape, dtype, seed=shape[0])
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    out = muon_orthogonalize(M, ns_steps=6, status=status)
    assert int(status) == 0
    ref = _ortho_ref(M, 6)
    err = torch.linalg.matrix_norm(out.double() - ref) / torch.linalg.matrix_norm(ref)
    assert float(err.max()) <= _ortho_tol(dtype, 6, *shape[1:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(300, 700), (3, 1100, 200)])
def test_ortho_wait_runs_out(cuda, shape, dtype):
    """A flag that nothing sets makes every wait run out (20 ms): the kernel returns, the status word says so, no
    result is left to be taken for one, with or without a status word, and the next call is sound."""
    M = _momentum(cuda, shape, dtype)
    want = muon_orthogonalize(M, ns_steps=4)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    hold = torch.zeros(1, dtype=torch.int32, device=cuda)
    torch.cuda.synchronize()
    try:
        S.soap_wait_limit(20_000_000, hold)
        got = [muon_orthogonalize(M, ns_steps=4, status=status), muon_orthogonalize(M, ns_steps=4)]
        torch.cuda.synchronize()
        hold.fill_(1)
        free = muon_orthogonalize(M, ns_steps=4)
        torch.cuda.synchronize()
    finally:
        S.soap_wait_limit(0, None)
    assert int(status) == S.STATUS_TIMEOUT
    assert all(x.isnan().all() for x in got)
    assert torch.equal(free, want)
    status.zero_()
    assert torch.equal(muon_orthogonalize(M, ns_steps=4, status=status), want) and int(status) == 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("shape", [(16, 40000), (50000, 16), (13, 48001), (64, 12000), (6000, 100), (2, 40, 9000)])
def test_accuracy_does_not_fall_with_a_long_side(cuda, shape, dtype):
    """A small side and a long one. The accumulator truncates, at most a unit of its last place (2^-23) per 16
    products, so split operands add it up in runs of 256 elements: 16 such units for any length. fp16's own
    rounding would hide that; the check is then of the scale alone, <out, ref> / <ref, ref>, in which roundings
    average out: 2^-11 / sqrt(elements), five times."""
    M = _momentum(cuda, shape, dtype, seed=shape[-1])
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    out, ref = muon_orthogonalize(M, ns_steps=6, status=status).double(), _ortho_ref(M, 6)
    assert int(status) == 0
    tol = 2 * math.sqrt(3 * 6) * 2.0 ** -22 + 16 * 2.0 ** -23
    if dtype == torch.float32:
        assert float(torch.linalg.norm(out - ref) / torch.linalg.norm(ref)) <= tol + 2.0 ** -24
    scale = float((out * ref).sum() / (ref * ref).sum())
    assert abs(scale - 1) <= tol + 5 * torch.finfo(dtype).eps / 2 / math.sqrt(ref.numel())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("e", [45, 46, 54, 55, 60, -41, -70])
def test_norm_of_large_and_small_elements(cuda, e, dtype):
    """Elements of 2^e to 2^(e + 1), 2^19 of them to a CTA: neither a square nor a sum of them leaves fp32's
    range unnoticed. X_0 does not depend on a power of two in M, so the result is that of e = 0. Beside the
    products' error: the sum of squares, whose longest chain has 16 + 128 + 5 + 8 + 17 fp32 additions (a
    thread's run, its runs, a warp, a CTA, the CTAs), at most 174 u, half of which reaches the norm."""
    g = torch.Generator(device=cuda).manual_seed(7)
    M = (1 + torch.rand(136, 65536, device=cuda, generator=g)).to(dtype).clamp_max(1.99)
    M *= torch.randint(0, 2, M.shape, device=cuda, generator=g).to(dtype) * 2 - 1
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    out = muon_orthogonalize(M * 2.0 ** e, ns_steps=2, eps=1e-37, status=status)
    assert int(status) == 0
    ref = _ortho_ref(M, 2)
    err = float(torch.linalg.norm(out.double() - ref) / torch.linalg.norm(ref))
    assert err <= _ortho_tol(dtype, 2, 136, 1024) + 87 * U  # K in runs of 1024 at most


# ---- layer norm ----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,width", [(40, 2048), (700, 1537), (5000, 1024)])
def test_norm_wait_runs_out(cuda, rows, width, dtype):
    """As for the orthogonalisation: no row comes while the flag is unset, the waits run out (20 ms), and
    what would have come from the rows is NaN."""
    g = torch.Generator(device=cuda).manual_seed(width)
    x, dy = (torch.randn(rows, width, device=cuda, generator=g).to(dtype) for _ in range(2))
    w = torch.randn(width, device=cuda, generator=g)
    y, mean, rstd = layer_norm_forward(x, w, w)
    want = (y, mean, rstd, *layer_norm_backward(dy, x, mean, rstd, w))

    def both(status=None):
        return (*layer_norm_forward(x, w, w, status=status),
                *layer_norm_backward(dy, x, mean, rstd, w, status=status))

    status = [torch.zeros(1, dtype=torch.int32, device=cuda) for _ in range(2)]
    hold = torch.zeros(1, dtype=torch.int32, device=cuda)
    torch.cuda.synchronize()
    try:
        S.soap_wait_limit(20_000_000, hold)
        layer_norm_forward(x, w, w, status=status[0])
        layer_norm_backward(dy, x, mean, rstd, w, status=status[1])
        got = both()
        torch.cuda.synchronize()
        hold.fill_(1)
        free = both()
        torch.cuda.synchronize()
    finally:
        S.soap_wait_limit(0, None)
    assert [int(s) for s in status] == [S.STATUS_TIMEOUT] * 2
    assert all(t.isnan().all() for t in got)
    assert all(torch.equal(a, b) for a, b in zip(free, want))
    clean = torch.zeros(1, dtype=torch.int32, device=cuda)
    assert all(torch.equal(a, b) for a, b in zip(both(clean), want)) and int(clean) == 0


# ---- layouts -------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("off,width", [(0, 64), (8, 64), (3, 61), (0, 512), (5, 507)])
def test_slices_of_every_row(cuda, off, width, dtype):
    """x[..., a:b] of more than two dimensions: read where it lies, with the dense tensor's bits where the rows'
    alignment leaves the same kernel, and its values to rounding where not."""
    g = torch.Generator(device=cuda).manual_seed(width)
    x, dy = (torch.randn(3, 5, 4, width + 16, device=cuda, generator=g).to(dtype)[..., off:off + width] for _ in range(2))
    assert not x.is_contiguous()
    w = torch.randn(width, device=cuda, generator=g)
    y, mean, rstd = layer_norm_forward(x, w, w)
    want = layer_norm_forward(x.contiguous(), w, w)
    assert y.shape == x.shape and y.is_contiguous() and mean.shape == x.shape[:-1]
    tol = dict(rtol=2 * torch.finfo(dtype).eps, atol=64 * U * 8)  # one rounding each; statistics within 64 u
    torch.testing.assert_close(y, want[0], **tol)
    got = layer_norm_backward(dy, x, mean, rstd, w)
    ref = layer_norm_backward(dy.contiguous(), x.contiguous(), *want[1:], w)
    torch.testing.assert_close(got[0], ref[0], **tol)
    for a, b in zip(got[1:], ref[1:]):  # 60 rows' sums of terms up to 30
        torch.testing.assert_close(a, b, rtol=0, atol=60 * 30 * 4 * U)
    r, q = route_forward(x, 4), route_forward(x.contiguous(), 4)
    assert all(torch.equal(a, b) for a, b in zip(r[:7], q[:7]))
    assert torch.equal(route_backward(x, r, dgates=r.gates), route_backward(x.contiguous(), q, dgates=q.gates))


# ---- streams -------------------------------------------------------------------------------

def _norm_args(cuda):
    x = torch.ones(3500, 1100, device=cuda)  # 15 MB: a block of its own, which the next such tensor would get
    w, m = torch.ones(1100, device=cuda), torch.ones(3500, device=cuda)
    return dict(x=x, w=w, m=m, dy=x.clone())


CALLS = {
    "x forward": ("x", _norm_args, lambda a, s: layer_norm_forward(a["x"], a["w"], a["w"], stream=s)),
    "x backward": ("x", _norm_args, lambda a, s: layer_norm_backward(a["dy"], a["x"], a["m"], a["m"], a["w"], stream=s)),
    "dy": ("dy", _norm_args, lambda a, s: layer_norm_backward(a["dy"], a["x"], a["m"], a["m"], a["w"], stream=s)),
    "logits": ("z", lambda cuda: dict(z=torch.ones(60000, 64, device=cuda)),
               lambda a, s: route_forward(a["z"], 4, stream=s)),
    "mask": ("mask", lambda cuda: dict(z=torch.ones(15000000, 1, device=cuda),
                                          mask=torch.ones(15000000, dtype=torch.bool, device=cuda)),
             lambda a, s: route_forward(a["z"], 1, mask=a["mask"], stream=s)),
    "M": ("M", lambda cuda: dict(M=torch.ones(40, 300, 320, device=cuda)),
          lambda a, s: muon_orthogonalize(a["M"], ns_steps=2, stream=s)),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_operands_outlive_the_call_on_its_stream(cuda, name):
    """The caller may drop an operand as soon as a call on another stream returns (a temporary: f(a + b,
    stream=s)): its memory is not given out again while that stream has yet to read it."""
    key, make, call = CALLS[name]
    args = make(cuda)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)  # 0.1 s: the call's kernels wait behind it
    call(args, s)
    shape, dtype, at = args[key].shape, args[key].dtype, args[key].data_ptr()
    del args[key]
    fresh = torch.empty(shape, dtype=dtype, device=cuda)
    busy = not s.query()
    same = fresh.data_ptr() == at
    s.synchronize()
    assert busy and not same


@pytest.mark.parametrize("key", ["logits", "dgates", "indices", "stats", "mask"])
def test_routing_outlives_the_backward_call_on_its_stream(cuda, key):
    t, e, k = 15000000, 2, 1
    z = torch.zeros(t, e, device=cuda)
    mask = torch.ones(t, dtype=torch.bool, device=cuda)
    r = route_forward(z, k, mask=mask)
    dg = torch.ones(t, k, device=cuda)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    route_backward(z, r, dgates=dg, stream=s)
    held = dict(logits=z, dgates=dg, indices=r.indices, stats=r.stats, mask=mask)
    shape, dtype, at = held[key].shape, held[key].dtype, held[key].data_ptr()
    drop = held.pop(key)
    if key in ("indices", "stats", "mask"):
        r = r._replace(**{key: None})
    if key == "logits":
        z = None
    elif key == "dgates":
        dg = None
    elif key == "mask":
        mask = None
    del drop
    fresh = torch.empty(shape, dtype=dtype, device=cuda)
    busy = not s.query()
    same = fresh.data_ptr() == at
    s.synchronize()
    assert busy and not same


# ---- results over operands -----------------------------------------------------------------
# What the headers allow of the C calls: the binding always makes new results.

def _call(fn, *args):
    args = [a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args]
    assert getattr(S.load_library(), fn)(*args, torch.cuda.current_stream().cuda_stream) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,width", [(3, 1), (500, 100), (4000, 1023), (700, 1537), (5000, 1024), (3000, 2051), (400, 8192),
                                        (200, 8191), (12, 16384), (5, 20000)])
def test_norm_in_place(cuda, rows, width, dtype):
    """y = x, dx = dy and dx = x, among them rows that share 16-byte units with their neighbours, which other
    CTAs read ahead and write: the bits of the calls with results of their own."""
    g = torch.Generator(device=cuda).manual_seed(rows)
    x, dy = (torch.randn(rows, width, device=cuda, generator=g).to(dtype) for _ in range(2))
    w = torch.randn(width, device=cuda, generator=g)
    t = S.DTYPES[dtype]
    y, mean, rstd = layer_norm_forward(x, w, w)
    dx, dw, db = layer_norm_backward(dy, x, mean, rstd, w)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    for _ in range(3):
        buf, m2, r2 = x.clone(), torch.empty_like(mean), torch.empty_like(rstd)
        _call("layer_norm_forward", rows, width, buf, width, t, w, w, 0, 1e-5, buf, width, m2, r2, status)
        assert torch.equal(buf, y) and torch.equal(m2, mean) and torch.equal(r2, rstd)
        need = S.load_library().layer_norm_workspace_bytes(rows, width)
        for over_x in (False, True):
            bx, bg, w2, b2 = x.clone(), dy.clone(), torch.empty_like(dw), torch.empty_like(db)
            ws = torch.empty(need, dtype=torch.uint8, device=cuda)
            out = bx if over_x else bg
            _call("layer_norm_backward", rows, width, bg, width, bx, width, t, mean, rstd, w, 0, out, width, w2, b2, ws,
                  need, status)
            assert torch.equal(out, dx) and torch.equal(w2, dw) and torch.equal(b2, db)
    assert int(status) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,e,k", [(37, 8, 2), (1000, 64, 8), (1000, 127, 6), (3000, 500, 10), (20000, 64, 8), (20001, 127, 6),
                                        (16000, 33, 3), (16000, 300, 4), (16000, 61, 9)])
def test_routing_gradient_over_the_logits(cuda, tokens, e, k, dtype):
    """dlogits = logits, dense and with a leading dimension: the gradient's bits, and nothing written between
    the rows."""
    g = torch.Generator(device=cuda).manual_seed(tokens)
    z = torch.randn(tokens, e, device=cuda, generator=g).to(dtype)
    mask = torch.rand(tokens, device=cuda, generator=g) < 0.8
    r = route_forward(z, k, mask=mask, coef=0.3)
    dg = torch.randn(tokens, k, device=cuda, generator=g)
    want = route_backward(z, r, dgates=dg, dloss=2.0)
    for pad in (0, 8, 3):
        big = torch.full((tokens, e + pad), 7.0, device=cuda, dtype=dtype)
        big[:, :e] = z
        _call("layer_route_backward", tokens, e, k, big, e + pad, S.DTYPES[dtype], mask, 1, 0.3, 2.0, r.indices, r.stats,
              r.counts, r.live, dg, big, e + pad)
        assert torch.equal(big[:, :e], want) and bool((big[:, e:] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("batch,rows,cols", [(1, 64, 2048), (3, 90, 130), (5, 200, 50), (2, 300, 700), (1, 2400, 300), (3, 333, 257)])
def test_orthogonalize_in_place(cuda, batch, rows, cols, dtype):
    """out = M, dense and with padded rows and matrices: the bits of the call with a result of its own."""
    M = _momentum(cuda, (batch, rows, cols), dtype, seed=rows)
    lib, t = S.load_library(), S.DTYPES[dtype]
    need = lib.muon_orthogonalize_workspace_bytes(batch, rows, cols, t)
    ws = torch.empty(need, dtype=torch.uint8, device=cuda)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    for pad in (0, 8, 3):
        ld, stride = cols + pad, (rows + 1) * (cols + pad)
        buf = torch.full((batch, rows + 1, ld), 7.0, device=cuda, dtype=dtype)
        buf[:, :rows, :cols] = M
        out = torch.empty(batch, rows + 1, ld, device=cuda, dtype=dtype)
        _call("muon_orthogonalize", batch, rows, cols, buf, ld, stride, t, None, 5, 1e-7, out, ld, stride, ws, need, status)
        _call("muon_orthogonalize", batch, rows, cols, buf, ld, stride, t, None, 5, 1e-7, buf, ld, stride, ws, need, status)
        assert torch.equal(buf[:, :rows, :cols], out[:, :rows, :cols])
        assert bool((buf[:, rows:] == 7.0).all()) and bool((buf[:, :rows, cols:] == 7.0).all())
        ref = _ortho_ref(M, 5)
        assert float(torch.linalg.norm(buf[:, :rows, :cols].double() - ref) / torch.linalg.norm(ref)) <= _ortho_tol(
            dtype, 5, rows, cols)
    assert int(status) == 0


# ---- sizes between the kernels' ------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("shape", [(2400, 300), (300, 2400), (2, 4500, 520), (5000, 1100), (128, 20000), (20000, 100), (65, 40000)])
def test_many_row_tiles_and_long_sides(cuda, shape, dtype):
    """More than eight row tiles, which are taken in groups of eight, and small sides too long for a cluster."""
    M = _momentum(cuda, shape, dtype, seed=shape[-1])
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    out = muon_orthogonalize(M, ns_steps=5, status=status)
    ref = _ortho_ref(M, 5)
    assert int(status) == 0
    # split operands: K in runs of at most 1024
    k = 1024 if dtype != torch.bfloat16 else max(shape[-2:])
    assert float(torch.linalg.norm(out.double() - ref) / torch.linalg.norm(ref)) <= _ortho_tol(dtype, 5, k, k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,width", [(6000, 8192), (5000, 8191), (3000, 12288), (2600, 16384), (2500, 16379), (40000, 520),
                                        (9000, 4096)])
def test_many_wide_rows(cuda, rows, width, dtype):
    """Many rows, so that every CTA's loop goes round often with many elements per thread. Bounds: a row's sums
    within 32 u of their terms' magnitudes and what follows within 64 u (as in test_gpu_layer_norm.py, here with
    |x - mu| below 6 deviations), one rounding to the type; column sums in runs of rows / 152 terms."""
    g = torch.Generator(device=cuda).manual_seed(rows)
    x, dy = (torch.randn(rows, width, device=cuda, generator=g).to(dtype) for _ in range(2))
    w = 1 + 0.2 * torch.randn(width, device=cuda, generator=g)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    y, mean, rstd = layer_norm_forward(x, w, w, status=status)
    dx, dw, db = layer_norm_backward(dy, x, mean, rstd, w, status=status)
    assert int(status) == 0
    half = torch.finfo(dtype).eps / 2
    rw, rb, aw, ab = (torch.zeros(width, dtype=torch.float64, device=cuda) for _ in range(4))
    for i in range(0, rows, 1000):
        xd, gd, wd = x[i:i + 1000].double(), dy[i:i + 1000].double(), w.double()
        var, mu = torch.var_mean(xd, 1, correction=0, keepdim=True)
        rs = (var + 1e-5).rsqrt()
        xh = (xd - mu) * rs
        want = xh * wd + wd
        assert bool(((y[i:i + 1000].double() - want).abs() <= (half * 1.001 + 4 * U) * want.abs()
                     + (32 + 64 * 8) * U * wd.abs()).all())
        gw = gd * wd
        want = rs * (gw - gw.mean(1, keepdim=True) - xh * (gw * xh).mean(1, keepdim=True))
        assert bool(((dx[i:i + 1000].double() - want).abs() <= half * 1.001 * want.abs()
                     + rs * 128 * U * (gw.abs() + gw.abs().mean(1, keepdim=True) + xh.abs() + 1)).all())
        rw += (gd * xh).sum(0)
        rb += gd.sum(0)
        aw += (gd * xh).abs().sum(0)
        ab += gd.abs().sum(0)
    k = (rows / 152 + 200) * U
    assert bool(((dw.double() - rw).abs() <= (k + 128 * U) * aw + 32 * U * ab).all())
    assert bool(((db.double() - rb).abs() <= k * ab).all())
