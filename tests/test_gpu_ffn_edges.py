"""The feed-forward block at its edges (include/layer.h, layer_ffn_*): roundings of 16-bit types, infinite elements, an
activation's tail, weights of different orders, calls without rows, waits that run out, long sums' workspaces."""
import pytest
import torch

from paper_2607_20548_gb300 import ffn_backward, ffn_forward
from paper_2607_20548_gb300 import soap as S
from tests.test_gpu_ffn import BF, F32, HALF, HF, TINY, U, _act, _operands

pytestmark = pytest.mark.gpu


def _both(x, dy, w, off=None, act="silu"):
    y, pre = ffn_forward(x, *w, offsets=off, act=act, keep=True)
    return [y, *ffn_backward(dy, x, pre, *w, offsets=off, act=act)]


def _exact(x, dy, w, lengths=None, act="silu"):
    """In 64 bits, one group after another: y, dx and the weights' gradients."""
    if lengths is not None:
        parts = [_exact(x[at:at + n], dy[at:at + n], [m[i] for m in w], act=act)
                 for i, (at, n) in enumerate(zip([sum(lengths[:i]) for i in range(len(lengths))], lengths))]
        return [torch.cat([p[i] for p in parts]) for i in range(2)] + [torch.stack([p[i] for p in parts]) for i in (2, 3, 4)]
    x, dy, wg, wu, wd = (v.double() for v in (x, dy, *w))
    g, u = x @ wg, x @ wu
    a, da = _act(g, act)
    h, dh = a * u, dy @ wd.mT
    dg, du = dh * u * da, dh * a
    return [h @ wd, dg @ wg.mT + du @ wu.mT, x.mT @ dg, x.mT @ du, h.mT @ dy]


def _mean_error(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("t", [BF, HF])
@pytest.mark.parametrize("lengths,hidden,width,roundings", [
    ([16], 1024, 1024, 1), ([17], 1024, 1024, 2), ([8], 2048, 4096, 1), ([8], 2048, 4104, 2),
    ([5, 11], 1024, 4096, 1), ([5, 11], 1024, 4104, 2)])
def test_roundings_by_size(cuda, lengths, hidden, width, roundings, t):
    """Up to 16384 elements of x and 2^23 of all groups' weights of a kind h, dg and du keep twice the type's bits, and a
    result has one rounding, else two independent ones, each of 0.578 of half a step in root mean square."""
    x, dy, w, off = _operands(cuda, lengths, hidden, width, t)
    dy = (dy * 10).to(t)  # (fp16's smallest steps do not count here)
    for a, b in zip(_both(x, dy, w, off), _exact(x, dy, w, lengths)):
        assert _mean_error(a, b) <= (0.6 if roundings == 1 else 0.82) * HALF[t] + 1e-5


@pytest.mark.parametrize("t", [BF, HF])
@pytest.mark.parametrize("lengths,hidden,width,act,columns", [
    ([300], 2048, 8192, "silu", (False, False)), ([1], 2048, 8192, "silu", (False, False)),
    ([24], 2048, 8192, "gelu", (True, False)), ([1000], 777, 1365, "gelu", (True, True)),
    ([60 + 17 * (i % 5) for i in range(64)], 2048, 768, "silu", (False, False)), ([3] * 64, 2048, 768, "silu", (False, True))])
def test_large_blocks_in_the_mean(cuda, lengths, hidden, width, act, columns, t):
    """Two independent roundings at most, of h (or dg and du) and of the result, each of 0.578 of half a step in root
    mean square, and sums in fp32: 1.415 x 0.578 = 0.82. (Bounds that add up magnitudes grow with the sums' length,
    these do not.)"""
    dense = len(lengths) == 1
    x, dy, w, off = _operands(cuda, lengths, hidden, width, t, columns=columns, dense=dense)
    dy = (dy * 10).to(t)  # (fp16's smallest steps do not count here)
    for a, b in zip(_both(x, dy, w, off, act), _exact(x, dy, w, None if dense else lengths, act)):
        assert _mean_error(a, b) <= 0.82 * HALF[t] + 1e-5


def _same(got, want, rel):
    """Infinities and NaN where the 64-bit values have them, the others near."""
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[got.isinf()].double(), want[want.isinf()])
    at = want.isfinite()
    assert bool(((got.double() - want)[at].abs() <= rel * want[at].abs() + 1e-37).all())


@pytest.mark.parametrize("hidden,width,lengths", [(64, 96, [40]), (300, 520, [40]), (72, 40, [5, 0, 300])])
@pytest.mark.parametrize("full", [False, True])
def test_infinite_elements(cuda, hidden, width, lengths, full):
    """fp32: an infinite element gives what products of infinities give, whether or not the others have more bits than
    a bf16 value. All terms are positive, so that no two infinities meet."""
    x, dy, w, off = _operands(cuda, lengths, hidden, width, F32)
    cut = (lambda v: v.abs() + 0.01) if full else (lambda v: (v.abs() + 0.01).bfloat16().float())
    x, dy, w = cut(x), cut(dy), [cut(m) for m in w]
    rel = 1000 * U  # all terms have one sign: 64 + K / 64 u in each of three sums in turn, a few products between them
    x0, dy0 = x.clone(), dy.clone()
    x[3, 5] = float("inf")
    want = _exact(x, dy, w, lengths)
    assert bool(want[0][3].isinf().all())
    _same(ffn_forward(x, *w, offsets=off)[0], want[0], rel)
    dy[2, 1] = -float("inf")
    want = _exact(x0, dy, w, lengths)
    assert bool(want[1][2].isinf().all()) and bool(want[2][0].isinf().all()) and bool(want[4][0, :, 1].isinf().all())
    for a, b in zip(_both(x0, dy, w, off), want):
        _same(a, b, rel)
    w[2][0, 2, 1] = float("inf")
    want = _exact(x0, dy0, w, lengths)
    for a, b in zip(_both(x0, dy0, w, off), want):
        _same(a, b, rel)
    w[0][0, 2, 1] = float("inf")
    x0[0, 2] = 0.0  # and no product with a zero
    _same(ffn_forward(x0, *w, offsets=off)[0], _exact(x0, dy0, w, lengths)[0], rel)


@pytest.mark.parametrize("hidden,width,lengths", [(520, 300, [40]), (72, 136, [300]), (520, 72, [30, 0, 200])])
@pytest.mark.parametrize("t", [BF, HF])
def test_infinite_elements_of_16_bits(cuda, hidden, width, lengths, t):
    """The same where h, dg and du are rounded to the type."""
    x, dy, w, off = _operands(cuda, lengths, hidden, width, t)
    x, dy, w = x.abs() + 0.01, dy.abs() + 0.01, [m.abs() + 0.01 for m in w]
    rel = 4 * HALF[t]  # all terms have one sign: two roundings (dx: of dg or du, and its own)
    for m, at in ((x, (3, 5)), (dy, (2, 1)), (w[2], (0, 2, 1)), (w[0], (0, 2, 1))):
        was = m[at].clone()
        m[at] = float("inf")
        want = _exact(x, dy, w, lengths)
        got = _both(x, dy, w, off)
        if m is x or m is w[0]:  # (silu' of an infinity is a NaN in 64 bits)
            got, want = got[:1], want[:1]
        assert not bool(want[0].isnan().any())
        for a, b in zip(got, want):
            _same(a, b, rel)
        m[at] = was


@pytest.mark.parametrize("t", [F32, BF])
def test_gelu_tail(cuda, t):
    """One element of h per row, whose g is given: y is act(g), dx is act'(g) and act(g). With u = 2^-24: Phi within
    4 steps of its argument's two roundings, which g^2 multiplies; the exponential within 2^-22 and g^2 / 2 roundings of
    its argument; a few more products; for 16-bit types their two roundings."""
    g = torch.linspace(-11, 11, 2003, device=cuda).to(t)
    x = torch.stack([g, torch.ones_like(g)], -1)
    w = [torch.tensor(v, device=cuda, dtype=t) for v in ([[1.0], [0.0]], [[0.0], [1.0]], [[1.0, 0.0]])]
    dy = torch.tensor([[1.0, 0.0]], device=cuda, dtype=t).expand(2003, 2)
    y, dx = _both(x, dy, w, act="gelu")[:2]
    g = g.double()
    normal, slope = 0.5 * torch.special.erfc(-g * 0.5 ** 0.5), (-g * g / 2).exp() / (2 * torch.pi) ** 0.5
    a, da, size = g * normal, normal + g * slope, normal + g.abs() * slope  # (ndtr is 1 + erf: it cancels in 64 bits too)
    steps = (3 * g * g + 24) * U
    half = 2.001 * HALF[t]
    for got, want, of in ((y[:, 0], a, a.abs()), (dx[:, 0], da, size), (dx[:, 1], a, a.abs())):
        assert bool(((got.double() - want).abs() <= steps * of + half * want.abs() + TINY[t]).all())


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("dense", [True, False])
@pytest.mark.parametrize("gate,up", [(True, False), (False, True)])
def test_orders_of_gate_and_up(cuda, gate, up, dense, t):
    """Weights of different orders: the results of one order, each gradient in its own weight's."""
    x, dy, w, off = _operands(cuda, [70] if dense else [30, 0, 40], 72, 136, t, dense=dense)
    want = _both(x, dy, w, off)
    turn = lambda m, columns: m.mT.contiguous().mT if columns else m  # noqa: E731
    mixed = [turn(w[0], gate), turn(w[1], up), w[2]]
    got = _both(x, dy, mixed, off)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for a, m in zip(got[2:], mixed):
        assert a.stride() == m.stride()


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("lengths", [[3], [300], [200, 0, 150], [1, 2, 3]])
def test_wait_runs_out_in_what_is_kept(cuda, t, lengths):
    """pre is a result too: after a wait that gave up (20 ms) it is NaN, and so is what a backward call makes of it."""
    x, dy, w, off = _operands(cuda, lengths, 64, 96, t)
    status, hold = (torch.zeros(1, dtype=torch.int32, device=cuda) for _ in range(2))
    torch.cuda.synchronize()
    try:
        S.soap_wait_limit(20_000_000, hold)
        y, pre = ffn_forward(x, *w, offsets=off, keep=True, status=status)
        torch.cuda.synchronize()
    finally:
        S.soap_wait_limit(0, None)
    assert int(status) == S.STATUS_TIMEOUT
    assert bool(y.isnan().all()) and bool(pre.isnan().all())
    grads = ffn_backward(dy, x, pre, *w, offsets=off)
    assert bool(grads[0].isnan().all())
    for m in grads[1:]:
        assert all(bool(m[i].isnan().all()) for i, n in enumerate(lengths) if n)


@pytest.mark.parametrize("t", [BF, F32])
def test_no_rows_and_bad_offsets(cuda, t):
    w = [torch.randn(2, *s, device=cuda).to(t) for s in ((8, 16), (8, 16), (16, 8))]
    x = torch.randn(0, 8, device=cuda).to(t)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    for off, told in (([0, 0, 0], 0), ([0, 3, 3], S.STATUS_RANGE), ([0, 0, -1], S.STATUS_RANGE)):
        off = torch.tensor(off, dtype=torch.int32, device=cuda)
        status.zero_()
        y, pre = ffn_forward(x, *w, offsets=off, keep=True, status=status)
        assert int(status) == told
        for params in (False, True):
            status.zero_()
            grads = ffn_backward(y, x, pre, *w, offsets=off, params=params, status=status)
            assert int(status) == told and grads[0].shape == x.shape
            assert not params or not any(bool(g.any()) for g in grads[1:])


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("lengths", [[140000], [65537] * 3, [5, 65600, 0, 131073]])
def test_long_sums_stay_in_the_workspace(cuda, t, lengths):
    """Sums along more rows than one accumulator takes: their parts fit the size that is asked for."""
    lib, dt, rows, hidden, width = S.load_library(), S.DTYPES[t], sum(lengths), 64, 72
    x, dy, w, off = _operands(cuda, lengths, hidden, width, t)
    want = _both(x, dy, w, off)
    _, pre = ffn_forward(x, *w, offsets=off, keep=True)
    dx, grads = torch.empty_like(x), [torch.empty_like(m) for m in w]
    mat = lambda m: S.layer_matrix(m.data_ptr(), m.shape[-1], m.shape[-1] * m.shape[-2], 0)  # noqa: E731
    size = lib.layer_ffn_workspace_bytes(rows, hidden, width, len(lengths), dt, 1, 1)
    ws = torch.full((size + (1 << 20),), 0xA5, dtype=torch.uint8, device=cuda)
    code = lib.layer_ffn_backward(
        rows, hidden, width, len(lengths), off.data_ptr(), dy.data_ptr(), hidden, x.data_ptr(), hidden, dt,
        *(mat(m) for m in w), 0, pre.data_ptr(), dx.data_ptr(), hidden, *(mat(m) for m in grads), None, ws.data_ptr(), size,
        torch.cuda.current_stream(cuda).cuda_stream)
    assert code == 0 and bool((ws[size:] == 0xA5).all())
    assert all(torch.equal(a, b) for a, b in zip([dx, *grads], want[1:]))
