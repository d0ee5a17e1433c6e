"""muon_orthogonalize (include/muon.h) against the iterations in fp64.

Tolerance (from the arithmetic, relative Frobenius norm): each of a step's three results is stored
with b bits (bf16: one fp16 value, b = 11; fp16 and fp32: a hi + lo pair, b = 22), a relative error
of at most 2^-b per element, independent from element to element. What is stored in step i
reaches the result through the later steps, whose gain relative to the signal's stays near 1 for
well-conditioned matrices; 2 is allowed. 3 n such errors add in quadrature. The fp32 accumulator
drops at most one unit (2^-23) per 16 products of a sum of K, and the result is rounded to its
type once. Inputs: a low-rank part over a noise floor, as momenta are.
"""
import math

import pytest
import torch

from paper_2607_20548_gb300 import muon_orthogonalize
from paper_2607_20548_gb300 import soap as S

pytestmark = pytest.mark.gpu

QUINTIC = (15 / 8, -10 / 8, 3 / 8)
ALL = [torch.bfloat16, torch.float16, torch.float32]


def _tol(dtype, steps, m, n):
    b = 11 if dtype == torch.bfloat16 else 22
    return torch.finfo(dtype).eps / 2 + 2 * math.sqrt(3 * steps) * 2.0 ** -b + math.ceil(max(m, n) / 16) * 2.0 ** -23


def _ref(M, coeffs, eps=1e-7):
    X = M.double()
    X = X / torch.linalg.matrix_norm(X, keepdim=True).clamp_min(eps)
    tall = X.shape[-2] > X.shape[-1]
    X = X.mT if tall else X
    for a, b, c in coeffs:
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.mT if tall else X


def _momentum(cuda, shape, dtype, seed=0, scale=1e-3):
    g = torch.Generator(device=cuda).manual_seed(seed)
    *lead, m, n = shape
    q = min(4, m, n)
    low = torch.randn(*lead, m, q, device=cuda, generator=g) @ torch.randn(*lead, q, n, device=cuda, generator=g)
    return ((low * (0.5 / math.sqrt(q)) + torch.randn(*lead, m, n, device=cuda, generator=g)) * scale).to(dtype)


def _rel(x, y):
    return float(torch.linalg.norm(x.double() - y) / torch.linalg.norm(y))


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("shape", [(64, 64 + 40), (128, 256), (256, 128), (1, 300), (300, 1), (7, 5), (5, 7), (129, 257),
                                   (257, 129), (3, 65, 200), (2, 200, 65), (2, 2, 40, 90), (640, 1500), (1501, 333)])
def test_shapes(cuda, shape, dtype):
    M = _momentum(cuda, shape, dtype)
    out = muon_orthogonalize(M, ns_steps=6)
    assert out.shape == M.shape and out.dtype == dtype
    assert _rel(out, _ref(M, [QUINTIC] * 6)) <= _tol(dtype, 6, *shape[-2:])


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("steps", [1, 2, 5, 16])
def test_steps(cuda, steps, dtype):
    M = _momentum(cuda, (2, 160, 420), dtype, seed=steps)
    assert _rel(muon_orthogonalize(M, ns_steps=steps), _ref(M, [QUINTIC] * steps)) <= _tol(dtype, steps, 160, 420)


@pytest.mark.parametrize("dtype", ALL)
def test_own_coefficients(cuda, dtype):
    # a steep first step, a step without its c and a step without its b and c; singular values pass 1
    coeffs = [(4.0, -9.0, 6.0), (2.0, -1.0, 0.0), (1.5, -0.5, 0.0), (1.0, 0.0, 0.0)]
    M = _momentum(cuda, (96, 320), dtype)
    assert _rel(muon_orthogonalize(M, coeffs=coeffs), _ref(M, coeffs)) <= 2 * _tol(dtype, 4, 96, 320)


@pytest.mark.parametrize("dtype", ALL)
def test_result_is_orthogonal(cuda, dtype):
    M = _momentum(cuda, (2, 100, 400), dtype)
    X = muon_orthogonalize(M, ns_steps=16).double()
    assert float((X @ X.mT - torch.eye(100, device=cuda, dtype=torch.float64)).abs().max()) <= 8 * _tol(dtype, 16, 100, 400)


@pytest.mark.parametrize("dtype", ALL)
def test_layouts(cuda, dtype):
    """Transposed views, padded rows, sliced batches and unaligned starts give the dense matrix's result, and
    leave what lies between their rows alone."""
    M = _momentum(cuda, (3, 130, 72), dtype)
    want = muon_orthogonalize(M, ns_steps=5)
    view = M.mT.contiguous().mT
    got = muon_orthogonalize(view, ns_steps=5)
    assert got.stride() == view.stride()
    tol = 2 * _tol(dtype, 5, 130, 72)
    assert _rel(got, want.double()) <= tol
    for pad in (1, 3, 8):
        big = torch.full((3, 130, 72 + pad), float("nan"), dtype=dtype, device=cuda)
        big[:, :, pad:] = M
        assert _rel(muon_orthogonalize(big[:, :, pad:], ns_steps=5), want.double()) <= tol
    wide = torch.full((6, 130, 72), float("nan"), dtype=dtype, device=cuda)
    wide[::2] = M
    assert _rel(muon_orthogonalize(wide[::2], ns_steps=5), want.double()) <= tol
    # neither order: copied
    odd = M.unsqueeze(-1).repeat(1, 1, 1, 2)[..., 0]
    assert _rel(muon_orthogonalize(odd, ns_steps=5), want.double()) <= tol


@pytest.mark.parametrize("dtype", ALL)
def test_zero_and_scale(cuda, dtype):
    M = _momentum(cuda, (3, 64, 96), dtype)
    M[1] = 0
    out = muon_orthogonalize(M, ns_steps=6)
    assert not out[1].any()
    assert _rel(out[2], _ref(M[2], [QUINTIC] * 6)) <= _tol(dtype, 6, 64, 96)
    # X_0 does not depend on a power of two in M ...
    # (fp16 takes no smaller one: 2^-4 M has subnormal elements, which are other numbers)
    for e in (4, 6) if dtype == torch.float16 else (60, -60, 100, -100):
        k = 2.0 ** e
        assert torch.equal(muon_orthogonalize(M[2] * k, ns_steps=6, eps=1e-37), out[2]), e
    # ... until the norm falls below eps
    small = muon_orthogonalize(M[2], ns_steps=3, eps=1e3)
    assert _rel(small, _ref(M[2], [QUINTIC] * 3, eps=1e3)) <= 64 * _tol(dtype, 3, 64, 96)


def test_nonfinite_stays_in_its_matrix(cuda):
    for dtype in ALL:
        M = _momentum(cuda, (4, 70, 50), dtype)
        want = muon_orthogonalize(M, ns_steps=4)
        M[1, 3, 4] = float("nan")
        M[2, 60, 49] = float("inf")
        status = torch.zeros(1, dtype=torch.int32, device=cuda)
        out = muon_orthogonalize(M, ns_steps=4, status=status)
        assert int(status) == S.STATUS_NONFINITE
        assert out[1].isnan().all() and out[2].isnan().all()
        assert torch.equal(out[0], want[0]) and torch.equal(out[3], want[3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_same_bits_and_other_stream(cuda, dtype):
    M = _momentum(cuda, (2, 300, 500), dtype)
    a = muon_orthogonalize(M)
    assert torch.equal(a, muon_orthogonalize(M))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = muon_orthogonalize(M, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a, b)


def test_agrees_with_the_step(cuda):
    """The operator on a momentum gives the Muon step's update (whose iterations are bf16, to their error)."""
    g = torch.Generator(device=cuda).manual_seed(3)
    G = torch.randn(256, 640, device=cuda, generator=g)
    W = torch.zeros(256, 640, device=cuda)
    opt = S.MuonOptimizer([(256, 640)], lr=1.0, weight_decay=0.0)
    opt.step([W], [G])
    assert opt.status() == 0
    want = -math.sqrt(640) * muon_orthogonalize(opt.state_get(0))
    assert _rel(W, want.double()) <= 2e-2


def test_refusals(cuda):
    M = torch.randn(8, 8, device=cuda)
    with pytest.raises(TypeError):
        muon_orthogonalize(M.cpu())
    with pytest.raises(TypeError):
        muon_orthogonalize(M.double())
    with pytest.raises(ValueError):
        muon_orthogonalize(M[0])
    with pytest.raises(ValueError):
        muon_orthogonalize(torch.zeros(1, 70000, device=cuda))
    for bad in (dict(ns_steps=0), dict(ns_steps=65), dict(eps=0.0), dict(coeffs=[]), dict(coeffs=[(1.0, float("nan"), 0.0)])):
        with pytest.raises(S.SoapError):
            muon_orthogonalize(M, **bad)
    with pytest.raises(TypeError):
        muon_orthogonalize(M, status=torch.zeros(1, device=cuda))
    assert muon_orthogonalize(torch.empty(0, 4, 4, device=cuda)).shape == (0, 4, 4)
