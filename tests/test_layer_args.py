"""The stand-alone operators' C entry points refuse invalid arguments on the host, before any device
work, and the binding refuses host tensors: no GPU is needed."""
import ctypes
import re

import pytest
import torch

from paper_2607_20548_gb300 import build, layer_norm_forward, muon_orthogonalize, route_forward
from paper_2607_20548_gb300 import soap as S
from tests.test_abi import _declared

PTR, ODD = 1 << 20, (1 << 20) + 2  # stand-ins: refused calls never read them


def _lib():
    build.build()
    return S.load_library()


def test_every_declared_symbol_is_exported():
    lib = _lib()
    names = _declared("layer.h", "layer_")
    assert set(names) == set(S.LAYER_EXPORTS)
    assert not [n for n in names if not hasattr(lib, n)]


def test_norm_refusals():
    f = _lib().layer_norm_forward
    ok = dict(rows=4, width=8, x=PTR, ld_x=8, x_type=1, w=PTR, b=PTR, w_type=0, eps=1e-5, y=PTR, ld_y=8, mean=PTR,
              rstd=PTR, status=None)
    for change in (dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=1 << 31), dict(x=None), dict(y=None),
                   dict(ld_x=7), dict(ld_y=7), dict(x_type=3), dict(x_type=-1), dict(w_type=2), dict(eps=-1.0),
                   dict(eps=float("nan")), dict(x=PTR + 1), dict(mean=ODD), dict(w=ODD), dict(x_type=0, x=ODD), dict(status=ODD)):
        assert f(*{**ok, **change}.values(), None) == 1, change
    assert f(*{**ok, "rows": 0, "x": None, "y": None}.values(), None) == 0
    g = _lib().layer_norm_backward
    need = _lib().layer_norm_workspace_bytes(4, 8)
    assert need >= 4 * 2 * 8 * 4 and _lib().layer_norm_workspace_bytes(-1, 8) == 0
    ok = dict(rows=4, width=8, dy=PTR, ld_dy=8, x=PTR, ld_x=8, x_type=1, mean=PTR, rstd=PTR, w=PTR, w_type=0, dx=PTR,
              ld_dx=8, dw=PTR, db=PTR, ws=PTR, bytes=need, status=None)
    for change in (dict(rows=-1), dict(width=0), dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None),
                   dict(rstd=None), dict(ld_dx=7), dict(ld_dy=1), dict(ws=None), dict(bytes=need - 1), dict(ws=PTR + 4),
                   dict(dw=ODD), dict(w_type=2)):
        assert g(*{**ok, **change}.values(), None) == 1, change


def test_route_refusals():
    lib = _lib()
    need = lib.layer_route_workspace_bytes(9, 16)
    assert need > 0
    assert lib.layer_route_workspace_bytes(9, 0) == lib.layer_route_workspace_bytes(9, 1025) == 0
    assert lib.layer_route_workspace_bytes(-1, 16) == 0
    ok = dict(tokens=9, experts=16, k=4, z=PTR, ld=16, type=0, mask=None, normalize=1, coef=0.1, idx=PTR, gates=PTR,
              stats=PTR, counts=PTR, live=PTR, mean=PTR, loss=PTR, status=None, ws=PTR, bytes=need)
    for change in (dict(tokens=-1), dict(tokens=1 << 31), dict(experts=0), dict(experts=1025), dict(k=0), dict(k=17),
                   dict(experts=64, ld=64, k=33, bytes=1 << 30), dict(z=None), dict(z=ODD), dict(ld=15), dict(type=3),
                   dict(coef=float("nan")), dict(idx=None), dict(gates=None), dict(counts=None), dict(live=None),
                   dict(stats=PTR + 4), dict(loss=None), dict(mean=ODD), dict(status=ODD), dict(ws=None), dict(ws=PTR + 8),
                   dict(bytes=need - 1)):
        assert lib.layer_route_forward(*{**ok, **change}.values(), None) == 1, change
    ok = dict(tokens=9, experts=16, k=4, z=PTR, ld=16, type=0, mask=None, normalize=1, coef=0.1, dloss=1.0, idx=PTR,
              stats=PTR, counts=PTR, live=PTR, dgates=PTR, dz=PTR, ld_d=16)
    for change in (dict(tokens=-1), dict(experts=0), dict(k=0), dict(z=None), dict(dz=None), dict(ld_d=15), dict(idx=None),
                   dict(stats=None), dict(counts=None), dict(live=None), dict(dgates=ODD), dict(dloss=float("inf"))):
        assert lib.layer_route_backward(*{**ok, **change}.values(), None) == 1, change
    assert lib.layer_route_backward(*{**ok, "tokens": 0}.values(), None) == 0


def test_orthogonalize_refusals():
    lib = _lib()
    need = lib.muon_orthogonalize_workspace_bytes(2, 5, 9, 0)
    assert need > 0
    for bad in ((0, 5, 9, 0), (65536, 5, 9, 0), (2, 0, 9, 0), (2, 5, 0, 0), (2, 65537, 1, 0), (1, 65536, 65536, 0),
                (2, 5, 9, 3), (2, 5, 9, -1)):
        assert lib.muon_orthogonalize_workspace_bytes(*bad) == 0, bad
    ok = dict(batch=2, rows=5, cols=9, M=PTR, ld=9, stride=45, type=0, coeffs=None, steps=4, eps=1e-7, out=PTR, ld_out=9,
              stride_out=45, ws=PTR, bytes=need, status=None)
    nan = (ctypes.c_float * 12)(*([1.0] * 11 + [float("nan")]))
    for change in (dict(batch=0), dict(rows=0), dict(cols=0), dict(M=None), dict(M=ODD), dict(ld=8), dict(stride=44),
                   dict(type=3), dict(coeffs=nan), dict(steps=0), dict(steps=65), dict(eps=0.0), dict(eps=float("inf")),
                   dict(out=None), dict(ld_out=8), dict(stride_out=1), dict(ws=None), dict(ws=PTR + 16),
                   dict(bytes=need - 1), dict(status=ODD)):
        assert lib.muon_orthogonalize(*{**ok, **change}.values(), None) == 1, change


def test_binding_refuses_host_tensors():
    _lib()
    x = torch.zeros(4, 8)
    for call in (lambda: layer_norm_forward(x), lambda: route_forward(x, 2), lambda: muon_orthogonalize(x),
                 lambda: layer_norm_forward(None)):
        with pytest.raises(TypeError, match="CUDA tensor"):
            call()


def test_headers_state_every_default():
    """The polynomial that NULL coefficients select is the optimizer's."""
    text = open(re.sub(r"tests.*", "include/muon.h", __file__)).read()
    assert "(15 - 10 x + 3 x^2) / 8" in text
