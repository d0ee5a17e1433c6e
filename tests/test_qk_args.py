"""The rotation's C entry points refuse invalid arguments on the host, before any device work: no GPU is needed."""
import pytest
import torch

from paper_2607_20548_gb300 import build, qk_rotary_backward, qk_rotary_forward
from paper_2607_20548_gb300 import soap as S

PTR, ODD = 1 << 20, (1 << 20) + 1  # stand-ins: refused calls never read them


def _heads(data=PTR, batch=4 * 5 * 8, token=5 * 8, head=8):
    return S.layer_heads(data, batch, token, head)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return S.load_library()


OK = dict(batch=2, length=4, heads=3, kv_heads=2, dim=8, rotary=8, interleaved=0, q=_heads(), k=_heads(), type=1,
          q_weight=PTR, k_weight=PTR, w_type=0, eps=1e-6, cos=PTR, sin=PTR, places=4, positions=PTR, positions_64=0,
          q_out=_heads(), k_out=_heads(), status=None)
WRONG = (dict(batch=-1), dict(length=-1), dict(length=1 << 31), dict(batch=1 << 16, length=1 << 16), dict(heads=-1),
         dict(heads=32769), dict(kv_heads=32769), dict(dim=7), dict(dim=0), dict(dim=514), dict(rotary=10), dict(rotary=3),
         dict(rotary=-2), dict(q=None), dict(k=_heads(None)), dict(q=_heads(ODD)), dict(q=_heads(token=-1)),
         dict(type=3), dict(type=-1), dict(w_type=2), dict(q_weight=ODD), dict(eps=-1.0), dict(eps=float("nan")),
         dict(cos=None), dict(sin=ODD), dict(places=-1), dict(positions=ODD), dict(positions=PTR + 4, positions_64=1),
         dict(status=ODD))


@pytest.mark.parametrize("change", WRONG + (dict(q_out=None), dict(k_out=_heads(head=7)), dict(q_out=_heads(token=7)),
                                            dict(q_out=_heads(batch=0))))
def test_forward_refuses(lib, change):
    assert lib.layer_qk_forward(*{**OK, **change}.values(), None) == 1


def test_nothing_to_do(lib):
    for change in (dict(batch=0), dict(length=0, q=None, cos=None), dict(heads=0, kv_heads=0, q=None, k=None)):
        assert lib.layer_qk_forward(*{**OK, **change}.values(), None) == 0


def _backward():
    c = dict(OK)
    out = {n: c.pop(n) for n in ("q_out", "k_out", "status")}
    head = {n: c.pop(n) for n in ("batch", "length", "heads", "kv_heads", "dim", "rotary", "interleaved")}
    return {**head, "dq": _heads(), "dk": _heads(), **c, "dx_q": out["q_out"], "dx_k": out["k_out"], "dwq": PTR,
            "dwk": PTR, "status": None, "ws": PTR, "bytes": 1 << 24}


@pytest.mark.parametrize("change", WRONG + (dict(dq=None), dict(dk=_heads(ODD)), dict(dx_q=None), dict(dx_k=_heads(head=7)),
                                            dict(dwq=None), dict(dwk=ODD), dict(ws=None), dict(ws=PTR + 8), dict(bytes=64)))
def test_backward_refuses(lib, change):
    assert lib.layer_qk_backward(*{**_backward(), **change}.values(), None) == 1


def test_workspace(lib):
    f = lib.layer_qk_workspace_bytes
    assert f(-1, 4, 1, 1, 8) == f(1, 4, -1, 1, 8) == f(1, 4, 1, 1, 7) == f(1 << 16, 1 << 16, 1, 1, 8) == 0
    assert 0 < f(1, 1, 1, 0, 8) <= f(1, 4096, 16, 4, 8) <= 4 * 8 * 1024


def test_binding_refuses_host_tensors():
    t = torch.zeros(2, 1, 8)
    with pytest.raises(TypeError):
        qk_rotary_forward(t, t)
    with pytest.raises(TypeError):
        qk_rotary_backward(t, t, t, t)
