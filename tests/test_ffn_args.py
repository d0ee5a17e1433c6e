"""The feed-forward block's C entry points refuse invalid arguments on the host, before any device work: no GPU is
needed."""
import pytest
import torch

from paper_2607_20548_gb300 import build, ffn_backward, ffn_forward
from paper_2607_20548_gb300 import soap as S

PTR, ODD = 1 << 20, (1 << 20) + 1  # stand-ins: refused calls never read them


def _mat(ld, stride=1 << 10, data=PTR, columns=0):
    return S.layer_matrix(data, ld, stride, columns)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return S.load_library()


OK = dict(rows=20, hidden=16, width=24, groups=2, offsets=PTR, x=PTR, ld_x=16, type=1, gate=_mat(24), up=_mat(24),
          down=_mat(16), act=0, y=PTR, ld_y=16, pre=PTR, status=None, ws=PTR, bytes=1 << 30)
WRONG = (dict(rows=-1), dict(rows=1 << 31), dict(hidden=0), dict(hidden=65537), dict(width=0), dict(width=65537),
         dict(groups=0), dict(groups=1025), dict(offsets=None), dict(offsets=ODD), dict(x=None), dict(x=ODD), dict(ld_x=15),
         dict(type=3), dict(type=-1), dict(gate=None), dict(gate=_mat(23)), dict(gate=_mat(24, stride=15 * 24 + 23)),
         dict(gate=_mat(24, columns=1)), dict(up=_mat(24, data=None)), dict(up=_mat(24, data=ODD)), dict(down=_mat(15)),
         dict(down=_mat(23, columns=1)), dict(act=2), dict(act=-1), dict(pre=PTR + 4), dict(status=ODD), dict(ws=None),
         dict(ws=PTR + 16), dict(bytes=256))


@pytest.mark.parametrize("change", WRONG + (dict(y=None), dict(y=ODD), dict(ld_y=15)))
def test_forward_refuses(lib, change):
    assert lib.layer_ffn_forward(*{**OK, **change}.values(), None) == 1


BACK = dict(rows=20, hidden=16, width=24, groups=2, offsets=PTR, dy=PTR, ld_dy=16, x=PTR, ld_x=16, type=1, gate=_mat(24),
            up=_mat(24), down=_mat(16), act=0, pre=PTR, dx=PTR, ld_dx=16, d_gate=_mat(24), d_up=_mat(24), d_down=_mat(16),
            status=None, ws=PTR, bytes=1 << 30)


@pytest.mark.parametrize("change", WRONG + (dict(dy=None), dict(dy=ODD), dict(ld_dy=15), dict(dx=None), dict(ld_dx=15),
                                            dict(pre=None), dict(d_gate=None), dict(d_down=None), dict(d_up=_mat(23)),
                                            dict(d_down=_mat(24, columns=1)), dict(d_gate=_mat(24, data=None))))
def test_backward_refuses(lib, change):
    assert lib.layer_ffn_backward(*{**BACK, **change}.values(), None) == 1


def test_sizes(lib):
    f, pre = lib.layer_ffn_workspace_bytes, lib.layer_ffn_pre_elems
    assert f(-1, 8, 8, 1, 0, 1, 0) == f(1, 0, 8, 1, 0, 1, 0) == f(1, 8, 65537, 1, 0, 1, 0) == f(1, 8, 8, 0, 0, 1, 0) == 0
    assert f(1, 8, 8, 1, 3, 1, 0) == pre(-1, 8, 1) == pre(1, 0, 1) == 0
    assert f(1, 8, 8, 1, 1, 1, 0) > 0 and pre(100, 24, 1) >= 2 * 100 * 24
    for type_ in range(3):  # results' intermediates, at least
        size = 4 if type_ == 0 else 2
        assert f(1000, 64, 96, 3, type_, 1, 0) >= 1000 * 96 * size
        assert f(1000, 64, 96, 3, type_, 1, 1) >= 3 * 1000 * 96 * size
        assert f(1000, 64, 96, 3, type_, 0, 1) >= f(1000, 64, 96, 3, type_, 1, 1)


def test_binding_refuses_host_tensors():
    x, w, d = torch.zeros(2, 8), torch.zeros(8, 8), torch.zeros(8, 8)
    with pytest.raises(TypeError):
        ffn_forward(x, w, w, d)
    with pytest.raises(TypeError):
        ffn_backward(x, x, x, w, w, d)
