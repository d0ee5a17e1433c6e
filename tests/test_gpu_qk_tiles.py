"""The rotation's kernel that takes heads in tiles (include/layer.h, layer_qk_*) against fp64: several sequences, both
kinds of pairs, units of 1 to 8 elements, heads over several tiles, positions. That a case reaches it shows in that its
waits run out while soap_wait_limit's flag is unset: calls of fewer heads wait for nothing. Tolerances: as in
test_gpu_qk."""
import pytest
import torch

from paper_2607_20548_gb300 import qk_rotary_backward, qk_rotary_forward
from paper_2607_20548_gb300 import soap as S
from tests.test_gpu_qk import BF, F32, HF, _check, _run, _table

pytestmark = pytest.mark.gpu


def _in_tiles(cuda, q, k, **how):
    """Whether both passes of these operands wait for tiles (5 ms)."""
    status = [torch.zeros(1, dtype=torch.int32, device=cuda) for _ in range(2)]
    hold = torch.zeros(1, dtype=torch.int32, device=cuda)
    torch.cuda.synchronize()
    try:
        S.soap_wait_limit(5_000_000, hold)
        qk_rotary_forward(q, k, status=status[0], **how)
        qk_rotary_backward(q, k, q, k, status=status[1], **how)
        torch.cuda.synchronize()
    finally:
        S.soap_wait_limit(0, None)
    return all(int(s) == S.STATUS_TIMEOUT for s in status)


def _make(cuda, name, lead, dim, t, seed=5):
    g = torch.Generator(device=cuda).manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=cuda, generator=g).to(t)  # noqa: E731

    def make(n):
        if name == "fused":
            return r(*lead, n + 3, dim)[..., 3:, :]
        if name == "heads_first":
            return r(*lead[:-1], n, lead[-1], dim).transpose(-2, -3)
        return r(*lead, n, dim)
    return make


CASES = pytest.mark.parametrize("name,lead,heads,kv,dim,rotary", [
    ("heads_first", (3, 4001), 4, 2, 64, 64),   # several sequences, cut at their ends
    ("fused", (3, 4001), 5, 1, 64, 64),
    ("fused", (9001,), 3, 3, 128, 96),
    ("heads_first", (9001,), 7, 2, 96, 48),
    ("dense", (2, 6111), 4, 2, 64, 62),         # units of 1 element
    ("heads_first", (5, 1777), 6, 3, 48, 36),   # of 2
    ("dense", (1200,), 70, 33, 256, 128),       # more heads than a tile holds
    ("fused", (2, 1500), 300, 0, 16, 16),
    ("heads_first", (16, 1), 9000, 512, 32, 32),  # a token a sequence
    ("heads_first", (700, 5), 40, 8, 64, 32),   # shorter than a tile
    ("dense", (50001,), 1, 1, 8, 8)])


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("t,wt", [(BF, BF), (BF, F32), (HF, HF), (F32, F32), (HF, None)])
@CASES
def test_against_fp64(cuda, name, lead, heads, kv, dim, rotary, t, wt, inter):
    _run(cuda, lead, heads, kv, dim, rotary, inter, t, wt, make=_make(cuda, name, lead, dim, t))


@pytest.mark.parametrize("t", [BF, F32])
@CASES
def test_cases_are_in_tiles(cuda, name, lead, heads, kv, dim, rotary, t):
    make = _make(cuda, name, lead, dim, t)
    cos, sin = _table(cuda, max(lead), rotary)
    tiled = _in_tiles(cuda, make(heads), make(kv), cos=cos, sin=sin)
    assert tiled


def test_few_heads_are_not_in_tiles(cuda):
    q, k = torch.randn(50, 4, 64, device=cuda), torch.randn(50, 2, 64, device=cuda)
    tiled = _in_tiles(cuda, q, k)
    assert not tiled


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("name", ["heads_first", "fused"])
def test_positions(cuda, t, name):
    """Default ones, one per token of a sequence, and some out of range far behind."""
    lead, dim = (3, 4001), 64
    make = _make(cuda, name, lead, dim, t)
    q, k = make(4), make(2)
    cos, sin = _table(cuda, 4001, dim)
    w = 1 + 0.1 * torch.randn(dim, device=cuda)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    own = torch.arange(4001, device=cuda)
    a = qk_rotary_forward(q, k, cos, sin, None, w, w, status=status)
    da = qk_rotary_backward(q, k, q, k, cos, sin, None, w, w, status=status)
    _check(q, k, cos, sin, own, w, w, 1e-6, False, q, k, a, da)
    for pos in (own, own.int(), own.expand(lead)):
        b = qk_rotary_forward(q, k, cos, sin, pos, w, w, status=status)
        db = qk_rotary_backward(q, k, q, k, cos, sin, pos, w, w, status=status)
        assert all(torch.equal(x, y) for x, y in zip(a + da, b + db))
    assert int(status) == 0
    pos = own.repeat(3, 1)
    pos[2, 3998], pos[1, 7] = 4001, -5
    bad = torch.zeros(lead, dtype=torch.bool, device=cuda)
    bad[2, 3998] = bad[1, 7] = True
    b = qk_rotary_forward(q, k, cos, sin, pos, w, w, status=status)
    assert int(status) == S.STATUS_RANGE
    status.zero_()
    db = qk_rotary_backward(q, k, q, k, cos, sin, pos, w, w, status=status)
    assert int(status) == S.STATUS_RANGE
    for x, y in zip(a + da[:2], b + db[:2]):
        assert torch.equal(x[~bad], y[~bad]) and bool(y[bad].isnan().all())
    assert bool(db[2].isnan().all()) and bool(db[3].isnan().all())
