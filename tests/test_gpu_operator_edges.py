"""The stand-alone operators where one part of a kernel hands data to another: lanes of a row, warps of a
CTA, CTAs of a pair."""
import pytest
import torch

from paper_2607_20548_gb300 import route_backward, route_forward

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
