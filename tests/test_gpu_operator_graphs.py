"""The stand-alone operators in a CUDA graph: every call only enqueues work on its stream, so a captured
step replays on new inputs with the bits that direct calls give."""
import pytest
import torch

from paper_2607_20548_gb300 import (layer_norm_backward, layer_norm_forward, muon_orthogonalize, route_backward,
                                    route_forward)

pytestmark = pytest.mark.gpu


def _step(x, w, z, mask, M, small):
    y, mean, rstd = layer_norm_forward(x, w, w)
    grads = layer_norm_backward(y, x, mean, rstd, w)
    r = route_forward(z, 3, mask)
    dz = route_backward(z, r, r.gates)
    return [y, *grads, *r[:7], dz, muon_orthogonalize(M, ns_steps=3), muon_orthogonalize(small, ns_steps=3)]


@pytest.mark.parametrize("rows,width,tokens,experts", [(5, 96, 7, 12), (40, 1001, 20000, 33)])
def test_replay(cuda, rows, width, tokens, experts):
    g = torch.Generator(cuda).manual_seed(rows)

    def inputs():
        r = lambda *s: torch.randn(*s, device=cuda, generator=g)  # noqa: E731
        return [r(rows, width).bfloat16(), r(width), r(tokens, experts),
                torch.rand(tokens, device=cuda, generator=g) < 0.8, r(2, 300, 520).half(), r(90, 60).bfloat16()]

    held = inputs()
    side = torch.cuda.Stream(cuda)
    side.wait_stream(torch.cuda.current_stream(cuda))
    with torch.cuda.stream(side):
        _step(*held)
    torch.cuda.current_stream(cuda).wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(*held)
    for _ in range(2):
        fresh = inputs()
        for a, b in zip(held, fresh):
            a.copy_(b)
        graph.replay()
        for got, want in zip(out, _step(*fresh)):
            assert torch.equal(got, want)
