"""The operators together, as examples/train_router.py runs them, against the same step in fp64.

Tolerance of the gradients (u = 2^-24, hidden = 128): a logit sums 128 products of magnitude sum near 11,
so it is within 150 u * 11 = 1e-4 of its value at worst, and a probability within 2e-4 relatively. A
gradient's terms hold at most four such factors (probability, gate, its quotient's sum, the gated error), and
the differences p (u - sum p u) lose at most a factor of a few: 2e-3 of the gradient's norm.
"""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_router.py")
TOKENS, HIDDEN, EXPERTS, K = 1000, 128, 16, 4


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_router", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture
def run(example, cuda):
    g = torch.Generator(cuda).manual_seed(5)
    return example.make_problem(TOKENS, HIDDEN, EXPERTS, K, g, cuda), example.Router(HIDDEN, EXPERTS, g, cuda)


def _objective(p, gain, bias, weight, indices, coef):
    """The pass in fp64, the choice given."""
    x, live = p.tokens.double(), p.mask.double()
    x = x - x.mean(1, keepdim=True)
    y = x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * gain + bias
    z = y @ weight
    prob = torch.softmax(z, 1)
    gates = prob.gather(1, indices)
    gates = gates / gates.sum(1, keepdim=True)
    off = torch.einsum("tk,tkw->tw", gates, p.outputs.double()[indices]) - p.wanted
    n = live.sum()
    error = (off.square().mean(1) * live).sum() / n
    counts = torch.zeros(EXPERTS, dtype=torch.float64, device=z.device)
    counts.index_add_(0, indices.flatten(), live[:, None].expand(-1, K).flatten())
    loss = coef * EXPERTS / (K * n) * (counts * (prob * live[:, None]).sum(0) / n).sum()
    return z, counts, error, loss


@pytest.mark.parametrize("coef", [0.0, 0.5])
def test_gradients_of_a_pass(example, run, coef):
    p, r = run
    error, routing, *grads = example.gradients(p, r, K, coef)
    params = [t.double().requires_grad_() for t in (r.weight, r.gain, r.bias)]
    indices = torch.where(p.mask[:, None], routing.indices, 0).long()
    z, counts, want, loss = _objective(p, params[1], params[2], params[0], indices, coef)
    assert routing.live.item() == p.mask.sum().item()
    assert torch.equal(routing.counts.double(), counts.detach())
    least = z.gather(1, indices).min(1).values                        # the choice is the k largest logits'
    rest = z.scatter(1, indices, float("-inf")).max(1).values
    assert ((least - rest)[p.mask] > -2e-4).all()
    assert abs(error.item() - want.item()) <= 2e-3 * want.item()
    assert abs(routing.loss.item() - loss.item()) <= 2e-3 * loss.item()
    (want + loss).backward()
    for got, param in zip(grads, params):
        assert (got.double() - param.grad).norm() <= 2e-3 * param.grad.norm()


def test_training_lowers_the_error(example, run):
    p, r = run
    status = torch.zeros(1, dtype=torch.int32, device=p.tokens.device)
    errors = [example.step(p, r, K, lr=3e-3, status=status)[0] for _ in range(60)]
    errors = [e.item() for e in errors]
    assert status.item() == 0
    assert errors[-1] < 0.5 * errors[0]
