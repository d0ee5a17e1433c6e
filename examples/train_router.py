#!/usr/bin/env python3
"""Trains the router of a mixture-of-experts layer with the library's operators: pre-norm, router
product, top-k routing with the balance loss, their gradients, and an orthogonalised-momentum
update of the router's weight.

    python examples/train_router.py [--steps 60] [--tokens 8192] [--hidden 2048] [--experts 64] [--k 8]

The experts are stood in for by fixed output vectors, and tokens come in groups that each want the
output of k experts of their own, so the loss can only fall by routing every group to its experts.
A tenth of the tokens is padding, which the mask leaves out. Nothing here waits for the device
but the report.
"""
import argparse
import math
import os
import sys
from typing import NamedTuple

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_20548_gb300 as lib  # noqa: E402


class Problem(NamedTuple):
    """tokens [T, hidden], mask [T], the experts' outputs [experts, width], wanted outputs [T, width]."""
    tokens: torch.Tensor
    mask: torch.Tensor
    outputs: torch.Tensor
    wanted: torch.Tensor


class Router:
    """Pre-norm weight and bias, the router's weight [hidden, experts] and its momentum."""

    def __init__(self, hidden, experts, generator, device):
        self.gain, self.bias = torch.ones(hidden, device=device), torch.zeros(hidden, device=device)
        self.weight = torch.randn(hidden, experts, generator=generator, device=device) / math.sqrt(hidden)
        self.momentum = torch.zeros_like(self.weight)


def make_problem(tokens, hidden, experts, k, generator, device, width=32):
    group = torch.randint(experts, (tokens,), generator=generator, device=device)
    centres = torch.randn(experts, hidden, generator=generator, device=device)
    x = centres[group] + 0.5 * torch.randn(tokens, hidden, generator=generator, device=device)
    outputs = torch.randn(experts, width, generator=generator, device=device)
    theirs = (group[:, None] + torch.arange(k, device=device)) % experts  # group g wants experts g .. g + k - 1
    mask = torch.rand(tokens, generator=generator, device=device) >= 0.1
    return Problem(x, mask, outputs, outputs[theirs].mean(1))


def gradients(p, r, k, coef=0.01, status=None):
    """(mean squared error, Routing, dweight, dgain, dbias) of one pass. The objective is
    the error of the gated outputs, averaged over the tokens that are not masked, plus the balance loss."""
    y, mean, rstd = lib.layer_norm_forward(p.tokens, r.gain, r.bias, status=status)
    z = lib.soap_gemm(y, r.weight)
    routing = lib.route_forward(z, k, p.mask, coef=coef, status=status)
    chosen = p.outputs[routing.indices.clamp(min=0).long()]          # [T, k, width]; no expert: index -1, gate 0
    off = torch.einsum("tk,tkw->tw", routing.gates, chosen) - p.wanted
    share = p.mask / (routing.live.clamp(min=1) * off.shape[1])      # a masked token's error does not count
    error = (off.square().sum(1) * share).sum()
    dgates = 2 * torch.einsum("tw,tkw->tk", off * share[:, None], chosen)
    dz = lib.route_backward(z, routing, dgates)
    dweight = lib.soap_gemm(y, dz, trans_a=True)
    dy = lib.soap_gemm(dz, r.weight, trans_b=True)
    _, dgain, dbias = lib.layer_norm_backward(dy, p.tokens, mean, rstd, r.gain, status=status)
    return error, routing, dweight, dgain, dbias


def step(p, r, k, lr=2e-4, beta=0.9, coef=0.01, status=None):
    """One pass and one update: the weight by its orthogonalised momentum, gain and bias by their gradients."""
    error, routing, dweight, dgain, dbias = gradients(p, r, k, coef, status)
    r.momentum.lerp_(dweight, 1 - beta)
    update = lib.muon_orthogonalize(r.momentum, status=status)
    r.weight.sub_(update, alpha=lr * math.sqrt(max(update.shape)))
    r.gain.sub_(dgain, alpha=lr)
    r.bias.sub_(dbias, alpha=lr)
    return error, routing


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("steps", 60), ("tokens", 8192), ("hidden", 2048), ("experts", 64), ("k", 8), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    dev = torch.device("cuda", 0)
    g = torch.Generator(dev).manual_seed(a.seed)
    p, r = make_problem(a.tokens, a.hidden, a.experts, a.k, g, dev), Router(a.hidden, a.experts, g, dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    for t in range(a.steps):
        error, routing = step(p, r, a.k, status=status)
        if t % 10 == 0 or t == a.steps - 1:
            counts = routing.counts.float()
            print(f"step {t:4d}  error {error.item():.4f}  balance loss {routing.loss.item():.5f}  "
                  f"busiest expert {(counts.max() / counts.mean()).item():.2f} x the mean")
    if status.item():
        sys.exit(f"device status {status.item():#x}")


if __name__ == "__main__":
    main()
