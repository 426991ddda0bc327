"""The example that runs the training and sampling calls together: the student's
loss falls, and one step's update equals the one that autograd gives."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_the_loss_falls(vie):
    from distill_student import train
    first, last = train(V=4001, streams=128, steps=120)
    assert last < 0.6 * first


def test_a_step_against_autograd(vie):
    """The tied matrix's gradient, from the same bf16 logits: the logits' gradient
    is rounded to bf16 (2^-8 of a value), so each sum may be off by 2^-8 of the
    sum of its terms' magnitudes (and half as much again for fp32 arithmetic)."""
    from distill_student import Student
    V, m, n, k = 997, 32, 64, 20
    g = torch.Generator(device="cuda").manual_seed(5)
    s = Student(V, m, 3)
    tokens = torch.randint(0, 50, (n,), generator=g, device="cuda", dtype=torch.int32)
    t_idx = torch.stack([torch.randperm(V, generator=g, device="cuda")[:k] for _ in range(n)]).int()
    t = torch.randn((n, k), generator=g, device="cuda")
    E = s.E.double().clone().requires_grad_(True)
    h = E[tokens.long()] * s.scale
    z = h @ E.t()
    z_seen = s.logits(tokens)[1].double()
    z = z + (z_seen - z).detach()  # the values that the step saw, the gradient of the product
    p = torch.softmax(t.double(), 1)
    loss = (p * (p.log() - torch.log_softmax(z, 1).gather(1, t_idx.long()))).sum(1)
    loss.mean().backward()
    got = s.step(tokens, t_idx, t, 0.0)
    assert (got.double() - loss.detach()).abs().max() < 1e-4
    dz = (torch.softmax(z_seen, 1).scatter_add(1, t_idx.long(), -p) / n).abs()
    terms = dz.t() @ h.detach().abs()
    terms.index_add_(0, tokens.long(), (dz @ E.detach().abs()) * s.scale)
    assert ((s.grad.double() - E.grad).abs() <= 1.5 * 2.0 ** -8 * terms + 1e-12).all()
