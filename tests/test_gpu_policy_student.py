"""The calls on drawn tokens and the 4-bit head together, as the example runs them:
it runs, its draws are those of the calls one by one, and the gradients of one
update are those that autograd gives in 64 bits."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_the_example_runs(vie, loss):
    from policy_student import train
    rewards = train(loss, V=1001, streams=32, steps=4)
    assert len(rewards) == 4 and all(0 <= r <= 1 for r in rewards)


def _drawn(vie, V=997, m=32, streams=24, length=5):
    from policy_student import Policy
    g = torch.Generator(device="cuda").manual_seed(7)
    p = Policy(V, m, 3)
    seen, old = p.draw(torch.randint(0, V, (streams,), generator=g, device="cuda", dtype=torch.int32), length, g)
    p.E += 0.02 * torch.randn(p.E.shape, generator=g, device="cuda")  # some updates later
    return p, seen, old, g


def test_draws_come_from_the_4_bit_head(vie):
    from policy_student import Policy
    p = Policy(997, 32, 3)
    tokens = torch.arange(40, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(9)
    seen, old = p.draw(tokens, 1, g)
    h = vie.e2m1_dequantize(vie.e2m1_quantize(vie.embed(p.E, tokens, scale=p.scale))).double()
    lp = torch.log_softmax(h @ vie.e2m1_dequantize(p.head).double().t(), 1)
    assert torch.equal(seen[:, 0], tokens) and ((seen[:, 1] >= 0) & (seen[:, 1] < 997)).all()
    assert (old[:, 0].double() - lp.gather(1, seen[:, 1:].long())[:, 0]).abs().max() < 1e-4


def _exact(p, seen):
    """lp of the drawn tokens with the values that the calls saw and the gradient of
    the model in 64 bits; E; the magnitudes that a gradient's rounding goes by."""
    before, drawn = seen[:, :-1].reshape(-1).long(), seen[:, 1:].reshape(-1).long()
    E = p.E.double().clone().requires_grad_(True)
    h = E[before] * p.scale
    z = h @ E.t()
    z = z + (p.logits(before.int())[1].double() - z).detach()
    return torch.log_softmax(z, 1).gather(1, drawn[:, None])[:, 0], E, h.detach(), z.detach(), before, drawn


def _check_grad(p, E, h, z, before, drawn, slope):
    """The logits' gradient is rounded to bf16 (2^-8 of a value), so each sum may be off by
    2^-8 of the sum of its terms' magnitudes (and half as much again for fp32 arithmetic)."""
    hot = torch.zeros_like(z).scatter_(1, drawn[:, None], 1.0)
    dz = (slope.abs()[:, None] * (hot + torch.softmax(z, 1)))
    terms = dz.t() @ h.abs()
    terms.index_add_(0, before, (dz @ E.detach().abs()) * p.scale)
    assert ((p.grad.double() - E.grad).abs() <= 1.5 * 2.0 ** -8 * terms + 1e-12).all()


def test_a_policy_update_against_autograd(vie):
    p, seen, old, g = _drawn(vie)
    advantage = torch.randn(old.shape, generator=g, device="cuda")
    lp, E, h, z, before, drawn = _exact(p, seen)
    ref = torch.log_softmax(p.logits(before.int(), p.first)[1].double(), 1).gather(1, drawn[:, None])[:, 0]
    r, A, x = torch.exp(lp - old.reshape(-1).double()), advantage.reshape(-1).double(), ref - lp
    losses = -torch.minimum(r * A, r.clamp(0.8, 1.28) * A) + 0.05 * (torch.exp(x) - x - 1)
    near = ((r - 0.8).abs() < 1e-4) | ((r - 1.28).abs() < 1e-4)
    assert not near.any()  # (rounding would choose the side)
    losses.mean().backward()
    slope = (A * r).abs() + 0.05 * (torch.exp(x) - 1).abs()
    got = p.policy_gradient(seen, old, advantage, 0.05)
    assert (got.double() - losses.detach()).abs().max() < 1e-4
    _check_grad(p, E, h, z, before, drawn, slope.detach() / len(r))


def test_a_preference_update_against_autograd(vie):
    p, seen, old, _ = _drawn(vie)
    lp, E, h, z, before, drawn = _exact(p, seen)
    ref = torch.log_softmax(p.logits(before.int(), p.first)[1].double(), 1).gather(1, drawn[:, None])[:, 0]
    D = (lp - ref).view(seen.shape[0], -1).sum(1).view(-1, 2)
    losses = -torch.nn.functional.logsigmoid(0.3 * (D[:, 0] - D[:, 1]))
    losses.mean().backward()
    got = p.preference_gradient(seen, 0.3)
    assert (got.double() - losses.detach()).abs().max() < 1e-4
    _check_grad(p, E, h, z, before, drawn, torch.full_like(lp, 0.3 / len(losses)).detach())
