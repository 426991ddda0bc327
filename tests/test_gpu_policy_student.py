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


def test_every_call_on_a_stream_of_its_own(vie):
    """The same results as on the current stream, ready when the stream is."""
    g = torch.Generator(device="cuda").manual_seed(11)
    n, V, d = 30, 5003, 200
    z = torch.randn((n, V), generator=g, device="cuda")
    tok = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    w, adv = torch.rand((n,), generator=g, device="cuda"), torch.randn((n,), generator=g, device="cuda")
    lp, stats = vie.token_logprobs(z, tok)
    ends = torch.tensor([0, 7, 11, 20, 28], dtype=torch.int32, device="cuda")
    margin, two = torch.tensor([0.3, -0.2], device="cuda"), torch.ones(2, device="cuda")
    x = torch.randn((n, d), generator=g, device="cuda")
    head = vie.e2m1_quantize(torch.randn((700, d), generator=g, device="cuda"))

    def parts(q):
        return q.codes, q.scales, q.row_scales

    calls = [lambda **k: vie.token_logprobs(z, tok, **k), lambda **k: vie.token_logprobs_grad(z, tok, stats, w, **k),
             lambda **k: vie.policy_loss(z, tok, lp, adv, **k),
             lambda **k: vie.policy_loss_grad(z, tok, lp, adv, lp, stats, w, **k),
             lambda **k: vie.policy_loss_step(z, tok, lp, adv, w, ref_logprob=lp, kl_coef=0.1, **k),
             lambda **k: vie.preference_loss(lp, ends, **k),
             lambda **k: vie.preference_loss_grad(margin, ends, two, n, **k),
             lambda **k: vie.preference_loss_step(lp, ends, two, **k),
             lambda **k: parts(vie.e2m1_quantize(x, **k)), lambda **k: vie.e2m1_dequantize(head, **k),
             lambda **k: vie.e2m1_logits(x, head, **k)]
    s = torch.cuda.Stream()
    for call in calls:
        want = call()
        s.wait_stream(torch.cuda.current_stream())
        got = call(stream=s)
        s.synchronize()
        want, got = ((v,) if torch.is_tensor(v) else v for v in (want, got))
        assert len(want) == len(got) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_run_of_calls_captured_and_replayed(vie):
    """Quantise the head, draw, score and step in one graph: other weights and states
    between replays give what the calls give one by one."""
    g = torch.Generator(device="cuda").manual_seed(13)
    V, m, n = 3001, 96, 40
    E, h = torch.empty((V, m), device="cuda"), torch.empty((n, m), device="cuda")
    u, adv = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda")
    weight = torch.full((n,), 1.0 / n, device="cuda")
    head, room = vie.E2m1.empty(V, m), vie.E2m1.empty(n, m)
    z = torch.empty((n, V), dtype=torch.bfloat16, device="cuda")

    def refill():
        for t in (E, h, adv):
            t.normal_(generator=g)
        u.uniform_(generator=g)

    def calls(z):
        vie.e2m1_quantize(E, out=head)
        vie.e2m1_logits(h, head, out=z, x_quantized=room)
        tok, _ = vie.sample_logits(z, u)
        old, _ = vie.token_logprobs(z, tok)
        loss, _, dz = vie.policy_loss_step(z, tok, old, adv, weight, out_grad=z)
        return tok, old, loss, dz

    refill()
    calls(z)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = calls(z)
    for _ in range(3):
        refill()
        graph.replay()
        torch.cuda.synchronize()
        seen = [t.clone() for t in got]
        want = calls(torch.empty_like(z))
        assert all(torch.equal(a, b) for a, b in zip(seen, want))
    assert vie.vie_device_status() == vie.VIE_OK
