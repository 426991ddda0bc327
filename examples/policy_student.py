"""A small model tuned on what it draws itself, with a 4-bit copy of its head.

The model has one tied matrix E [V, m]: its hidden state is the embedding of the
last token, its logits are E times that.  All of it on the device:

  quantise  the head's rows to 4 bits after each update (e2m1_quantize);
  draw      a few tokens for every stream: look up (embed), full logits of the
            4-bit head (e2m1_logits), one token each (sample_logits), and its
            log-probability under the policy that drew it (token_logprobs);
  reward    each answer: here the share of its tokens in the first tenth of the
            vocabulary;
  update    either by the clipped policy loss, with a KL term against the model
            before tuning (policy_loss_step), or by preferring the better half of
            the answers over the worse one, in pairs (preference_loss_step, whose
            gradient by token goes on through token_logprobs_grad);
  sum       the tied matrix's gradient: the logits' side (a matrix product) and
            the lookup's side, added to it by token (embed_grad).

    python examples/policy_student.py [--loss policy|preference] [--steps 60]

prints the mean reward.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2608_27460_gb300 as vie


class Policy:
    def __init__(self, V, m, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.scale = m ** 0.5
        self.E = 0.1 * torch.randn((V, m), generator=g, device="cuda")
        self.first = self.E.clone()  # the reference
        self.grad = torch.zeros_like(self.E)
        self.head = vie.e2m1_quantize(self.E)

    def logits(self, tokens, E=None):
        """Hidden states and bf16 logits of the rows after `tokens`."""
        E = self.E if E is None else E
        h = vie.embed(E, tokens, scale=self.scale)
        return h, (h @ E.t()).bfloat16()

    def draw(self, tokens, length, generator):
        """`length` tokens for every stream: (prompts and tokens [streams, length + 1],
        log-probabilities of the tokens [streams, length])."""
        seen, lps = [tokens], []
        for _ in range(length):
            z = vie.e2m1_logits(vie.embed(self.E, tokens, scale=self.scale), self.head)
            tokens, _ = vie.sample_logits(z, torch.rand((len(tokens),), generator=generator, device="cuda"))
            lps.append(vie.token_logprobs(z, tokens)[0])
            seen.append(tokens)
        return torch.stack(seen, 1), torch.stack(lps, 1)

    def backward(self, tokens, h, dz):
        """The tied matrix's gradient from the logits' one."""
        dz = dz.float()
        torch.matmul(dz.t(), h, out=self.grad)
        vie.embed_grad(tokens, dz @ self.E, len(self.E), scale=self.scale, out=self.grad, accumulate=True)

    def policy_gradient(self, seen, old, advantage, kl):
        """Gradient of the mean policy loss of all drawn tokens; returns the losses."""
        before, drawn = seen[:, :-1].reshape(-1), seen[:, 1:].reshape(-1)
        ref = vie.token_logprobs(self.logits(before, self.first)[1], drawn)[0]
        h, z = self.logits(before)
        weight = torch.full((len(drawn),), 1.0 / len(drawn), device="cuda")
        loss, _, dz = vie.policy_loss_step(z, drawn, old.reshape(-1), advantage.reshape(-1), weight, ref_logprob=ref,
                                           clip_high=0.28, kl_coef=kl, out_grad=z)
        self.backward(before, h, dz)
        return loss

    def preference_gradient(self, seen, beta):
        """Gradient of the mean preference loss of answers 2p over 2p + 1; returns the losses."""
        n, length = seen.shape[0], seen.shape[1] - 1
        before, drawn = seen[:, :-1].reshape(-1), seen[:, 1:].reshape(-1)
        ends = torch.arange(0, n * length + 1, length, dtype=torch.int32, device="cuda")
        ref = vie.token_logprobs(self.logits(before, self.first)[1], drawn)[0]
        h, z = self.logits(before)
        lp, stats = vie.token_logprobs(z, drawn)
        weight = torch.full((n // 2,), 2.0 / n, device="cuda")
        loss, _, dlp = vie.preference_loss_step(lp, ends, weight, ref_logprob=ref, beta=beta)
        self.backward(before, h, vie.token_logprobs_grad(z, drawn, stats, dlp, out_grad=z))
        return loss

    def update(self, lr):
        self.E.sub_(lr * self.grad / self.grad.square().mean().sqrt().add(1e-12))
        vie.e2m1_quantize(self.E, out=self.head)


def train(loss="policy", V=4001, m=64, streams=128, length=8, steps=60, lr=0.003, seed=0, report=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    policy = Policy(V, m, seed + 1)
    rewards = []
    for step in range(steps):
        prompts = torch.randint(0, V, (streams,), generator=g, device="cuda", dtype=torch.int32)
        seen, old = policy.draw(prompts, length, g)
        reward = (seen[:, 1:] < V // 10).float().mean(1)
        if loss == "policy":
            advantage = (reward - reward.mean()) / (reward.std() + 1e-6)
            policy.policy_gradient(seen, old, advantage[:, None].expand(-1, length).contiguous(), 0.01)
        else:
            order = torch.argsort(reward, descending=True)
            pairs = torch.stack([order[:streams // 2], order[streams // 2:]], 1).reshape(-1)
            policy.preference_gradient(seen[pairs].contiguous(), 0.1)
        policy.update(lr)
        rewards.append(reward.mean())
        if report and (step % report == 0 or step == steps - 1):
            print(f"step {step:4d}  reward {float(rewards[-1]):.4f}", flush=True)
    vie.check(vie.vie_device_status())
    return [float(r) for r in rewards]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--loss", choices=("policy", "preference"), default="policy")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--streams", type=int, default=128)
    a = ap.parse_args()
    train(a.loss, streams=a.streams, steps=a.steps, report=max(1, a.steps // 20))


if __name__ == "__main__":
    main()
