"""A small student model trained on what an exact output head says.

The teacher is a `Head`: fixed bf16 rows W [V, d] on hidden states that follow
the context (here a random function of the last token).  The student has one
tied matrix E [V, m]: its hidden state is the embedding of the last token, its
logits are E times that.  One step, all of it on the device:

  draw      the student's next token for every stream, from its full logits
            (sample_logits);
  look up   the hidden states of the new tokens (embed);
  ask       the teacher for its top-k logits there (Head.topk_many);
  compare   loss of the student's full logits against that list, and its
            gradient, in place of the logits (distill_topk_step);
  sum       the gradient of the tied matrix: the logits' side (a matrix product)
            and the lookup's side, added to it by token (embed_grad).

    python examples/distill_student.py [--steps 200]

prints the mean loss as it falls.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2608_27460_gb300 as vie


class Student:
    def __init__(self, V, m, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.scale = m ** 0.5
        self.E = 0.02 * torch.randn((V, m), generator=g, device="cuda")
        self.grad = torch.empty_like(self.E)
        self.mean, self.square, self.steps = torch.zeros_like(self.E), torch.zeros_like(self.E), 0
        self.workspace = None

    def logits(self, tokens):
        h = vie.embed(self.E, tokens, scale=self.scale)
        return h, (h @ self.E.t()).bfloat16()

    def step(self, tokens, t_idx, t_logits, lr):
        """One update from the teacher's lists at `tokens`; returns the loss of each row."""
        n, (V, m) = tokens.shape[0], self.E.shape
        if self.workspace is None:
            _, need = vie.vie_embed_grad_workspace(n, V, m)
            self.workspace = torch.empty((need,), dtype=torch.uint8, device="cuda")
        h, z = self.logits(tokens)
        weight = torch.full((n,), 1.0 / n, device="cuda")
        loss, dz = vie.distill_topk_step(z, t_idx, t_logits, weight, out_grad=z)
        dz = dz.float()
        torch.matmul(dz.t(), h, out=self.grad)                 # the logits' side of the tied matrix
        vie.embed_grad(tokens, dz @ self.E, V, scale=self.scale, out=self.grad, accumulate=True,
                       workspace=self.workspace)               # the lookup's side joins it
        # Adam
        self.steps += 1
        self.mean.lerp_(self.grad, 0.1)
        self.square.lerp_(self.grad.square(), 0.01)
        size = (self.square / (1 - 0.99 ** self.steps)).sqrt_().add_(1e-8)
        self.E.addcdiv_(self.mean, size, value=-lr / (1 - 0.9 ** self.steps))
        return loss


def train(V=20011, d=256, m=64, streams=256, k=50, steps=200, lr=0.02, contexts=16, top_k=100, seed=0, report=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = (0.06 * torch.randn((V, d), generator=g, device="cuda")).bfloat16()
    context = torch.randn((contexts, d), generator=g, device="cuda")  # the teacher's hidden state: by token mod contexts
    student = Student(V, m, seed + 1)
    tokens = torch.randint(0, V, (streams,), generator=g, device="cuda", dtype=torch.int32)
    means = []
    with vie.Head(W) as head:
        for step in range(steps):
            _, z = student.logits(tokens)
            u = torch.rand((streams,), generator=g, device="cuda")
            settings = dict(temperature=torch.full((streams,), 1.0, device="cuda"),
                            top_k=torch.full((streams,), top_k, dtype=torch.int32, device="cuda"),
                            top_p=torch.full((streams,), 0.95, device="cuda"))
            tokens, _ = vie.sample_logits(z, u, **settings)
            t_idx, t_logits = head.topk_many(context[(tokens % contexts).long()], k)
            loss = student.step(tokens, t_idx, t_logits, lr)
            if report and (step % report == 0 or step == steps - 1):
                means.append(float(loss.mean()))
                print(f"step {step:4d}  loss {means[-1]:.4f}", flush=True)
            elif not report and step in (0, steps - 1):
                means.append(float(loss.mean()))
        vie.check(head.device_status())
    return means


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--streams", type=int, default=256)
    a = ap.parse_args()
    train(streams=a.streams, steps=a.steps, report=max(1, a.steps // 20))


if __name__ == "__main__":
    main()
