"""The training and sampling calls around the head from their definitions, in
64 bits (torch on the CPU or numpy), and how far fp32 arithmetic may be off.

U = 2^-24 is the largest relative error of one fp32 rounding.  A value
exp((z - m) / T) has an argument of up to X (subtraction, division or product
with a rounded reciprocal, conversion to the base-2 exponential: at most four
roundings of X) and an exponential of at most 2 ulp (4 U): relative error
(4 X + 4) U.  A sum of V positive terms over at least 256 threads adds at most
V / 256 + 32 roundings."""
import math

import numpy as np
import torch

U = 2.0 ** -24
BF16_HALF_ULP = torch.finfo(torch.bfloat16).eps / 2  # 8 significant bits: 2^-8 of a value


def out_round(dtype):
    """Relative error of the rounding to the output's type."""
    return BF16_HALF_ULP if dtype == torch.bfloat16 else U


def distill(z, idx, t, T, grad_loss):
    """(loss [n], stats [n, 2], gradient [n, V], tolerances of the three) from
    CPU tensors.  Rows with NaN or +inf logits: NaN."""
    n, V = z.shape
    z, t = z.double(), t.double()
    loss, stats, grad = torch.zeros(n).double(), torch.zeros(n, 2).double(), torch.zeros(n, V).double()
    loss_tol, s_tol, grad_tol = torch.zeros(n).double(), torch.zeros(n).double(), torch.zeros(n, V).double()
    for r in range(n):
        valid = [j for j in range(idx.shape[1]) if 0 <= int(idx[r, j]) < V and not t[r, j] == -math.inf]
        if not valid:
            continue
        at, tv = idx[r, valid].long(), t[r, valid]
        x = (tv - tv.max()) / T
        p = torch.exp(x) / torch.exp(x).sum()
        m = z[r].max()
        y = (z[r] - m) / T if m > -math.inf else torch.where(torch.isnan(z[r]), z[r], torch.full_like(z[r], -math.inf))
        e = torch.exp(y)
        s = e.sum()
        q = e / s if s != 0 else e
        cost = p * (x - torch.log(torch.exp(x).sum()) - y[at] + torch.log(s))
        loss[r] = T * T * cost[p.float() > 0].sum() if s != 0 else math.inf
        stats[r, 0], stats[r, 1] = m, s
        g = q.clone().index_add_(0, at, -p)
        grad[r] = T * grad_loss[r].double() * g
        # the largest argument that matters: below -120 an fp32 exp is 0
        args = torch.cat([y[torch.isfinite(y)].clamp(min=-120), x.clamp(min=-120), y[at][(p.float() > 0) & torch.isfinite(y[at])]])
        X = float(-args[~torch.isnan(args)].min()) if args.numel() else 0.0
        rel = (4 * X + 4 + V / 256 + 32) * U
        loss_tol[r] = T * T * (2 * rel + 4 * U * (2 * X + math.log(V + 1) + math.log(len(valid) + 1)) * 4)
        s_tol[r] = rel * s
        mass = q.clone().index_add_(0, at, p)
        grad_tol[r] = abs(T * grad_loss[r].double()) * (2 * rel + 4 * U) * mass + 1e-37
    return loss, stats, grad, loss_tol, s_tol, grad_tol


def embed_grad(tokens, grad, V, scale, base):
    """(gradient [V, d], sum of magnitudes [V, d], rows per token [V]) in 64 bits."""
    ok = (tokens >= 0) & (tokens < V)
    at, rows = tokens[ok].long(), grad[ok].double() * scale
    zero = torch.zeros(V, grad.shape[1], dtype=torch.float64, device=grad.device)
    out = (zero if base is None else base.double()).clone().index_add_(0, at, rows)
    mag = zero.clone().index_add_(0, at, rows.abs())
    return out, mag, torch.bincount(at, minlength=V)


class Draw:
    """One row's distribution: the ranked tokens and their weights in 64 bits."""

    def __init__(self, z, T):
        z = np.asarray(z, dtype=np.float64)
        drawable = np.flatnonzero(z > -math.inf)
        self.order = drawable[np.lexsort((drawable, -z[drawable]))]
        zs = z[self.order]
        self.rank = {int(v): i for i, v in enumerate(self.order)}
        if len(zs) == 0:
            return
        with np.errstate(invalid="ignore"):
            x = np.where(zs == zs[0], 0.0, (zs - zs[0]) / T if T > 0 else -math.inf)
        self.w = np.exp(x)
        self.w[self.w < 2.0 ** -40] = 0.0
        self.C = np.cumsum(self.w)
        # error of a weight (arguments up to 28: 1.5 roundings of them, 4 U for
        # the exponential), of the 2^-40 steps and of u and top_p (2^-24 each)
        self.eps = (1.5 * 28 + 4 + 4) * U + len(zs) * 2.0 ** -40

    def kept_mass(self, T, top_k, top_p, min_p, nudge):
        n = len(self.w) if top_k <= 0 else min(top_k, len(self.w))
        if not T > 0:
            n = 1
        S = self.C[n - 1]
        M = S
        if top_p < 1:
            M = min(M, self.C[min(int(np.searchsorted(self.C[:n], max(top_p, 0) * S * (1 + nudge))), n - 1)])
        if min_p > 0:
            k = int(np.count_nonzero(self.w >= min_p * (1 - nudge)))
            M = min(M, self.C[k - 1] if k else 0.0)
        return max(M, 1.0)

    def problems(self, T, top_k, top_p, min_p, u, token, prob):
        if len(self.order) == 0:
            return [] if (token, prob) == (-1, 0.0) else [f"nothing to draw, got {token} {prob}"]
        if token not in self.rank:
            return [f"token {token} is masked out"]
        j = self.rank[token]
        Ms = [self.kept_mass(T, top_k, top_p, min_p, s) for s in (-self.eps, 0.0, self.eps)]
        lo, hi = min(Ms), max(Ms)
        u = min(max(u, 0.0), 1 - 2.0 ** -24)
        before = self.C[j - 1] if j else 0.0
        out = []
        if before > u * hi + self.eps * hi or self.C[j] < u * lo - self.eps * hi or self.w[j] == 0:
            out.append(f"token {token} (rank {j}) covers [{before}, {self.C[j]}], the draw is {u * lo}..{u * hi}")
        if not self.w[j] / hi * (1 - 4 * self.eps) <= prob <= self.w[j] / lo * (1 + 4 * self.eps):
            out.append(f"probability {prob}, want {self.w[j] / hi}..{self.w[j] / lo}")
        return out
