"""The calls on drawn tokens and on 4-bit rows from their definitions, in 64 bits
on the CPU, and how far fp32 arithmetic may be off.

U = 2^-24 is the largest relative error of one fp32 rounding.  exp((z - m) / T) =
2^((z - m) c) has an argument of y = (z - m) / T with a subtraction, c's two
roundings and a product in it, at most 4 U |y| of absolute error, and an
exponential of at most 2 ulp (4 U): a relative error of (4 |y| + 4) U, where
arguments below -120 give 0 and e^-120 at most.  The softmax's sum s = sum e
joins V positive terms over at least 256 threads' running sums (V / 256 roundings,
each rescaled once per step of the maximum: counted twice) and 32 more for the
joins: rel_s = (mean of 4 |y| + 4 under the softmax + 2 V / 256 + 32) U.
lp = y_t - log s: 3 U |y_t| (difference, division, and the last subtraction's
share), rel_s for the logarithm's argument, 3 U |log s| for the logarithm (1 ulp)
and the last subtraction."""
import math

import torch

U = 2.0 ** -24
FLOOR = 2.0 ** -126  # results below it may be flushed to 0
HALF = {torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2, torch.float32: U}


class Rows:
    """lp, stats, q and their tolerances of every row."""

    def __init__(self, z, tok, T):
        n, V = z.shape
        self.dtype, self.T = z.dtype, T
        z, tok = z.double(), tok.long()
        self.live = (tok >= 0) & (tok < V)
        self.tok = torch.where(self.live, tok, 0)
        m = z.amax(1)
        none = m == -math.inf
        y = (z - torch.where(none, 0.0, m)[:, None]) / T
        e = torch.exp(y)
        s = e.sum(1)
        self.q = torch.where(none[:, None], torch.zeros_like(e), e / s[:, None])
        at = z.gather(1, self.tok[:, None])[:, 0]
        yt = torch.where(none, -math.inf, (at - m) / T)
        logs = torch.where(none, 0.0, torch.log(s))
        self.lp = torch.where(self.live, yt - logs, 0.0)
        self.m, self.s = torch.where(self.live, m, 0.0), torch.where(self.live, s, 0.0)
        ya = y.abs().clamp(max=120)
        self.rel_e = (4 * torch.nan_to_num(ya, 0.0) + 4) * U
        self.rel_s = (self.q.nan_to_num(0.0) * self.rel_e).sum(1) + (2 * V / 256 + 32) * U
        self.lp_tol = torch.where(self.live, 3 * U * yt.abs() + self.rel_s + 3 * U * logs.abs() + U * self.lp.abs(), 0.0)
        self.lp_tol = torch.where(torch.isinf(yt), 0.0, self.lp_tol)
        self.s_tol = torch.where(self.live, self.rel_s * s, 0.0)

    def gradient(self, slope, slope_tol):
        """(gradient of sum slope lp, tolerance) by row; slope_tol: its absolute error."""
        slope = torch.where(self.live, slope.double(), 0.0) / self.T
        slope_tol = torch.where(self.live, slope_tol, 0.0) / self.T
        hot = torch.zeros_like(self.q).scatter_(1, self.tok[:, None], 1.0)
        g = slope[:, None] * (hot - self.q)
        # 6 U: T, 1 / s, slope / s and the last product, and the difference from 1 at the token
        tol = (slope.abs()[:, None] * (self.q * (self.rel_e + self.rel_s[:, None] + 6 * U) + 2 * U * hot)
               + slope_tol[:, None] * (hot + self.q))
        g = torch.where((slope == 0)[:, None], torch.zeros_like(g), g)
        tol = torch.where((slope == 0)[:, None], torch.zeros_like(tol), tol)
        return g, tol + HALF[self.dtype] * g.abs() + FLOOR * self.live[:, None]


def policy(rows, old, adv, ref, low, high, kl):
    """(loss, its tolerance, slope, its tolerance) of every row from 64-bit lp."""
    old, A = old.double(), adv.double()
    lp, tol = rows.lp, rows.lp_tol
    d = lp - old
    r = torch.exp(d)
    rel = tol + U * d.abs() + 4 * U  # lp, the difference, exp (2 ulp)
    low, high = 1 - low, 1 + high
    held = r.clamp(low, high)
    free = torch.where(A == 0, 0.0, r * A)
    bound = torch.where(A == 0, 0.0, held * A)
    first = free <= bound
    loss = torch.where(first, -free, -bound)
    slope = torch.where(first, -free, 0.0)
    loss_tol = torch.where(first, free.abs() * rel, 0.0) + 3 * U * loss.abs() + 2 * U * A.abs()
    slope_tol = slope.abs() * (rel + 2 * U)
    if kl:
        x = ref.double() - lp
        e = torch.expm1(x)
        k3 = torch.where(torch.isinf(e), math.inf, e - x)
        x_tol = tol + U * x.abs()
        loss = loss + kl * k3
        fine = torch.isfinite(loss)
        loss_tol = loss_tol + torch.where(fine, kl * (e.abs() * x_tol + 4 * U * e.abs() + 2 * U * (x.abs() + k3)) + 2 * U * loss.abs(), 0.0)
        slope = slope - kl * e
        slope_tol = slope_tol + torch.where(torch.isfinite(e), kl * ((e + 1) * x_tol + 6 * U * e.abs()) + 2 * U * slope.abs(), 0.0)
    zero = torch.zeros_like(loss)
    return tuple(torch.where(rows.live, v, zero) for v in (loss, loss_tol, slope, slope_tol))


def preference(lp, ref, offsets, beta, smoothing):
    """(loss, margin, slope of a chosen token, and the tolerances of the three)."""
    lp = lp.double()
    r = lp - (0.0 if ref is None else ref.double())
    ends = offsets.tolist()
    D = torch.zeros(len(ends) - 1, dtype=torch.float64)
    D_tol = torch.zeros_like(D)
    for j, (a, b) in enumerate(zip(ends[:-1], ends[1:])):
        D[j] = r[a:b].sum()
        # one rounding per difference; at most (length / 256 + 32) roundings of partial sums
        D_tol[j] = r[a:b].abs().sum() * (1 + (b - a) / 256 + 32) * U
    D, D_tol = D.view(-1, 2), D_tol.view(-1, 2)
    h = beta * (D[:, 0] - D[:, 1])
    h_tol = abs(beta) * D_tol.sum(1) + 3 * U * h.abs()
    sp, sn = torch.nn.functional.softplus(h), torch.nn.functional.softplus(-h)
    loss = (1 - smoothing) * sn + smoothing * sp
    slope = beta * (smoothing - torch.sigmoid(-h))
    loss_tol = h_tol + 8 * U * (loss + h.abs() + 1) + FLOOR
    slope_tol = abs(beta) * (h_tol * 0.25 + 8 * U * (smoothing + torch.sigmoid(-h)) + 4 * U * h.abs() * torch.sigmoid(-h)) + FLOOR
    return loss, h, slope, loss_tol, h_tol, slope_tol


# ---- 4 bits -------------------------------------------------------------------

VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]).double()


def _nearest(y, grid):
    """The index of the nearest grid value (ascending), ties to the even index."""
    hi = torch.searchsorted(grid, y.contiguous()).clamp(1, len(grid) - 1)
    lo = hi - 1
    dl, dh = y - grid[lo], grid[hi] - y
    return torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def quantize(x):
    """(codes [n, d] as 0 .. 15, e4m3 bytes [n, blocks], s [n], values [n, d]), in 64 bits."""
    n, d = x.shape
    x = x.double()
    good = torch.isfinite(x).all(1)
    x = torch.where(good[:, None], x, 0.0)
    top = x.abs().amax(1)
    E = torch.full((n,), -126)
    for e in range(-126, 118):
        E[top > 2688 * 2.0 ** e] = e + 1
    s = 2.0 ** E.double()
    blocks = (d + 15) // 16
    xb = torch.zeros(n, blocks * 16, dtype=torch.float64)
    xb[:, :d] = x / s[:, None]
    xb = xb.view(n, blocks, 16)
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()  # 0 .. 448, ascending
    byte = _nearest(xb.abs().amax(2) / 6, e4m3)
    sigma = e4m3[byte]
    y = torch.where(sigma[:, :, None] > 0, xb / torch.where(sigma > 0, sigma, 1.0)[:, :, None], 0.0)
    code = _nearest(y.abs().clamp(max=6), VALUES[:8])
    code = torch.where((y < 0) & (sigma[:, :, None] > 0), code + 8, code)
    values = (VALUES[code] * (sigma * s[:, None])[:, :, None]).view(n, -1)[:, :d]
    values = torch.where(good[:, None], values, math.nan)
    return code.view(n, -1)[:, :d], byte.to(torch.uint8), torch.where(good, s, math.nan), values


def unpack(q):
    """(codes [n, padded], e4m3 bytes [padded rows, padded blocks], s) of an E2m1, on the CPU."""
    c = q.codes.cpu()
    codes = torch.stack([c & 15, c >> 4], 2).view(c.shape[0], -1)
    sc = q.scales.cpu().view(torch.uint8)
    scales = sc.permute(0, 3, 2, 1, 4).reshape(sc.shape[0] * 128, -1)
    return codes, scales, q.row_scales.cpu()
