"""Tuning a small model on what it has drawn itself, as timed cases: the losses on
the drawn tokens' log-probabilities, and a head held in 4 bits that draws cheaply.

A case is one call of a public entry point on inputs made from a seed:

  logprob          log-probabilities of given tokens under full logits, with the
                   softmax statistics that a gradient needs (``token_logprobs``);
  logprob_grad     the gradient of a weighted sum of them (``token_logprobs_grad``);
  policy           clipped policy loss with a KL term (``policy_loss``);
  policy_grad      its gradient with respect to the logits (``policy_loss_grad``);
  policy_step      both in one call (``policy_loss_step``);
  preference       loss of pairs of sequences, the chosen one and the rejected one,
                   from their tokens' log-probabilities (``preference_loss``);
  preference_step  with the gradient of each token (``preference_loss_step``);
  quantize         rows to 4-bit floating point with a scale per 16 values, and the
                   values that this leaves (``e2m1_quantize``);
  logits           full logits of a 4-bit head: hidden states are quantised as its
                   rows are, and multiplied with them (``e2m1_logits``).

Formulas.  Per row of logits, z: V values, t: its token, T: the temperature:

  lp = (z_t - m) / T - log s,  m = max z,  s = sum_v exp((z_v - m) / T);
  q = softmax(z / T),  d lp / d z_v = ([v = t] - q_v) / T;
  a row whose token is negative has lp 0, statistics (0, 0), loss 0 and gradient 0.

  policy:  r = exp(lp - old),  A: the advantage,
  loss = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(ref - lp) - (ref - lp) - 1),
  d loss / d lp = -A r where r A is the smaller one, else 0, + kl (1 - exp(ref - lp)).

  preference:  sequence j has tokens offsets[j] to offsets[j + 1]; D_j: its sum of
  lp - ref;  pair p is sequence 2p, chosen, and 2p + 1, rejected;
  h = beta (D_2p - D_2p+1),
  loss = -(1 - e) log sigmoid(h) - e log sigmoid(-h)   (e: label smoothing),
  d loss / d lp = beta (e - sigmoid(-h)) for chosen tokens, the negative for rejected
  ones, 0 for tokens of no sequence.

  4 bits:  a row x of d values has a power of two, 2^E, with E the least whole number
  (-126 at the least) with max |x| <= 2688 2^E; each 16 values have a scale, sigma =
  e4m3(max |x| over them / (6 2^E)), rounded to nearest, ties to even; a value's code
  is e2m1(x / (2^E sigma)), rounded likewise, at most 6 in magnitude (0 where sigma is
  0), and stands for code sigma 2^E.  Codes lie by rows, two to a byte, the even
  column in the low half, rows of ceil(d / 32) * 16 bytes; scales lie in tiles of 128
  rows by 4 scales, [ceil(rows / 128), ceil(d / 64), 32, 4, 4]: a tile's element
  [a, b, c] is the scale c of row 32 b + a.  What a row or tile has beyond its matrix
  is 0.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
_DT = {BF16: torch.bfloat16, F32: torch.float32}
_SIZE = {BF16: 2, F32: 4}


def _rows(name, kind, n, V, dtype, T):
    return {"name": name, "kind": kind, "n": n, "V": V, "dtype": dtype, "T": T}


def _policy(name, kind, n, V, dtype, T, low, high, kl):
    return dict(_rows(name, kind, n, V, dtype, T), low=low, high=high, kl=kl)


def _preference(name, kind, pairs, mean, beta, smoothing):
    return {"name": name, "kind": kind, "pairs": pairs, "mean": mean, "beta": beta, "smoothing": smoothing}


def _quantize(name, n, d, dtype, weights):
    return {"name": name, "kind": "quantize", "n": n, "d": d, "dtype": dtype, "weights": weights}


def _logits(name, n, V, d, dtype, out):
    return {"name": name, "kind": "logits", "n": n, "V": V, "d": d, "dtype": dtype, "out": out}


def listed():
    return [
        # a handful of positions scored, odd vocabulary
        _rows("logprob_20011_n7_f32", "logprob", 7, 20011, F32, 1.0),
        # behaviour log-probabilities of a batch of rollouts on the largest vocabulary
        _rows("logprob_262144_n2048", "logprob", 2048, 262144, BF16, 1.0),
        # backward pass of an autograd program (a preference loss, a likelihood)
        _rows("logprob_grad_128256_n2048", "logprob_grad", 2048, 128256, BF16, 1.0),
        # training steps: a ragged small one in fp32, and a full batch
        _policy("policy_step_20011_n61_f32", "policy_step", 61, 20011, F32, 0.7, 0.2, 0.2, 0.05),
        _policy("policy_step_151936_n4096", "policy_step", 4096, 151936, BF16, 1.0, 0.2, 0.28, 0.02),
        # a small step's pairs, and a batch of long answers
        _preference("preference_step_4x300", "preference_step", 4, 300, 0.1, 0.0),
        _preference("preference_step_256x2048", "preference_step", 256, 2048, 0.05, 0.1),
        # the hidden states of a decode step; a head's weights after an update
        _quantize("quantize_32x1152_f32", 32, 1152, F32, False),
        _quantize("quantize_262144x1152", 262144, 1152, BF16, True),
        # a decode step of 32 streams; an odd head and batch; many positions at once
        _logits("logits_262144x1152_n32", 32, 262144, 1152, F32, F32),
        _logits("logits_100003x1000_n129", 129, 100003, 1000, BF16, F32),
        _logits("logits_128256x2048_n2048", 2048, 128256, 2048, BF16, BF16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    d = _log(rng, lo, hi)
    return (d + 63) // 64 * 64 if rng.random() < 0.7 else d  # most models' widths; the others are odd sizes


def draw(rng):
    kind = rng.choice(["logprob", "logprob_grad", "policy", "policy_grad", "policy_step", "preference",
                       "preference_step", "quantize", "logits", "logits"])
    dtype = rng.choice([BF16, F32])
    if kind.startswith("preference"):
        mean = _log(rng, 8, 16384)
        case = _preference("", kind, min(_log(rng, 1, 512), 2 ** 19 // mean), mean,
                           rng.choice([0.05, 0.1, 0.5]), rng.choice([0.0, 0.0, 0.1]))
    elif kind == "quantize":
        d = _width(rng, 64, 8192)
        case = _quantize("", min(_log(rng, 1, 262144), 262144 * 1152 // d), d, dtype, rng.random() < 0.5)
    elif kind == "logits":
        V, d = _log(rng, 16000, 262144), _width(rng, 64, 4096)
        d = min(d, 2 ** 29 // V)
        n = min(_log(rng, 1, 2048), 2048 * 128256 // V, 2048 * 128256 * 2048 // (V * d))
        case = _logits("", n, V, d, dtype, rng.choice([BF16, F32]))
    else:
        V = _log(rng, 16000, 262144)
        n = min(_log(rng, 1, 4096), int(4096 * 151936 * 2 // (V * _SIZE[dtype])))
        T = rng.choice([1.0, 1.0, 0.7, 1.3])
        case = _rows("", kind, n, V, dtype, T) if kind.startswith("logprob") else \
            _policy("", kind, n, V, dtype, T, 0.2, rng.choice([0.2, 0.28]), rng.choice([0.0, 0.02, 0.1]))
    del case["name"]
    return case


# ---- inputs -----------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _row_inputs(case, g):
    """Logits whose drawn tokens are likely ones; one row in ten is a prompt's or padding."""
    n, V = case["n"], case["V"]
    tok = torch.randint(0, V, (n,), generator=g, device="cuda")
    z = 2.0 * torch.randn((n, V), generator=g, device="cuda")
    z.scatter_(1, tok[:, None], 6.0 + 2.5 * torch.randn((n, 1), generator=g, device="cuda"))
    z = z.to(_DT[case["dtype"]])
    tok[1:][torch.rand((n - 1,), generator=g, device="cuda") < 0.1] = -1
    weight = (1.0 / n) * (0.5 + torch.rand((n,), generator=g, device="cuda"))
    return z, tok.int(), weight


def _statistics(z, tok, T):
    """lp, m and s of each row in 64 bits."""
    out = torch.zeros((z.shape[0], 3), dtype=torch.float64, device="cuda")
    for r0 in range(0, z.shape[0], 256):
        x, t = z[r0:r0 + 256].double(), tok[r0:r0 + 256].long()
        m = x.amax(1)
        s = torch.exp((x - m[:, None]) / T).sum(1)
        lp = (x.gather(1, t.clamp(min=0)[:, None])[:, 0] - m) / T - torch.log(s)
        out[r0:r0 + 256] = torch.where((t >= 0)[:, None], torch.stack([lp, m, s], 1), 0.0)
    return out


def _policy_inputs(case, lp, g):
    """A policy some steps away from the one that drew the tokens and from the
    reference.  A ratio on the border of the clip, whose gradient is the one of
    either side, is no more likely in fp32 than any other number: none is within a
    thousandth of it, where a rounding of lp would choose the side."""
    n = case["n"]

    def normal():
        return torch.randn((n,), generator=g, device="cuda", dtype=torch.float64)

    delta = 0.15 * normal()
    for border in (math.log(1 - case["low"]), math.log(1 + case["high"])):
        delta = torch.where((delta - border).abs() < 1e-3, delta + 3e-3, delta)
    return (lp - delta).float(), normal().float(), (lp + 0.3 * normal()).float()


def _preference_inputs(case, g):
    """Pairs of answers of 0.1 to 1.9 times the mean length, a stretch of tokens before them and one behind."""
    pairs, mean = case["pairs"], case["mean"]
    n = 2 * pairs * mean + 24
    offsets = 11.0 + mean * torch.arange(2 * pairs + 1, device="cuda", dtype=torch.float64)
    offsets[1:-1] += 0.9 * mean * (torch.rand((2 * pairs - 1,), generator=g, device="cuda").double() - 0.5)
    offsets = offsets.round().int()
    lp = -2.0 * torch.rand((n,), generator=g, device="cuda") ** 2
    ref = lp + 0.05 * torch.randn((n,), generator=g, device="cuda")
    weight = (1.0 / pairs) * (0.5 + torch.rand((pairs,), generator=g, device="cuda"))
    return lp, ref, offsets, weight


def _weights(V, d, dtype, g):
    """Rows of a head, of norms that differ."""
    return (0.02 * torch.exp(0.3 * torch.randn((V, 1), generator=g, device="cuda"))
            * torch.randn((V, d), generator=g, device="cuda")).to(_DT[dtype])


def _states(n, d, dtype, g):
    """Hidden states with a few columns that stand out."""
    x = torch.randn((n, d), generator=g, device="cuda")
    x[:, torch.randint(0, d, (max(1, d // 200),), generator=g, device="cuda")] *= 20.0
    return x.to(_DT[dtype])


def _matrix(case, g):
    make = _weights if case["weights"] else _states
    return make(case["n"], case["d"], case["dtype"], g)


def prepare(case, seed):
    g, kind = _generator(seed), case["kind"]
    s = dict(case)

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if kind.startswith("preference"):
        s["lp"], s["ref"], s["offsets"], s["weight"] = _preference_inputs(case, g)
        s["loss"], s["margin"] = empty((case["pairs"],), torch.float32), empty((case["pairs"],), torch.float32)
        if kind == "preference_step":
            s["to"] = torch.empty_like(s["lp"])
    elif kind == "quantize":
        s["x"] = _matrix(case, g)
        s["codes"], s["scales"], s["powers"] = _room(case["n"], case["d"])
        s["to"] = empty((case["n"], case["d"]), torch.bfloat16)
    elif kind == "logits":
        V, d = case["V"], case["d"]
        s["codes"], s["scales"], s["powers"] = _packed(_weights(V, d, BF16, g))
        s["x"] = _states(case["n"], d, case["dtype"], g)
        s["x_codes"], s["x_scales"], s["x_powers"] = _room(case["n"], d)
        s["to"] = empty((case["n"], V), _DT[case["out"]])
    else:
        s["z"], s["tok"], s["weight"] = _row_inputs(case, g)
        exactly = _statistics(s["z"], s["tok"], case["T"])
        s["stats"] = exactly[:, 1:].float().contiguous()  # what a forward pass has left, as s["lp"], or room for it
        if kind.startswith("policy"):
            s["old"], s["adv"], s["ref"] = _policy_inputs(case, exactly[:, 0], g)
            s["loss"] = empty((case["n"],), torch.float32)
        s["lp"] = exactly[:, 0].float()
        if kind.endswith(("grad", "step")):
            s["to"] = torch.empty_like(s["z"])
    return s


# ---- the plain forms --------------------------------------------------------

def _plain_softmax(s, forward):
    """lp, m, s of each row (those of the forward pass, if this is not one), exp((z - m) / T), tokens and live rows."""
    z, T = s["z"].float(), s["T"]
    tok = s["tok"].long()
    live = (tok >= 0) & (tok < s["V"])
    m = z.amax(1) if forward else s["stats"][:, 0]
    e = torch.exp((z - m[:, None]) / T)
    total = e.sum(1) if forward else s["stats"][:, 1]
    tok = torch.where(live, tok, torch.zeros_like(tok))
    lp = (z.gather(1, tok[:, None])[:, 0] - m) / T - torch.log(total) if forward else s["lp"]
    return torch.where(live, lp, torch.zeros_like(lp)), m, total, e, tok, live


def _plain_rows(s):
    kind = s["kind"]
    zero = torch.zeros((), device="cuda")
    lp, m, total, e, tok, live = _plain_softmax(s, not kind.endswith("grad"))
    stats = torch.where(live[:, None], torch.stack([m, total], 1), zero)
    if kind == "logprob":
        return lp, stats
    if kind == "logprob_grad":
        slope = s["weight"]
    else:
        r = torch.exp(lp - s["old"])
        free = r * s["adv"]
        held = torch.clamp(r, 1.0 - s["low"], 1.0 + s["high"]) * s["adv"]
        x = s["ref"] - lp
        loss = -torch.minimum(free, held) + s["kl"] * (torch.expm1(x) - x)
        loss = torch.where(live, loss, zero)
        if kind == "policy":
            return loss, lp, stats
        slope = s["weight"] * (torch.where(free <= held, -free, zero) - s["kl"] * torch.expm1(x))
    slope = torch.where(live, slope / s["T"], zero)
    grad = e * torch.where(live, -slope / total, zero)[:, None]
    grad.scatter_add_(1, tok[:, None], slope[:, None])
    grad = torch.where(live[:, None], grad, zero).to(s["z"].dtype)
    return (loss, lp, grad) if kind == "policy_step" else (grad,)


def _plain_preference(s):
    lp, n, pairs = s["lp"], s["lp"].shape[0], s["pairs"]
    ends = s["offsets"].long()
    C = torch.zeros((n + 1,), dtype=torch.float64, device="cuda")  # running sums: far tokens' need 64 bits
    C[1:] = torch.cumsum(lp.double() - s["ref"].double(), 0)
    D = (C[ends[1:]] - C[ends[:-1]]).view(pairs, 2)
    h = (s["beta"] * (D[:, 0] - D[:, 1])).float()
    low = torch.log1p(torch.exp(-h.abs()))
    e = s["smoothing"]
    loss = (1.0 - e) * (low - h.clamp(max=0)) + e * (low + h.clamp(min=0))
    if s["kind"] == "preference":
        return loss, h
    slope = s["beta"] * s["weight"] * (e - 1.0 / (1.0 + torch.exp(h)))
    per = torch.stack([slope, -slope], 1).view(-1)
    j = torch.searchsorted(ends, torch.arange(n, device="cuda"), right=True) - 1
    grad = torch.where((j >= 0) & (j < 2 * pairs), per[j.clamp(0, 2 * pairs - 1)], torch.zeros((), device="cuda"))
    return loss, h, grad


def _room(n, d):
    """Codes, scales and powers of n rows of d values."""
    return (torch.empty((n, (d + 31) // 32 * 16), dtype=torch.uint8, device="cuda"),
            torch.empty(((n + 127) // 128, (d + 63) // 64, 32, 4, 4), dtype=torch.uint8, device="cuda"),
            torch.empty((n,), dtype=torch.float32, device="cuda"))


def _plain_quantize(x):
    """(codes as 0 .. 15 [n, blocks, 16], scales [n, blocks], powers of two [n]) of a matrix."""
    x = x.float()
    n, d = x.shape
    top = x.abs().amax(1).double() / 2688.0
    half, power = torch.frexp(top)
    power = torch.where(half == 0.5, power - 1, power)
    power = torch.where(top == 0, torch.full_like(power, -126), power.clamp(min=-126))
    powers = ((power + 127) << 23).view(torch.float32)  # 2^power
    x = (x.double() / powers.double()[:, None]).float()
    x = torch.nn.functional.pad(x, (0, -d % 16)).view(n, -1, 16)
    sigma = (x.abs().amax(2) / 6.0).to(torch.float8_e4m3fn).float()
    y = x / torch.where(sigma == 0, torch.ones_like(sigma), sigma)[:, :, None]
    a = torch.where(sigma[:, :, None] == 0, torch.zeros_like(y), y.abs())
    code = (a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() \
        + (a >= 3.5).byte() + (a > 5.0).byte()
    return code + 8 * (y < 0).byte(), sigma, powers


def _value(code):
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                        device="cuda")[code.int()]


def _plain_values(x):
    code, sigma, powers = _plain_quantize(x)
    return (_value(code) * sigma[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]], powers


def _packed(x):
    """Codes, scales and powers of a matrix's rows as they are stored."""
    n, d = x.shape
    codes, scales, powers = _room(n, d)
    for r0 in range(0, n, 32768):  # (a multiple of 128 rows, for memory's sake)
        r = slice(r0, min(n, r0 + 32768))
        code, sigma, powers[r] = _plain_quantize(x[r])
        rows = code.shape[0]
        code = torch.nn.functional.pad(code.view(rows, -1), (0, 2 * codes.shape[1] - 16 * code.shape[1]))
        codes[r] = code[:, 0::2] | (code[:, 1::2] << 4)
        sigma = torch.nn.functional.pad(sigma, (0, 4 * scales.shape[1] - sigma.shape[1], 0, -rows % 128))
        sigma = sigma.to(torch.float8_e4m3fn).view(torch.uint8).view(-1, 4, 32, scales.shape[1], 4)
        scales[r0 // 128:r0 // 128 + sigma.shape[0]] = sigma.permute(0, 3, 2, 1, 4)
    return codes, scales, powers


def _plain_logits(s):
    V, d = s["V"], s["d"]
    codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], 2).view(V, -1)
    sigma = s["scales"].view(torch.float8_e4m3fn).float().permute(0, 3, 2, 1, 4).reshape(-1, 4 * s["scales"].shape[1])
    w = _value(codes[:, :d]) * sigma[:V].repeat_interleave(16, 1)[:, :d]
    x, powers = _plain_values(s["x"])
    return ((x @ w.t()) * powers[:, None] * s["powers"]).to(_DT[s["out"]])


def run(s):
    kind = s["kind"]
    if not own:
        if kind.startswith("preference"):
            return _plain_preference(s)
        if kind == "quantize":
            x, powers = _plain_values(s["x"])
            return (x * powers[:, None]).to(torch.bfloat16), powers
        if kind == "logits":
            return _plain_logits(s)
        return _plain_rows(s)
    import paper_2608_27460_gb300 as vie
    if kind == "logprob":
        return vie.token_logprobs(s["z"], s["tok"], temperature=s["T"], out_logprob=s["lp"], out_stats=s["stats"])
    if kind == "logprob_grad":
        return (vie.token_logprobs_grad(s["z"], s["tok"], s["stats"], s["weight"], temperature=s["T"],
                                        out_grad=s["to"]),)
    if kind == "quantize":
        q = vie.e2m1_quantize(s["x"], out=vie.E2m1(s["codes"], s["scales"], s["powers"], s["d"]), out_values=s["to"])
        return s["to"], q.row_scales
    if kind == "logits":
        return vie.e2m1_logits(s["x"], vie.E2m1(s["codes"], s["scales"], s["powers"], s["d"]), out=s["to"],
                               x_quantized=vie.E2m1(s["x_codes"], s["x_scales"], s["x_powers"], s["d"]))
    if kind == "preference":
        return vie.preference_loss(s["lp"], s["offsets"], ref_logprob=s["ref"], beta=s["beta"],
                                   label_smoothing=s["smoothing"], out_loss=s["loss"], out_margin=s["margin"])
    if kind == "preference_step":
        return vie.preference_loss_step(s["lp"], s["offsets"], s["weight"], ref_logprob=s["ref"], beta=s["beta"],
                                        label_smoothing=s["smoothing"], out_loss=s["loss"], out_margin=s["margin"],
                                        out_grad=s["to"])
    how = {"ref_logprob": s["ref"], "clip_low": s["low"], "clip_high": s["high"], "kl_coef": s["kl"],
           "temperature": s["T"]}
    if kind == "policy":
        return vie.policy_loss(s["z"], s["tok"], s["old"], s["adv"], out_loss=s["loss"], out_logprob=s["lp"],
                               out_stats=s["stats"], **how)
    if kind == "policy_grad":
        return (vie.policy_loss_grad(s["z"], s["tok"], s["old"], s["adv"], s["lp"], s["stats"], s["weight"],
                                     out_grad=s["to"], **how),)
    return vie.policy_loss_step(s["z"], s["tok"], s["old"], s["adv"], s["weight"], out_loss=s["loss"],
                                out_logprob=s["lp"], out_grad=s["to"], **how)


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    kind = case["kind"]
    if kind.startswith("preference"):
        tokens = 2 * case["pairs"] * case["mean"] + 24
        return {"bytes": tokens * (12 if kind == "preference_step" else 8) + 20 * case["pairs"], "flops": 3 * tokens}
    if kind == "quantize":
        n, d = case["n"], case["d"]
        return {"bytes": n * d * (_SIZE[case["dtype"]] + 0.5625 + 2), "flops": 4 * n * d}
    if kind == "logits":
        n, V, d = case["n"], case["V"], case["d"]
        return {"bytes": V * (d * 0.5625 + 4) + n * d * _SIZE[case["dtype"]] + n * V * _SIZE[case["out"]],
                "flops": 2 * n * V * d}
    n, V, size = case["n"], case["V"], _SIZE[case["dtype"]]
    live = 0.9 * n  # rows without a token need not be read
    if kind in ("logprob", "policy"):
        return {"bytes": live * V * size + 28 * n, "flops": 4 * live * V}
    return {"bytes": (live + n) * V * size + 32 * n, "flops": 6 * live * V}


# ---- the same in 64 bits ----------------------------------------------------

def _exact_rows(case, seed):
    g, kind, n, T = _generator(seed), case["kind"], case["n"], case["T"]
    z, tok, weight = _row_inputs(case, g)
    live = tok >= 0
    stats = torch.zeros((n, 2), dtype=torch.float64, device="cuda")
    lp = torch.zeros((n,), dtype=torch.float64, device="cuda")
    grad = torch.empty(z.shape, dtype=torch.float64, device="cuda") if kind.endswith(("grad", "step")) else None
    loss = slope = None
    for r0 in range(0, n, 256):
        r = slice(r0, r0 + 256)
        zr = z[r].double()
        norm = torch.logsumexp(zr / T, 1)
        top = zr.max(1).values
        lp[r] = torch.where(live[r], zr.gather(1, tok[r].long().clamp(min=0)[:, None])[:, 0] / T - norm, 0.0)
        stats[r, 0] = torch.where(live[r], top, 0.0)
        stats[r, 1] = torch.where(live[r], torch.exp(norm - top / T), 0.0)
    if kind.startswith("policy"):
        old, A, ref = (v.double() for v in _policy_inputs(case, _statistics(z, tok, T)[:, 0], g))
        ratio = torch.exp(lp - old)
        inside = torch.where(A > 0, ratio <= 1 + case["high"], ratio >= 1 - case["low"])
        bound = torch.where(A > 0, torch.full_like(A, 1 + case["high"]), torch.full_like(A, 1 - case["low"]))
        over = torch.exp(ref - lp)
        loss = case["kl"] * (over - 1 - (ref - lp)) - A * torch.where(inside, ratio, bound)
        loss = torch.where(live, loss, 0.0)
        slope = case["kl"] * (1 - over) - torch.where(inside, A * ratio, 0.0)
    if kind == "logprob":
        return lp, stats
    if kind == "policy":
        return loss, lp, stats
    slope = torch.where(live, weight.double() * (1.0 if slope is None else slope), 0.0) / T
    for r0 in range(0, n, 256):
        r = slice(r0, r0 + 256)
        q = torch.softmax(z[r].double() / T, 1)
        q.scatter_add_(1, tok[r].long().clamp(min=0)[:, None], torch.full_like(q[:, :1], -1.0))
        grad[r] = -slope[r, None] * q
    return (loss, lp, grad) if kind == "policy_step" else (grad,)


def _exact_preference(case, seed):
    lp, ref, offsets, weight = _preference_inputs(case, _generator(seed))
    ends, ratio = offsets.tolist(), lp.double() - ref.double()
    D = torch.stack([ratio[a:b].sum() for a, b in zip(ends[:-1], ends[1:])]).view(-1, 2)
    h, e = case["beta"] * (D[:, 0] - D[:, 1]), case["smoothing"]
    loss = -(1 - e) * torch.nn.functional.logsigmoid(h) - e * torch.nn.functional.logsigmoid(-h)
    if case["kind"] == "preference":
        return loss, h
    slope = (case["beta"] * weight.double() * (e * torch.sigmoid(h) - (1 - e) * torch.sigmoid(-h))).tolist()
    grad = torch.zeros_like(ratio)
    for p, v in enumerate(slope):
        grad[ends[2 * p]:ends[2 * p + 1]] = v
        grad[ends[2 * p + 1]:ends[2 * p + 2]] = -v
    return loss, h, grad


def _exact_power(E):
    return ((E.long() + 1023) << 52).view(torch.float64)


def _exact_values(x):
    """What a matrix's rows stand for in 4 bits, with their powers of two apart."""
    n, d = x.shape
    x = x.double()
    top = x.abs().max(1).values
    E = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 2688)).clamp(min=-126)
    E += (top > 2688 * _exact_power(E)).double()  # (a logarithm's rounding)
    E -= ((top <= 2688 * _exact_power(E - 1)) & (E > -126)).double()
    x = torch.cat([x * _exact_power(-E)[:, None], x.new_zeros((n, -d % 16))], 1).view(n, -1, 16)
    share = x.abs().max(2).values / 6
    unit = _exact_power(torch.frexp(share)[1].clamp(min=-5) - 4)  # three bits behind the leading one
    sigma = (share / unit).round() * unit
    y = torch.where(sigma[:, :, None] > 0, x / sigma[:, :, None].clamp(min=1e-3), 0.0).clamp(-6, 6)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return ((y / step).round() * step * sigma[:, :, None]).view(n, -1)[:, :d], _exact_power(E)


def _exact_blocks(x):
    parts = [_exact_values(x[r0:r0 + 16384]) for r0 in range(0, x.shape[0], 16384)]
    return torch.cat([v for v, _ in parts]), torch.cat([p for _, p in parts])


def _exact_logits(case, seed):
    g = _generator(seed)
    W = _weights(case["V"], case["d"], BF16, g)
    x, px = _exact_values(_states(case["n"], case["d"], case["dtype"], g))
    out = torch.empty((case["n"], case["V"]), dtype=torch.float64, device="cuda")
    for r0 in range(0, case["V"], 16384):
        w, pw = _exact_values(W[r0:r0 + 16384])
        out[:, r0:r0 + 16384] = (x * px[:, None]) @ (w * pw[:, None]).t()
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind.startswith("preference"):
        return _exact_preference(case, seed)
    if kind == "quantize":
        values, powers = _exact_blocks(_matrix(case, _generator(seed)))
        return values * powers[:, None], powers
    if kind == "logits":
        return _exact_logits(case, seed)
    return _exact_rows(case, seed)
