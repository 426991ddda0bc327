"""The work around the output head when a small model is trained on what the exact
head says (the top-k logits of ``Head.topk_many``), as timed cases.

A case is one call of a public entry point on inputs made from a seed:

  embed         token rows of an embedding table, scaled (``embed``);
  embed_grad    the table's gradient from the rows' gradients, summed per token
                (``embed_grad``): a whole gradient table, or added to one;
  distill       loss of a student's logits against a teacher's top-k logits, with
                the softmax statistics that its gradient needs (``distill_topk``);
  distill_grad  the gradient of that loss with respect to the student's logits
                (``distill_topk_grad``);
  distill_step  both in one call (``distill_topk_step``);
  sample        tokens drawn from a student's full logits with temperature, top-k,
                top-p and min-p of each row, from given uniform numbers
                (``sample_logits``).

Formulas, per row (z: V student logits, T: temperature):

  p = softmax(t / T) over the teacher's valid entries (index in [0, V), t not -inf);
  q = softmax(z / T) over the vocabulary;
  loss = T^2 sum_j p_j (log p_j - log q_(index j)),  d loss / d z = T (q - p);
  a row without valid entries has loss 0 and gradient 0.

  Sampling ranks by (z descending, index ascending) and holds weights as whole
  numbers, w = floor(2^40 exp((z - max z) (1 / T))), so that sums do not depend on
  their order; top_k keeps the first top_k tokens, of mass S; top_p the shortest
  prefix of mass >= top_p S; min_p those with w >= min_p 2^40; the kept tokens are
  the shortest of these prefixes (at least one), of mass M; the token is the first
  whose running mass exceeds u M.  top_p and u count in steps of 2^-24.
  Temperature 0 takes the best token.
"""
import math

import numpy as np
import torch

own = False

BF16, F32 = "bf16", "f32"
_DT = {BF16: torch.bfloat16, F32: torch.float32}
_SIZE = {BF16: 2, F32: 4}


def _embed(name, n, V, d, table, out, scaled):
    return {"name": name, "kind": "embed", "n": n, "V": V, "d": d, "table": table, "out": out, "scaled": scaled}


def _embed_grad(name, n, V, d, grad, out, add, scaled):
    return {"name": name, "kind": "embed_grad", "n": n, "V": V, "d": d, "grad": grad, "out": out, "add": add,
            "scaled": scaled}


def _distill(name, kind, n, V, k, dtype, T):
    return {"name": name, "kind": kind, "n": n, "V": V, "k": k, "dtype": dtype, "T": T}


def _sample(name, batch, V, dtype):
    return {"name": name, "kind": "sample", "batch": batch, "V": V, "dtype": dtype}


def listed():
    return [
        # a decode step's token embeddings, scaled by sqrt(d), in the head's fp32
        _embed("embed_262144x1152_n32", 32, 262144, 1152, BF16, F32, True),
        # a training batch of 16 sequences of 1024 tokens
        _embed("embed_151936x1024_n16384", 16384, 151936, 1024, BF16, BF16, False),
        # the table's gradient on its own: a table of zeros but for the batch's tokens
        _embed_grad("embed_grad_262144x640_n8192", 8192, 262144, 640, BF16, F32, False, True),
        # a tied table: the batch's rows join the gradient that the output head has left there
        _embed_grad("embed_grad_add_151936x1024_n16384", 16384, 151936, 1024, BF16, F32, True, False),
        # evaluation of a handful of positions, odd vocabulary
        _distill("distill_20011_n7_k50_f32", "distill", 7, 20011, 50, F32, 1.0),
        # held-out loss on the largest vocabulary
        _distill("distill_262144_n2048_k64", "distill", 2048, 262144, 64, BF16, 1.0),
        # backward passes of an autograd program: a batch, and odd sizes with wide teacher lists
        _distill("distill_grad_128256_n2048_k50", "distill_grad", 2048, 128256, 50, BF16, 1.0),
        _distill("distill_grad_100003_n333_k300_f32", "distill_grad", 333, 100003, 300, F32, 2.0),
        # training steps: a ragged small one in fp32, and a full batch
        _distill("distill_step_20011_n61_k50_f32", "distill_step", 61, 20011, 50, F32, 2.0),
        _distill("distill_step_151936_n4096_k50", "distill_step", 4096, 151936, 50, BF16, 1.0),
        # tokens of one stream, and of a rollout batch whose rows have settings of their own
        _sample("sample_151936_b1", 1, 151936, F32),
        _sample("sample_262144_b64", 64, 262144, F32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "distill", "distill_grad", "distill_step", "sample"])
    V = _log(rng, 16000, 262144)
    if kind == "sample":
        batch = _log(rng, 1, 256)
        case = _sample("", batch, V, rng.choice([F32, BF16]))
    elif kind.startswith("embed"):
        d = _log(rng, 64, 4096)
        if rng.random() < 0.7:
            d = (d + 63) // 64 * 64  # most models' widths; the others are odd sizes
        d = min(d, int(2 ** 29 // V))
        n = min(_log(rng, 1, 65536), int(2 ** 27 // d))
        a, b, scaled = rng.choice([BF16, F32]), rng.choice([BF16, F32]), rng.random() < 0.5
        case = _embed("", n, V, d, a, b, scaled) if kind == "embed" else \
            _embed_grad("", n, V, d, a, b, rng.random() < 0.5, scaled)
    else:
        dtype = rng.choice([BF16, F32])
        n = min(_log(rng, 1, 4096), int(4096 * 151936 * 2 // (V * _SIZE[dtype])))
        case = _distill("", kind, n, V, _log(rng, 1, 1024), dtype, rng.choice([1.0, 1.0, 2.0, 0.7]))
    del case["name"]
    return case


# ---- inputs -----------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _tokens(case, g):
    """int32 [n]: ids about as frequent as 1 / (1 + id), and one empty slot (-1) in 20."""
    n, V = case["n"], case["V"]
    tok = torch.exp(torch.rand((n,), generator=g, device="cuda", dtype=torch.float64) * math.log(V + 1.0)).long() - 1
    tok = tok.clamp_(0, V - 1).int()
    tok[torch.rand((n,), generator=g, device="cuda") < 0.05] = -1
    return tok


def _scale(case):
    return math.sqrt(case["d"]) if case["scaled"] else 1.0


def _embed_inputs(case, g):
    table = (0.02 * torch.randn((case["V"], case["d"]), generator=g, device="cuda")).to(_DT[case["table"]])
    return _tokens(case, g), table


def _embed_grad_inputs(case, g):
    rows = (0.05 * torch.randn((case["n"], case["d"]), generator=g, device="cuda")).to(_DT[case["grad"]])
    tok = _tokens(case, g)
    base = None
    if case["add"]:
        base = (0.05 * torch.randn((case["V"], case["d"]), generator=g, device="cuda")).to(_DT[case["out"]])
    return tok, rows, base


def _distill_inputs(case, g):
    """Teacher lists sorted best first, as the exact head returns them (one row in
    ten without any entry: a prompt's positions; one in ten with a short list), and
    student logits that follow the teacher's at its tokens."""
    n, V, k = case["n"], case["V"], case["k"]
    step = V // k
    t_idx = torch.randint(0, step, (n, k), generator=g, device="cuda") + torch.arange(k, device="cuda") * step
    t_idx = t_idx.gather(1, torch.argsort(torch.rand((n, k), generator=g, device="cuda"), dim=1))
    t = torch.sort(6.0 + 2.5 * torch.randn((n, k), generator=g, device="cuda"), dim=1, descending=True).values
    z = 2.0 * torch.randn((n, V), generator=g, device="cuda")
    z.scatter_(1, t_idx, t + torch.randn((n, k), generator=g, device="cuda"))
    z = z.to(_DT[case["dtype"]])
    kind = torch.rand((n, 1), generator=g, device="cuda")
    length = (torch.rand((n, 1), generator=g, device="cuda") * k).int()
    drop = (kind < 0.1) | ((kind > 0.9) & (torch.arange(k, device="cuda") >= length))
    t_idx = torch.where(drop, torch.full_like(t_idx, -1), t_idx).int()
    grad_loss = (1.0 / n) * (0.5 + torch.rand((n,), generator=g, device="cuda"))
    return z, t_idx, t, grad_loss


def _sample_inputs(case, g):
    """Logits with a head of likely tokens, a tenth of them masked out, and settings
    as requests bring them: temperature 0 or 0.6 to 1.2; top-k off or 20 to 200;
    top-p off or 0.8 to 0.98; min-p off or 0.02 to 0.1."""
    b, V = case["batch"], case["V"]

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    z = 2.5 * torch.randn((b, V), generator=g, device="cuda")
    z[:, :V // 10] = -math.inf
    z = z[:, torch.randperm(V, generator=g, device="cuda")].to(_DT[case["dtype"]])
    temperature = torch.where(rand(b) < 0.1, torch.zeros(b, device="cuda"), 0.6 + 0.6 * rand(b))
    top_k = torch.where(rand(b) < 0.5, torch.zeros(b, device="cuda"), 20 + 180 * rand(b)).int()
    top_p = torch.where(rand(b) < 0.3, torch.ones(b, device="cuda"), 0.8 + 0.18 * rand(b))
    min_p = torch.where(rand(b) < 0.5, torch.zeros(b, device="cuda"), 0.02 + 0.08 * rand(b))
    return z, rand(b), temperature, top_k, top_p, min_p


def prepare(case, seed):
    g, kind = _generator(seed), case["kind"]
    s = dict(case)

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if kind == "embed":
        s["tokens"], s["weights"] = _embed_inputs(case, g)
        s["to"] = empty((case["n"], case["d"]), _DT[case["out"]])
    elif kind == "embed_grad":
        s["tokens"], s["rows"], s["to"] = _embed_grad_inputs(case, g)
        if s["to"] is None:
            s["to"] = empty((case["V"], case["d"]), _DT[case["out"]])
        # scratch of a training program, kept from step to step (bytes, ample for any n tokens)
        s["workspace"] = empty((64 * case["n"] + 8 * ((case["n"] + 7) // 8) * case["d"] + (1 << 21),), torch.uint8)
    elif kind == "sample":
        s["z"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"] = _sample_inputs(case, g)
        s["token"], s["prob"] = empty((case["batch"],), torch.int32), empty((case["batch"],), torch.float32)
    else:
        z, s["t_idx"], s["t"], s["grad_loss"] = _distill_inputs(case, g)
        s["z"] = z
        s["loss"], s["to"] = empty((case["n"],), torch.float32), None
        if kind == "distill":
            s["stats"] = empty((case["n"], 2), torch.float32)
        else:
            s["to"] = torch.empty_like(z)
        if kind == "distill_grad":  # what the forward pass has left: max z and sum exp((z - max z) / T)
            has = ((s["t_idx"] >= 0) & (s["t"] > -math.inf)).any(1)
            zf = z.float()
            m = zf.amax(1)
            total = torch.exp((zf - m[:, None]) / case["T"]).sum(1)
            s["stats"] = torch.where(has[:, None], torch.stack([m, total], 1), torch.zeros((), device="cuda"))
    return s


# ---- the plain forms --------------------------------------------------------

def _plain_embed(s):
    tok = s["tokens"].long()
    rows = s["weights"][tok.clamp(0, s["V"] - 1)].float() * _scale(s)
    inside = (tok >= 0) & (tok < s["V"])
    return torch.where(inside[:, None], rows, torch.zeros_like(rows)).to(_DT[s["out"]])


def _plain_embed_grad(s):
    tok = s["tokens"].long()
    inside = (tok >= 0) & (tok < s["V"])
    rows = s["rows"].float() * _scale(s)
    rows = torch.where(inside[:, None], rows, torch.zeros_like(rows))
    tok = tok.clamp(0, s["V"] - 1)
    if s["add"]:
        if s["to"].dtype == torch.float32:
            return s["to"].index_add_(0, tok, rows)
        return s["to"].copy_(s["to"].float().index_add_(0, tok, rows))
    out = torch.zeros((s["V"], s["d"]), device="cuda")
    return out.index_add_(0, tok, rows).to(_DT[s["out"]])


def _plain_teacher(s):
    """p and log p [n, k] (0 for entries that do not count), usable indices, rows that have any."""
    idx, t = s["t_idx"].long(), s["t"]
    valid = (idx >= 0) & (idx < s["V"]) & (t != -math.inf)
    t = torch.where(valid, t, torch.full_like(t, -math.inf))
    has = valid.any(1, keepdim=True)
    m = torch.where(has, t.amax(1, keepdim=True), torch.zeros_like(t[:, :1]))
    x = (t - m) / s["T"]
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    p = torch.where(has, e / total, torch.zeros_like(e))
    logp = torch.where(valid, x - torch.log(total), torch.zeros_like(e))
    return p, logp, idx.clamp(0, s["V"] - 1), has


def _plain_distill(s, forward, backward):
    T, z = s["T"], s["z"].float()
    p, logp, idx, has = _plain_teacher(s)
    zero = torch.zeros((), device="cuda")
    if forward:
        m = z.amax(1, keepdim=True)
        e = torch.exp((z - torch.where(m == -math.inf, zero, m)) / T)
        total = e.sum(1, keepdim=True)
    else:
        m, total = s["stats"][:, :1], s["stats"][:, 1:]
        e = torch.exp((z - torch.where(m == -math.inf, zero, m)) / T)
    out = []
    if forward:
        logq = (z.gather(1, idx) - m) / T - torch.log(total)
        loss = T * T * torch.where(p > 0, p * (logp - logq), zero).sum(1)
        out.append(torch.where(has[:, 0], loss, zero))
        if not backward:
            out.append(torch.where(has, torch.cat([m, total], 1), zero))
    if backward:
        q = torch.where(total == 0, zero, e / total)
        q.scatter_add_(1, idx, -p)
        q *= T * s["grad_loss"][:, None]
        out.append(torch.where(has, q, zero).to(s["z"].dtype))
    return tuple(out)


def _share(mass, count):
    """floor(mass count / 2^24) and the rest's presence, for mass < 2^62 and count <= 2^24."""
    low = (mass & 0xFFFFFF) * count
    return (mass >> 24) * count + (low >> 24), (low & 0xFFFFFF) != 0


def _plain_sample(s):
    z, order = torch.sort(s["z"].float(), dim=1, descending=True, stable=True)
    V = z.shape[1]
    warm = (s["temperature"] > 0)[:, None]
    inv = (1.0 / s["temperature"])[:, None]
    best = z[:, :1]
    x = torch.where(z == best, torch.zeros_like(z), torch.where(warm, (z - best) * inv, torch.full_like(z, -math.inf)))
    w = torch.where(z == -math.inf, torch.zeros_like(z), torch.exp(x) * 2.0 ** 40).long()
    top_k = torch.where((s["top_k"] <= 0) | (s["top_k"] > V), torch.full_like(s["top_k"], V), s["top_k"]).long()
    top_k = torch.where(warm[:, 0], top_k, torch.ones_like(top_k))[:, None]
    C = torch.cumsum(w, 1)
    S = C.gather(1, top_k - 1)
    least, more = _share(S, torch.ceil(s["top_p"].clamp(0, 1) * 2.0 ** 24).long()[:, None])
    n_p = (C < least + more).sum(1, keepdim=True) + 1
    n_m = (w >= torch.ceil(s["min_p"] * 2.0 ** 40).long()[:, None]).sum(1, keepdim=True)
    n = torch.minimum(top_k, torch.minimum(n_p, n_m)).clamp(min=1)
    M = C.gather(1, n - 1)
    target, _ = _share(M, (s["u"] * 2.0 ** 24).long().clamp(0, 2 ** 24 - 1)[:, None])
    j = (C <= target).sum(1, keepdim=True)
    return order.gather(1, j)[:, 0].int(), w.gather(1, j)[:, 0].float() / M[:, 0].float()


def run(s):
    kind = s["kind"]
    if not own:
        if kind == "embed":
            return _plain_embed(s)
        if kind == "embed_grad":
            return _plain_embed_grad(s)
        if kind == "sample":
            return _plain_sample(s)
        return _plain_distill(s, kind != "distill_grad", kind != "distill")
    import paper_2608_27460_gb300 as vie
    if kind == "embed":
        return vie.embed(s["weights"], s["tokens"], scale=_scale(s), out=s["to"])
    if kind == "embed_grad":
        return vie.embed_grad(s["tokens"], s["rows"], s["V"], scale=_scale(s), out=s["to"], accumulate=s["add"],
                              workspace=s["workspace"])
    if kind == "sample":
        return vie.sample_logits(s["z"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                 min_p=s["min_p"], out_token=s["token"], out_prob=s["prob"])
    if kind == "distill":
        return vie.distill_topk(s["z"], s["t_idx"], s["t"], temperature=s["T"], out_loss=s["loss"], out_stats=s["stats"])
    if kind == "distill_grad":
        return (vie.distill_topk_grad(s["z"], s["t_idx"], s["t"], s["stats"], s["grad_loss"], temperature=s["T"],
                                      out_grad=s["to"]),)
    return vie.distill_topk_step(s["z"], s["t_idx"], s["t"], s["grad_loss"], temperature=s["T"], out_loss=s["loss"],
                                 out_grad=s["to"])


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    kind, V = case["kind"], case["V"]
    if kind == "sample":
        return {"bytes": case["batch"] * (V * _SIZE[case["dtype"]] + 28), "flops": 0}
    if kind.startswith("embed"):
        # distinct tokens expected: ids drawn with density 1 / (1 + id)
        n, d = case["n"], case["d"]
        ids = np.arange(1, V + 1, dtype=np.float64)
        share = np.log((ids + 1) / ids) / math.log(V + 1.0)
        distinct = float(np.sum(-np.expm1(0.95 * n * np.log1p(-share))))
        if kind == "embed":
            return {"bytes": 4 * n + distinct * d * _SIZE[case["table"]] + n * d * _SIZE[case["out"]], "flops": n * d}
        written = 2 * distinct if case["add"] else V
        return {"bytes": 4 * n + 0.95 * n * d * _SIZE[case["grad"]] + written * d * _SIZE[case["out"]], "flops": n * d}
    n, k, size = case["n"], case["k"], _SIZE[case["dtype"]]
    live = 0.9 * n  # rows without a teacher's entries need not be read
    out = 8 * n * k + (12 * n if kind == "distill" else 4 * n)
    if kind == "distill":
        return {"bytes": live * V * size + out, "flops": 4 * live * V}
    return {"bytes": (live + n) * V * size + out, "flops": 6 * live * V}


# ---- the same in 64 bits ----------------------------------------------------

def _exact_embed(case, seed):
    tok, table = _embed_inputs(case, _generator(seed))
    out = torch.zeros((case["n"], case["d"]), dtype=torch.float64, device="cuda")
    at = torch.nonzero((tok >= 0) & (tok < case["V"]))[:, 0]
    out[at] = table.index_select(0, tok[at].long()).double().mul(_scale(case))
    return out


def _exact_embed_grad(case, seed):
    tok, rows, base = _embed_grad_inputs(case, _generator(seed))
    at = torch.nonzero((tok >= 0) & (tok < case["V"]))[:, 0]
    ids, where = torch.unique(tok[at].long(), return_inverse=True)
    sums = torch.zeros((ids.numel(), case["d"]), dtype=torch.float64, device="cuda")
    sums.index_add_(0, where, rows[at].double())
    out = torch.zeros((case["V"], case["d"]), dtype=torch.float64, device="cuda") if base is None else base.double()
    out[ids] += _scale(case) * sums
    return out


def _exact_distill(case, seed):
    z, idx, t, grad_loss = _distill_inputs(case, _generator(seed))
    n, V, T, kind = case["n"], case["V"], case["T"], case["kind"]
    loss = torch.zeros((n,), dtype=torch.float64, device="cuda")
    stats = torch.zeros((n, 2), dtype=torch.float64, device="cuda")
    grad = torch.zeros((n, V), dtype=torch.float64, device="cuda") if kind != "distill" else None
    for r0 in range(0, n, 256):
        r = slice(r0, min(n, r0 + 256))
        zr, tr = z[r].double() / T, t[r].double() / T
        tr = tr.masked_fill((idx[r] < 0) | (idx[r] >= V), -math.inf)
        live = torch.isfinite(tr).any(1)
        p = torch.softmax(tr, 1)
        p[~live] = 0
        at = idx[r].long().clamp(0, V - 1)
        logq = torch.log_softmax(zr, 1)
        some = torch.xlogy(p, p) - p * logq.gather(1, at)
        loss[r] = T * T * some.sum(1)
        top = zr.max(1).values
        stats[r, 0] = torch.where(live, z[r].double().max(1).values, 0.0)
        stats[r, 1] = torch.where(live, torch.exp(torch.logsumexp(zr, 1) - top), 0.0)
        if grad is not None:
            d = torch.exp(logq).scatter_add(1, at, -p)
            grad[r] = d * (T * grad_loss[r].double() * live)[:, None]
    if kind == "distill":
        return loss, stats
    return (grad,) if kind == "distill_grad" else (loss, grad)


def _exact_sample(case, seed):
    z, u, temperature, top_k, top_p, min_p = (x.double().cpu().numpy() for x in _sample_inputs(case, _generator(seed)))
    b, V = z.shape
    token, prob = np.empty(b, np.int32), np.empty(b)
    for r in range(b):
        order = np.argsort(-z[r], kind="stable")
        zs = z[r][order]
        if not temperature[r] > 0:
            token[r], prob[r] = order[0], 1.0
            continue
        w = np.floor(np.ldexp(np.exp((zs - zs[0]) / temperature[r]), 40)).astype(np.int64)
        keep = int(top_k[r]) if 0 < top_k[r] < V else V
        C = np.cumsum(w[:keep])
        least = -(-int(C[-1]) * math.ceil(top_p[r] * 2 ** 24) // 2 ** 24)
        keep = max(1, min(keep, int(np.searchsorted(C, least)) + 1, int(np.count_nonzero(w >= min_p[r] * 2.0 ** 40))))
        M = int(C[keep - 1])
        j = int(np.searchsorted(C[:keep], M * int(u[r] * 2 ** 24) // 2 ** 24, side="right"))
        token[r], prob[r] = order[j], int(w[j]) / M
    return torch.from_numpy(token), torch.from_numpy(prob)


def exact(case, seed):
    kind = case["kind"]
    if kind == "embed":
        return _exact_embed(case, seed)
    if kind == "embed_grad":
        return _exact_embed_grad(case, seed)
    if kind == "sample":
        return _exact_sample(case, seed)
    return _exact_distill(case, seed)
