"""GPU parity of the calls on drawn tokens (token_logprobs, policy_loss and their
gradients) against their definitions in 64 bits (tests/policy_ref.py, with the
tolerances derived there), and the gradients against differences."""
import math

import pytest
import torch

import policy_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(n, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    z = (spread * torch.randn(n, V, generator=g)).to(DT[dtype])
    tok = torch.randint(0, V, (n,), generator=g).int()
    return z, tok, torch.randn(n, generator=g), g


def _terms(rows, g, low, high):
    """old, advantage and reference; no ratio within 2^-8 of a border of the clip, where
    the roundings of lp would choose the side."""
    n = rows.lp.shape[0]
    lp = torch.where(torch.isfinite(rows.lp), rows.lp, -50.0)
    d = 0.2 * torch.randn(n, generator=g).double()
    for b in (math.log(max(1 - low, 1e-6)), math.log(1 + high)):
        d = torch.where((d - b).abs() < 2.0 ** -8, d + 2.0 ** -6, d)
    return (lp - d).float(), torch.randn(n, generator=g), (lp + 0.3 * torch.randn(n, generator=g).double()).float()


def _close(got, want, tol, what):
    got = got.double().cpu()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bad.any(), (what, got[bad][:4], want[bad][:4], (bad.nonzero()[:4]).tolist())


def _copy(zc):
    """The same values at the same alignment and pitch: a row's sums are taken by 16-byte
    vectors at 16-byte addresses, so their order, and their last bits, depend on those."""
    shift = zc.data_ptr() % 16 // zc.element_size()
    n, ld = zc.shape[0], zc.stride(0)
    buf = torch.empty((n * ld + shift + 16,), dtype=zc.dtype, device="cuda")
    out = buf[shift:shift + n * ld].view(n, ld)[:, :zc.shape[1]]
    return out.copy_(zc)


def _check(vie, z, tok, T, grad, g, low=0.2, high=0.3, kls=(0.0, 0.05), zc=None, terms=None):
    rows = ref.Rows(z, tok, T)
    zc = z.cuda() if zc is None else zc
    tc, gc = tok.cuda(), grad.cuda()
    lp, stats = vie.token_logprobs(zc, tc, temperature=T)
    _close(lp, rows.lp, rows.lp_tol, "logprob")
    _close(stats[:, 0], rows.m, 0, "m")
    _close(stats[:, 1], rows.s, rows.s_tol, "s")
    want, tol = rows.gradient(grad, torch.zeros(len(grad)).double())
    dz = vie.token_logprobs_grad(zc, tc, stats, gc, temperature=T)
    assert dz.dtype == z.dtype
    _close(dz, want, tol, "logprob gradient")
    own = _copy(zc)
    assert torch.equal(vie.token_logprobs_grad(own, tc, stats, gc, temperature=T, out_grad=own), dz)
    old, adv, r = terms if terms is not None else _terms(rows, g, low, high)
    oc, ac, rc = old.cuda(), adv.cuda(), r.cuda()
    for kl in kls:
        loss_w, loss_t, slope, slope_t = ref.policy(rows, old, adv, r, low, high, kl)
        how = dict(clip_low=low, clip_high=high, kl_coef=kl, temperature=T, ref_logprob=rc if kl else None)
        gd = grad.double()
        weighted = torch.where(gd == 0, 0.0, gd * slope)  # (a weight of 0 masks a row, whatever its slope)
        want, tol = rows.gradient(weighted, gd.abs() * slope_t + 2 * ref.U * weighted.abs())
        loss, lp2, stats2 = vie.policy_loss(zc, tc, oc, ac, **how)
        assert torch.equal(lp2, lp) and torch.equal(stats2, stats)
        _close(loss, loss_w, loss_t, ("loss", kl))
        dz = vie.policy_loss_grad(zc, tc, oc, ac, lp2, stats2, gc, **how)
        _close(dz, want, tol, ("policy gradient", kl))
        own = _copy(zc)
        assert torch.equal(vie.policy_loss_grad(own, tc, oc, ac, lp2, stats2, gc, out_grad=own, **how), dz)
        out = torch.full((len(tok), 2), 7.0, device="cuda")
        loss, lp3, dz = vie.policy_loss_step(zc, tc, oc, ac, gc, out_stats=out, **how)
        _close(lp3, rows.lp, rows.lp_tol, "step logprob")
        _close(out[:, 1], rows.s, rows.s_tol, "step s")
        _close(loss, loss_w, loss_t, ("step loss", kl))
        _close(dz, want, tol, ("step gradient", kl))
        own = _copy(zc)
        again = vie.policy_loss_step(own, tc, oc, ac, gc, out_grad=own, **how)
        assert torch.equal(again[2], dz) and torch.equal(again[0], loss) and again[2].data_ptr() == own.data_ptr()
    assert vie.vie_device_status() == vie.VIE_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,T", [(1, 1, 1.0), (3, 2, 1.0), (2, 7, 0.5), (5, 33, 2.0), (4, 257, 1.0), (3, 4099, 1.3),
                                   (9, 20011, 1.0), (2, 65537, 0.7), (10, 131071, 1.0), (300, 515, 1.0),
                                   (2, 262144, 1.0)])
def test_sizes(vie, dtype, n, V, T):
    z, tok, grad, g = _inputs(n, V, dtype, seed=V)
    tok[0] = V - 1
    if n > 1:
        tok[1] = 0
    _check(vie, z, tok, T, grad, g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_longer_than_any_slice(vie, dtype):
    z, tok, grad, g = _inputs(2, 1000003, dtype, seed=3)
    _check(vie, z, tok, 1.0, grad, g, kls=(0.05,))


@pytest.mark.parametrize("n,V,dtype", [(8, 51001, "bf16"), (9, 51001, "bf16"), (72, 51001, "bf16"), (73, 51001, "bf16"),
                                       (85, 33001, "bf16"), (86, 33001, "bf16"), (145, 25003, "f32"), (146, 25003, "f32"),
                                       (304, 13001, "bf16"), (305, 13001, "bf16"), (342, 8200, "f32"), (343, 8200, "f32"),
                                       (608, 7001, "f32"), (609, 7001, "f32"), (1217, 7001, "bf16")])
def test_rows_on_both_sides_of_a_round(vie, n, V, dtype):
    """As many rows as one round of CTAs takes in each number of slices, and one more."""
    z, tok, grad, g = _inputs(n, V, dtype, seed=n)
    tok[::11] = -1
    tok[1] = V - 1
    _check(vie, z, tok, 1.0, grad, g, kls=(0.05,))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_place_of_the_token(vie, dtype):
    """All tokens of a small row, at every alignment: the edges' vectors and those between."""
    V = 2077
    z, _, _, g = _inputs(1, V, dtype, seed=5)
    grad = torch.ones(V)
    tok = torch.arange(V).int()
    for off in range(3):
        big = torch.zeros((off + V + 8,), dtype=DT[dtype], device="cuda")
        zc = big[off:off + V].view(1, V)
        zc.copy_(z)
        rows = ref.Rows(z.expand(V, V), tok, 1.0)
        want, tol = rows.gradient(grad, torch.zeros(V).double())
        many = zc.expand(V, V).contiguous()
        lp, stats = vie.token_logprobs(many, tok.cuda())
        _close(lp, rows.lp, rows.lp_tol, off)
        _close(vie.token_logprobs_grad(many, tok.cuda(), stats, grad.cuda()), want, tol, off)
        one = torch.tensor([V // 2 + off], dtype=torch.int32, device="cuda")
        lp, stats = vie.token_logprobs(zc, one)
        got = vie.token_logprobs_grad(zc, one, stats, grad[:1].cuda())
        _close(got[0], want[V // 2 + off], tol[V // 2 + off], off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_empty_rows(vie, dtype):
    z, tok, grad, g = _inputs(7, 3001, dtype, seed=7)
    tok[0], tok[3] = -1, -2 ** 31
    z[0] = float("nan")  # not read
    z[3, 7] = float("inf")
    rows = ref.Rows(z, tok, 1.0)
    old, adv, r = _terms(rows, g, 0.2, 0.3)
    old[0], adv[0], r[0] = float("nan"), float("nan"), float("inf")
    grad[3] = float("nan")
    _check(vie, z, tok, 1.0, grad, g, terms=(old, adv, r))


def test_tokens_beyond_the_vocabulary_are_reported(vie):
    z, tok, grad, g = _inputs(5, 100, "f32", seed=9)
    tok[1], tok[4] = 100, 2 ** 31 - 1
    lp, stats = vie.token_logprobs(z.cuda(), tok.cuda())
    assert vie.vie_device_status() == vie.VIE_ERR_DEVICE and "token" in vie.vie_last_error()
    assert (lp[[1, 4]] == 0).all() and (stats[[1, 4]] == 0).all() and (lp[[0, 2, 3]] < 0).all()
    dz = vie.token_logprobs_grad(z.cuda(), tok.cuda(), stats, grad.cuda())
    assert not dz[[1, 4]].any() and dz[[0, 2, 3]].any(1).all()
    assert vie.vie_device_status() == vie.VIE_ERR_DEVICE
    assert vie.vie_device_status() == vie.VIE_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_masked_logits(vie, dtype, T):
    """-inf and the type's lowest value in masked places, at the token, and in whole rows."""
    low = torch.finfo(DT[dtype]).min
    z, tok, grad, g = _inputs(9, 1537, dtype, seed=11)
    z[0, ::3] = -math.inf
    z[0, tok[0]] = 1.0
    z[1, ::3] = low
    z[1, tok[1]] = 1.0
    z[2] = low                    # equal logits: uniform
    z[3] = -math.inf              # no softmax: lp is -inf, q is 0
    z[4] = -math.inf
    z[4, tok[4]] = 1.0            # the token alone: lp 0
    z[5] = low
    z[5, 7] = -math.inf
    z[5, tok[5]] = low
    z[6, tok[6]] = -math.inf      # a masked token: lp is -inf
    z[7] = torch.finfo(DT[dtype]).max
    z[8, :700] = low
    z[8, 700:] = -math.inf
    tok[8] = 3
    rows = ref.Rows(z, tok, T)
    assert rows.lp[3] == -math.inf and rows.lp[6] == -math.inf and rows.lp[4] == 0
    _check(vie, z, tok, T, grad, g, kls=(0.0,))
    # with a KL term, such a token's loss is +inf; the other rows are as they were
    old, adv, r = _terms(rows, g, 0.2, 0.3)
    loss_w, loss_t, _, _ = ref.policy(rows, old, adv, r, 0.2, 0.3, 0.1)
    loss = vie.policy_loss(z.cuda(), tok.cuda(), old.cuda(), adv.cuda(), ref_logprob=r.cuda(), clip_high=0.3,
                           kl_coef=0.1, temperature=T)[0]
    _close(loss, loss_w, loss_t, "kl")
    assert loss[3] == math.inf and loss[6] == math.inf


def test_nan_and_inf_stay_in_their_row(vie):
    z, tok, grad, g = _inputs(5, 999, "f32", seed=13)
    z[1, 500] = float("nan")
    z[3, 2] = float("inf")
    old, adv, r = _terms(ref.Rows(torch.nan_to_num(z, 0.0, 0.0), tok, 1.0), g, 0.2, 0.2)
    adv[:] = 1.0
    adv[4] = float("nan")
    loss, lp, dz = vie.policy_loss_step(z.cuda(), tok.cuda(), old.cuda(), adv.cuda(), grad.cuda(), ref_logprob=r.cuda(),
                                        kl_coef=0.1)
    assert torch.isfinite(lp).tolist() == [True, False, True, False, True]
    for row in range(5):
        assert bool(torch.isfinite(loss[row])) == (row in (0, 2))
        assert bool(torch.isfinite(dz[row]).all()) == (row in (0, 2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_and_inf_beside_a_masked_token(vie, dtype):
    """A token at -inf: -inf beside numbers and where no logit is above it, NaN beside a NaN or +inf, at any place."""
    V = 5003
    z, tok, grad, g = _inputs(7, V, dtype, seed=53)
    tok[:] = 100
    z[:, 100] = -math.inf
    z[1], z[2, 0], z[3, V - 1], z[4, 2500], z[5, 101] = -math.inf, math.nan, math.nan, math.inf, math.inf
    z[6], z[6, 99] = -math.inf, math.nan
    lp, stats = vie.token_logprobs(z.cuda(), tok.cuda())
    assert (lp[:2] == -math.inf).all() and torch.isnan(lp[2:]).all()
    assert stats[1, 0] == -math.inf and stats[1, 1] == 0


def test_extreme_terms(vie):
    """Ratios of 0 and infinity, advantages of 0, references that rule a token out."""
    z, tok, grad, g = _inputs(8, 300, "f32", seed=17)
    rows = ref.Rows(z, tok, 1.0)
    old = (rows.lp - 0.05).float()
    adv = torch.tensor([1.0, -1.0, 0.0, 0.0, 1.0, -1.0, 2.0, 0.0])
    r = (rows.lp + 0.1).float()
    old[0] = old[1] = old[2] = -1000.0     # r is infinite: clipped, +inf, none
    old[4] = old[5] = 1000.0               # r is 0: none, clipped
    _check(vie, z, tok, 1.0, torch.where(torch.arange(8) == 1, 0.0, grad), g, terms=(old, adv, r), kls=(0.0,))
    loss, _, stats = vie.policy_loss(z.cuda(), tok.cuda(), old.cuda(), adv.cuda())
    assert loss[1] == math.inf and loss[2] == 0 and abs(float(loss[0]) + 1.2) < 1e-6
    r[6] = -math.inf                       # the reference never draws this token
    loss = vie.policy_loss(z.cuda(), tok.cuda(), old.cuda(), adv.cuda(), ref_logprob=r.cuda(), kl_coef=0.5)[0]
    assert loss[6] == math.inf and torch.isfinite(loss[[0, 2, 3, 4, 5, 7]]).all()


def test_a_ratio_of_one_on_both_borders(vie):
    """The tokens' own policy, no clip range at all: r A is the smaller one as well."""
    z, tok, grad, g = _inputs(6, 500, "f32", seed=19)
    adv = torch.tensor([1.0, -1.0, 2.0, -2.0, 0.5, 0.0])
    zc, tc = z.cuda(), tok.cuda()
    old, _ = vie.token_logprobs(zc, tc)
    loss, lp, stats = vie.policy_loss(zc, tc, old, adv.cuda(), clip_low=0.0, clip_high=0.0)
    assert torch.equal(lp, old) and torch.equal(loss.cpu(), -adv)
    dz = vie.policy_loss_grad(zc, tc, old, adv.cuda(), lp, stats, grad.cuda(), clip_low=0.0, clip_high=0.0)
    assert torch.equal(dz, vie.token_logprobs_grad(zc, tc, stats, grad.cuda() * -adv.cuda()))


def test_clipped_tokens_have_no_gradient(vie):
    z, tok, grad, g = _inputs(4, 5000, "bf16", seed=23)
    rows = ref.Rows(z, tok, 1.0)
    old = (rows.lp - torch.tensor([0.5, 0.5, -0.5, -0.5]).double()).float()
    adv = torch.tensor([1.0, -1.0, 1.0, -1.0])
    dz = vie.policy_loss_step(z.cuda(), tok.cuda(), old.cuda(), adv.cuda(), grad.cuda())[2]
    assert not dz[[0, 3]].any() and dz[[1, 2]].any(1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ld,off", [(1000, 0), (1003, 0), (1001, 1), (1024, 3), (1013, 7)])
def test_strides_and_alignment(vie, dtype, ld, off):
    n, V = 5, 999
    z, tok, grad, g = _inputs(n, V, dtype, seed=ld + off)
    big = torch.full((n * ld + off + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    zc = big[off:off + n * ld].view(n, ld)[:, :V]
    zc.copy_(z)
    _check(vie, z, tok, 1.0, grad, g, zc=zc)
    lp, stats = vie.token_logprobs(zc, tok.cuda())
    want = vie.token_logprobs_grad(zc, tok.cuda(), stats, grad.cuda())
    for o, l in ((0, V), (1, V + 2), (5, V + 9)):  # nothing outside an output's rows is written
        buf = torch.full((n * l + 16,), 7.0, dtype=DT[dtype], device="cuda")
        out = buf[o:o + n * l].view(n, l)[:, :V]
        got = vie.token_logprobs_grad(zc, tok.cuda(), stats, grad.cuda(), out_grad=out)
        assert got.data_ptr() == out.data_ptr() and torch.equal(got, want)
        out.fill_(7.0)
        assert (buf == 7.0).all()
    got = vie.token_logprobs(z.t().contiguous().cuda().t(), tok.cuda())[0]  # other layouts are copied
    assert torch.equal(got, vie.token_logprobs(z.cuda(), tok.cuda())[0])


@pytest.mark.parametrize("T", [1.0, 2.0])
def test_gradients_against_differences(vie, T):
    """From differences of the GPU's own results: logits spaced so that a step of
    2^-7 is exact; a central difference is off by h^2 / 6 of the third derivative
    (of lp at most 1 / T^3; of a loss with |A| r and kl of at most 2 at most 8 of
    them) plus the result's error over h."""
    V, h = 64, 2.0 ** -7
    g = torch.Generator().manual_seed(29)
    z = torch.round(torch.randn(1, V, generator=g) * 64) / 64
    tok = torch.tensor([17], dtype=torch.int32)
    many = torch.cat([z + torch.eye(V) * h, z - torch.eye(V) * h]).cuda()
    rows = ref.Rows(z, tok, T)
    tol = float(rows.lp_tol[0])
    one = torch.ones(1, device="cuda")
    lp = vie.token_logprobs(many, tok.expand(2 * V).cuda(), temperature=T)[0].double().cpu()
    stats = vie.token_logprobs(z.cuda(), tok.cuda(), temperature=T)[1]
    dz = vie.token_logprobs_grad(z.cuda(), tok.cuda(), stats, one, temperature=T).double().cpu()[0]
    assert (dz - (lp[:V] - lp[V:]) / (2 * h)).abs().max() <= h * h / 6 / T ** 3 + tol / h
    old, r = (rows.lp - 0.03).float(), (rows.lp + 0.3).float()
    for A, kl in ((1.0, 0.0), (-0.7, 0.5), (0.0, 1.0)):
        a = torch.tensor([A])
        how = dict(ref_logprob=r.cuda(), kl_coef=kl, temperature=T)
        wide = {k: (v.expand(2 * V) if k == "ref_logprob" else v) for k, v in how.items()}
        loss = vie.policy_loss(many, tok.expand(2 * V).cuda(), old.expand(2 * V).cuda(), a.expand(2 * V).cuda(),
                               **wide)[0].double().cpu()
        dz = vie.policy_loss_step(z.cuda(), tok.cuda(), old.cuda(), a.cuda(), one, **how)[2].double().cpu()[0]
        loss_tol = float(ref.policy(rows, old, a, r, 0.2, 0.2, kl)[1][0])
        assert (dz - (loss[:V] - loss[V:]) / (2 * h)).abs().max() <= 8 * h * h / 6 / T ** 3 + 2 * loss_tol / h


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1e-38, 1e-30, 1e-20, 1e20, 1e30])
def test_temperatures_far_from_one(vie, dtype, T):
    T = float(torch.tensor(T, dtype=torch.float32))
    z, tok, grad, g = _inputs(5, 64, dtype, seed=31)
    tok[0] = z[0].float().argmax()
    rows = ref.Rows(z, tok, T)
    lp, stats = vie.token_logprobs(z.cuda(), tok.cuda(), temperature=T)
    want = rows.lp.float().double()  # (-inf where it is beyond fp32)
    got = lp.double().cpu()
    assert ((got == want) | ((got - want).abs() <= rows.lp_tol)).all() and not torch.isnan(lp).any()
    dz = vie.token_logprobs_grad(z.cuda(), tok.cuda(), stats, grad.cuda() * T, temperature=T)
    gt = (grad.cuda() * T).cpu()
    want, tol = rows.gradient(gt, torch.zeros(5).double())
    _close(dz, want, tol + 2.0 ** -148 / T, "gradient")  # (a product with T that is subnormal)


def test_the_same_bits_again_on_a_stream_and_in_a_graph(vie):
    z, tok, grad, g = _inputs(9, 30011, "bf16", seed=37)
    old, adv, r = (x.cuda() for x in _terms(ref.Rows(z, tok, 1.0), g, 0.2, 0.2))
    z, tok, grad = z.cuda(), tok.cuda(), grad.cuda()
    how = dict(ref_logprob=r, kl_coef=0.1)
    want = vie.policy_loss_step(z, tok, old, adv, grad, **how)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = vie.policy_loss_step(z, tok, old, adv, grad, stream=s, **how)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = [torch.empty_like(x) for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        vie.policy_loss_step(z, tok, old, adv, grad, out_loss=out[0], out_logprob=out[1], out_grad=out[2], **how)
    for _ in range(2):
        for x in out:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_offsets_beyond_32_bits(vie):
    V = 262144
    n = 2 ** 31 // V + 3
    big = torch.zeros((n, V), dtype=torch.bfloat16, device="cuda")
    z, tok, grad, g = _inputs(2, V, "bf16", seed=41)
    old, adv, r = _terms(ref.Rows(z, tok, 1.0), g, 0.2, 0.2)
    want = vie.policy_loss_step(z.cuda(), tok.cuda(), old.cuda(), adv.cuda(), grad.cuda())
    big[-2:] = z.cuda()
    tok_all = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    rest = [torch.ones(n, device="cuda") for _ in range(3)]
    tok_all[-2:] = tok.cuda()
    for x, y in zip(rest, (old, adv, grad)):
        x[-2:] = y.cuda()
    loss, lp, dz = vie.policy_loss_step(big, tok_all, *rest, out_grad=big)
    assert torch.equal(loss[-2:], want[0]) and torch.equal(dz[-2:], want[2])
    assert (loss[:-2] == 0).all() and not dz[:-2].any()


def test_changes_in_place_are_counted(vie):
    _, tok, grad, _ = (x.cuda() if torch.is_tensor(x) else x for x in _inputs(4, 100, "f32", seed=43))
    leaf = torch.randn(4, 100, device="cuda", requires_grad=True)
    for form in ("logprobs", "grad", "step"):
        z = leaf * 1.0
        square = (z * z).sum()  # saves z
        before = z._version
        lp, stats = vie.token_logprobs(z, tok)
        vie.token_logprobs_grad(z, tok, stats, grad)
        assert z._version == before
        own = z.detach()
        if form == "logprobs":
            vie.token_logprobs_grad(own, tok, stats, grad, out_grad=own)
        elif form == "grad":
            vie.policy_loss_grad(own, tok, lp, grad, lp, stats, grad, out_grad=own)
        else:
            vie.policy_loss_step(own, tok, lp, grad, grad, out_grad=own)
        assert z._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            square.backward()


def test_no_rows_and_refusals(vie):
    z, tok, grad, _ = (x.cuda() if torch.is_tensor(x) else x for x in _inputs(4, 100, "f32", seed=47))
    lp, stats = vie.token_logprobs(z[:0], tok[:0])
    assert lp.shape == (0,) and stats.shape == (0, 2)
    assert vie.policy_loss_step(z[:0], tok[:0], grad[:0], grad[:0], grad[:0])[2].shape == (0, 100)
    lp, stats = vie.token_logprobs(z, tok)
    for call in (lambda: vie.token_logprobs(z.half(), tok), lambda: vie.token_logprobs(z, tok.long()),
                 lambda: vie.token_logprobs(z, tok[:3]), lambda: vie.token_logprobs(z[0], tok),
                 lambda: vie.token_logprobs(z, tok.cpu()),
                 lambda: vie.token_logprobs(z, tok, out_logprob=torch.empty(8, device="cuda")[::2]),
                 lambda: vie.token_logprobs_grad(z, tok, stats[:, :1], grad),
                 lambda: vie.token_logprobs_grad(z, tok, stats, grad.double()),
                 lambda: vie.token_logprobs_grad(z, tok, stats, grad, out_grad=z.t()),
                 lambda: vie.token_logprobs_grad(z, tok, stats, grad, out_grad=z.bfloat16()),
                 lambda: vie.policy_loss(z, tok, lp, grad, kl_coef=0.1),
                 lambda: vie.policy_loss(z, tok, lp[:3], grad),
                 lambda: vie.policy_loss(z, tok, lp, grad, ref_logprob=lp.half(), kl_coef=0.1),
                 lambda: vie.policy_loss_grad(z, tok, lp, grad, lp[:2], stats, grad),
                 lambda: vie.policy_loss_step(z, tok, lp, grad, grad[:3])):
        with pytest.raises(ValueError):
            call()
    for kw in (dict(temperature=0.0), dict(clip_low=1.5), dict(clip_low=-0.1), dict(clip_high=-0.1),
               dict(clip_high=math.inf), dict(kl_coef=-1.0, ref_logprob=lp), dict(kl_coef=math.nan, ref_logprob=lp)):
        with pytest.raises(vie.VieError):
            vie.policy_loss(z, tok, lp, grad, **kw)
