"""GPU parity of the preference loss and its gradient against their definitions in
64 bits (tests/policy_ref.py, with the tolerances derived there), and against
differences."""
import math

import pytest
import torch

import policy_ref as ref

pytestmark = pytest.mark.gpu


def _inputs(lengths, before, behind, seed, spread=0.1):
    g = torch.Generator().manual_seed(seed)
    ends = torch.cat([torch.tensor([before]), before + torch.cumsum(torch.tensor(lengths, dtype=torch.long), 0)])
    n = int(ends[-1]) + behind
    lp = -3.0 * torch.rand(n, generator=g)
    return lp, lp + spread * torch.randn(n, generator=g), ends.int(), torch.randn(len(lengths) // 2, generator=g)


def _check(vie, lp, r, ends, grad, beta, smoothing):
    loss_w, h_w, slope, loss_t, h_t, slope_t = ref.preference(lp, r, ends, beta, smoothing)
    rc = None if r is None else r.cuda()
    how = dict(beta=beta, label_smoothing=smoothing)
    loss, h = vie.preference_loss(lp.cuda(), ends.cuda(), ref_logprob=rc, **how)
    out = torch.full_like(lp.cuda(), 7.0)
    loss2, h2, dlp = vie.preference_loss_step(lp.cuda(), ends.cuda(), grad.cuda(), ref_logprob=rc, out_grad=out, **how)
    assert torch.equal(loss, loss2) and torch.equal(h, h2)
    assert torch.equal(vie.preference_loss_grad(h, ends.cuda(), grad.cuda(), len(lp), **how), dlp)
    assert ((loss.double().cpu() - loss_w).abs() <= loss_t).all()
    assert ((h.double().cpu() - h_w).abs() <= h_t).all()
    want, tol = torch.zeros(len(lp)).double(), torch.zeros(len(lp)).double()
    e = ends.tolist()
    for p in range(len(grad)):
        for a, b, sign in ((e[2 * p], e[2 * p + 1], 1), (e[2 * p + 1], e[2 * p + 2], -1)):
            want[a:b] = sign * grad[p].double() * slope[p]
            tol[a:b] = grad[p].double().abs() * slope_t[p]
    assert ((dlp.double().cpu() - want).abs() <= tol).all()
    assert vie.vie_device_status() == vie.VIE_OK


@pytest.mark.parametrize("lengths", [
    [1, 1], [0, 0], [0, 5], [7, 0], [3, 2, 0, 0, 1, 9], [255, 256, 257, 31, 32, 33], [1000, 1] * 40, [5, 300] * 200,
    [20000, 13], [70001, 65536], [300000, 1, 2, 3],
], ids=str)
@pytest.mark.parametrize("before,behind", [(0, 0), (3, 5), (777, 40001)])
def test_sizes(vie, lengths, before, behind):
    lp, r, ends, grad = _inputs(lengths, before, behind, seed=len(lengths) + before)
    _check(vie, lp, r, ends, grad, 0.1, 0.0)
    _check(vie, lp, None, ends, grad, 0.05, 0.2)


@pytest.mark.parametrize("beta", [0.0, -0.3, 1.0, 50.0, 1000.0])
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 0.5, 1.0])
def test_margins_of_any_size(vie, beta, smoothing):
    lp, r, ends, grad = _inputs([40, 60, 13, 0, 100, 101], 1, 1, seed=3)
    _check(vie, lp, r, ends, grad, beta, smoothing)


def test_gradient_against_differences(vie):
    """Steps of 2^-6 of one token at a time: a central difference of the GPU's loss is
    off by h^2 / 6 of the third derivative (beta^3 at most) plus the loss's error over h."""
    h, beta = 2.0 ** -6, 0.5
    lp, r, ends, _ = _inputs([5, 7, 4, 6], 2, 3, seed=5)
    lp = torch.round(lp * 64) / 64
    one = torch.ones(2, device="cuda")
    dlp = vie.preference_loss_step(lp.cuda(), ends.cuda(), one, ref_logprob=r.cuda(), beta=beta)[2].double().cpu()
    tol = float(ref.preference(lp, r, ends, beta, 0.0)[3].max())
    for i in range(len(lp)):
        d = torch.zeros(len(lp))
        d[i] = h
        up = vie.preference_loss((lp + d).cuda(), ends.cuda(), ref_logprob=r.cuda(), beta=beta)[0].double().sum()
        down = vie.preference_loss((lp - d).cuda(), ends.cuda(), ref_logprob=r.cuda(), beta=beta)[0].double().sum()
        assert abs(float(up - down) / (2 * h) - float(dlp[i])) <= h * h / 6 * beta ** 3 + 4 * tol / h


def test_infinite_log_probabilities_stay_in_their_pair(vie):
    lp, r, ends, grad = _inputs([9, 9, 9, 9, 9, 9], 0, 0, seed=7)
    lp[3] = -math.inf          # a token that the policy rules out, in a chosen answer
    lp[30] = -math.inf         # in a rejected one
    loss, h, dlp = vie.preference_loss_step(lp.cuda(), ends.cuda(), torch.ones(3, device="cuda"), ref_logprob=r.cuda())
    assert loss[0] == math.inf and h[0] == -math.inf and loss[1] == 0 and h[1] == math.inf
    assert torch.allclose(dlp[:9], torch.full((9,), -0.1, device="cuda")) and not dlp[18:36].any()
    assert torch.isfinite(loss[2]) and torch.isfinite(dlp).all()
    lp[3] = float("nan")
    loss = vie.preference_loss(lp.cuda(), ends.cuda(), ref_logprob=r.cuda())[0]
    assert torch.isnan(loss).tolist() == [True, False, False]


def test_a_weight_of_zero_masks_a_pair(vie):
    lp, r, ends, grad = _inputs([9, 9, 9, 9], 0, 0, seed=11)
    lp[2] = float("nan")
    w = torch.tensor([0.0, 1.0], device="cuda")
    _, h, dlp = vie.preference_loss_step(lp.cuda(), ends.cuda(), w, ref_logprob=r.cuda())
    assert torch.isnan(h[0]) and not dlp[:18].any() and dlp[18:].all()
    assert torch.equal(vie.preference_loss_grad(h, ends.cuda(), w, len(lp)), dlp)


def test_bad_offsets_are_held_inside_and_reported(vie):
    """Host and kernel keep every access inside the n tokens."""
    lp, r, ends, grad = _inputs([9, 9, 9, 9], 2, 2, seed=9)
    for bad in ([-5, 9, 18, 27, 36], [2, 11, 5, 29, 38], [2, 11, 20, 29, 2 ** 31 - 1], [50, 60, 70, 80, 90]):
        o = torch.tensor(bad, dtype=torch.int32, device="cuda")
        buf = torch.full((len(lp) + 64,), 7.0, device="cuda")
        vie.preference_loss_step(lp.cuda(), o, torch.ones(2, device="cuda"), ref_logprob=r.cuda(),
                                 out_grad=buf[32:-32])
        assert (buf[:32] == 7.0).all() and (buf[-32:] == 7.0).all()
        assert vie.vie_device_status() == vie.VIE_ERR_DEVICE and "offsets" in vie.vie_last_error()
    assert vie.vie_device_status() == vie.VIE_OK


def test_a_stream_a_graph_and_nothing_to_do(vie):
    lp, r, ends, grad = (x.cuda() for x in _inputs([500, 700] * 9, 3, 4, seed=11))
    want = vie.preference_loss_step(lp, ends, grad, ref_logprob=r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = vie.preference_loss_step(lp, ends, grad, ref_logprob=r, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = [torch.empty_like(x) for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        vie.preference_loss_step(lp, ends, grad, ref_logprob=r, out_loss=out[0], out_margin=out[1], out_grad=out[2])
    for x in out:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, h, dlp = vie.preference_loss_step(lp, none, grad[:0])
    assert loss.shape == (0,) and dlp.shape == lp.shape and not dlp.any()
    loss = vie.preference_loss(lp[:0], torch.zeros(3, dtype=torch.int32, device="cuda"))[0]
    assert abs(float(loss[0]) - math.log(2)) < 1e-6


def test_refusals(vie):
    lp, r, ends, grad = (x.cuda() for x in _inputs([5, 7, 4, 6], 2, 3, seed=5))
    for call in (lambda: vie.preference_loss(lp.double(), ends), lambda: vie.preference_loss(lp, ends.long()),
                 lambda: vie.preference_loss(lp, ends[:4]), lambda: vie.preference_loss(lp[None], ends),
                 lambda: vie.preference_loss(lp, ends, ref_logprob=r[:-1]), lambda: vie.preference_loss(lp, ends.cpu()),
                 lambda: vie.preference_loss_step(lp, ends, grad[:1]),
                 lambda: vie.preference_loss_grad(grad[:1], ends, grad, 20),
                 lambda: vie.preference_loss_step(lp, ends, grad, out_grad=lp[:-1])):
        with pytest.raises(ValueError):
            call()
    for kw in (dict(beta=math.inf), dict(beta=math.nan), dict(label_smoothing=-0.1), dict(label_smoothing=1.1)):
        with pytest.raises(vie.VieError):
            vie.preference_loss(lp, ends, **kw)
