"""GPU parity of distillation from a teacher's top logits (vie_distill_topk,
_grad, _step) against its definition in 64 bits (tests/student_ref.py, with the
tolerances derived there), and the gradient against differences of the loss."""
import math

import pytest
import torch

import student_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(n, V, k, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    z = (spread * torch.randn(n, V, generator=g)).to(DT[dtype])
    idx = torch.stack([torch.randperm(V, generator=g)[:k] if k <= V else torch.randint(0, V, (k,), generator=g)
                       for _ in range(n)]).int()
    t = 3.0 + 2.0 * torch.randn(n, k, generator=g)
    gl = torch.randn(n, generator=g)
    return z, idx, t, gl


def _check(vie, z, idx, t, T, gl, zc=None, forms=("apart", "step", "in place")):
    """Every form of the call on the GPU tensor of z (or zc: the same values laid out otherwise)."""
    want_loss, want_stats, want_grad, loss_tol, s_tol, grad_tol = ref.distill(z, idx, t, T, gl)
    zc = z.cuda() if zc is None else zc
    ic, tc, gc = idx.cuda(), t.cuda(), gl.cuda()

    def close(got, want, tol, what):
        got = got.double().cpu()
        same = (got == want) | (torch.isnan(got) & torch.isnan(want))
        bad = ~(same | ((got - want).abs() <= tol))
        assert not bad.any(), (what, got[bad][:4], want[bad][:4], (bad.nonzero()[:4]).tolist())

    rnd = ref.out_round(z.dtype)
    for form in forms:
        if form == "apart":
            loss, stats = vie.distill_topk(zc, ic, tc, temperature=T)
            keep = stats.clone()
            close(stats[:, 0], want_stats[:, 0], 0, form)
            close(stats[:, 1], want_stats[:, 1], s_tol, form)
            grad = vie.distill_topk_grad(zc, ic, tc, stats, gc, temperature=T)
            assert torch.equal(keep.view(torch.int32), stats.view(torch.int32))
        elif form == "step":
            loss, grad = vie.distill_topk_step(zc, ic, tc, gc, temperature=T)
        else:
            own = zc.clone()
            loss, grad = vie.distill_topk_step(own, ic, tc, gc, temperature=T, out_grad=own)
            assert grad.data_ptr() == own.data_ptr()
            own = zc.clone()
            grad2 = vie.distill_topk_grad(own, ic, tc, vie.distill_topk(own, ic, tc, temperature=T)[1], gc,
                                          temperature=T, out_grad=own)
            close(grad2, want_grad, grad_tol + (rnd + ref.U) * want_grad.abs(), form)
        assert grad.dtype == z.dtype
        close(loss, want_loss, loss_tol, form)
        close(grad, want_grad, grad_tol + (rnd + ref.U) * want_grad.abs(), form)
    assert vie.vie_device_status() == vie.VIE_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,k,T", [
    (1, 1, 1, 1.0), (3, 2, 1, 1.0), (2, 7, 7, 0.5), (5, 33, 8, 2.0), (4, 257, 50, 1.0), (3, 1000, 64, 1.0),
    (2, 4099, 1024, 1.5), (7, 20011, 50, 1.0), (3, 40000, 129, 4.0), (2, 65536, 50, 1.0), (2, 131071, 300, 1.0),
    (300, 515, 13, 1.0), (2, 262144, 50, 0.7),
])
def test_sizes(vie, dtype, n, V, k, T):
    z, idx, t, gl = _inputs(n, V, k, dtype, seed=V + k)
    _check(vie, z, idx, t, T, gl)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_one_launch_cannot_keep_on_chip(vie, dtype):
    """Rows longer than the shared memory of any cluster that the step uses."""
    z, idx, t, gl = _inputs(1, 1000003, 50, dtype, seed=3)
    _check(vie, z, idx, t, 1.0, gl)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_empty_slots_and_rows(vie, dtype):
    z, idx, t, gl = _inputs(12, 3001, 40, dtype, seed=5)
    idx[0] = -1                       # no entries at all
    idx[1, 3:] = -1                   # a short list
    t[1, 3:] = float("nan")           # what stands in empty slots does not matter
    idx[2, ::2] = 3001                # out of range: empty
    t[2, 0] = float("inf")
    t[3] = -math.inf                  # entries without weight: an empty row
    t[4, 1:] = -math.inf
    idx[5] = -7
    z[5] = float("nan")               # an empty row's logits are not read
    idx[6] = 2 ** 31 - 1
    idx[7, 0] = 3000
    idx[8, 0] = 0
    z[0, 5] = float("inf")
    _check(vie, z, idx, t, 1.0, gl)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k", [2, 50, 1024])
def test_repeated_indices_add_up(vie, dtype, k):
    z, idx, t, gl = _inputs(6, 2003, k, dtype, seed=7)
    idx[0, 1] = idx[0, 0]
    idx[1] = 77                       # all the same
    idx[2] = (torch.arange(k) % 5).int()
    idx[3, -1] = idx[3, 0]
    _check(vie, z, idx, t, 1.3, gl)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_masked_logits(vie, dtype, T):
    """-inf and the type's lowest value in masked places, rows of nothing else."""
    low = torch.finfo(DT[dtype]).min
    z, idx, t, gl = _inputs(10, 1537, 20, dtype, seed=11)
    z[0, ::3] = -math.inf
    z[1, ::3] = low
    z[1, idx[1].long()] = 0.5         # (a teacher's token there: a loss of about the type's largest value)
    z[2] = low                        # equal logits: uniform
    z[3] = -math.inf                  # no softmax: q = 0, the loss is +inf
    z[4] = -math.inf
    z[4, idx[4].long()] = 1.0         # only the teacher's tokens
    z[5] = low
    z[5, 7] = -math.inf
    z[6, idx[6, 0].long()] = -math.inf  # the teacher wants a masked token: +inf
    z[7] = torch.finfo(DT[dtype]).max
    z[8, :700] = low
    z[8, 700:] = -math.inf
    _check(vie, z, idx, t, T, gl)


def test_nan_and_inf_stay_in_their_row(vie):
    z, idx, t, gl = _inputs(5, 999, 10, "f32", seed=13)
    z[1, 500] = float("nan")
    z[3, 2] = float("inf")
    t[4, 0] = float("nan")
    loss, grad = vie.distill_topk_step(z.cuda(), idx.cuda(), t.cuda(), gl.cuda())
    for r in range(5):
        ok = r in (0, 2)
        assert bool(torch.isfinite(loss[r])) == ok
        if ok:
            assert torch.isfinite(grad[r]).all()
        elif r == 4:
            assert torch.isnan(grad[r, idx[4].long()]).all()  # p is NaN, q is not
        else:
            assert torch.isnan(grad[r]).any()


def test_extreme_teachers_and_temperatures(vie):
    z, idx, t, gl = _inputs(6, 2000, 30, "f32", seed=17, spread=30.0)
    t[0] = 1e30 * torch.arange(30)
    t[1] = -3e38
    t[2] = 0.0
    for T in (0.05, 20.0):
        _check(vie, z, idx, t, T, gl)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ld,off", [(1000, 0), (1003, 0), (1001, 1), (1024, 3), (1013, 7)])
def test_strides_and_alignment(vie, dtype, ld, off):
    n, V, k = 5, 999, 20
    z, idx, t, gl = _inputs(n, V, k, dtype, seed=ld + off)
    big = torch.full((n * ld + off + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    zc = big[off:off + n * ld].view(n, ld)[:, :V]
    zc.copy_(z)
    _check(vie, z, idx, t, 1.0, gl, zc=zc, forms=("apart", "step"))
    # an output with a pitch and alignment of its own: nothing outside its rows is written
    want = vie.distill_topk_step(zc, idx.cuda(), t.cuda(), gl.cuda())[1]
    for o, l in ((0, V), (1, V + 2), (5, V + 9)):
        buf = torch.full((n * l + 16,), 7.0, dtype=DT[dtype], device="cuda")
        out = buf[o:o + n * l].view(n, l)[:, :V]
        got = vie.distill_topk_step(zc, idx.cuda(), t.cuda(), gl.cuda(), out_grad=out)[1]
        assert got.data_ptr() == out.data_ptr() and torch.equal(got, want)
        buf[o:o + n * l].view(n, l)[:, :V] = 7.0
        assert (buf == 7.0).all()
    # other layouts are copied
    got = vie.distill_topk_step(z.t().contiguous().cuda().t(), idx.cuda(), t.cuda(), gl.cuda())[1]
    assert torch.equal(got, vie.distill_topk_step(z.cuda(), idx.cuda(), t.cuda(), gl.cuda())[1])


def test_gradient_against_differences(vie):
    """d loss / d z from differences of the GPU's own loss: logits spaced so that
    a step of 2^-7 is exact; the error of a central difference is h^2 / 6 of the
    third derivative (at most 1 / T) plus twice the loss's error over 2 h."""
    n, V, k, h = 1, 64, 6, 2.0 ** -7
    for T in (1.0, 2.0):
        g = torch.Generator().manual_seed(3)
        z = torch.round(torch.randn(n, V, generator=g) * 64) / 64
        idx = torch.randperm(V, generator=g)[:k][None].int()
        t = torch.randn(n, k, generator=g)
        eye = torch.eye(V) * h
        many = torch.cat([z + eye, z - eye]).cuda()
        loss = vie.distill_topk(many, idx.expand(2 * V, k).cuda(), t.expand(2 * V, k).cuda(), temperature=T)[0].double().cpu()
        diff = (loss[:V] - loss[V:]) / (2 * h)
        grad = vie.distill_topk_step(z.cuda(), idx.cuda(), t.cuda(), torch.ones(1, device="cuda"), temperature=T)[1]
        tol = h * h / 6 / T + 2 * float(ref.distill(z, idx, t, T, torch.ones(1))[3][0]) / (2 * h)
        assert (grad.double().cpu()[0] - diff).abs().max() <= tol


def test_rows_sum_to_zero_and_repeat_bit_for_bit(vie):
    z, idx, t, gl = _inputs(40, 5001, 50, "f32", seed=23)
    a = vie.distill_topk_step(z.cuda(), idx.cuda(), t.cuda(), gl.cuda())
    b = vie.distill_topk_step(z.cuda(), idx.cuda(), t.cuda(), gl.cuda())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # sum of q - p is 0: 5001 roundings of values that sum to at most 2
    total = a[1].double().sum(1).cpu().abs() / gl.abs().double()
    assert (total <= 2 * (4 * 20 + 4 + 5001 / 256 + 64) * ref.U).all()


def test_another_stream_and_a_graph(vie):
    z, idx, t, gl = (x.cuda() for x in _inputs(9, 30011, 50, "bf16", seed=29))
    want = vie.distill_topk_step(z, idx, t, gl)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = vie.distill_topk_step(z, idx, t, gl, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    loss, grad = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        vie.distill_topk_step(z, idx, t, gl, out_loss=loss, out_grad=grad)
    for _ in range(2):
        loss.zero_()
        grad.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[1])


def test_no_rows_and_refusals(vie):
    z, idx, t, gl = (x.cuda() for x in _inputs(4, 100, 5, "f32", seed=31))
    loss, stats = vie.distill_topk(z[:0], idx[:0], t[:0])
    assert loss.shape == (0,) and stats.shape == (0, 2)
    assert vie.distill_topk_step(z[:0], idx[:0], t[:0], gl[:0])[1].shape == (0, 100)
    with pytest.raises(ValueError):
        vie.distill_topk(z.half(), idx, t)
    with pytest.raises(ValueError):
        vie.distill_topk(z, idx.long(), t)
    with pytest.raises(ValueError):
        vie.distill_topk(z, idx[:3], t[:3])
    with pytest.raises(ValueError):
        vie.distill_topk(z, idx, t[:, :4])
    with pytest.raises(ValueError):
        vie.distill_topk_step(z, idx, t, gl.double())
    with pytest.raises(ValueError):
        vie.distill_topk_step(z, idx, t, gl, out_grad=torch.empty(4, 99, device="cuda"))
    with pytest.raises(ValueError):
        vie.distill_topk_step(z, idx, t, gl, out_grad=torch.empty(4, 100, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        vie.distill_topk_step(z, idx, t, gl, out_grad=torch.empty(100, 4, device="cuda").t())
    with pytest.raises(vie.VieError):
        vie.distill_topk(z, idx, t, temperature=0.0)


def test_offsets_beyond_32_bits(vie):
    """The last rows of a matrix of more than 2^31 values."""
    V, k = 262144, 50
    n = 2 ** 31 // V + 3
    big = torch.zeros((n, V), dtype=torch.bfloat16, device="cuda")
    z, idx, t, gl = _inputs(2, V, k, "bf16", seed=37)
    big[-2:] = z.cuda()
    idx_all = torch.full((n, k), -1, dtype=torch.int32, device="cuda")
    idx_all[-2:] = idx.cuda()
    t_all = torch.zeros((n, k), device="cuda")
    t_all[-2:] = t.cuda()
    gl_all = torch.ones(n, device="cuda")
    gl_all[-2:] = gl.cuda()
    want = vie.distill_topk_step(z.cuda(), idx.cuda(), t.cuda(), gl.cuda())
    loss, grad = vie.distill_topk_step(big, idx_all, t_all, gl_all, out_grad=big)
    assert torch.equal(loss[-2:], want[0]) and torch.equal(grad[-2:], want[1])
    assert (loss[:-2] == 0).all() and not grad[:-2].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1e-38, 1e-30, 1e-24, 1e-20, 1e18, 1e20, 1e30])
def test_temperatures_whose_square_leaves_fp32(vie, dtype, T):
    """Any positive finite temperature: T^2 is 0 or infinite in fp32 at most of
    these, the loss (about T times a difference of logits where T is small) is not.
    Where T^2 times the roundings' error is beyond fp32, only its sign of NaN is looked at."""
    T = float(torch.tensor(T, dtype=torch.float32))
    n, V = 4, 64
    z, idx, t, gl = _inputs(n, V, V, dtype, seed=41)
    z[1, idx[1, t[1].argmax()].long()] = -math.inf  # the teacher wants a masked token: +inf
    idx[2, 5:] = -1
    t[3] = z[3, idx[3].long()].float()              # the same distribution
    want_loss, _, want_grad, loss_tol, _, grad_tol = ref.distill(z, idx, t, T, gl)
    zc, ic, tc, gc = z.cuda(), idx.cuda(), t.cuda(), gl.cuda()
    least = 2.0 ** -149  # spacing of the smallest fp32 values
    largest = torch.finfo(torch.float32).max
    for loss, grad in (vie.distill_topk_step(zc, ic, tc, gc, temperature=T),
                       (vie.distill_topk(zc, ic, tc, temperature=T)[0], None)):
        loss = loss.double().cpu()
        assert not torch.isnan(loss).any() and loss[1] == math.inf
        for r in (0, 2, 3):
            want = float(want_loss[r].float())  # (+inf where the loss itself is beyond fp32)
            if float(loss_tol[r]) < largest:
                assert float(loss[r]) == want or abs(float(loss[r]) - want) <= float(loss_tol[r]) + 2 * least, r
        if grad is not None:
            grad = grad.double().cpu()
            tol = grad_tol + (ref.out_round(z.dtype) + ref.U) * want_grad.abs() + 2 * least
            assert ((grad - want_grad).abs() <= tol).all()


def test_a_stream_of_another_device_is_refused(vie):
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    z, idx, t, _ = (x.cuda(0) for x in _inputs(4, 100, 5, "f32", seed=31))
    with pytest.raises(ValueError, match="stream"):
        vie.distill_topk(z, idx, t, stream=torch.cuda.Stream(device=1))


def test_changes_in_place_are_counted(vie):
    """A gradient in place of the logits is a change that autograd has to know
    of: a graph that has saved them refuses to go on.  Other calls change none."""
    _, idx, t, gl = (x.cuda() for x in _inputs(4, 100, 5, "f32", seed=43))
    leaf = torch.randn(4, 100, device="cuda", requires_grad=True)
    for form in ("step", "apart"):
        z = leaf * 1.0
        square = (z * z).sum()  # saves z
        before = z._version
        stats = vie.distill_topk(z, idx, t)[1]
        vie.distill_topk_step(z, idx, t, gl, out_grad=torch.empty_like(z))
        assert z._version == before
        own = z.detach()
        if form == "step":
            vie.distill_topk_step(own, idx, t, gl, out_grad=own)
        else:
            vie.distill_topk_grad(own, idx, t, stats, gl, out_grad=own)
        assert z._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            square.backward()
    with torch.inference_mode():  # such tensors have no count
        z = torch.randn(4, 100, device="cuda")
        vie.distill_topk_step(z, idx, t, gl, out_grad=z)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_step_hands_out_its_statistics(vie, dtype):
    z, idx, t, gl = _inputs(5, 3001, 20, dtype, seed=47)
    idx[2] = -1
    _, want_stats, want_grad, _, s_tol, grad_tol = ref.distill(z, idx, t, 1.5, gl)
    zc, ic, tc, gc = z.cuda(), idx.cuda(), t.cuda(), gl.cuda()
    out = torch.full((5, 2), 7.0, device="cuda")
    loss, grad = vie.distill_topk_step(zc, ic, tc, gc, temperature=1.5, out_stats=out)
    plain = vie.distill_topk_step(zc, ic, tc, gc, temperature=1.5)
    assert torch.equal(loss, plain[0]) and torch.equal(grad, plain[1])
    got = out.double().cpu()
    assert torch.equal(got[:, 0], want_stats[:, 0]) and ((got[:, 1] - want_stats[:, 1]).abs() <= s_tol).all()
    again = vie.distill_topk_grad(zc, ic, tc, out, gc, temperature=1.5)  # what they are for
    tol = grad_tol + (ref.out_round(z.dtype) + ref.U) * want_grad.abs()
    assert ((again.double().cpu() - want_grad).abs() <= tol).all()
    for bad in (torch.empty(5, 3, device="cuda"), torch.empty(5, 2, dtype=torch.float64, device="cuda"),
                torch.empty(5, 2), torch.empty(2, 5, device="cuda").t()):
        with pytest.raises(ValueError, match="out_stats"):
            vie.distill_topk_step(zc, ic, tc, gc, out_stats=bad)


@pytest.mark.parametrize("T", [0.01, 0.1, 0.5, 0.9])
def test_teachers_of_nothing_but_masked_tokens(vie, T):
    """All of a teacher's tokens at the type's lowest value: a loss of about T times
    that, within fp32, though the lowest value over T is not."""
    n, V, k = 200, 300, 40
    z, idx, t, gl = _inputs(n, V, k, "f32", seed=53)
    z.scatter_(1, idx.long(), torch.finfo(torch.float32).min)
    T = float(torch.tensor(T, dtype=torch.float32))
    want, _, _, tol, _, _ = ref.distill(z, idx, t, T, gl)
    assert float(want.max()) < 0.95 * torch.finfo(torch.float32).max
    for loss in (vie.distill_topk(z.cuda(), idx.cuda(), t.cuda(), temperature=T)[0],
                 vie.distill_topk_step(z.cuda(), idx.cuda(), t.cuda(), gl.cuda(), temperature=T)[0]):
        assert ((loss.double().cpu() - want).abs() <= tol).all()
