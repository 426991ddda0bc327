"""Host-side argument checks of the calls on drawn tokens and 4-bit rows: status
codes and messages before any CUDA call, and what the torch binding refuses."""
import math
import os
import re

import pytest
import torch

import paper_2608_27460_gb300 as vie
import policy_ref as ref

P = 0x10000
BF16, F32 = vie.VIE_DTYPE_BF16, vie.VIE_DTYPE_F32
INVALID, UNSUPPORTED = vie.VIE_ERR_INVALID_ARG, vie.VIE_ERR_UNSUPPORTED


def _call(fn, ok, **kw):
    return fn(*dict(ok, **kw).values())


ROWS = dict(logits=P, dtype=F32, n=4, V=100, ld=100, tokens=P, temperature=1.0)
TERMS = dict(ROWS, old_logprob=P, advantage=P, ref_logprob=P, clip_low=0.2, clip_high=0.2, kl_coef=0.1)
FORMS = {
    "vie_token_logprobs": dict(ROWS, out_logprob=P, out_stats=0),
    "vie_token_logprobs_grad": dict(ROWS, stats=P, grad_logprob=P, out_grad=P, ld_grad=100),
    "vie_policy_loss": dict(TERMS, out_loss=P, out_logprob=P, out_stats=0),
    "vie_policy_loss_grad": dict(TERMS, logprob=P, stats=P, grad_loss=P, out_grad=P, ld_grad=100),
    "vie_policy_loss_step": dict(TERMS, grad_loss=P, out_loss=P, out_logprob=P, out_stats=0, out_grad=P, ld_grad=100),
}
BAD = [dict(logits=0), dict(tokens=0), dict(n=-1), dict(n=vie.VIE_MANY_MAX + 1), dict(V=0), dict(V=2 ** 31 - 1),
       dict(ld=99), dict(ld=2 ** 60), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.inf),
       dict(temperature=math.nan), dict(logits=P + 2), dict(logits=P + 1, dtype=BF16), dict(tokens=P + 2)]
BAD_TERMS = [dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=math.nan), dict(clip_high=-0.1),
             dict(clip_high=math.inf), dict(clip_high=math.nan), dict(kl_coef=-0.1), dict(kl_coef=math.inf),
             dict(kl_coef=math.nan), dict(ref_logprob=0), dict(ref_logprob=P + 1)]


@pytest.mark.parametrize("name", FORMS)
def test_row_refusals(name):
    fn, ok = getattr(vie, name), FORMS[name]
    for bad in BAD + (BAD_TERMS if "kl_coef" in ok else []):
        assert _call(fn, ok, **bad) == INVALID, bad
        assert name in vie.vie_last_error()
    assert _call(fn, ok, dtype=2) == UNSUPPORTED
    for p in ("out_loss", "out_logprob", "logprob", "stats", "grad_loss", "grad_logprob", "out_grad", "old_logprob",
              "advantage"):
        if p in ok:
            assert _call(fn, ok, **{p: 0}) == INVALID, p
            assert _call(fn, ok, **{p: P + 2}) == INVALID, p
    if "out_stats" in ok:
        assert _call(fn, ok, out_stats=P + 2) == INVALID
    if "ld_grad" in ok:
        assert _call(fn, ok, ld_grad=99) == INVALID
    none = {p: 0 for p in ok if ok[p] == P}
    assert _call(fn, ok, n=0, **none) == vie.VIE_OK  # nothing to do: no buffer is looked at


@pytest.mark.parametrize("name", ["vie_policy_loss", "vie_policy_loss_step"])
def test_results_in_place_of_terms_are_refused(name):
    """Other CTAs of a row may still read them."""
    fn = getattr(vie, name)
    ok = dict(FORMS[name], out_loss=P + 16, out_logprob=P + 32, out_stats=P + 64)
    for out in ("out_loss", "out_logprob", "out_stats"):
        for term in ("old_logprob", "advantage", "ref_logprob"):
            bad = dict(ok, **{term: P + 128, out: P + 128})
            assert _call(fn, bad) == INVALID and "in place" in vie.vie_last_error()


PAIRS = dict(n=20, offsets=P, pairs=2, beta=0.1, label_smoothing=0.0)
PREFERENCE = {
    "vie_preference_loss": dict(dict(logprob=P, ref_logprob=P), **PAIRS, out_loss=P, out_margin=P),
    "vie_preference_loss_grad": dict(dict(margin=P), **PAIRS, grad_loss=P, out_grad=P),
    "vie_preference_loss_step": dict(dict(logprob=P, ref_logprob=0), **PAIRS, grad_loss=P, out_loss=P, out_margin=P,
                                     out_grad=P),
}


@pytest.mark.parametrize("name", PREFERENCE)
def test_preference_refusals(name):
    fn, ok = getattr(vie, name), PREFERENCE[name]
    for bad in (dict(n=-1), dict(n=vie.VIE_PREFERENCE_N_MAX + 1), dict(pairs=-1), dict(pairs=vie.VIE_MANY_MAX + 1),
                dict(offsets=0), dict(offsets=P + 2), dict(beta=math.inf), dict(beta=math.nan),
                dict(label_smoothing=-0.1), dict(label_smoothing=1.1), dict(label_smoothing=math.nan)):
        assert _call(fn, ok, **bad) == INVALID, bad
        assert name in vie.vie_last_error()
    for p in ("logprob", "margin", "grad_loss", "out_loss", "out_margin", "out_grad"):
        if p in ok:
            assert _call(fn, ok, **{p: 0}) == INVALID, p
            assert _call(fn, ok, **{p: P + 2}) == INVALID, p
    if "ref_logprob" in ok:
        assert _call(fn, ok, ref_logprob=P + 1) == INVALID


QUANTIZE = dict(x=P, dtype=BF16, n=4, d=50, ld=50, codes=P, scales=P, row_scales=P, values=P, values_dtype=F32,
                ld_values=50)
DEQUANTIZE = dict(codes=P, scales=P, row_scales=P, n=4, d=50, out=P, out_dtype=F32, ld_out=50)
LOGITS = dict(x_codes=P, x_scales=P, x_row_scales=P, n=4, w_codes=P, w_scales=P, w_row_scales=P, V=100, d=50, out=P,
              out_dtype=F32, ld_out=100)


W = P + 0x1000
BOTH = dict(x=P, dtype=F32, n=4, ld=50, x_codes=P, x_scales=P, x_row_scales=P, w_codes=W, w_scales=W, w_row_scales=W,
            V=100, d=50, out=P, out_dtype=F32, ld_out=100)


def test_e2m1_refusals():
    shape = [dict(n=-1), dict(n=vie.VIE_E2M1_N_MAX + 1), dict(d=0), dict(d=vie.VIE_D_MAX + 1)]
    parts = [dict(codes=0), dict(scales=0), dict(row_scales=0), dict(codes=P + 8), dict(scales=P + 4),
             dict(row_scales=P + 2)]
    for fn, ok, bads in (
            (vie.vie_e2m1_quantize, QUANTIZE, shape + parts + [dict(x=0), dict(x=P + 1), dict(ld=49),
                                                               dict(values=P + 2), dict(ld_values=49)]),
            (vie.vie_e2m1_dequantize, DEQUANTIZE, shape + parts + [dict(out=0), dict(out=P + 2), dict(ld_out=49)]),
            (vie.vie_e2m1_logits, LOGITS,
             [dict(n=-1), dict(n=vie.VIE_MANY_MAX + 1), dict(V=0), dict(V=vie.VIE_E2M1_N_MAX + 1), dict(d=0),
              dict(d=vie.VIE_D_MAX + 1), dict(out=0), dict(out=P + 2), dict(ld_out=99)]
             + [{p + k: v for k, v in b.items()} for p in ("x_", "w_") for b in parts]),
            (vie.vie_e2m1_quantize_logits, BOTH,
             [dict(n=-1), dict(n=vie.VIE_MANY_MAX + 1), dict(V=0), dict(V=vie.VIE_E2M1_N_MAX + 1), dict(d=0),
              dict(d=vie.VIE_D_MAX + 1), dict(out=0), dict(out=P + 2), dict(ld_out=99), dict(x=0), dict(x=P + 2),
              dict(ld=49)] + [{p + k: v for k, v in b.items()} for p in ("x_", "w_") for b in parts])):
        for bad in bads:
            assert _call(fn, ok, **bad) == INVALID, bad
            assert fn.__name__ in vie.vie_last_error()
    assert _call(vie.vie_e2m1_quantize_logits, BOTH, dtype=2) == UNSUPPORTED
    assert _call(vie.vie_e2m1_quantize, QUANTIZE, dtype=2) == UNSUPPORTED
    assert _call(vie.vie_e2m1_quantize, QUANTIZE, values_dtype=2) == UNSUPPORTED
    assert _call(vie.vie_e2m1_dequantize, DEQUANTIZE, out_dtype=5) == UNSUPPORTED
    assert _call(vie.vie_e2m1_logits, LOGITS, out_dtype=2) == UNSUPPORTED
    for fn, ok in ((vie.vie_e2m1_quantize, QUANTIZE), (vie.vie_e2m1_dequantize, DEQUANTIZE),
                   (vie.vie_e2m1_logits, LOGITS), (vie.vie_e2m1_quantize_logits, BOTH)):
        assert _call(fn, ok, n=0, **{p: 0 for p in ok if ok[p] in (P, W)}) == vie.VIE_OK


def test_results_in_place_of_inputs():
    """Where they may be, and with the layout that makes it safe."""
    for name in ("vie_token_logprobs_grad", "vie_policy_loss_grad", "vie_policy_loss_step"):
        apart = {r: W for r in ("out_loss", "out_logprob") if r in FORMS[name]}
        bad = dict(FORMS[name], **apart, logits=P + 64, out_grad=P + 64, ld_grad=104)
        assert _call(getattr(vie, name), bad) == INVALID and "pitch" in vie.vie_last_error()
    apart = dict(QUANTIZE, values=P + 64)
    for bad in (dict(x=P + 64, dtype=F32, ld_values=51), dict(x=P + 64)):  # (another pitch; another type)
        assert _call(vie.vie_e2m1_quantize, apart, **bad) == INVALID and "in place" in vie.vie_last_error()
    for part in ("codes", "scales", "row_scales"):
        assert _call(vie.vie_e2m1_quantize_logits, BOTH, **{"x_" + part: W}) == INVALID
        assert "in place" in vie.vie_last_error()


def test_e2m1_results_in_place_of_inputs_or_of_one_another():
    def apart(ok):
        return {k: P + 256 * i if v in (P, W) else v for i, (k, v) in enumerate(ok.items())}

    parts = ("codes", "scales", "row_scales")
    for fn, ok, pairs in (
            (vie.vie_e2m1_quantize, QUANTIZE, [(p, o) for p in ("x", "values") for o in parts]),
            (vie.vie_e2m1_dequantize, DEQUANTIZE, [("out", o) for o in parts]),
            (vie.vie_e2m1_logits, LOGITS, [("out", m + o) for m in ("x_", "w_") for o in parts]),
            (vie.vie_e2m1_quantize_logits, BOTH, [("out", m + o) for m in ("x_", "w_") for o in parts]
             + [("x", "x_" + o) for o in parts])):
        for a, b in pairs:
            assert _call(fn, apart(ok), **{a: W, b: W}) == INVALID, (a, b)
            assert "in place" in vie.vie_last_error() and fn.__name__ in vie.vie_last_error()


def test_policy_results_in_place_of_weights():
    ok = dict(FORMS["vie_policy_loss_step"], out_loss=P + 16, out_logprob=P + 32, out_stats=P + 64, grad_loss=W)
    for out in ("out_loss", "out_logprob", "out_stats"):
        assert _call(vie.vie_policy_loss_step, ok, **{out: W}) == INVALID and "in place" in vie.vie_last_error()


@pytest.mark.parametrize("name", PREFERENCE)
def test_preference_results_in_place_of_inputs(name):
    fn, args = getattr(vie, name), PREFERENCE[name]
    ok = {k: P + 16 * i if v == P else v for i, (k, v) in enumerate(args.items())}
    for out in (k for k in ok if k.startswith("out_")):
        for term in ("logprob", "ref_logprob", "margin", "grad_loss"):
            if term in ok:
                assert _call(fn, ok, **{out: W, term: W}) == INVALID and "in place" in vie.vie_last_error()


def test_e2m1_bytes():
    assert vie.load().vie_e2m1_bytes(4, 100, None, None) == INVALID
    for n, d in ((-1, 5), (5, 0), (5, vie.VIE_D_MAX + 1), (vie.VIE_E2M1_N_MAX + 1, 5)):
        assert vie.vie_e2m1_bytes(n, d)[0] == INVALID
    for n, d in ((0, 1), (1, 1), (128, 64), (129, 65), (262144, 1152), (vie.VIE_E2M1_N_MAX, vie.VIE_D_MAX)):
        assert vie.vie_e2m1_bytes(n, d) == (vie.VIE_OK, n * ((d + 31) // 32 * 16),
                                            (n + 127) // 128 * ((d + 63) // 64) * 512)
    q = vie.E2m1.empty(129, 65, device="cpu")
    assert (vie.VIE_OK, q.codes.numel(), q.scales.numel()) == vie.vie_e2m1_bytes(129, 65) and q.shape == (129, 65)


def test_the_reference_rounds_as_the_types_do():
    """The 64-bit definition's nearest values against torch's conversion to e4m3, and ties by hand."""
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    v = torch.cat([e4m3, (e4m3[1:] + e4m3[:-1]) / 2, torch.rand(1000).double() * 448])
    assert torch.equal(e4m3[ref._nearest(v, e4m3)], v.float().to(torch.float8_e4m3fn).double())
    y = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.2501]).double()
    assert ref.VALUES[ref._nearest(y, ref.VALUES[:8])].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 0.5]


def test_binding_refuses_cpu_tensors():
    z, t, f = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    o = torch.zeros(3, dtype=torch.int32)
    for call in (lambda: vie.token_logprobs(z, t), lambda: vie.token_logprobs_grad(z, t, torch.zeros(2, 2), f),
                 lambda: vie.policy_loss(z, t, f, f), lambda: vie.policy_loss_grad(z, t, f, f, f, torch.zeros(2, 2), f),
                 lambda: vie.policy_loss_step(z, t, f, f, f), lambda: vie.preference_loss(f, o),
                 lambda: vie.preference_loss_grad(f, o, f, 2), lambda: vie.preference_loss_step(f, o, f),
                 lambda: vie.e2m1_quantize(z), lambda: vie.e2m1_dequantize(vie.E2m1.empty(2, 8, device="cpu")),
                 lambda: vie.e2m1_logits(z, vie.E2m1.empty(2, 8, device="cpu"))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_binding_refuses_room_for_states_that_are_quantised_already():
    q, room, w = (vie.E2m1.empty(n, 8, device="cpu") for n in (2, 2, 5))
    with pytest.raises(ValueError, match="x_quantized"):
        vie.e2m1_logits(q, w, x_quantized=room)
    for same in (None, q):  # (as far as the next check)
        with pytest.raises(ValueError, match="CUDA"):
            vie.e2m1_logits(q, w, x_quantized=same)


class _Tensor:
    """A tensor of device 0, as far as the binding asks before it launches."""
    is_cuda, dtype = True, torch.float32

    def get_device(self):
        return 0


class _Stream:
    def __init__(self, index):
        self.device, self.cuda_stream = torch.device("cuda", index), 0


def test_binding_refuses_a_stream_of_another_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x = y = _Tensor()
    q = vie.E2m1(x, x, x, 8)
    for call in (lambda s: vie.token_logprobs(x, y, stream=s), lambda s: vie.token_logprobs_grad(x, y, y, y, stream=s),
                 lambda s: vie.policy_loss(x, y, y, y, stream=s),
                 lambda s: vie.policy_loss_grad(x, y, y, y, y, y, y, stream=s),
                 lambda s: vie.policy_loss_step(x, y, y, y, y, stream=s), lambda s: vie.preference_loss(x, y, stream=s),
                 lambda s: vie.preference_loss_grad(x, y, y, 5, stream=s),
                 lambda s: vie.preference_loss_step(x, y, y, stream=s), lambda s: vie.e2m1_quantize(x, stream=s),
                 lambda s: vie.e2m1_dequantize(q, stream=s), lambda s: vie.e2m1_logits(x, q, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call(_Stream(1))


def test_limits_match_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "vie_head.h")).read()
    assert re.search(r"#define\s+VIE_PREFERENCE_N_MAX\s+\(1 << 30\)", text) and vie.VIE_PREFERENCE_N_MAX == 1 << 30
    assert re.search(r"#define\s+VIE_E2M1_N_MAX\s+\(1 << 28\)", text) and vie.VIE_E2M1_N_MAX == 1 << 28
