"""Host-side argument checks of the training and sampling calls: status codes
and messages before any CUDA call, and what the torch binding refuses."""
import pytest
import torch

import paper_2608_27460_gb300 as vie

P = 0x10000
BF16, F32 = vie.VIE_DTYPE_BF16, vie.VIE_DTYPE_F32
INVALID, UNSUPPORTED = vie.VIE_ERR_INVALID_ARG, vie.VIE_ERR_UNSUPPORTED


def _call(fn, ok, **kw):
    a = dict(ok)
    a.update(kw)
    return fn(*a.values())


DISTILL = dict(logits=P, dtype=F32, n=4, V=100, ld=100, t_idx=P, t_logits=P, k=5, temperature=1.0)
FORMS = {
    "vie_distill_topk": dict(DISTILL, out_loss=P, out_stats=0),
    "vie_distill_topk_grad": dict(DISTILL, stats=P, grad_loss=P, out_grad=P, ld_grad=100),
    "vie_distill_topk_step": dict(DISTILL, grad_loss=P, out_loss=P, out_stats=0, out_grad=P, ld_grad=100),
}
BAD = [dict(logits=0), dict(t_idx=0), dict(t_logits=0), dict(n=-1), dict(n=vie.VIE_MANY_MAX + 1), dict(V=0),
       dict(V=2 ** 31 - 1), dict(ld=99), dict(k=0), dict(k=vie.VIE_K_MAX + 1), dict(temperature=0.0),
       dict(temperature=-1.0), dict(temperature=float("inf")), dict(temperature=float("nan")), dict(logits=P + 2),
       dict(logits=P + 1, dtype=BF16), dict(t_idx=P + 2), dict(t_logits=P + 2), dict(ld=2 ** 60)]


@pytest.mark.parametrize("name", FORMS)
def test_distill_refusals(name):
    fn, ok = getattr(vie, name), FORMS[name]
    for bad in BAD:
        assert _call(fn, ok, **bad) == INVALID, bad
        assert name in vie.vie_last_error()
    assert _call(fn, ok, dtype=2) == UNSUPPORTED
    for p in ("out_loss", "stats", "grad_loss", "out_grad"):
        if p in ok:
            assert _call(fn, ok, **{p: 0}) == INVALID, p
            assert _call(fn, ok, **{p: P + 2}) == INVALID, p
    if "out_stats" in ok:
        assert _call(fn, ok, out_stats=P + 2) == INVALID
    if "ld_grad" in ok:
        assert _call(fn, ok, ld_grad=99) == INVALID
    # nothing to do: no buffer is looked at
    none = {p: 0 for p in ok if ok[p] == P}
    assert _call(fn, ok, n=0, **none) == vie.VIE_OK


EMBED = dict(table=P, dtype=BF16, V=100, d=16, ld=16, tokens=P, n=4, scale=1.0, out=P, out_dtype=F32, ld_out=16)


def test_embed_refusals():
    for bad in [dict(table=0), dict(tokens=0), dict(out=0), dict(V=0), dict(V=2 ** 31 - 1), dict(d=0),
                dict(d=vie.VIE_D_MAX + 1), dict(ld=15), dict(ld_out=15), dict(n=-1), dict(n=vie.VIE_MANY_MAX + 1),
                dict(tokens=P + 2), dict(table=P + 1), dict(out=P + 2)]:
        assert _call(vie.vie_embed, EMBED, **bad) == INVALID, bad
        assert "vie_embed" in vie.vie_last_error()
    assert _call(vie.vie_embed, EMBED, dtype=2) == UNSUPPORTED
    assert _call(vie.vie_embed, EMBED, out_dtype=7) == UNSUPPORTED
    assert _call(vie.vie_embed, EMBED, n=0, tokens=0, out=0) == vie.VIE_OK


GRAD = dict(tokens=P, n=4, grad=P, dtype=BF16, ld_grad=16, scale=1.0, V=100, d=16, out=P, out_dtype=F32, ld=16,
            accumulate=1, workspace=P, workspace_bytes=1 << 20)


def test_embed_grad_refusals():
    for bad in [dict(tokens=0), dict(grad=0), dict(out=0), dict(V=0), dict(d=0), dict(d=vie.VIE_D_MAX + 1),
                dict(ld=15), dict(ld_grad=15), dict(n=-1), dict(n=vie.VIE_MANY_MAX + 1), dict(tokens=P + 2),
                dict(grad=P + 1), dict(out=P + 2), dict(workspace=0), dict(workspace=P + 8),
                dict(workspace_bytes=vie.vie_embed_grad_workspace(4, 100, 16)[1] - 1)]:
        assert _call(vie.vie_embed_grad, GRAD, **bad) == INVALID, bad
        assert "vie_embed_grad" in vie.vie_last_error()
    assert _call(vie.vie_embed_grad, GRAD, dtype=2) == UNSUPPORTED
    assert _call(vie.vie_embed_grad, GRAD, out_dtype=2) == UNSUPPORTED
    assert _call(vie.vie_embed_grad, GRAD, n=0, tokens=0, grad=0, workspace=0, workspace_bytes=0) == vie.VIE_OK


def test_embed_grad_workspace():
    assert vie.load().vie_embed_grad_workspace(4, 100, 16, None) == INVALID
    assert vie.vie_embed_grad_workspace(-1, 100, 16)[0] == INVALID
    assert vie.vie_embed_grad_workspace(4, 0, 16)[0] == INVALID
    assert vie.vie_embed_grad_workspace(4, 100, 0)[0] == INVALID
    last = 0
    for n in (0, 1, 31, 1000, 65536, 65537, vie.VIE_MANY_MAX):  # no call that needs more for fewer tokens
        st, need = vie.vie_embed_grad_workspace(n, 262144, 1024)
        assert st == vie.VIE_OK and need >= last
        last = need


SAMPLE = dict(logits=P, dtype=F32, batch=2, V=100, ld=100, u=P, temperature=0, top_k=0, top_p=0, min_p=0, out_token=P,
              out_prob=P)


def test_sample_logits_refusals():
    for bad in [dict(logits=0), dict(u=0), dict(out_token=0), dict(out_prob=0), dict(batch=-1),
                dict(batch=vie.VIE_MANY_MAX + 1), dict(V=0), dict(V=vie.VIE_SAMPLE_V_MAX + 1, ld=2 ** 23), dict(ld=99),
                dict(logits=P + 2), dict(u=P + 1), dict(temperature=P + 1), dict(top_k=P + 2), dict(top_p=P + 2),
                dict(min_p=P + 2), dict(out_token=P + 2), dict(out_prob=P + 2)]:
        assert _call(vie.vie_sample_logits, SAMPLE, **bad) == INVALID, bad
        assert "vie_sample_logits" in vie.vie_last_error()
    assert _call(vie.vie_sample_logits, SAMPLE, dtype=3) == UNSUPPORTED
    assert _call(vie.vie_sample_logits, SAMPLE, batch=0, logits=0, u=0, out_token=0, out_prob=0) == vie.VIE_OK


def test_binding_refuses_cpu_tensors():
    z, i, t = torch.zeros(2, 8), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    with pytest.raises(ValueError, match="logits"):
        vie.distill_topk(z, i, t)
    with pytest.raises(ValueError, match="logits"):
        vie.distill_topk_grad(z, i, t, torch.zeros(2, 2), torch.zeros(2))
    with pytest.raises(ValueError, match="logits"):
        vie.distill_topk_step(z, i, t, torch.zeros(2))
    with pytest.raises(ValueError, match="table"):
        vie.embed(z, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="grad"):
        vie.embed_grad(torch.zeros(2, dtype=torch.int32), z, 10)
    with pytest.raises(ValueError, match="logits"):
        vie.sample_logits(z, torch.zeros(2))


def test_limits_and_types_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "vie_head.h")).read()
    assert re.search(r"#define\s+VIE_SAMPLE_V_MAX\s+\(1 << 22\)", text) and vie.VIE_SAMPLE_V_MAX == 1 << 22
    assert re.search(r"VIE_DTYPE_F32\s*=\s*1", text) and vie.VIE_DTYPE_F32 == 1


class _Tensor:
    """A tensor of device 0, as far as the binding asks before it launches."""
    is_cuda, dtype = True, torch.float32

    def get_device(self):
        return 0


class _Stream:
    def __init__(self, index):
        self.device, self.cuda_stream = torch.device("cuda", index), 0


def test_binding_refuses_a_stream_of_another_device(monkeypatch):
    """Not to run on a stream that the caller has not named."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x, y = _Tensor(), _Tensor()
    for call in (lambda s: vie.distill_topk(x, y, y, stream=s), lambda s: vie.distill_topk_grad(x, y, y, y, y, stream=s),
                 lambda s: vie.distill_topk_step(x, y, y, y, stream=s), lambda s: vie.embed(x, y, stream=s),
                 lambda s: vie.embed_grad(y, x, 10, stream=s), lambda s: vie.sample_logits(x, y, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call(_Stream(1))


def test_embed_grad_workspace_where_the_sort_changes():
    """From 131073 tokens on the whole array is sorted, with counters of its own:
    no workspace there is smaller than one for fewer tokens."""
    for V, d in ((262144, 1), (262144, 1024), (2 ** 31 - 2, vie.VIE_D_MAX)):
        need = [vie.vie_embed_grad_workspace(n, V, d) for n in range(131000, 131200)]
        assert all(st == vie.VIE_OK for st, _ in need)
        sizes = [b for _, b in need]
        assert sizes == sorted(sizes) and sizes[73] > sizes[72]  # 131073 and 131072
