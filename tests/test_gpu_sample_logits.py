"""GPU parity of sampling from full logits (vie_sample_logits): every draw must
be one that the definition in 64 bits allows (tests/student_ref.py), and where
the weights are exact (equal logits) it must be that very token."""
import math

import numpy as np
import pytest
import torch

import student_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _settings(b, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda: torch.rand(b, generator=g)  # noqa: E731
    T = torch.where(r() < 0.1, torch.zeros(b), 0.3 + 1.5 * r())
    k = torch.where(r() < 0.4, torch.zeros(b), 1 + 120 * r()).int()
    p = torch.where(r() < 0.3, torch.ones(b), 0.05 + 0.95 * r())
    m = torch.where(r() < 0.5, torch.zeros(b), 0.2 * r())
    return r(), T, k, p, m


def _check(vie, z, u, T, k, p, m, zc=None):
    zc = z.cuda() if zc is None else zc
    tok, prob = vie.sample_logits(zc, u.cuda(), *(x.cuda() for x in (T, k, p, m)))
    tok, prob = tok.cpu().tolist(), prob.cpu().tolist()
    zn = z.float().numpy()
    for r in range(z.shape[0]):
        d = ref.Draw(zn[r], float(T[r]))
        bad = d.problems(float(T[r]), int(k[r]), float(p[r]), float(m[r]), float(u[r]), tok[r], prob[r])
        assert not bad, (r, float(T[r]), int(k[r]), float(p[r]), float(m[r]), float(u[r]), bad)
    assert vie.vie_device_status() == vie.VIE_OK
    return tok, prob


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,V,spread", [
    (1, 1, 1.0), (5, 2, 1.0), (9, 33, 2.0), (40, 1000, 2.0), (3, 4096, 0.1), (33, 20011, 2.5), (4, 65537, 1.0),
    (6, 151936, 2.5), (3, 262144, 0.01), (2, 262143, 4.0), (300, 257, 1.5), (2, 1000003, 2.0),
])
def test_draws_match_the_definition(vie, dtype, b, V, spread):
    g = torch.Generator().manual_seed(V)
    z = (spread * torch.randn(b, V, generator=g)).to(DT[dtype])
    _check(vie, z, *_settings(b, seed=b + V))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_logits(vie, dtype):
    low = torch.finfo(DT[dtype]).min
    z = (2 * torch.randn(12, 3000, generator=torch.Generator().manual_seed(1))).to(DT[dtype])
    z[0] = -math.inf                  # nothing to draw
    z[1] = float("nan")
    z[2, 1:] = -math.inf              # one token
    z[3, :2999] = -math.inf
    z[4] = low                        # equal, though the lowest of the type
    z[5, ::2] = -math.inf
    z[6, 10:] = low
    z[7, 5] = float("nan")            # NaN is never drawn
    z[8, 50:60] = float("inf")        # share the whole mass
    z[9] = float("inf")
    z[10, ::3] = low
    zr = z.clone()
    zr[torch.isnan(zr)] = -math.inf
    for seed in range(4):
        u, T, k, p, m = _settings(12, seed)
        tok, prob = vie.sample_logits(z.cuda(), u.cuda(), *(x.cuda() for x in (T, k, p, m)))
        assert tok[:2].tolist() == [-1, -1] and prob[:2].tolist() == [0.0, 0.0]
        assert tok[2] == 0 and tok[3] == 2999 and prob[2] == 1 and prob[3] == 1
        assert 50 <= int(tok[8]) < 60
        want, _ = _check(vie, zr, u, T, k, p, m)
        assert tok.tolist() == want


@pytest.mark.parametrize("V", [1, 31, 1000, 65536, 262144])
def test_equal_logits_draw_by_index(vie, V):
    """Equal weights are exact, and so is the draw: token floor(floor(u 2^24) n / 2^24)
    of the n that are kept, whatever the split of the row."""
    b = 64
    g = torch.Generator().manual_seed(V)
    u = torch.rand(b, generator=g)
    u[0], u[1], u[2], u[3] = 0.0, 1.0 - 2.0 ** -24, 1.0, -0.5
    k = torch.randint(0, V + 2, (b,), generator=g).int()
    p = torch.where(torch.rand(b, generator=g) < 0.5, torch.ones(b), torch.rand(b, generator=g))
    z = torch.full((b, V), -1.25)
    tok, prob = vie.sample_logits(z.cuda(), u.cuda(), top_k=k.cuda(), top_p=p.cuda())
    for r in range(b):
        n = V if not 0 < k[r] < V else int(k[r])
        if p[r] < 1:
            p24 = math.ceil(float(p[r]) * 2 ** 24)
            n = max(1, -(-(-(-(n << 40) * p24 // 2 ** 24)) // 2 ** 40))
        u24 = min(max(int(float(u[r]) * 2 ** 24), 0), 2 ** 24 - 1)
        assert int(tok[r]) == (((n << 40) * u24) >> 24) >> 40, (r, n, float(u[r]))
        assert float(prob[r]) == pytest.approx(1.0 / n, rel=4 * ref.U)


def test_ties_rank_by_index_and_zeros_are_equal(vie):
    z = torch.full((1, 4000), -50.0)
    at = [3999, 17, 2048, 900, 901]
    z[0, at] = 0.0
    z[0, [17, 901]] = -0.0
    order = sorted(at)
    for j, uu in enumerate((0.1, 0.3, 0.5, 0.7, 0.9)):
        tok, prob = vie.sample_logits(z.cuda(), torch.tensor([uu]).cuda())
        assert int(tok) == order[j] and float(prob) == pytest.approx(0.2, rel=1e-6)
    for k in range(1, 6):  # top-k cuts through the ties by index
        tok, _ = vie.sample_logits(z.cuda(), torch.tensor([0.9999]).cuda(), top_k=torch.tensor([k]).int().cuda())
        assert int(tok) == order[k - 1]


def test_greedy_rows(vie):
    z = torch.randn(8, 5000, generator=torch.Generator().manual_seed(3))
    z[4, 100] = z[4, 50] = 9.0
    T = torch.tensor([0.0, -1.0, float("nan"), 1e-38, 0.0, 1e-42, 0.0, 1e-6])
    u = torch.full((8,), 0.999)
    tok, prob = vie.sample_logits(z.cuda(), u.cuda(), temperature=T.cuda())
    want = z.argmax(1)
    want[4] = 50
    assert tok.cpu().tolist() == want.tolist() and prob.cpu().tolist() == [1.0] * 8


def test_infinite_temperature_is_uniform(vie):
    z = torch.randn(4, 1000, generator=torch.Generator().manual_seed(4))
    z[:, ::2] = -math.inf
    _check(vie, z, torch.rand(4), torch.full((4,), math.inf), torch.zeros(4).int(), torch.ones(4), torch.zeros(4))
    prob = vie.sample_logits(z.cuda(), torch.rand(4).cuda(), temperature=torch.full((4,), math.inf).cuda())[1]
    assert (prob == 1.0 / 500).all()


def test_filters_at_their_limits(vie):
    b, V = 9, 2000
    z = torch.randn(b, V, generator=torch.Generator().manual_seed(5))
    u = torch.full((b,), 0.99999)
    T = torch.ones(b)
    off = torch.zeros(b)
    k = torch.tensor([-5, 0, 1, 2, V - 1, V, V + 1, 2 ** 31 - 1, 3]).int()
    _check(vie, z, u, T, k, torch.ones(b), off)
    p = torch.tensor([0.0, -1.0, 1e-30, 2.0 ** -24, 0.5, 1.0, 2.0, float("inf"), 1 - 2.0 ** -24])
    tok, _ = _check(vie, z, u, T, off.int(), p, off)
    assert tok[:4] == z.argmax(1)[:4].tolist()
    m = torch.tensor([0.0, -1.0, 1e-30, 1.0, 2.0, float("inf"), 0.5, 1e-8, 0.999])
    tok, prob = _check(vie, z, u, T, off.int(), torch.ones(b), m)
    assert tok[3:6] == z.argmax(1)[3:6].tolist() and prob[3:6] == [1.0] * 3
    nan = torch.full((b,), float("nan"))  # a filter that is not a number is off
    assert [x.tolist() for x in vie.sample_logits(z.cuda(), u.cuda(), top_p=nan.cuda(), min_p=nan.cuda())] == \
        [x.tolist() for x in vie.sample_logits(z.cuda(), u.cuda())]
    assert vie.sample_logits(z.cuda(), nan.cuda())[0].tolist() == z.argmax(1).tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,ld,off", [(999, 999, 0), (1000, 1001, 1), (33000, 33003, 3), (40000, 40008, 5)])
def test_strides_and_alignment(vie, dtype, V, ld, off):
    b = 7
    z = (2 * torch.randn(b, V, generator=torch.Generator().manual_seed(6))).to(DT[dtype])
    buf = torch.full((b * ld + off + 8,), float("inf"), dtype=DT[dtype], device="cuda")
    zc = buf[off:off + b * ld].view(b, ld)[:, :V]
    zc.copy_(z)
    s = _settings(b, 8)
    got = _check(vie, z, *s, zc=zc)
    assert got == _check(vie, z, *s)
    assert got == _check(vie, z, *s, zc=z.t().contiguous().cuda().t())
    if dtype == "bf16":  # the same values in fp32: the same draws
        assert got == _check(vie, z.float(), *s)


def test_frequencies_follow_the_distribution(vie):
    V, b = 50, 4000
    z = torch.randn(V, generator=torch.Generator().manual_seed(7))
    u = (torch.arange(b) + 0.5) / b  # evenly spread: counts are within one of b p
    tok, _ = vie.sample_logits(z.expand(b, V).contiguous().cuda(), u.cuda(), temperature=torch.full((b,), 0.8).cuda())
    p = torch.softmax(z.double() / 0.8, 0)
    assert (torch.bincount(tok.cpu().long(), minlength=V).double() - b * p).abs().max() <= 1.01


def test_sparse_logits_of_the_head(vie):
    """The head's sparse tensor (-inf but k logits), drawn from directly."""
    from gpu_cases import to_device_bits, workload
    V, d, b, k = 30011, 256, 6, 50
    W, h = workload(V, d, b, seed=19)
    with vie.Head(to_device_bits(W)) as head:
        idx, val, sp = head.topk_sparse(torch.from_numpy(h).cuda(), k)
        u, T, tk, p, m = _settings(b, 10)
        tok, _ = _check(vie, sp.cpu(), u, T, tk, p, m)
        for r in range(b):
            assert tok[r] in idx[r].tolist()


def test_stream_graph_defaults_and_no_rows(vie):
    z = torch.randn(5, 30000, device="cuda")
    u = torch.rand(5, device="cuda")
    want = vie.sample_logits(z, u)
    one, zero = torch.ones(5, device="cuda"), torch.zeros(5, device="cuda")
    same = vie.sample_logits(z, u, one, zero.int(), one, zero)
    assert torch.equal(same[0], want[0]) and torch.equal(same[1], want[1])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = vie.sample_logits(z, u, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    tok, prob = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        vie.sample_logits(z, u, out_token=tok, out_prob=prob)
    for _ in range(2):
        tok.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tok, want[0]) and torch.equal(prob, want[1])
    assert vie.sample_logits(z[:0], u[:0])[0].shape == (0,)
    for bad in (lambda: vie.sample_logits(z.half(), u), lambda: vie.sample_logits(z, u[:4]),
                lambda: vie.sample_logits(z, u.double()), lambda: vie.sample_logits(z, u, top_k=one),
                lambda: vie.sample_logits(z, u, temperature=one[:4]), lambda: vie.sample_logits(z[0], u),
                lambda: vie.sample_logits(z, u, out_token=torch.empty(5, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            bad()


def test_offsets_beyond_32_bits(vie):
    V = 262144
    n = 2 ** 31 // V + 2
    big = torch.zeros((n, V), dtype=torch.bfloat16, device="cuda")
    z = torch.randn(2, V, device="cuda").bfloat16()
    big[-2:] = z
    u = torch.rand(n, device="cuda")
    got = vie.sample_logits(big, u)[0]
    assert torch.equal(got[-2:], vie.sample_logits(z, u[-2:].contiguous())[0])
    np.testing.assert_array_equal(got[:-2].cpu().numpy(), ((u[:-2].double() * 2 ** 24).long() * V >> 24).cpu().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,V,spread", [(6, 60000, 2.0), (3, 262144, 0.05), (4, 262144, 3.0), (700, 3000, 1.0)])
def test_large_top_k(vie, dtype, b, V, spread):
    """More tokens than are ranked at once, and than there are threads."""
    g = torch.Generator().manual_seed(V + b)
    z = (spread * torch.randn(b, V, generator=g)).to(DT[dtype])
    u, T, k, p, m = _settings(b, seed=b)
    k = (V * torch.rand(b, generator=g) ** 3).int() + 1
    _check(vie, z, u, torch.where(T > 0, T, torch.ones(b)), k, p, m)


def test_the_split_of_a_row_does_not_matter(vie):
    """The same row alone, among few and among many others: the same draw."""
    V = 100000
    z = 2.0 * torch.randn(1, V, generator=torch.Generator().manual_seed(9)).cuda()
    for top_k, top_p, min_p in ((0, 0.9, 0.0), (40, 1.0, 0.0), (0, 1.0, 0.02), (20000, 0.7, 0.0), (0, 0.9, 0.001)):
        got = set()
        for b in (1, 5, 40, 300, 800):
            row = lambda x, dt=torch.float32: torch.full((b,), x, dtype=dt, device="cuda")  # noqa: E731
            tok, prob = vie.sample_logits(z.expand(b, V).contiguous(), row(0.37), row(0.9), row(top_k, torch.int32),
                                          row(top_p), row(min_p))
            got |= set(zip(tok.tolist(), prob.tolist()))
        assert len(got) == 1, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_batches_of_rows_that_differ_in_work(vie, dtype):
    """Rows without a top-k go first in large batches: the draws are those of small ones."""
    b, V = 1100, 3001
    z = (2 * torch.randn(b, V, generator=torch.Generator().manual_seed(12))).to(DT[dtype]).cuda()
    u, T, k, p, m = (x.cuda() for x in _settings(b, 13))
    tok, prob = vie.sample_logits(z, u, T, k, p, m)
    for lo in range(0, b, 50):
        rows = slice(lo, min(lo + 50, b))
        one = vie.sample_logits(z[rows], u[rows], T[rows], k[rows], p[rows], m[rows])
        assert torch.equal(tok[rows], one[0]) and torch.equal(prob[rows], one[1])
    no_k = vie.sample_logits(z, u, T, None, p, m)
    zero = vie.sample_logits(z, u, T, torch.zeros_like(k), p, m)
    assert torch.equal(no_k[0], zero[0]) and torch.equal(no_k[1], zero[1])


@pytest.mark.parametrize("V,step", [(5000, 0.0), (5000, 1e-6), (20000, 1e-7), (3000, 0.01)])
def test_many_candidates_that_differ_little(vie, V, step):
    """Hundreds to thousands of tokens of one bin: few keys, each of many tokens or of one."""
    b = 24
    z = -step * torch.randint(0, 40, (b, V), generator=torch.Generator().manual_seed(V)).float()
    _check(vie, z, *_settings(b, 14))
    _check(vie, z.bfloat16(), *_settings(b, 15))
