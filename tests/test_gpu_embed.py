"""GPU parity of the embedding lookup and its gradient (vie_embed,
vie_embed_grad) against their definitions in 64 bits."""
import math

import pytest
import torch

import student_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tokens(n, V, seed, kind="skewed"):
    g = torch.Generator().manual_seed(seed)
    if kind == "skewed":
        tok = (torch.exp(torch.rand(n, generator=g).double() * math.log(V + 1.0)).long() - 1).clamp(0, V - 1)
    elif kind == "one":
        tok = torch.full((n,), V - 1)
    elif kind == "two":
        tok = torch.randint(0, 2, (n,), generator=g) * (V - 1)
    elif kind == "distinct":
        tok = torch.randperm(max(n, V), generator=g)[:n] % V
    else:
        tok = torch.randint(0, V, (n,), generator=g)
    tok = tok.int()
    if kind == "skewed":
        tok[torch.rand(n, generator=g) < 0.1] = -1
    return tok


@pytest.mark.parametrize("a", ["bf16", "f32"])
@pytest.mark.parametrize("b", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,d,scale", [
    (1, 1, 1, 1.0), (3, 5, 7, 2.5), (33, 1000, 64, 8.0), (257, 20011, 640, math.sqrt(640)), (32, 5000, 1152, 1.0),
    (100, 300, 1001, -0.3), (5, 40, 16384, 1.0), (2000, 100, 72, 1.0),
])
def test_lookup(vie, a, b, n, V, d, scale):
    g = torch.Generator().manual_seed(n + d)
    table = torch.randn(V, d, generator=g).to(DT[a])
    tok = _tokens(n, V, seed=d)
    out = vie.embed(table.cuda(), tok.cuda(), scale=scale, out_dtype=DT[b])
    assert out.dtype == DT[b] and tuple(out.shape) == (n, d)
    s32 = float(torch.tensor(scale, dtype=torch.float32))
    want = table.double()[tok.long().clamp(0)] * s32
    want[tok < 0] = 0
    # one fp32 product, one rounding to the output's type
    assert ((out.double().cpu() - want).abs() <= (ref.U + ref.out_round(DT[b])) * want.abs()).all()
    assert vie.vie_device_status() == vie.VIE_OK


def test_lookup_keeps_bits_without_a_scale(vie):
    table = torch.randn(300, 130, device="cuda").bfloat16()
    table[7, 3], table[7, 4], table[7, 5] = float("inf"), float("nan"), -0.0
    tok = torch.tensor([7, 0, 299, 7], dtype=torch.int32, device="cuda")
    assert torch.equal(vie.embed(table, tok).view(torch.int16), table[tok.long()].view(torch.int16))


def test_tokens_out_of_range(vie):
    table = torch.randn(50, 40, device="cuda")
    table[0] = float("nan")  # nothing of the table may leak into an empty slot
    tok = torch.tensor([-1, 3, -2 ** 31, 49], dtype=torch.int32, device="cuda")
    out = vie.embed(table, tok)
    assert not out[0].any() and not out[2].any() and torch.equal(out[1], table[3]) and torch.equal(out[3], table[49])
    assert vie.vie_device_status() == vie.VIE_OK  # negative: an empty slot
    for bad in (50, 2 ** 31 - 1):
        tok[0] = bad
        out = vie.embed(table, tok)
        assert not out[0].any() and torch.equal(out[1], table[3])
        assert vie.vie_device_status() == vie.VIE_ERR_DEVICE and "token" in vie.vie_last_error()
        assert vie.vie_device_status() == vie.VIE_OK
        g = vie.embed_grad(tok, torch.ones(4, 40, device="cuda"), 50)
        assert (g[3] == 1).all() and (g[49] == 1).all() and float(g.sum()) == 80
        assert vie.vie_device_status() == vie.VIE_ERR_DEVICE
        assert vie.vie_device_status() == vie.VIE_OK


def _check_grad(vie, tok, grad, V, scale, out_dtype, base=None, out=None, workspace=None):
    s32 = float(torch.tensor(scale, dtype=torch.float32))
    tc, gc = tok.cuda(), grad.cuda()
    want, mag, count = ref.embed_grad(tc, gc, V, s32, base)
    if out is None:
        out = base.clone() if base is not None else None
    got = vie.embed_grad(tc, gc, V, scale=scale, out=out, accumulate=base is not None, out_dtype=out_dtype,
                         workspace=workspace)
    assert got.dtype == out_dtype
    # a token's sum of c rows: c - 1 additions, the scale, the addition to what was there; one rounding to the type
    tol = (count.double()[:, None] + 2) * ref.U * mag + (2 * ref.U + ref.out_round(out_dtype)) * want.abs()
    err = (got.double() - want).abs()
    assert (err <= tol).all(), (float(err.max()), (err > tol).nonzero()[:4].tolist())
    untouched = count == 0
    if base is not None:
        assert torch.equal(got[untouched], base[untouched])
    else:
        assert not got[untouched].any()
    again = vie.embed_grad(tc, gc, V, scale=scale, out=base.clone() if base is not None else None,
                           accumulate=base is not None, out_dtype=out_dtype)
    assert torch.equal(again, got)  # the same bits
    assert vie.vie_device_status() == vie.VIE_OK


@pytest.mark.parametrize("a", ["bf16", "f32"])
@pytest.mark.parametrize("b", ["bf16", "f32"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("n,V,d", [(1, 1, 1), (1, 100, 64), (2, 1, 9), (31, 7, 33), (32, 300, 640), (1000, 256, 257),
                                   (2049, 20011, 640), (5000, 65536, 100), (9000, 151936, 1024), (300, 50, 4100)])
def test_gradient(vie, a, b, add, n, V, d):
    g = torch.Generator().manual_seed(n + d)
    grad = torch.randn(n, d, generator=g).to(DT[a])
    base = torch.randn(V, d, generator=g).to(DT[b]).cuda() if add else None
    _check_grad(vie, _tokens(n, V, seed=n), grad, V, 1.7 if add else 1.0, DT[b], base)


@pytest.mark.parametrize("kind", ["one", "two", "distinct", "uniform"])
@pytest.mark.parametrize("n,V", [(777, 1000), (4096, 8192), (20000, 262144), (70001, 3000), (140000, 262144)])
def test_gradient_distributions(vie, kind, n, V):
    g = torch.Generator().manual_seed(n)
    grad = torch.randn(n, 96, generator=g)
    _check_grad(vie, _tokens(n, V, seed=n, kind=kind), grad, V, 1.0, torch.float32)


def test_gradient_all_slots_empty(vie):
    tok = torch.full((500,), -1, dtype=torch.int32, device="cuda")
    grad = torch.full((500, 24), float("nan"), device="cuda")
    assert not vie.embed_grad(tok, grad, 100).any()
    base = torch.randn(100, 24, device="cuda")
    assert torch.equal(vie.embed_grad(tok, grad, 100, out=base.clone(), accumulate=True), base)


def test_gradient_large_vocabulary_ids(vie):
    """Ids of more than 24 bits take a fourth sorting pass."""
    V, n = 2 ** 24 + 5, 3000
    tok = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(1)).int()
    tok[::7] = V - 1
    tok[3] = 0
    _check_grad(vie, tok, torch.randn(n, 4), V, 1.0, torch.float32)


@pytest.mark.parametrize("a,b", [("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("d,pad,off", [(64, 0, 1), (64, 8, 0), (100, 3, 2), (130, 2, 0), (513, 7, 5)])
def test_strides_and_alignment(vie, a, b, d, pad, off):
    n, V, ld = 300, 200, d + pad
    tok = _tokens(n, V, seed=d)
    buf = torch.randn(n * ld + off, device="cuda").to(DT[a])
    grad = buf[off:off + n * ld].view(n, ld)[:, :d]
    o = torch.full((V * ld + off + 8,), 7.0, device="cuda").to(DT[b])
    out = o[off:off + V * ld].view(V, ld)[:, :d]
    _check_grad(vie, tok, grad, V, 1.0, DT[b], out=out)
    rows = torch.full((n * ld + off + 8,), 7.0, device="cuda").to(DT[a])
    dst = rows[off:off + n * ld].view(n, ld)[:, :d]
    got = vie.embed(out, tok.cuda(), out=dst)
    want = out.double()[tok.long().clamp(0).cuda()] * (tok >= 0).cuda()[:, None]
    assert ((got.double() - want).abs() <= (ref.U + ref.out_round(DT[a])) * want.abs()).all()
    for t, v in ((o, out), (rows, dst)):  # nothing outside the rows is written
        v.fill_(7.0)
        assert (t == 7.0).all()


def test_lookup_and_gradient_are_adjoint(vie):
    """<embed(W), G> = <W, embed_grad(G)>, exactly: small whole numbers."""
    g = torch.Generator().manual_seed(9)
    W = torch.randint(-3, 4, (500, 80), generator=g).float().cuda()
    G = torch.randint(-3, 4, (4000, 80), generator=g).float().cuda()
    tok = _tokens(4000, 500, seed=2).cuda()
    left = (vie.embed(W, tok, scale=2.0).double() * G.double()).sum()
    right = (W.double() * vie.embed_grad(tok, G, 500, scale=2.0).double()).sum()
    assert float(left) == float(right)


def test_workspace_streams_and_graph(vie):
    n, V, d = 5000, 3000, 128
    tok, grad = _tokens(n, V, seed=4).cuda(), torch.randn(n, d, device="cuda")
    want = vie.embed_grad(tok, grad, V)
    need = vie.vie_embed_grad_workspace(n, V, d)[1]
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    got = vie.embed_grad(tok, grad, V, workspace=ws[:need])
    assert torch.equal(got, want) and (ws[need:] == 255).all()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [vie.embed_grad(tok, grad, V, stream=s) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph, out, rows = torch.cuda.CUDAGraph(), torch.empty_like(want), torch.empty(n, d, device="cuda")
    with torch.cuda.graph(graph, stream=streams[0]):
        vie.embed_grad(tok, grad, V, out=out, workspace=ws)
        vie.embed(out, tok, out=rows)
    for _ in range(2):
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(rows, vie.embed(want, tok))


def test_no_tokens_and_refusals(vie):
    table = torch.randn(10, 8, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert vie.embed(table, none).shape == (0, 8)
    out = torch.full((10, 8), 5.0, device="cuda")
    assert not vie.embed_grad(none, torch.empty(0, 8, device="cuda"), 10, out=out).any()
    out.fill_(5.0)
    assert (vie.embed_grad(none, torch.empty(0, 8, device="cuda"), 10, out=out, accumulate=True) == 5.0).all()
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    grad = torch.zeros(4, 8, device="cuda")
    for bad in (lambda: vie.embed(table, tok.long()), lambda: vie.embed(table.half(), tok),
                lambda: vie.embed(table[0], tok), lambda: vie.embed(table, tok[None]),
                lambda: vie.embed(table, tok, out=torch.empty(4, 9, device="cuda")),
                lambda: vie.embed_grad(tok[:3], grad, 10), lambda: vie.embed_grad(tok, grad, 10, accumulate=True),
                lambda: vie.embed_grad(tok, grad, 10, out=torch.empty(11, 8, device="cuda")),
                lambda: vie.embed_grad(tok, grad, 10, out=torch.empty(10, 8, device="cuda", dtype=torch.float16)),
                lambda: vie.embed_grad(tok, grad, 10, workspace=torch.empty(1 << 20, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(vie.VieError):
        vie.embed_grad(tok, grad, 0)


def test_offsets_beyond_32_bits(vie):
    """The last rows of a table of more than 2^31 values, as source and as gradient."""
    d = 16384
    V = 2 ** 31 // d + 5
    table = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    rows = torch.randn(3, d, device="cuda").bfloat16()
    table[-3:] = rows
    tok = torch.tensor([V - 1, V - 3, V - 2, V - 1], dtype=torch.int32, device="cuda")
    assert torch.equal(vie.embed(table, tok), rows[torch.tensor([2, 0, 1, 2], device="cuda")])
    vie.embed_grad(tok, rows[torch.tensor([2, 0, 1, 2], device="cuda")], V, out=table)
    assert torch.equal(table[-3:-1], rows[:2]) and torch.equal(table[-1].float(), 2 * rows[2].float())
    assert not table[:-3].any()


@pytest.mark.parametrize("n", [131072, 131073, 200003])
def test_gradient_of_long_batches(vie, n):
    """Either side of the number of tokens from which the whole array is sorted,
    with most of them one token."""
    g = torch.Generator().manual_seed(n)
    tok = torch.where(torch.rand(n, generator=g) < 0.7, torch.full((n,), 12345), torch.randint(0, 50000, (n,), generator=g)).int()
    _check_grad(vie, tok, torch.randn(n, 24, generator=g), 50000, 1.0, torch.float32)


def test_gradient_of_one_bucket(vie):
    """Tokens that are all alike modulo 128: one CTA sorts them, beyond its shared memory."""
    g = torch.Generator().manual_seed(3)
    tok = (torch.randint(0, 2000, (30000,), generator=g) * 128 + 5).int()
    _check_grad(vie, tok, torch.randn(30000, 16, generator=g), 262144, 1.0, torch.float32)
    _check_grad(vie, tok[1:], torch.randn(29999, 16, generator=g), 262144, 1.0, torch.bfloat16,
                torch.zeros(262144, 16, dtype=torch.bfloat16, device="cuda"))


def test_additions_in_place_are_counted(vie):
    """What a call adds to has changed, and autograd can tell."""
    tok, rows = torch.tensor([1, 1, 3], dtype=torch.int32, device="cuda"), torch.ones(3, 8, device="cuda")
    table = torch.ones(5, 8, device="cuda")
    weight = torch.ones(5, 8, device="cuda", requires_grad=True)
    product = (weight * table).sum()  # saves table
    before = table._version
    vie.embed(table, tok)
    assert table._version == before
    vie.embed_grad(tok, rows, 5, out=table, accumulate=True)
    assert table._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()
    with torch.inference_mode():
        vie.embed_grad(tok, rows, 5, out=torch.ones(5, 8, device="cuda"), accumulate=True)


@pytest.mark.parametrize("V,passes", [(2 ** 19 + 3, 3), (2 ** 25 + 9, 4)])
def test_gradient_of_grouped_tokens_with_many_digits(vie, V, passes):
    """Up to 131072 tokens are spread over 128 lists by their low 7 bits, and each
    list is sorted 6 bits at a time: both parities of the number of passes, with
    lists that fit shared memory (2048 entries) and lists that do not."""
    assert -(-((V - 1) >> 7).bit_length() // 6) == passes
    g = torch.Generator().manual_seed(V)
    n, top = 12000, (V - 1) >> 7
    tok = torch.randint(0, V, (n,), generator=g)
    tok[::3] = torch.randint(0, top, (n // 3,), generator=g) * 128 + 77      # a list of about 4000
    tok[1::3] = (torch.randint(0, top >> 6, (n // 3,), generator=g) << 13) + 5  # ids that differ in the upper digits only
    tok[2::3] %= V - 128                                                     # the other lists hold about 30
    tok[2::300] = V - 1
    tok[5], tok[8] = 0, (1 << (V - 1).bit_length() - 1)                      # the top digit alone
    tok = tok.int()
    tok[11::50] = -1
    assert (tok % 128 == 77).sum() > 2048 and (tok % 128 == 5).sum() > 2048
    _check_grad(vie, tok, torch.randn(n, 2, generator=g), V, 1.0, torch.bfloat16)


@pytest.mark.parametrize("n", [131072, 131073])
def test_gradient_of_long_batches_with_large_ids(vie, n):
    """Ids of more than 24 bits on either side of the number of tokens from which the
    whole array is sorted: a fourth pass of 8 bits there, a fourth of 6 here."""
    V = 2 ** 25 + 9
    g = torch.Generator().manual_seed(n)
    tok = torch.randint(0, V, (n,), generator=g)
    tok[::4] = (torch.randint(0, 2, (tok[::4].numel(),), generator=g) << 24) + 3  # the top digit alone
    tok[1::4] = torch.randint(V - 50, V, (tok[1::4].numel(),), generator=g)
    tok = tok.int()
    tok[2::40] = -1
    _check_grad(vie, tok, torch.randn(n, 1, generator=g), V, 1.0, torch.bfloat16)
