"""GPU parity of 4-bit rows (e2m1_quantize, e2m1_dequantize, e2m1_logits) against
their definitions in 64 bits (tests/policy_ref.py).  Quantisation and its values
are exact; a logit is a sum of exact products in fp32, at most one rounding per
product, and is rounded once more to its type."""
import math

import pytest
import torch

import policy_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rows(n, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, d, generator=g) * torch.exp(2.0 * torch.randn(n, 1, generator=g))
    x[torch.rand(n, d, generator=g) < 0.05] = 0.0
    return x.to(DT[dtype])


def _check_rows(vie, x, xc=None, q=None):
    n, d = x.shape
    code, byte, s, values = ref.quantize(x.cpu())
    values_out = torch.empty((n, d), device="cuda")
    q = vie.e2m1_quantize(x.cuda() if xc is None else xc, out=q, out_values=values_out)
    codes, scales, row = ref.unpack(q)
    good = torch.isfinite(s)
    got = ref.VALUES[codes.long()]  # (a zero may have a sign)
    assert torch.equal(got[:, :d][good], ref.VALUES[code][good])
    assert not codes[:, d:].any() and not codes[~good].any()
    blocks = byte.shape[1]
    assert torch.equal(scales[:n, :blocks][good], byte[good])
    assert not scales[n:].any() and not scales[:, blocks:].any() and not scales[:n][~good].any()
    assert torch.equal(torch.isnan(row), ~good) and torch.equal(row[good].double(), s[good])
    assert torch.equal(values_out.double().cpu().nan_to_num(9.0), values.float().double().nan_to_num(9.0))
    for dt in (torch.float32, torch.bfloat16):
        got = vie.e2m1_dequantize(q, out_dtype=dt).cpu().nan_to_num(9.0)
        assert torch.equal(got, values.to(dt).nan_to_num(9.0))
    return q, values


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(1, 1), (1, 16), (3, 17), (2, 31), (5, 64), (127, 33), (128, 65), (129, 100),
                                 (300, 640), (33, 1152), (260, 257), (4, 5000), (9, 16384), (1000, 48)])
def test_sizes(vie, dtype, n, d):
    _check_rows(vie, _rows(n, d, dtype, seed=n + d))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(1300, 33), (1290, 64), (2100, 257), (2500, 300), (5200, 1001), (9300, 2048), (3000, 16)])
def test_many_rows(vie, dtype, n, d):
    """Rows that a warp takes each, 32 of a tile to a CTA; the last tile is not full."""
    x = _rows(n, d, dtype, seed=n + d)
    x[n - 2] = float("inf")
    _check_rows(vie, x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 9, 16, 33, 64, 97, 250, 257, 300, 640, 767, 768, 769, 1001, 1024, 1025, 1152, 1280, 1281, 1400,
                               1536, 1537, 1800, 2040, 2048])
def test_many_rows_of_every_width(vie, dtype, d):
    """Rows that a warp takes each, on both sides of the widths at which its lanes keep another number of vectors,
    with both kinds of values, apart and in place of the rows, at and off 16-byte addresses: the definition's
    bytes in the first and last tile, and those of calls of few rows (a CTA each) in all others."""
    n = 3 * (2000 + 12 * min(d, 768)) + 200
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(n, d, generator=g, device="cuda") * torch.exp(2.0 * torch.randn(n, 1, generator=g, device="cuda"))
    x = x.to(DT[dtype])
    x[n - 2, d - 1], x[5, 0], x[131] = math.inf, math.nan, 0.0
    x[n - 1, d - 1] = 300.0  # a row's largest at its end
    for (off, ld), (o, l) in (((0, (d + 7) // 8 * 8), (0, (d + 7) // 8 * 8)), ((3, d + 1), (3, d + 1)), ((1, d), (7, d + 2))):
        big = torch.full((off + n * ld + 16,), float("nan"), dtype=DT[dtype], device="cuda")
        xc = big[off:off + n * ld].view(n, ld)[:, :d]
        xc.copy_(x)
        q = vie.e2m1_quantize(xc)
        for rows in (slice(0, 128), slice((n - 1) // 128 * 128, n)):
            code, byte, s, want = ref.quantize(x[rows].cpu())
            tiles = slice(rows.start // 128, rows.start // 128 + 1)
            codes, scales, row = ref.unpack(vie.E2m1(q.codes[rows], q.scales[tiles], q.row_scales[rows], d))
            good = torch.isfinite(s)
            assert torch.equal(codes[good][:, :d].long(), torch.where(code == 8, 0, code)[good]) and not codes[:, d:].any()
            m, blocks = byte.shape
            assert torch.equal(scales[:m, :blocks][good], byte[good]) and not scales[m:].any() and not scales[:, blocks:].any()
            assert torch.equal(torch.isnan(row), ~good) and torch.equal(row[good].double(), s[good])
        few = torch.empty((n, d), device="cuda")
        for r0 in range(0, n, 1024):
            part = vie.e2m1_quantize(xc[r0:r0 + 1024], out_values=few[r0:r0 + 1024])
            m = part.codes.shape[0]
            assert torch.equal(q.codes[r0:r0 + m], part.codes)
            assert torch.equal(q.scales[r0 // 128:(r0 + m + 127) // 128], part.scales)
            assert torch.equal(q.row_scales[r0:r0 + m].nan_to_num(9.0), part.row_scales.nan_to_num(9.0))
        few = few.nan_to_num(9.0)
        for values in ("bf16", "f32"):
            out = torch.full((o + n * l + 16,), 7.0, dtype=DT[values], device="cuda")
            view = out[o:o + n * l].view(n, l)[:, :d]
            q2 = vie.e2m1_quantize(xc, out_values=view)
            assert torch.equal(q2.codes, q.codes) and torch.equal(q2.scales, q.scales)
            assert torch.equal(view.nan_to_num(9.0), few.to(DT[values]))
            view.fill_(7.0)
            assert (out == 7.0).all()
        vie.e2m1_quantize(xc, out_values=xc)
        assert torch.equal(xc.nan_to_num(9.0), few.to(DT[dtype]))


@pytest.mark.parametrize("n", [40, 1500])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("values", ["bf16", "f32"])
def test_rows_and_values_at_every_address(vie, n, dtype, values):
    """Every alignment of a row of x with one of the values, widths that end anywhere in a vector."""
    for d, (off, ld), (o, l) in ((99, (1, 99), (3, 101)), (97, (0, 97), (0, 97)), (104, (4, 104), (0, 104)),
                                 (103, (5, 106), (7, 107)), (9, (2, 9), (1, 11)), (64, (0, 65), (0, 64)),
                                 (250, (3, 251), (6, 253))):
        x = _rows(n, d, dtype, seed=d)
        want = ref.quantize(x)[3].to(DT[values])
        big = torch.full((off + n * ld + 8,), float("nan"), dtype=DT[dtype], device="cuda")
        xc = big[off:off + n * ld].view(n, ld)[:, :d]
        xc.copy_(x)
        out = torch.full((o + n * l + 16,), 7.0, dtype=DT[values], device="cuda")
        view = out[o:o + n * l].view(n, l)[:, :d]
        q = vie.e2m1_quantize(xc, out_values=view)
        assert torch.equal(view.cpu(), want)
        assert torch.equal(vie.e2m1_dequantize(q, out_dtype=DT[values]).cpu(), want)
        view.fill_(7.0)
        assert (out == 7.0).all()
        if dtype == values:
            own = xc.clone(memory_format=torch.preserve_format)
            vie.e2m1_quantize(own, out_values=own)
            assert torch.equal(own.cpu(), want)
            vie.e2m1_quantize(xc, out_values=xc)
            assert torch.equal(xc.cpu(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1793, 2049, 2500, 3585, 4097, 5376, 7169, 8193, 8200, 10240, 10241, 12289, 16383])
def test_long_rows(vie, dtype, d):
    """Rows about the widths at which a CTA has another number of warps or of vectors per lane."""
    n = 5
    for off, ld in ((0, (d + 15) // 16 * 16), (1, d), (6, d + 5)):
        x = _rows(n, d, dtype, seed=d + off)
        x[1, d - 1] = 300.0  # a row's largest at its end
        big = torch.full((off + n * ld + 16,), float("nan"), dtype=DT[dtype], device="cuda")
        xc = big[off:off + n * ld].view(n, ld)[:, :d]
        xc.copy_(x)
        _check_rows(vie, x, xc)
        want = ref.quantize(x)[3].to(DT[dtype])
        vie.e2m1_quantize(xc, out_values=xc)
        assert torch.equal(xc.cpu(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(1, 5), (2, 1023), (33, 1024), (130, 1025), (257, 1030), (3, 2052), (300, 64), (1, 16384)])
def test_values_at_every_address(vie, dtype, n, d):
    """Widths about the 1024 columns that a warp reads at once, rows at and off 16-byte addresses; what lies
    beside and behind them stays."""
    x = _rows(n, d, "f32", seed=3 * n + d)
    x[n // 2, d // 2] = float("nan")
    want = ref.quantize(x)[3].to(DT[dtype]).nan_to_num(9.0)
    q = vie.e2m1_quantize(x.cuda())
    for o, pad in ((0, 0), (0, 8 - d % 8), (1, 0), (4, 3), (7, 5), (8, 4 - d % 4), (2, 16 - d % 16)):
        ld = d + pad
        out = torch.full((o + n * ld + 16,), 7.0, dtype=DT[dtype], device="cuda")
        view = out[o:o + n * ld].view(n, ld)[:, :d]
        vie.e2m1_dequantize(q, out=view)
        assert torch.equal(view.cpu().nan_to_num(9.0), want)
        view.fill_(7.0)
        assert (out == 7.0).all()


def test_ties_and_borders(vie):
    """Values on and beside the midpoints of codes and of scales, in blocks whose scale is known."""
    g = torch.Generator().manual_seed(3)
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 5.9, 0.5, 3.0])
    rows = []
    for sigma in (1.0, 1.125, 1.25, 1.375, 1.5, 1.625, 1.75, 1.875, 0.0625, 448.0, 13.0):
        v = mids[torch.randint(0, len(mids), (4, 64), generator=g)] * sigma
        v = v * torch.where(torch.rand(4, 64, generator=g) < 0.5, -1.0, 1.0)
        v[:, ::16] = 6.0 * sigma
        up, down = torch.nextafter(v, v * 2), torch.nextafter(v, v * 0)
        pick = torch.randint(0, 3, v.shape, generator=g)
        v = torch.where(pick == 0, v, torch.where(pick == 1, up, down))
        v[:, ::16] = 6.0 * sigma
        v[:, 48] = 2688.0  # the row's power of two is 1
        rows.append(v)
    x = torch.cat(rows)
    _check_rows(vie, x)
    _check_rows(vie, x.bfloat16())
    # largest magnitudes around the midpoints of scales, and around 2688 powers of two
    top = torch.tensor([6.375, 6.125, 7.125, 11.625, 2688.0, 2687.9998, 2688.0002, 1344.0001, 1344.0, 5376.0])
    x = torch.zeros(len(top) * 3, 48)
    for i, t in enumerate(top):
        for j, v in enumerate((t, torch.nextafter(t, t * 2), torch.nextafter(t, t * 0))):
            x[3 * i + j, 5], x[3 * i + j, 20] = -v, 2000.0 if i < 4 else 1.0
            x[3 * i + j, 21] = v / 3
    _check_rows(vie, x)


@pytest.mark.parametrize("n,d", [(5, 200), (40, 3000), (2100, 257), (1500, 96)])
def test_zeros_have_one_code(vie, n, d):
    """Values of both signs that round to 0, zeros of both signs, blocks whose scale is 0: code 0, and the same
    bytes from bf16 and from fp32 rows, at and off 16-byte addresses."""
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, d, generator=g) * 2.0 ** torch.randint(-40, 1, (n, d), generator=g).float()
    x[:, ::7] = torch.where(torch.rand(n, (d + 6) // 7, generator=g) < 0.5, -0.0, 0.0)
    x[:, 32:64] = -(2.0 ** -60)
    x[:, 64::16] *= 2.0 ** 12
    x = x.bfloat16()
    want = ref.quantize(x)[0]
    want = torch.where(want == 8, 0, want)
    for off, ld in ((0, (d + 7) // 8 * 8), (1, d)):
        first = None
        for dtype in (torch.bfloat16, torch.float32):
            big = torch.zeros((off + n * ld + 16,), dtype=dtype, device="cuda")
            xc = big[off:off + n * ld].view(n, ld)[:, :d]
            xc.copy_(x)
            values = torch.empty((n, d), device="cuda")
            for q in (vie.e2m1_quantize(xc), vie.e2m1_quantize(xc, out_values=values)):
                codes = ref.unpack(q)[0]
                assert torch.equal(codes[:, :d].long(), want) and not codes[:, d:].any()
                assert not torch.signbit(vie.e2m1_dequantize(q)[vie.e2m1_dequantize(q) == 0]).any()
                if first is None:
                    first = q
                assert torch.equal(q.codes, first.codes) and torch.equal(q.scales, first.scales)
                assert torch.equal(q.row_scales, first.row_scales)
            assert not torch.signbit(values[values == 0]).any()


def test_ranges(vie):
    """Rows from subnormal numbers to the largest ones, rows of zeros, blocks that vanish beside others."""
    x = _rows(60, 96, "f32", seed=5)
    x = x / x.abs().amax(1, keepdim=True) * (2.0 ** torch.linspace(-149, 127.9, 60).double()[:, None]).float()
    x[7] = 0.0
    x[8] = -0.0
    x[9, :90] = 0.0
    _check_rows(vie, x)
    y = _rows(40, 64, "f32", seed=7)
    y[:, 16:32] *= 2.0 ** -torch.arange(40.0)[:, None]
    y[:, 40] = 2.0 ** torch.arange(40.0) * 10
    _check_rows(vie, y)
    x = torch.full((3, 20), torch.finfo(torch.float32).max)
    _check_rows(vie, x)
    _check_rows(vie, torch.full((3, 20), torch.finfo(torch.bfloat16).max, dtype=torch.bfloat16))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_not_finite(vie, dtype):
    x = _rows(6, 100, dtype, seed=9)
    x[1, 99], x[3, 0], x[4, 50] = float("nan"), math.inf, -math.inf
    q, values = _check_rows(vie, x)
    assert torch.isnan(values[[1, 3, 4]]).all() and torch.isfinite(values[[0, 2, 5]]).all()
    w = vie.e2m1_quantize(_rows(70, 100, dtype, seed=10).cuda())
    out = vie.e2m1_logits(q, w)
    assert torch.isnan(out[[1, 3, 4]]).all() and torch.isfinite(out[[0, 2, 5]]).all()
    out = vie.e2m1_logits(w, q)
    assert torch.isnan(out[:, [1, 3, 4]]).all() and torch.isfinite(out[:, [0, 2, 5]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_places_and_values_in_place(vie, dtype):
    n, d = 37, 99
    x = _rows(n, d, dtype, seed=11)
    for off, ld in ((0, 104), (1, 99), (3, 101), (8, 128)):
        big = torch.full((off + n * ld,), float("nan"), dtype=DT[dtype], device="cuda")
        xc = big[off:].view(n, ld)[:, :d]
        xc.copy_(x)
        _check_rows(vie, x, xc=xc)
        out = torch.full((n * ld + 16,), 7.0, dtype=DT[dtype], device="cuda")
        view = out[off:off + n * ld].view(n, ld)[:, :d]
        vie.e2m1_quantize(xc, out_values=view)
        want = ref.quantize(x)[3].to(DT[dtype])
        assert torch.equal(view.cpu(), want)
        view.fill_(7.0)
        assert (out == 7.0).all()
    own = x.cuda().clone()
    before = own._version
    vie.e2m1_quantize(own, out_values=own)
    assert torch.equal(own.cpu(), ref.quantize(x)[3].to(DT[dtype])) and own._version > before
    _check_rows(vie, x, xc=x.t().contiguous().cuda().t())
    # codes and scales that were something else before
    q = vie.E2m1.empty(n, d)
    q.codes.fill_(255)
    q.scales.fill_(255)
    _check_rows(vie, x, q=q)


def _whole(n, d, seed):
    """Rows whose codes are their values times a power of two, each block's another:
    all products and sums are whole numbers below 2^24."""
    g = torch.Generator().manual_seed(seed)
    v = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0, -1.0, -2.0, -3.0, -4.0, -6.0])
    x = v[torch.randint(0, len(v), (n, d), generator=g)]
    blocks = (d + 15) // 16
    x[:, ::16] = 6.0
    power = 2.0 ** torch.randint(0, 2, (n, blocks), generator=g).float()
    return x * power.repeat_interleave(16, 1)[:, :d] * 2.0 ** torch.randint(-9, 9, (n, 1), generator=g).float()


SHAPES = [(1, 1, 1), (3, 7, 5), (16, 128, 64), (17, 129, 65), (33, 300, 100), (64, 1000, 640), (65, 515, 1152),
          (8, 4096, 128), (129, 2048, 257), (257, 4099, 300), (5, 20011, 96), (300, 384, 4096), (2, 257, 16384),
          (100, 40000, 192), (1, 30000, 1000), (513, 1024, 512), (1030, 3001, 64)]


@pytest.mark.parametrize("n,V,d", SHAPES)
def test_logits_of_whole_numbers_are_exact(vie, n, V, d):
    x, w = _whole(n, d, seed=n), _whole(V, d, seed=V + 1)
    want = x.cuda().double() @ w.cuda().double().t()
    wq, xq = vie.e2m1_quantize(w.cuda()), vie.e2m1_quantize(x.cuda())
    assert torch.equal(vie.e2m1_dequantize(wq).cpu(), w) and torch.equal(vie.e2m1_dequantize(xq).cpu(), x)
    assert torch.equal(vie.e2m1_logits(xq, wq).double(), want)
    assert torch.equal(vie.e2m1_logits(x.cuda(), wq, out_dtype=torch.bfloat16), want.float().bfloat16())
    assert vie.vie_device_status() == vie.VIE_OK


@pytest.mark.parametrize("n,V,d", [(1, 60001, 4096), (16, 60001, 4096), (40, 60001, 4096), (100, 60001, 4096), (257, 60001, 4096),
                                   (600, 40000, 1152)])
def test_scales_of_their_own_stage(vie, n, V, d):
    """Block scales that differ from each 64 columns to the next, by powers that cancel between the two
    matrices, so that a sum is a whole number again only if each product meets the scales of its own
    columns: tens of stages a tile and several tiles a CTA, whose scales go through the same columns of
    tensor memory in turn."""
    g = torch.Generator().manual_seed(61)
    power = 2.0 ** torch.randint(-3, 4, ((d + 63) // 64,), generator=g).float().repeat_interleave(64)[:d]
    v = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0, -1.0, -2.0, -3.0, -4.0, -6.0])
    x, w = (v[torch.randint(0, len(v), (rows, d), generator=g)] for rows in (n, V))
    x[:, ::16], w[:, ::16] = 6.0, -6.0
    want = x.cuda().double() @ w.cuda().double().t()
    xq, wq = vie.e2m1_quantize((x * power).cuda()), vie.e2m1_quantize((w / power).cuda())
    assert torch.equal(vie.e2m1_dequantize(wq), (w / power).cuda()) and torch.equal(vie.e2m1_dequantize(xq), (x * power).cuda())
    for _ in range(3):
        assert torch.equal(vie.e2m1_logits(xq, wq).double(), want)
    assert vie.vie_device_status() == vie.VIE_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,d", SHAPES[:14])
def test_logits_of_any_rows(vie, dtype, n, V, d):
    x, w = _rows(n, d, dtype, seed=n + d), _rows(V, d, "bf16", seed=V)
    wq = vie.e2m1_quantize(w.cuda())
    room = vie.E2m1.empty(n, d)
    got = vie.e2m1_logits(x.cuda(), wq, x_quantized=room)
    assert torch.equal(got, vie.e2m1_logits(room, wq))
    xv, wv = vie.e2m1_dequantize(room).double(), vie.e2m1_dequantize(wq).double()
    want, mass = xv @ wv.t(), xv.abs() @ wv.abs().t()
    tol = (d + 2) * ref.U * mass
    assert ((got.double() - want).abs() <= tol).all()
    got = vie.e2m1_logits(x.cuda(), wq, out_dtype=torch.bfloat16)
    assert ((got.double() - want).abs() <= tol + (ref.HALF[torch.bfloat16] + ref.U) * want.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_into_rows_with_a_pitch(vie, dtype):
    n, V, d = 19, 333, 80
    x, w = _whole(n, d, seed=1).cuda(), _whole(V, d, seed=2).cuda()
    wq = vie.e2m1_quantize(w)
    want = vie.e2m1_logits(x, wq, out_dtype=DT[dtype])
    for off, ld in ((0, 333), (1, 336), (3, 341), (8, 512)):
        buf = torch.full((off + n * ld + 40,), 7.0, dtype=DT[dtype], device="cuda")
        view = buf[off:off + n * ld].view(n, ld)[:, :V]
        got = vie.e2m1_logits(x, wq, out=view)
        assert got.data_ptr() == view.data_ptr() and torch.equal(got, want)
        view.fill_(7.0)
        assert (buf == 7.0).all()


def test_logits_of_far_powers(vie):
    """Rows near the ends of fp32 whose products are within it, and products beyond it.
    A sum of codes and block scales, at most d 2688^2, is multiplied with s t, the product
    of the rows' powers of two, which is exact but where it is below 2^-149: there it
    becomes 0, and what is lost is less than d 2688^2 2^-149."""
    x, w = _whole(5, 96, seed=51), _whole(40, 96, seed=52)
    x = x / x.abs().amax(1, keepdim=True) * 6
    w = w / w.abs().amax(1, keepdim=True) * 6
    a = 2.0 ** torch.tensor([120.0, -120.0, 60.0, 0.0, -140.0])
    b = 2.0 ** torch.tensor([-120.0, 120.0, 100.0, -20.0]).repeat(10)
    x, w = x * a[:, None], w * b[:, None]
    want = (x.double() @ w.double().t()).float()
    got = vie.e2m1_logits(x.cuda(), vie.e2m1_quantize(w.cuda())).cpu()
    values = ref.quantize(x)[3].double() @ ref.quantize(w)[3].double().t()  # (subnormal rows lose digits)
    st = ref.quantize(x)[2][:, None] * ref.quantize(w)[2]
    lost = torch.where(st < 2.0 ** -149, 96 * 2688.0 ** 2 * 2.0 ** -149, 0.0)
    far = torch.isinf(want) | torch.isinf(got)
    assert torch.equal(got[far], values.float()[far])
    scale = (x.double().abs() @ w.double().abs().t()).float()
    assert ((got - values).abs()[~far] <= 98 * ref.U * scale[~far] + 2.0 ** -148 + lost[~far]).all()


@pytest.mark.parametrize("n,copies", [(7, 1), (16, 1), (30, 1), (60, 1), (66, 1), (200, 1), (600, 61), (20, 999)])
def test_logits_of_all_powers_are_exact(vie, n, copies):
    """Rows from one end of fp32 to the other, whose sums of codes are whole numbers, small ones, and 0 (rows
    that share no column, products that cancel): the definition's values rounded to fp32, then to bf16.  With
    copies of the vocabulary's rows, and plain rows between them, CTAs have tiles with and without such rows."""
    d = 96
    powers = torch.tensor([-149, -140, -130, -126, -120, -110, -101, -100, -99, -90, -64, -30, 0, 17, 40, 64, 75, 90, 91, 100,
                           110, 124])
    g = torch.Generator().manual_seed(71)
    v = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0, -1.0, -2.0, -3.0, -4.0, -6.0])

    def rows(sign):
        x = v[torch.randint(0, len(v), (3 * len(powers), d), generator=g)]
        x[:, ::16] = 6.0
        x[0::3, :16], x[0::3, 16:32] = 1.0, sign
        x[0::3, 32:] = 0.0                              # 0 in the product of two such rows, or 16 * 2
        x[1::3].view(-1, d // 16, 16)[:, 1::2] = 0.0    # blocks that the next row has not
        x[2::3].view(-1, d // 16, 16)[:, 0::2] = 0.0
        return (x.double() * 2.0 ** powers.double().repeat_interleave(3)[:, None]).float()

    x, w = rows(1.0).repeat(10, 1)[torch.randperm(10 * 3 * len(powers), generator=g)[:n]], rows(-1.0)
    if copies > 1:
        plain = torch.zeros((1, d))
        plain[0, 5] = 3.0
        w = torch.cat([w, plain.expand(255, d)]).repeat(copies, 1)
    want = (ref.quantize(x)[3] @ ref.quantize(w)[3].t()).float()
    assert (want == 0).any() and torch.isinf(want).any() and (want.abs() > 2.0 ** 100).any()
    wq = vie.e2m1_quantize(w.cuda())
    assert torch.equal(vie.e2m1_logits(x.cuda(), wq).cpu(), want)
    assert torch.equal(vie.e2m1_logits(x.cuda(), wq, out_dtype=torch.bfloat16).cpu(), want.bfloat16())


def test_the_same_bits_again_on_streams_and_in_a_graph(vie):
    n, V, d = 40, 30011, 640
    x, w = _rows(n, d, "f32", seed=21).cuda(), _rows(V, d, "bf16", seed=22).cuda()
    wq = vie.e2m1_quantize(w)
    want = vie.e2m1_logits(x, wq)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        for s in streams:  # two calls at once
            got.append(vie.e2m1_logits(x, wq, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got)
    out, room = torch.empty_like(want), vie.E2m1.empty(n, d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        vie.e2m1_logits(x, wq, out=out, x_quantized=room)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_rows_beyond_32_bits(vie):
    """Codes of more than 2^31 values, and logits of more than 2^31 values."""
    d = 16384
    n = 2 ** 31 // d + 130
    x = torch.zeros((n, d), dtype=torch.bfloat16, device="cuda")
    x[-3:] = _rows(3, d, "bf16", seed=31).cuda()
    q = vie.e2m1_quantize(x)
    want = vie.e2m1_quantize(x[-3:].clone())
    assert torch.equal(q.codes[-3:], want.codes) and torch.equal(q.row_scales[-3:], want.row_scales)
    assert torch.equal(vie.e2m1_dequantize(q, out_dtype=torch.bfloat16)[-3:],
                       vie.e2m1_dequantize(want, out_dtype=torch.bfloat16))
    y = vie.e2m1_quantize(_rows(2, d, "f32", seed=32).cuda())
    assert torch.equal(vie.e2m1_logits(y, q)[:, -3:], vie.e2m1_logits(y, want))
    del x, q
    V, n = 262144, 2 ** 31 // 262144 + 3
    w, h = vie.e2m1_quantize(_whole(V, 64, seed=33).cuda()), vie.e2m1_quantize(_whole(n, 64, seed=34).cuda())
    out = vie.e2m1_logits(h, w, out_dtype=torch.bfloat16)
    last = vie.e2m1_quantize(vie.e2m1_dequantize(h)[-2:])
    assert torch.equal(out[-2:], vie.e2m1_logits(last, w, out_dtype=torch.bfloat16))


def test_no_rows_and_refusals(vie):
    x, w = _rows(4, 50, "f32", seed=41).cuda(), _rows(60, 50, "f32", seed=42).cuda()
    q = vie.e2m1_quantize(x[:0])
    assert q.shape == (0, 50) and vie.e2m1_dequantize(q).shape == (0, 50)
    wq = vie.e2m1_quantize(w)
    assert vie.e2m1_logits(q, wq).shape == (0, 60) and vie.e2m1_logits(x[:0], wq).shape == (0, 60)
    for call in (lambda: vie.e2m1_quantize(x.half()), lambda: vie.e2m1_quantize(x[0]), lambda: vie.e2m1_quantize(x.cpu()),
                 lambda: vie.e2m1_quantize(x, out=vie.E2m1.empty(5, 50)),
                 lambda: vie.e2m1_quantize(x, out=vie.E2m1.empty(4, 51)),
                 lambda: vie.e2m1_quantize(x, out=vie.E2m1.empty(4, 50, device="cpu")),
                 lambda: vie.e2m1_quantize(x, out_values=x[:3]), lambda: vie.e2m1_quantize(x, out_values=x.t()),
                 lambda: vie.e2m1_quantize(x, out_values=x.half()),
                 lambda: vie.e2m1_logits(x[:, :49], wq), lambda: vie.e2m1_logits(x.cpu(), wq),
                 lambda: vie.e2m1_logits(vie.e2m1_quantize(x[:, :48]), wq),
                 lambda: vie.e2m1_logits(x, wq, x_quantized=vie.E2m1.empty(5, 50)),
                 lambda: vie.e2m1_logits(x, wq, out=torch.empty(4, 61, device="cuda")),
                 lambda: vie.e2m1_logits(x, wq, out=torch.empty(4, 60, device="cuda", dtype=torch.float16)),
                 lambda: vie.e2m1_logits(x, wq, out=torch.empty(60, 4, device="cuda").t())):
        with pytest.raises(ValueError):
            call()
