"""The operators around the LM head on the GPU: final norm, microscaled formats, product on them; each against the plain
64-bit statement in mx_reference.py."""
import math

import pytest
import torch

import mx_reference as ref
import paper_2511_02620_b200 as difr

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def randn(*shape, seed=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g) * std


def mx_of(rows, d, fmt):
    """A tensor whose buffers are full of a value that nothing writes."""
    mx = difr.MxTensor.allocate(rows, d, fmt)
    mx.codes.fill_(0x5A)
    mx.scales.fill_(0xA5)
    return mx


def assert_mx_equal(mx, y, fmt):
    """Codes and scales are those of the 64-bit statement, bit for bit; bytes of rows behind the last are untouched."""
    c, byte = ref.quantize(y, fmt)
    assert torch.equal(mx.codes.cpu(), ref.pack(c, fmt))
    assert torch.equal(mx.scales.cpu(), ref.tile_scales(byte, fill=0xA5))


# ------------------------------------------------------------------ quantisation
@pytest.mark.parametrize("fmt", [8, 4])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 32), (3, 31), (5, 33), (2, 100), (129, 128), (130, 1056), (257, 1749),
                                    (9, 70), (20, 1030), (7, 4096), (1, 8192)])
def test_quantisation_is_bit_exact(rows, d, dtype, fmt):
    x = randn(rows, d, seed=rows + d).to(DTYPES[dtype])
    mx = mx_of(rows, d, fmt)
    difr.difr_mx_quantize(x.cuda(), mx)
    assert_mx_equal(mx, x, fmt)


@pytest.mark.parametrize("fmt", [8, 4])
def test_every_rounding_border_of_the_format(fmt):
    """All code values, all midpoints (ties) and their fp32 neighbours, both signs, under scales over the whole range."""
    t = ref.table(fmt)
    mid = (t[1:] + t[:-1]) / 2
    top = t[-1]
    pts = torch.cat([t, mid, torch.tensor([float(top) * 1.05, float(top) * 1.14, 2.0 ** (ref.EMAX[fmt] + 1) * (1 - 2.0 ** -24)],
                                          dtype=torch.float64)]).float()
    pts = torch.cat([pts, torch.nextafter(pts, torch.tensor(math.inf)), torch.nextafter(pts, torch.tensor(0.0))])
    pts = torch.cat([pts, -pts])
    pts = pts[pts.abs() < 2.0 ** (ref.EMAX[fmt] + 1)]
    rows = []
    for e in (-126 + ref.EMAX[fmt] + 8, -60, -1, 0, 3, 60, 127 - ref.EMAX[fmt]):
        for i in range(0, pts.numel(), 30):
            p = pts[i:i + 30]
            row = torch.zeros(32)
            row[:p.numel()] = p
            row[31] = 2.0 ** ref.EMAX[fmt]  # fixes the scale at 2^e
            rows.append(torch.ldexp(row, torch.tensor(e)))
    x = torch.stack(rows)
    assert torch.isfinite(x).all()
    mx = mx_of(x.shape[0], 32, fmt)
    difr.difr_mx_quantize(x.cuda(), mx)
    assert_mx_equal(mx, x, fmt)


@pytest.mark.parametrize("fmt", [8, 4])
def test_extreme_blocks(fmt):
    """Zero blocks, subnormals, the largest numbers, signed zeros; NaN and infinities spoil their block only."""
    x = randn(12, 96, seed=5)
    x[0] = 0.0
    x[1] = -0.0
    x[2] = torch.finfo(torch.float32).max
    x[3, :32] = 1e-45
    x[3, 32:64] = -3e-39
    x[4] = x[4] * 1e-42
    x[5, 40] = math.nan
    x[6, 0] = math.inf
    x[7, 95] = -math.inf
    x[8] = -torch.finfo(torch.float32).max
    x[9] = torch.finfo(torch.float32).tiny
    x[10, 32:] = 0.0
    mx = mx_of(12, 96, fmt)
    difr.difr_mx_quantize(x.cuda(), mx)
    assert_mx_equal(mx, x, fmt)
    out = torch.empty(12, 96, device="cuda")
    difr.difr_mx_dequantize(mx, out)
    c, byte = ref.quantize(x, fmt)
    want = ref.values(c, byte, fmt, 96)
    assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out.cpu().double()), torch.nan_to_num(want))
    nan_blocks = torch.isnan(want).view(12, 3, 32)
    assert nan_blocks.any(-1).sum() == 3 and torch.equal(nan_blocks.any(-1), nan_blocks.all(-1))


@pytest.mark.parametrize("fmt", [8, 4])
@pytest.mark.parametrize("out_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,ld", [(1, 1, 1), (3, 31, 40), (129, 256, 256), (70, 1749, 1749), (5, 4096, 4104), (9, 70, 70), (20, 1030, 1034)])
def test_dequantisation_is_exact(rows, d, ld, out_dtype, fmt):
    g = torch.Generator().manual_seed(d)
    nb = (d + 31) // 32
    c = torch.randint(0, 2 ** fmt, (rows, nb * 32), generator=g)
    if fmt == 8:
        c[(c & 127) == 127] = 0  # NaN codes: below
    c[:, d:] = 0
    byte = torch.randint(20, 230, (rows, nb), generator=g)
    mx = difr.MxTensor(ref.pack(c, fmt).cuda(), ref.tile_scales(byte).cuda(), fmt, rows, d)
    buf = torch.full((rows, ld), -7.0, dtype=DTYPES[out_dtype], device="cuda")
    difr.difr_mx_dequantize(mx, buf[:, :d])
    assert torch.equal(buf[:, :d].cpu().double(), ref.values(c, byte, fmt, d))
    assert torch.all(buf[:, d:] == -7.0)


def test_nan_codes_stay_nan():
    c = torch.zeros(1, 32, dtype=torch.long)
    c[0, 3], c[0, 9] = 127, 255
    mx = difr.MxTensor(ref.pack(c, 8).cuda(), ref.tile_scales(torch.full((1, 1), 127)).cuda(), 8, 1, 32)
    out = torch.empty(1, 32, device="cuda")
    difr.difr_mx_dequantize(mx, out)
    assert torch.isnan(out).nonzero()[:, 1].tolist() == [3, 9]


@pytest.mark.parametrize("fmt", [8, 4])
@pytest.mark.parametrize("offset,ld", [(0, 72), (1, 72), (0, 67), (8, 80)])
def test_quantisation_of_strided_rows(offset, ld, fmt):
    buf = randn(40, ld + 8, seed=ld).to(torch.bfloat16)
    flat = buf.cuda()
    x = flat[:, offset:offset + 65]
    mx = mx_of(40, 65, fmt)
    difr.difr_mx_quantize(x, mx)
    assert_mx_equal(mx, buf[:, offset:offset + 65], fmt)


def test_a_last_row_that_ends_its_allocation():
    """Rows as the tail of a buffer, with a stride longer than what is left behind the last row."""
    buf = randn(3 * 100 + 33, seed=2)
    x = torch.as_strided(buf.cuda(), (4, 33), (100, 1))
    mx = mx_of(4, 33, 8)
    difr.difr_mx_quantize(x, mx)
    assert_mx_equal(mx, torch.as_strided(buf, (4, 33), (100, 1)), 8)


# ------------------------------------------------------------------ norm
# Error of y in fp32, relative: the squares' sum has at most 32 terms per thread, 5 + 32 more additions (each 2^-24), the
# root halves that; mean, + eps, root, reciprocal and two products add six roundings.
Y_ERR = (32 + 37) / 2 * 2.0 ** -24 + 6 * 2.0 ** -24


def assert_close_h(h, y):
    err = (h.double().cpu() - y).abs()
    assert torch.all(err <= (2.0 ** -8 + Y_ERR * (1 + 2.0 ** -8)) * y.abs() + 2.0 ** -134)


def assert_mx_nearest(mx, y, fmt):
    """The scale is that of the 64-bit row (the neighbour where its maximum is within Y_ERR of a power of two), and
    each value is as near to y as the format allows, up to y's own error."""
    rows, d = y.shape
    nb = (d + 31) // 32
    byte = ref.untile_scales(mx.scales.cpu(), rows, nb)
    b = ref.blocks(y)
    ok = torch.zeros_like(byte, dtype=torch.bool)
    for f in (1 - Y_ERR, 1.0, 1 + Y_ERR):
        ok |= byte == ref.scale_exponents(b * f, fmt) + 127
    assert ok.all()
    c = ref.unpack(mx.codes.cpu(), fmt)
    assert torch.all(c[:, d:] == 0)
    got = ref.values(c, byte, fmt, nb * 32).view(rows, nb, 32)
    s = torch.exp2(byte.double() - 127).unsqueeze(-1)
    grid = ref.table(fmt) * 1.0
    best = (b.abs() / s).clamp(max=float(grid[-1]))
    i = torch.bucketize(best, grid).clamp(max=grid.numel() - 1)
    near = torch.minimum((grid[i] - best).abs(), (best - grid[(i - 1).clamp(min=0)]).abs()) * s
    err = (got.abs() - torch.minimum(b.abs(), grid[-1] * s)).abs()
    assert torch.all(err <= near + 2 * Y_ERR * b.abs())
    assert torch.all((got == 0) | (torch.sign(got) == torch.sign(b)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", [0, 8, 4])
@pytest.mark.parametrize("T,d,residual", [(1, 1, False), (1, 4096, True), (3, 100, True), (9, 31, False), (130, 160, True),
                                          (5, 1749, True), (9, 70, True), (7, 1030, True), (17, 2048, False), (33, 5120, True), (2, 9001, True),
                                          (1, 32768, True), (3, 16384, False)])
def test_norm(T, d, residual, fmt, dtype):
    x = randn(T, d, seed=1).to(DTYPES[dtype])
    r = (randn(T, d, seed=2, std=3.0)).to(DTYPES[dtype]) if residual else None
    w = (1 + 0.2 * randn(d, seed=3)).to(DTYPES[dtype])
    out = difr.NormOut(h=torch.empty(T, d, dtype=torch.bfloat16, device="cuda"),
                       residual=torch.empty(T, d, dtype=DTYPES[dtype], device="cuda") if residual else None,
                       mx=mx_of(T, d, fmt) if fmt else None)
    difr.difr_rms_norm(x.cuda(), w.cuda(), 1e-6, out, residual=r.cuda() if residual else None)
    stream, y = ref.rms_norm(x, r, w, 1e-6)
    if residual:
        assert torch.equal(out.residual.cpu(), stream)
    assert_close_h(out.h, y)
    if fmt:
        assert_mx_nearest(out.mx, y, fmt)
        again = mx_of(T, d, fmt)  # without h, and without the stream: the same codes
        difr.difr_rms_norm(x.cuda(), w.cuda(), 1e-6, difr.NormOut(mx=again), residual=r.cuda() if residual else None)
        assert torch.equal(again.codes, out.mx.codes) and torch.equal(again.scales, out.mx.scales)


def test_norm_in_place_and_strided():
    """The stream over the residual, h over x; rows of wider matrices, aligned to 16 bytes and not."""
    for pad, off in ((8, 0), (7, 0), (16, 8), (9, 3), (2, 0), (6, 2), (4, 4)):
        T, d = 37, 520
        xb, rb = randn(T, d + pad + off, seed=4).bfloat16(), randn(T, d + pad + off, seed=5).bfloat16()
        w = (1 + 0.1 * randn(d, seed=6)).bfloat16()
        x, r = xb.cuda()[:, off:off + d], rb.cuda()[:, off:off + d]
        stream, y = ref.rms_norm(xb[:, off:off + d], rb[:, off:off + d], w, 1e-5)
        difr.difr_rms_norm(x, w.cuda(), 1e-5, difr.NormOut(h=x, residual=r), residual=r)
        assert torch.equal(r.cpu(), stream)
        assert_close_h(x, y)
        assert torch.equal(x._base[:, :off].cpu(), xb[:, :off]) and torch.equal(x._base[:, off + d:].cpu(), xb[:, off + d:])


def test_norm_of_huge_tiny_and_broken_rows():
    T, d = 8, 1000
    x = randn(T, d, seed=7)
    x[0] *= 1e25      # squares beyond fp32
    x[1] *= 1e37
    x[2] *= 1e-30     # eps decides
    x[3] = 0.0
    x[4, 17] = math.nan
    x[5, 18] = math.inf
    x[6, :500] = 0.0
    w = torch.ones(d)
    h = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    mx = mx_of(T, d, 8)
    difr.difr_rms_norm(x.cuda(), w.cuda(), 1e-6, difr.NormOut(h=h, mx=mx))
    _, y = ref.rms_norm(x, None, w, 1e-6)
    good = [0, 1, 2, 3, 6, 7]
    assert_close_h(h[good], y[good])
    assert torch.isnan(h[4]).all()
    assert torch.isnan(h[5]).nonzero().flatten().tolist() == [18] and torch.nan_to_num(h[5]).abs().max() == 0
    byte = ref.untile_scales(mx.scales.cpu(), T, 32)
    assert torch.all(byte[4] == 255) and (byte[5] == 255).nonzero().flatten().tolist() == [0]
    assert not (byte[good] == 255).any()


# ------------------------------------------------------------------ product
def random_mx(rows, d, fmt, seed, exponents=(-1, 2)):
    """Random codes (no NaN) with scales 2^e, e in [exponents): (MxTensor on the GPU, 64-bit values)."""
    g = torch.Generator().manual_seed(seed)
    nb = (d + 31) // 32
    c = torch.randint(0, 2 ** fmt, (rows, nb * 32), generator=g)
    if fmt == 8:
        c[(c & 127) == 127] = 0
    c[:, d:] = 0
    byte = torch.randint(127 + exponents[0], 127 + exponents[1], (rows, nb), generator=g)
    return (difr.MxTensor(ref.pack(c, fmt).cuda(), ref.tile_scales(byte, fill=0xFF).cuda(), fmt, rows, d),
            ref.values(c, byte, fmt, d))


def logits_bound(h, W, fmt, out_dtype):
    """Every tensor-core step adds 32 (8 bits) or 64 (4 bits) exact products to the fp32 accumulator; a step may drop up to
    two units in the last place (2^-23) of the largest magnitude it meets, which sum |h W| bounds."""
    steps = (h.shape[1] + (31 if fmt == 8 else 63)) // (32 if fmt == 8 else 64)
    mass = h.abs() @ W.abs().T
    bound = (2 * steps + 2) * 2.0 ** -23 * mass
    exact = h @ W.T
    if out_dtype == torch.bfloat16:
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * exact.abs()
    return exact, bound


@pytest.mark.parametrize("fmt", [4, 8])
@pytest.mark.parametrize("T,d,V", [(1, 256, 256), (16, 128, 512), (32, 512, 300), (64, 4096, 257), (128, 96, 1000),
                                   (256, 256, 256), (300, 1749, 515), (513, 640, 2049), (300, 1749, 5000), (513, 640, 4200),
                                   (200, 4096, 9800)])
def test_logits_of_small_integers_are_exact(T, d, V, fmt):
    """Codes that are small multiples of 1/2 under scales 1/2 .. 2: every partial sum fits fp32, so any error is a
    misplaced code or scale."""
    g = torch.Generator().manual_seed(T + d)
    nb = (d + 31) // 32

    def make(rows):
        c4 = torch.randint(0, 16, (rows, nb * 32), generator=g)
        c4[:, d:] = 0
        c = c4
        if fmt == 8:  # the same values in e4m3
            mag = ref.table(4)[c4 & 7]
            c = torch.searchsorted(ref.table(8), mag) | ((c4 >> 3) << 7)
        byte = torch.randint(126, 129, (rows, nb), generator=g)
        return (difr.MxTensor(ref.pack(c, fmt).cuda(), ref.tile_scales(byte, fill=0xFF).cuda(), fmt, rows, d),
                ref.values(c, byte, fmt, d))

    h, hv = make(T)
    W, Wv = make(V)
    out = torch.full((T, V), math.nan, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    difr.difr_mx_logits(h, W, out, status)
    assert int(status.item()) == 0
    assert torch.equal(out.cpu().double(), hv @ Wv.T)


@pytest.mark.parametrize("fmt", [4, 8])
@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d,V", [(1, 1, 1), (1, 32, 31), (2, 4096, 1003), (17, 2080, 777), (40, 64, 256), (100, 992, 3001),
                                   (129, 1000, 511), (260, 5120, 1025), (1000, 333, 4097), (129, 1000, 9731), (260, 2048, 4999)])
def test_logits(T, d, V, out_dtype, fmt):
    h, hv = random_mx(T, d, fmt, seed=d, exponents=(-6, 3))
    W, Wv = random_mx(V, d, fmt, seed=V, exponents=(-12, -3))
    dt = DTYPES[out_dtype]
    out = torch.full((T, V), math.nan, dtype=dt, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    difr.difr_mx_logits(h, W, out, status)
    assert int(status.item()) == 0
    exact, bound = logits_bound(hv, Wv, fmt, dt)
    assert torch.all((out.cpu().double() - exact).abs() <= bound)


@pytest.mark.parametrize("fmt", [4, 8])
@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,ld", [(3, 300, 300), (140, 520, 528), (300, 1000, 1008), (300, 1001, 1001), (530, 777, 800),
                                    (257, 130, 131), (300, 5000, 5008), (300, 5001, 5001), (530, 4097, 4104), (257, 4998, 5000)])
def test_logits_rows_of_a_wider_matrix(T, V, ld, out_dtype, fmt):
    """Row strides that do and do not allow tile stores; nothing is written behind a row or behind the last one."""
    d = 160
    h, hv = random_mx(T, d, fmt, seed=1)
    W, Wv = random_mx(V, d, fmt, seed=2)
    dt = DTYPES[out_dtype]
    buf = torch.full((T + 2, ld), -7.0, dtype=dt, device="cuda")
    difr.difr_mx_logits(h, W, buf[:T, :V])
    exact, bound = logits_bound(hv, Wv, fmt, dt)
    assert torch.all((buf[:T, :V].cpu().double() - exact).abs() <= bound)
    assert torch.all(buf[:T, V:] == -7.0) and torch.all(buf[T:] == -7.0)


@pytest.mark.parametrize("T", [15, 16, 17, 31, 33, 63, 65, 127, 129, 255, 257, 272, 384, 511, 512, 769])
@pytest.mark.parametrize("V", [1100, 10000])  # few tiles and many: 128 and 256 tokens per tile
def test_logits_at_the_borders_of_token_tiles(T, V):
    for fmt in (4, 8):
        h, hv = random_mx(T, 96, fmt, seed=T)
        W, Wv = random_mx(V, 96, fmt, seed=T + 1)
        out = torch.full((T, V), math.nan, device="cuda")
        difr.difr_mx_logits(h, W, out)
        exact, bound = logits_bound(hv, Wv, fmt, torch.float32)
        assert torch.all((out.cpu().double() - exact).abs() <= bound)


@pytest.mark.parametrize("fmt", [4, 8])
@pytest.mark.parametrize("T,V", [(1, 700), (200, 700), (200, 9800)])
def test_broken_blocks_make_their_logits_nan(T, V, fmt):
    """A NaN or an infinity in a hidden state makes its row NaN, one in the head its column; the rest is untouched."""
    d = 200
    x, w = randn(T, d, seed=8), randn(V, d, seed=9)
    w[13, 199], w[600, 0] = math.inf, math.nan
    if T > 1:
        x[77, 5] = -math.inf
    h, W = mx_of(T, d, fmt), mx_of(V, d, fmt)
    difr.difr_mx_quantize(x.cuda(), h)
    difr.difr_mx_quantize(w.cuda(), W)
    out = torch.empty(T, V, device="cuda")
    difr.difr_mx_logits(h, W, out)
    nan = torch.zeros(T, V, dtype=torch.bool)
    nan[:, 13] = nan[:, 600] = True
    if T > 1:
        nan[77] = True
    assert torch.equal(torch.isnan(out).cpu(), nan)


def test_extreme_scales_in_the_product():
    """Scales up to the ends of fp32: products that fit come out to the bound, those beyond as infinities."""
    for fmt in (4, 8):
        d = 128
        c = torch.zeros(4, d, dtype=torch.long)
        one = int((ref.table(fmt) == 1.0).nonzero())
        c[:, 0] = one
        hb = torch.tensor([[127 + 60], [127 - 60], [127 + 100], [127]]).expand(4, 4)
        wb = torch.tensor([[127 + 60], [127 - 60], [127 + 100], [127]]).expand(4, 4)
        h = difr.MxTensor(ref.pack(c, fmt).cuda(), ref.tile_scales(hb).cuda(), fmt, 4, d)
        W = difr.MxTensor(ref.pack(c, fmt).cuda(), ref.tile_scales(wb).cuda(), fmt, 4, d)
        out = torch.empty(4, 4, device="cuda")
        difr.difr_mx_logits(h, W, out)
        e = torch.tensor([60, -60, 100, 0])
        want = torch.exp2((e.view(-1, 1) + e.view(1, -1)).double()).float()
        assert torch.equal(out.cpu(), want)


def test_scales_at_the_ends_of_their_range():
    """Scale bytes 0 (2^-127) and 254 (2^127) against each other."""
    for fmt in (4, 8):
        c = torch.zeros(3, 32, dtype=torch.long)
        c[:, 5] = int((ref.table(fmt) == 1.0).nonzero())
        hb, wb = torch.tensor([[0], [254], [127]]), torch.tensor([[254], [0], [127]])
        h = difr.MxTensor(ref.pack(c, fmt).cuda(), ref.tile_scales(hb).cuda(), fmt, 3, 32)
        W = difr.MxTensor(ref.pack(c, fmt).cuda(), ref.tile_scales(wb).cuda(), fmt, 3, 32)
        out = torch.empty(3, 3, device="cuda")
        difr.difr_mx_logits(h, W, out)
        assert out[0, 0].item() == 1.0 and out[1, 1].item() == 1.0 and out[2, 2].item() == 1.0
        assert math.isinf(out[1, 0].item()) and out[2, 0].item() == 2.0 ** 127 and out[1, 2].item() == 2.0 ** 127


def test_random_shapes():
    """Seeded random problems over the operators' ranges, small sizes more often."""
    import random

    rng = random.Random(2026)

    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    for i in range(60):
        fmt, dtype = rng.choice((4, 8)), rng.choice(list(DTYPES))
        T, V, d = size(1, 700), size(1, 3000), size(1, 3000)
        pad, res = rng.choice((0, 0, 1, 8)), rng.random() < 0.5
        x = randn(T, d + pad, seed=i).to(DTYPES[dtype])
        r = randn(T, d, seed=1000 + i, std=4.0).to(DTYPES[dtype]) if res else None
        w = (1 + 0.3 * randn(d, seed=2000 + i)).to(DTYPES[dtype])
        o = difr.NormOut(h=torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), mx=mx_of(T, d, fmt),
                         residual=torch.empty(T, d, dtype=DTYPES[dtype], device="cuda") if res else None)
        difr.difr_rms_norm(x.cuda()[:, :d], w.cuda(), 1e-5, o, residual=r.cuda() if res else None)
        stream, y = ref.rms_norm(x[:, :d], r, w, 1e-5)
        assert_close_h(o.h, y)
        assert_mx_nearest(o.mx, y, fmt)
        if res:
            assert torch.equal(o.residual.cpu(), stream)
        Wp = (randn(V, d, seed=3000 + i) * d ** -0.5).to(DTYPES[dtype])
        W = mx_of(V, d, fmt)
        difr.difr_mx_quantize(Wp.cuda(), W)
        assert_mx_equal(W, Wp, fmt)
        out_dtype = rng.choice((torch.float32, torch.bfloat16))
        out = torch.full((T, V), math.nan, dtype=out_dtype, device="cuda")
        difr.difr_mx_logits(o.mx, W, out)
        nb = (d + 31) // 32
        hv = ref.values(ref.unpack(o.mx.codes.cpu(), fmt), ref.untile_scales(o.mx.scales.cpu(), T, nb), fmt, d)
        c, byte = ref.quantize(Wp, fmt)
        exact, bound = logits_bound(hv, ref.values(c, byte, fmt, d), fmt, out_dtype)
        assert torch.all((out.cpu().double() - exact).abs() <= bound), (i, T, V, d, fmt, dtype)


def test_the_first_call_of_a_process_may_be_captured():
    """No call before it has loaded a kernel or asked the device anything."""
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import sys; sys.path.insert(0, %r)
import torch
import paper_2511_02620_b200 as difr
x = torch.randn(40, 96, device="cuda").bfloat16(); w = torch.ones(96, dtype=torch.bfloat16, device="cuda")
o = difr.NormOut(mx=difr.MxTensor.allocate(40, 96, 4)); W = difr.MxTensor.allocate(300, 96, 4)
v = torch.randn(300, 96, device="cuda"); out = torch.zeros(40, 300, device="cuda"); back = torch.zeros(300, 96, device="cuda")
def run():
    difr.difr_rms_norm(x, w, 1e-6, o); difr.difr_mx_quantize(v, W); difr.difr_mx_logits(o.mx, W, out); difr.difr_mx_dequantize(W, back)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    run()
g.replay(); torch.cuda.synchronize(); a = out.clone(), back.clone(); out.zero_(); back.zero_()
run(); torch.cuda.synchronize()
assert torch.equal(a[0], out) and torch.equal(a[1], back) and float(out.abs().max()) > 0
""" % root
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def test_outputs_beyond_32_bits():
    """Logits of more than 2^32 values and a matrix of more than 2^32 elements: the last rows are where they belong."""
    T, V, d = 33000, 131072 + 6, 32
    h, hv = random_mx(T, d, 4, seed=3)
    W, Wv = random_mx(V, d, 4, seed=4)
    out = torch.empty(T, V, dtype=torch.bfloat16, device="cuda")
    assert out.numel() > 2 ** 32
    difr.difr_mx_logits(h, W, out)
    rows = [0, 1, 16383, 16384, 32767, 32768, T - 1]
    exact, bound = logits_bound(hv[rows], Wv, 4, torch.bfloat16)
    assert torch.all((out[rows].cpu().double() - exact).abs() <= bound)
    del out
    rows, d = (1 << 20) + 3, 4104
    x = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 32
    tail = randn(3, d, seed=6).bfloat16()
    x[-3:] = tail.cuda()
    mx = difr.MxTensor.allocate(rows, d, 8)
    difr.difr_mx_quantize(x, mx)
    c, byte = ref.quantize(tail, 8)
    assert torch.equal(mx.codes[-3:].cpu(), ref.pack(c, 8)) and int(mx.codes[:-3].max()) == 0
    x.zero_()
    difr.difr_mx_dequantize(mx, x)
    assert torch.equal(x[-3:].cpu().double(), ref.values(c, byte, 8, d)) and float(x[:-3].abs().max()) == 0
    x[:-3] = 0
    x[-3:] = tail.cuda()
    difr.difr_rms_norm(x, torch.ones(d, dtype=torch.bfloat16, device="cuda"), 1e-6, difr.NormOut(h=x))
    _, y = ref.rms_norm(tail, None, torch.ones(d), 1e-6)
    assert_close_h(x[-3:], y)


# ------------------------------------------------------------------ together, and as programs call it
@pytest.mark.parametrize("fmt", [4, 8])
def test_a_quantised_head_from_the_residual_stream_to_the_scores(fmt):
    """Norm -> microscaled h -> logits of the quantised head; the same head dequantised goes through the scoring calls, and
    both agree: logits with difr_logits, the greedy replay's token with the largest logit."""
    T, d, V = 300, 512, 4096
    x, r = randn(T, d, seed=1).bfloat16().cuda(), randn(T, d, seed=2, std=2.0).bfloat16().cuda()
    w = (1 + 0.1 * randn(d, seed=3)).bfloat16().cuda()
    Wb = (randn(V, d, seed=4) * d ** -0.5).bfloat16().cuda()
    W = difr.difr_mx_quantize(Wb, difr.MxTensor.allocate(V, d, fmt))
    o = difr.NormOut(residual=r, mx=difr.MxTensor.allocate(T, d, fmt))
    difr.difr_rms_norm(x, w, 1e-6, o, residual=r)
    logits = difr.difr_mx_logits(o.mx, W, torch.empty(T, V, device="cuda"))
    h = difr.difr_mx_dequantize(o.mx, torch.empty(T, d, dtype=torch.bfloat16, device="cuda"))
    Wd = difr.difr_mx_dequantize(W, torch.empty(V, d, dtype=torch.bfloat16, device="cuda"))
    exact, bound = logits_bound(h.cpu().double(), Wd.cpu().double(), fmt, torch.float32)
    assert torch.all((logits.cpu().double() - exact).abs() <= bound)
    plain = difr.difr_logits(h, Wd, torch.empty(T, V, device="cuda"))
    # (the bf16 product accumulates 16 values a step: twice the steps at most)
    assert torch.all((logits - plain).abs().cpu() <= 5 * bound)
    out = difr.DifrOut.allocate(T, d, V, 0.05)
    top = logits.topk(2, dim=1)
    tokens = top.indices[:, 0].int().contiguous()
    difr.difr_score_gm(h, Wd, tokens, torch.arange(T, device="cuda"), torch.arange(T, device="cuda", dtype=torch.int32), 0.0, out)
    clear = (top.values[:, 0] - top.values[:, 1]).cpu() > 2 * bound.max(dim=1).values
    assert clear.float().mean() > 0.9
    assert torch.equal(out.argmax.cpu()[clear], tokens.cpu()[clear])
    assert torch.all(out.margin.cpu()[clear] >= 0)


def test_capture_and_replay():
    """A captured run of the operators, replayed on other inputs in the same buffers, gives what the calls give."""
    T, d, V, fmt = 200, 416, 1000, 4
    x, r = torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    Wb = randn(V, d, seed=1).bfloat16().cuda()

    def make():
        return (difr.NormOut(h=torch.empty_like(x), residual=torch.empty_like(x), mx=difr.MxTensor.allocate(T, d, fmt)),
                difr.MxTensor.allocate(V, d, fmt), torch.empty(T, V, device="cuda"), torch.empty_like(x))

    def run(o, W, logits, back):
        difr.difr_mx_quantize(Wb, W)
        difr.difr_rms_norm(x, w, 1e-6, o, residual=r)
        difr.difr_mx_logits(o.mx, W, logits)
        difr.difr_mx_dequantize(o.mx, back)

    x.copy_(randn(T, d, seed=2)); r.copy_(randn(T, d, seed=3))
    a, b = make(), make()
    run(*a)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):  # two graphs of the same work, replayed one after the other
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(*a)
        graphs.append(g)
    for seed in (5, 6, 7):
        x.copy_(randn(T, d, seed=seed)); r.copy_(randn(T, d, seed=seed + 10)); Wb.copy_(randn(V, d, seed=seed + 20))
        for g in graphs:
            g.replay()
        run(*b)
        torch.cuda.synchronize()
        for p, q in zip((a[0].h, a[0].residual, a[0].mx.codes, a[0].mx.scales, a[2], a[3]),
                        (b[0].h, b[0].residual, b[0].mx.codes, b[0].mx.scales, b[2], b[3])):
            assert torch.equal(p, q)


def test_two_streams_at_once():
    """Calls on two streams, and on a stream that is not the current one, each with buffers of their own."""
    T, d, V = 500, 1024, 30000
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    sets = []
    for k, fmt in enumerate((4, 8)):
        h, hv = random_mx(T, d, fmt, seed=k)
        W, Wv = random_mx(V, d, fmt, seed=10 + k)
        sets.append((h, W, torch.empty(T, V, device="cuda"), difr.difr_mx_logits(h, W, torch.empty(T, V, device="cuda"))))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (h, W, out, _) in zip(streams, sets):
            difr.difr_mx_logits(h, W, out, stream=s)
    torch.cuda.synchronize()
    for _, _, out, want in sets:
        assert torch.equal(out, want)


def test_repeated_calls_give_the_same_bits():
    for fmt in (4, 8):
        T, d, V = 700, 1000, 5000
        x, w = randn(T, d, seed=1).cuda(), torch.ones(d, device="cuda")
        W = difr.difr_mx_quantize(randn(V, d, seed=2).cuda(), difr.MxTensor.allocate(V, d, fmt))
        first = None
        for _ in range(30):
            o = difr.NormOut(h=torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), mx=difr.MxTensor.allocate(T, d, fmt))
            difr.difr_rms_norm(x, w, 1e-6, o)
            out = difr.difr_mx_logits(o.mx, W, torch.empty(T, V, device="cuda"))
            now = (o.h, o.mx.codes, o.mx.scales, out)
            first = first or now
            assert all(torch.equal(p, q) for p, q in zip(now, first))


@pytest.mark.parametrize("fmt", [4, 8])
def test_a_row_does_not_depend_on_its_batch(fmt):
    """The same rows alone, in small and in large batches: the same bits from the norm and from the product."""
    d, V = 1504, 3000
    x, r = randn(2000, d, seed=1).bfloat16().cuda(), randn(2000, d, seed=2, std=2.0).bfloat16().cuda()
    w = (1 + 0.1 * randn(d, seed=3)).bfloat16().cuda()
    W = difr.difr_mx_quantize(randn(V, d, seed=4).cuda(), difr.MxTensor.allocate(V, d, fmt))

    def run(T):
        o = difr.NormOut(h=torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), mx=difr.MxTensor.allocate(T, d, fmt))
        difr.difr_rms_norm(x[:T], w, 1e-6, o, residual=r[:T])
        return o.h, o.mx.codes, difr.difr_mx_logits(o.mx, W, torch.empty(T, V, device="cuda"))

    full = run(2000)
    for T in (1, 2, 17, 33, 65, 129, 300, 700):
        for part, whole in zip(run(T), full):
            assert torch.equal(part, whole[:T]), T


def test_empty_batches():
    d, V = 64, 300
    x = torch.empty(0, d, device="cuda")
    mx = difr.MxTensor.allocate(0, d, 4)
    difr.difr_mx_quantize(x, mx)
    difr.difr_mx_dequantize(mx, x)
    difr.difr_rms_norm(x, torch.ones(d, device="cuda"), 1e-6, difr.NormOut(h=torch.empty(0, d, dtype=torch.bfloat16, device="cuda"), mx=mx))
    W, _ = random_mx(V, d, 4, seed=1)
    difr.difr_mx_logits(mx, W, torch.empty(0, V, device="cuda"))
    torch.cuda.synchronize()


def test_the_binding_refuses_what_does_not_fit():
    d = 64
    x = torch.zeros(8, d, device="cuda")
    w = torch.ones(d, device="cuda")
    h16 = torch.empty(8, d, dtype=torch.bfloat16, device="cuda")
    mx = difr.MxTensor.allocate(8, d, 4)
    W = difr.MxTensor.allocate(100, d, 4)
    logits = torch.empty(8, 100, device="cuda")
    bad = [
        lambda: difr.difr_mx_quantize(x.double(), mx),
        lambda: difr.difr_mx_quantize(x.cpu(), mx),
        lambda: difr.difr_mx_quantize(x[0], mx),
        lambda: difr.difr_mx_quantize(x[:4], mx),
        lambda: difr.difr_mx_quantize(x.t(), difr.MxTensor.allocate(d, 8, 4)),
        lambda: difr.difr_mx_quantize(x[:1].expand(8, d), mx),
        lambda: difr.difr_mx_quantize(x, difr.MxTensor(mx.codes, mx.scales, 8, 8, d)),
        lambda: difr.difr_mx_quantize(x, difr.MxTensor(mx.codes, mx.scales[:-1], 4, 8, d)),
        lambda: difr.difr_mx_quantize(x, difr.MxTensor(mx.codes.cpu(), mx.scales, 4, 8, d)),
        lambda: difr.difr_mx_quantize(x, difr.MxTensor(mx.codes, mx.scales, 6, 8, d)),
        lambda: difr.difr_mx_dequantize(mx, x.half()),
        lambda: difr.difr_mx_dequantize(mx, x[:, :32]),
        lambda: difr.difr_rms_norm(x, w, 1e-6, difr.NormOut(h=x)),                       # h is bf16
        lambda: difr.difr_rms_norm(x, w.bfloat16(), 1e-6, difr.NormOut(h=h16)),
        lambda: difr.difr_rms_norm(x, w[:32], 1e-6, difr.NormOut(h=h16)),
        lambda: difr.difr_rms_norm(x, w, 1e-6, difr.NormOut(h=h16), residual=x.bfloat16()),
        lambda: difr.difr_rms_norm(x, w, 1e-6, difr.NormOut(h=h16), residual=x[:4]),
        lambda: difr.difr_rms_norm(x, w, 1e-6, difr.NormOut(mx=W)),
        lambda: difr.difr_mx_logits(mx, difr.MxTensor.allocate(100, d, 8), logits),      # mixed formats
        lambda: difr.difr_mx_logits(mx, difr.MxTensor.allocate(100, 32, 4), logits),
        lambda: difr.difr_mx_logits(mx, W, logits.half()),
        lambda: difr.difr_mx_logits(mx, W, logits[:, :99]),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(TypeError):
            call()
            pytest.fail(f"call {k} was accepted")
    refused = [
        lambda: difr.difr_rms_norm(x, w, 0.0, difr.NormOut(h=h16)),
        lambda: difr.difr_rms_norm(x, w, math.nan, difr.NormOut(h=h16)),
        lambda: difr.difr_rms_norm(x, w, 1e-6, difr.NormOut()),                           # nothing asked for
        lambda: difr.difr_rms_norm(x, w, 1e-6, difr.NormOut(h=h16, residual=x)),          # a stream without a residual
        lambda: difr.difr_rms_norm(torch.zeros(1, 32776, device="cuda"), torch.ones(32776, device="cuda"), 1e-6,
                                   difr.NormOut(h=torch.empty(1, 32776, dtype=torch.bfloat16, device="cuda"))),
    ]
    for call in refused:
        with pytest.raises(difr.DifrError):
            call()
    unaligned = torch.empty(8 * 32 + 1, dtype=torch.uint8, device="cuda")[1:].view(8, 32)
    with pytest.raises(difr.DifrError):
        difr.difr_mx_quantize(x, difr.MxTensor(unaligned, mx.scales, 4, 8, d))
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", [4, 8])
@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
def test_logits_at_every_alignment_of_their_rows(out_dtype, fmt):
    """First elements at every place inside 16 bytes, strides that move it from row to row, vocabularies that end anywhere
    inside a block of 128 ids: all values are there and their neighbours are left alone."""
    dt = DTYPES[out_dtype]
    T, d = 261, 64
    h, hv = random_mx(T, d, fmt, seed=1)
    for k, (V, pad) in enumerate([(256, 0), (257, 0), (383, 1), (385, 2), (130, 3), (255, 5), (512, 7), (640, 1), (769, 0),
                                  (5120, 0), (5121, 0), (4991, 1), (4993, 2), (5119, 5), (4866, 6)]):
        W, Wv = random_mx(V, d, fmt, seed=2 + k)
        exact, bound = logits_bound(hv, Wv, fmt, dt)
        for off in (0, 1, 3, 6):
            flat = torch.full((T * (V + pad) + 64,), -7.0, dtype=dt, device="cuda")
            out = torch.as_strided(flat, (T, V), (V + pad, 1), off)
            difr.difr_mx_logits(h, W, out)
            assert torch.all((out.cpu().double() - exact).abs() <= bound)
            out.fill_(-7.0)
            assert torch.all(flat == -7.0)


# ------------------------------------------------------------------ the ends of fp32's range
@pytest.mark.parametrize("d", [1, 520, 1001, 32768])
def test_eps_counts_in_rows_whose_squares_leave_fp32(d):
    """Any finite eps: as large as squares beyond 3.4e38, and so large that the mean and it leave fp32 together."""
    scale = torch.tensor([1e-10, 1.0, 1e17, 3e18, 1.7e19, 2e19, 1e21, 1e30, 1e37])
    x = (0.5 + torch.rand(scale.numel(), d, generator=torch.Generator().manual_seed(d))) * scale.view(-1, 1)
    x[:, ::2] *= -1
    w = 1 + 0.2 * randn(d, seed=3)
    for eps in (1e-6, 1e10, 1e30, 1e34, 1e36, 1e38, 2e38, 3.4e38):
        h = torch.empty(scale.numel(), d, dtype=torch.bfloat16, device="cuda")
        difr.difr_rms_norm(x.cuda(), w.cuda(), eps, difr.NormOut(h=h))
        _, y = ref.rms_norm(x, None, w, eps)
        assert_close_h(h, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 520, 1001, 9000])
def test_rows_whose_squares_are_subnormal(d, dtype):
    """With an eps that is smaller still the formula holds down to the smallest numbers; zero rows stay zero."""
    scale = torch.tensor([0.0, 1e-44, 1e-40, 1e-30, 1e-24, 1e-22, 1e-21, 1e-20, 1e-19, 1e-15, 1e-10, 1.0])
    x = (0.5 + torch.rand(scale.numel(), d, generator=torch.Generator().manual_seed(d))) * scale.view(-1, 1)
    x[:, ::2] *= -1
    x = x.to(DTYPES[dtype])
    w = (1 + 0.2 * randn(d, seed=3)).to(DTYPES[dtype])
    for eps in (1e-45, 1e-42, 1e-40, 1e-36, 1e-31, 1e-29, 1e-6):
        h = torch.empty(scale.numel(), d, dtype=torch.bfloat16, device="cuda")
        mx = mx_of(scale.numel(), d, 8)
        difr.difr_rms_norm(x.cuda(), w.cuda(), eps, difr.NormOut(h=h, mx=mx))
        _, y = ref.rms_norm(x, None, w, eps)
        assert_close_h(h, y)
        assert torch.all(h[0] == 0)
        keep = y.abs().amax(1) > 1e-30  # (below, y itself is close to fp32's subnormal numbers)
        got = difr.difr_mx_dequantize(mx, torch.empty(scale.numel(), d, device="cuda")).cpu().double()
        top = ref.blocks(y).abs().amax(-1, keepdim=True).expand(-1, -1, 32).flatten(1)[:, :d]
        # e4m3: half a step is 2^-4 of the value, 448 for up to 512 is 2^-3; among its subnormals half a step is 2^-10 of
        # the scale, which is at most 2^-8 of the block's largest
        assert torch.all(((got - y).abs() <= (2.0 ** -3 + 2 * Y_ERR) * y.abs() + 2.0 ** -18 * (1 + Y_ERR) * top)[keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [700, 1001, 20000])
def test_small_values_in_huge_and_tiny_rows(d, dtype):
    """Values of all magnitudes beside those that fix the root: y is as exact as anywhere while it is a normal number."""
    x = torch.exp2(torch.rand(6, d, generator=torch.Generator().manual_seed(d)) * 110 - 100)
    x[0] = torch.exp2(torch.rand(d, generator=torch.Generator().manual_seed(d + 1)) * 20 - 70)
    x[:, 0] = torch.tensor([3e19, 1e21, 1e30, 1e38, 1e-25, 1e-30])
    x[4:, 1:] *= 2.0 ** -95
    x[4:] = x[4:].clamp(max=1e-25)
    x = x.to(DTYPES[dtype])
    w = (1 + 0.2 * randn(d, seed=3)).to(DTYPES[dtype])
    h = torch.empty(6, d, dtype=torch.bfloat16, device="cuda")
    difr.difr_rms_norm(x.cuda(), w.cuda(), 1e-42, difr.NormOut(h=h))
    _, y = ref.rms_norm(x, None, w, 1e-42)
    assert w.abs().max() < 2  # r / sqrt(..) is a normal number, too
    normal = y.abs() > 2.0 ** -125
    assert normal[:4].any(1).all()
    err = (h.double().cpu() - y).abs()
    assert torch.all((err <= (2.0 ** -8 + Y_ERR * (1 + 2.0 ** -8)) * y.abs())[normal])


# ------------------------------------------------------------------ waits that run out
@pytest.mark.parametrize("fmt", [4, 8])
@pytest.mark.parametrize("T,V,d,ld,out_dtype", [
    (600, 9800, 160, 9800, "bf16"), (600, 9801, 160, 9801, "f32"), (300, 1100, 160, 1104, "f32"), (40, 9800, 96, 9803, "bf16"),
    (20, 50000, 96, 50000, "bf16"), (7, 30000, 96, 30000, "f32"), (2700, 9800, 1 << 20, 9800, "bf16")])
def test_logits_that_a_wait_keeps_from_being_computed_are_nan(T, V, d, ld, out_dtype, fmt):
    """The way out of the product's epilogue after waits that ran out, at every tile width: the warps of a half give up
    together, all logits but those of the finished tiles are NaN, the status word says so, and the next call is as good
    as ever."""
    buf = torch.full((T + 1, ld), -7.0, dtype=DTYPES[out_dtype], device="cuda")
    part = buf[:T, :V]
    left = []
    for done in (0, 1, 2, 3, 1000):
        buf.fill_(-7.0)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        difr.difr_selftest_mx_wait(fmt, d, part, done, 1_000_000, status)
        nan = torch.isnan(part)
        assert int(status.item()) == (0 if done == 1000 else -7 if bool(nan.any()) else 0)
        assert torch.all(part[~nan] == -7.0)
        assert torch.all(buf[:T, V:] == -7.0) and torch.all(buf[T:] == -7.0)
        left.append(~nan)
        buf.fill_(-7.0)
        difr.difr_selftest_mx_wait(fmt, d, part, done, 1_000_000)  # no status word: the logits tell
        assert torch.equal(torch.isnan(part), nan)
    assert not left[0].any() and left[-1].all()
    width = 256 if T > 128 and (V + 255) // 256 * ((T + 255) // 256) > 37 else 128 if T > 64 else 64 if T > 32 else 32 if T > 16 else 16
    for less, more in zip(left, left[1:]):
        new = more & ~less
        assert not (less & ~more).any()
        # whole tiles, at most one for every pair of the 74
        rows = torch.nn.functional.pad(new, (0, -V % 256, 0, -T % width)).view(-1, width, (V + 255) // 256, 256)
        tiles = rows.any(3).any(1)
        assert more.all() or int(tiles.sum()) <= 74
        inside = torch.nn.functional.pad(torch.ones_like(new), (0, -V % 256, 0, -T % width)).view_as(rows)
        assert torch.equal(rows, inside & tiles.view(-1, 1, tiles.shape[1], 1))
    h, _ = random_mx(70, 96, fmt, seed=1)
    W, _ = random_mx(1000, 96, fmt, seed=2)
    want = difr.difr_mx_logits(h, W, torch.empty(70, 1000, device="cuda"))
    assert not torch.isnan(want).any()


# ------------------------------------------------------------------ long rows, several raster groups, heads beyond L2
def exact_mx(rows, d, fmt, seed):
    """Values of the 4-bit format under scales 1/2 .. 2, made on the GPU: (MxTensor, the values it holds exactly)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.randint(0, 16, (rows, d), generator=g, device="cuda", dtype=torch.uint8)
    v = ref.table(4).float().cuda()[(c & 7).int()] * (1 - 2 * (c >> 3).float())
    e = torch.randint(-1, 2, (rows, (d + 31) // 32), generator=g, device="cuda").float()
    v *= torch.exp2(e).repeat_interleave(32, 1)[:, :d]
    mx = difr.difr_mx_quantize(v, difr.MxTensor.allocate(rows, d, fmt))
    assert torch.equal(difr.difr_mx_dequantize(mx, torch.empty_like(v)), v)
    return mx, v


@pytest.mark.parametrize("T,d,V,fmt", [
    (1300, 131072, 2500, 4),   # 6 token tiles in groups of 2
    (1100, 131072, 2500, 4),   # 5: the last group has one
    (1300, 65536, 2500, 8),
    (1100, 65537, 2500, 8),
    (600, 262177, 4100, 4),    # groups of one tile
    (300, 1 << 20, 700, 4),    # the longest rows, tiles of 128 tokens
    (300, 1 << 20, 700, 8),
    (48, 1024, 110000, 8),     # one token tile, heads that L2 does not hold
    (5, 2048, 120007, 4),
    (48, 2048, 110001, 8),
])
def test_logits_of_long_rows_and_large_heads_are_exact(T, d, V, fmt):
    """Every product is a multiple of 1/16 and a row's sums stay far below 2^20 (the products' deviation is below 24, and
    2^20 terms make 2.5e4): each partial sum fits fp32, so any error is a misplaced tile, code or scale."""
    h, hv = exact_mx(T, d, fmt, seed=1)
    W, Wv = exact_mx(V, d, fmt, seed=2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = difr.difr_mx_logits(h, W, torch.full((T, V), math.nan, device="cuda"), status)
    assert int(status.item()) == 0
    want = torch.zeros(T, V, dtype=torch.float64, device="cuda")
    for k in range(0, d, 65536):
        want += hv[:, k:k + 65536].double() @ Wv[:, k:k + 65536].double().T
    assert float(want.abs().max()) < 2.0 ** 20
    assert torch.equal(out.double(), want)


# ------------------------------------------------------------------ the norm's steps
# Relative error of y: a group of eight squares passes four roundings along two chains and one where they meet, the
# groups are joined in 64 bits; the cast, 1 / d, the mean and + eps make four more; the root halves the nine.  rsqrtf is
# within 2 units in the last place (four of 2^-24), two products follow: 10.5 of 2^-24, and 0.5 for terms of second order.
Y_STEPS = 11 * 2.0 ** -24


@pytest.mark.parametrize("fmt", [4, 8])
@pytest.mark.parametrize("T,d,dtype", [(400, 5120, "bf16"), (300, 8192, "f32"), (900, 1749, "f32"), (60, 32768, "bf16")])
def test_codes_differ_from_the_exact_rows_next_to_a_border_only(T, d, dtype, fmt):
    """Codes lie between those of y (1 - Y_STEPS) and y (1 + Y_STEPS); rows of one large and many small squares, each
    lost beside the large one in 32 bits, among them."""
    x = randn(T, d, seed=1)
    x[::3] = 2.0 ** -12 * (1 + 0.25 * torch.rand(x[::3].shape, generator=torch.Generator().manual_seed(2)))
    x[::3, 0] = 1.0
    x = x.to(DTYPES[dtype])
    w = (1 + 0.2 * randn(d, seed=3)).to(DTYPES[dtype])
    mx = mx_of(T, d, fmt)
    difr.difr_rms_norm(x.cuda(), w.cuda(), 1e-6, difr.NormOut(mx=mx))
    _, y = ref.rms_norm(x, None, w, 1e-6)
    nb = (d + 31) // 32
    byte = ref.untile_scales(mx.scales.cpu(), T, nb)
    low, high = (ref.quantize(y * f, fmt) for f in (1 - Y_STEPS, 1 + Y_STEPS))
    assert torch.all((byte == low[1]) | (byte == high[1]))
    sure = (low[1] == high[1]).unsqueeze(-1).expand(-1, -1, 32).flatten(1)  # (two scales: codes of two grids)
    assert sure.double().mean() > 0.999
    mag = 2 ** (fmt - 1) - 1
    c = ref.unpack(mx.codes.cpu(), fmt)
    assert torch.equal((c >> (fmt - 1))[sure], (low[0] >> (fmt - 1))[sure])
    assert torch.all((((c & mag) >= (low[0] & mag)) & ((c & mag) <= (high[0] & mag)))[sure])
    assert ((low[0] != high[0]) & sure).sum() <= 1e-4 * c.numel()
