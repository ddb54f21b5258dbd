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
                                    (7, 4096), (1, 8192)])
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
@pytest.mark.parametrize("rows,d,ld", [(1, 1, 1), (3, 31, 40), (129, 256, 256), (70, 1749, 1749), (5, 4096, 4104)])
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
                                          (5, 1749, True), (17, 2048, False), (33, 5120, True), (2, 9001, True),
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
    for pad, off in ((8, 0), (7, 0), (16, 8), (9, 3)):
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
                                   (256, 256, 256), (300, 1749, 515), (513, 640, 2049)])
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
                                   (129, 1000, 511), (260, 5120, 1025), (1000, 333, 4097)])
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
