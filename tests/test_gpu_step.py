"""A decoding step's operators on the GPU: block norm, 4-bit head with group scales, verification of drafted tokens; each
against the plain 64-bit statement in step_reference.py."""
import math

import pytest
import torch

import paper_2511_02620_b200 as difr
import step_reference as ref
from test_gpu_mx import assert_mx_nearest

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF = {k: torch.finfo(v).eps / 2 for k, v in DTYPES.items()}


def randn(*shape, seed=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g) * std


# ------------------------------------------------------------------ block norm
# Relative error of a normed value in fp32: the final norm's (69 additions and 6 more roundings, halved by the root where they
# are under it: test_gpu_mx.py) and the addition of the offset.
N_ERR = (32 + 37) / 2 * 2.0 ** -24 + 7 * 2.0 ** -24


def run_block(x, residual, weight, eps, post_weight=None, post_eps=None, gate=None, fmt=0, h=True, stream=True, **kw):
    T, d = x.shape
    c = lambda t: None if t is None else t.cuda()
    out = difr.NormOut(h=torch.full((T, d), 7.0, dtype=torch.bfloat16, device="cuda") if h else None,
                       residual=torch.full((T, d), 7.0, dtype=x.dtype, device="cuda") if stream else None,
                       mx=difr.MxTensor.allocate(T, d, fmt) if fmt else None)
    difr.difr_block_norm(c(x), c(residual), c(weight), eps, out, post_weight=c(post_weight), post_eps=post_eps, gate=c(gate), **kw)
    return out


def check_stream(got, x, residual, dtype, post_weight=None, post_eps=1e-6, gate=None, scale=1.0, residual_scale=1.0,
                 weight_offset=0.0):
    want, size = ref.block_stream(x, residual, post_weight, post_eps, gate, scale, residual_scale, weight_offset)
    # fp32: the normed value, two or three products and the sum (one rounding each); then the type's rounding
    fp32 = (N_ERR + 4 * 2.0 ** -24) * size
    err = (got.double().cpu() - want).abs()
    tiny = 2.0 ** -25 if dtype == "f16" else 2.0 ** -134
    assert torch.all(err <= fp32 + HALF[dtype] * (want.abs() + fp32) + tiny)


def check_h(h, stream, weight, eps, offset=0.0):
    y = ref.rms(stream.double().cpu(), eps) * (weight.double() + ref.f32(offset))
    # (an offset near the weight's opposite cancels: its rounding counts by the sizes)
    size = ref.rms(stream.double().cpu(), eps).abs() * (weight.double().abs() + abs(offset))
    err = (h.double().cpu() - y).abs()
    assert torch.all(err <= 2.0 ** -8 * y.abs() + N_ERR * (1 + 2.0 ** -8) * size + 2.0 ** -134)


def block_inputs(T, d, dtype, gate):
    dt = DTYPES[dtype]
    x, r = randn(T, d, seed=1).to(dt), randn(T, d, seed=2, std=3.0).to(dt)
    w, pw = (1 + 0.2 * randn(d, seed=3)).to(dt), (1 + 0.2 * randn(d, seed=4)).to(dt)
    g = {"none": None, "channel": torch.tanh(randn(1, d, seed=5)).to(dt), "token": torch.tanh(randn(T, d, seed=5)).to(dt)}[gate]
    return x, r, w, pw, g


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("T,d,gate,fmt", [(1, 1, "none", 0), (1, 4096, "channel", 0), (3, 100, "token", 8), (9, 31, "channel", 4),
                                          (130, 160, "token", 0), (5, 1749, "token", 4), (9, 70, "none", 0), (7, 1030, "channel", 8),
                                          (17, 2048, "token", 0), (3, 5120, "none", 4), (2, 9001, "token", 0),
                                          (1, 32768, "token", 8), (3, 16384, "none", 0), (2, 6002, "channel", 0)])
def test_block_norm(T, d, gate, fmt, post, dtype):
    x, r, w, pw, g = block_inputs(T, d, dtype, gate)
    kw = dict(scale=0.22, residual_scale=1.5, weight_offset=0.25)
    out = run_block(x, r, w, 1e-6, pw if post else None, 1e-5, g, fmt, **kw)
    check_stream(out.residual, x, r, dtype, pw if post else None, 1e-5, g, **kw)
    check_h(out.h, out.residual, w, 1e-6, 0.25)
    if fmt:
        plain = run_block(x, r, w, 1e-6, pw if post else None, 1e-5, g, 0, **kw)
        assert torch.equal(plain.residual, out.residual) and torch.equal(plain.h, out.h)
        # (that check allows twice the final norm's error, which is more than the offset's one rounding adds)
        assert_mx_nearest(out.mx, ref.rms(out.residual.double().cpu(), 1e-6) * (w.double() + 0.25), fmt)


def test_block_norm_equals_the_final_norm_where_they_meet():
    """Without a norm after the block, gate and scales: bit for bit difr_rms_norm with the residual's addition."""
    for T, d, dtype in ((5, 4096, "bf16"), (9, 1749, "f32"), (130, 256, "f16")):
        x, r, w, _, _ = block_inputs(T, d, dtype, "none")
        for fmt in (8, 4):
            out = run_block(x, r, w, 1e-6, fmt=fmt)
            o = difr.NormOut(h=torch.empty_like(out.h), residual=torch.empty_like(out.residual), mx=difr.MxTensor.allocate(T, d, fmt))
            difr.difr_rms_norm(x.cuda(), w.cuda(), 1e-6, o, residual=r.cuda())
            for a, b in ((out.h, o.h), (out.residual, o.residual), (out.mx.codes, o.mx.codes), (out.mx.scales, o.mx.scales)):
                assert torch.equal(a, b)


def test_block_norm_stream_alone():
    x, r, w, pw, g = block_inputs(7, 640, "bf16", "token")
    both = run_block(x, r, w, 1e-6, pw, None, g, scale=0.5)
    alone = run_block(x, r, None, 1e-6, pw, None, g, h=False, scale=0.5)
    assert torch.equal(both.residual, alone.residual)
    no_stream = run_block(x, r, w, 1e-6, pw, None, g, stream=False, scale=0.5)
    assert torch.equal(both.h, no_stream.h)


def test_block_norm_in_place_and_strided():
    """The stream over the residual or over x, h over x; rows apart from each other, a gate row without a stride."""
    T, d, ld = 37, 1032, 1040
    x, r, w, pw, g = block_inputs(T, d, "bf16", "channel")
    want = run_block(x, r, w, 1e-6, pw, None, g)
    place = lambda t: torch.as_strided(torch.full((T * ld,), -3.0, dtype=t.dtype, device="cuda"), (T, d), (ld, 1)).copy_(t.cuda())
    for over in ("residual", "x"):
        xs, rs = place(x), place(r)
        out = difr.NormOut(h=xs if over == "residual" else rs, residual=rs if over == "residual" else xs)
        difr.difr_block_norm(xs, rs, w.cuda(), 1e-6, out, post_weight=pw.cuda(), gate=g.cuda())
        assert torch.equal(out.h, want.h) and torch.equal(out.residual, want.residual)
        assert torch.all(torch.as_strided(xs, (T - 1, ld - d), (ld, 1), xs.storage_offset() + d) == -3.0)
    gates = g.expand(T, d).contiguous()
    assert torch.equal(run_block(x, r, w, 1e-6, pw, None, gates).h, want.h)


@pytest.mark.parametrize("d", [128, 4096, 1749])
def test_block_norm_rows_do_not_notice_their_batch(d):
    x, r, w, pw, g = block_inputs(33, d, "bf16", "token")
    cut = lambda t, i: t.cuda()[i:i + 1]
    out = lambda n: difr.NormOut(h=torch.empty(n, d, dtype=torch.bfloat16, device="cuda"))
    whole, one = out(33), out(1)
    difr.difr_block_norm(x.cuda(), r.cuda(), w.cuda(), 1e-6, whole, post_weight=pw.cuda(), gate=g.cuda())
    for i in (0, 7, 32):
        difr.difr_block_norm(cut(x, i), cut(r, i), w.cuda(), 1e-6, one, post_weight=pw.cuda(), gate=cut(g, i))
        assert torch.equal(one.h[0], whole.h[i])


def test_block_norm_rows_at_the_ends_of_fp32():
    """Blocks whose squares leave fp32's range or its normal numbers, zero rows, rows with a NaN or an infinity."""
    d = 512
    x, r, w, pw, _ = block_inputs(8, d, "f32", "none")
    x[0] *= 1e25
    x[1] *= 1e-30
    x[2] = 0.0
    x[3] *= 3e38 / 8
    x[4, 5] = math.nan
    x[5, 9] = math.inf
    r[6] *= 1e25
    out = run_block(x, r, w, 1e-6, pw, 1e-45)
    good = torch.tensor([0, 1, 2, 3, 6, 7])
    check_stream(out.residual[good.cuda()], x[good], r[good], "f32", pw, 1e-45)
    check_h(out.h[good.cuda()], out.residual[good.cuda()], w, 1e-6)
    assert torch.isnan(out.h[4]).all() and torch.isnan(out.residual[4]).all()
    assert torch.isnan(out.residual[5, 9]) and torch.equal(out.residual[5, :9].cpu(), r[5, :9])


def test_block_norm_refusals():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = difr.NormOut(h=torch.empty_like(x))
    for bad in (dict(gate=torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda")), dict(gate=x.float()), dict(gate=w),
                dict(post_weight=w.float()), dict(post_weight=w[:32]), dict(gate=x.cpu())):
        with pytest.raises(TypeError):
            difr.difr_block_norm(x, x, w, 1e-6, out, **bad)
    with pytest.raises(TypeError):
        difr.difr_block_norm(x, x[:2], w, 1e-6, out)
    for bad in (dict(scale=math.nan), dict(residual_scale=math.inf), dict(weight_offset=-math.inf), dict(post_weight=w, post_eps=0.0)):
        with pytest.raises(difr.DifrError) as e:
            difr.difr_block_norm(x, x, w, 1e-6, out, **bad)
        assert e.value.status == -1
    for weight, o in ((None, out), (w, difr.NormOut(residual=torch.empty_like(x))), (None, difr.NormOut())):
        with pytest.raises(difr.DifrError):
            difr.difr_block_norm(x, x, weight, 1e-6, o)
    empty = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    difr.difr_block_norm(empty, empty, w, 1e-6, difr.NormOut(h=empty))
