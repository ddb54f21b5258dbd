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


# ------------------------------------------------------------------ verification of drafted tokens
def make_drafts(B, K, V, dtype, probs, temperature, seed=0, ragged=True, near=0.6):
    """Target logits, drafts sampled near them, words; `temperature` per request or one for all."""
    g = torch.Generator().manual_seed(seed)
    n = [int(torch.randint(0, K + 1, (1,), generator=g)) if ragged else K for _ in range(B)]
    off = torch.tensor([0] + n).cumsum(0).to(torch.int32)
    D = int(off[-1])
    logits = (2.5 * torch.randn(D + B, V, generator=g)).to(DTYPES[dtype])
    t = torch.as_tensor(temperature, dtype=torch.float32).expand(B)
    drafted = torch.zeros(D, dtype=torch.int32)
    q = torch.zeros(D, V)
    for b in range(B):
        for j in range(n[b]):
            i = int(off[b]) + j
            z = (logits[i + b].float() + near * torch.randn(V, generator=g)) / (float(t[b]) or 0.5)
            q[i] = torch.softmax(z, 0)
            drafted[i] = int(torch.multinomial(q[i], 1, generator=g))
    words = lambda k: torch.randint(-2 ** 31, 2 ** 31, (k,), generator=g, dtype=torch.int64).to(torch.int32)
    return dict(logits=logits, drafted=drafted, offsets=off, accept=words(D), sample=words(B), t=t, K=K,
                probs=q if probs else None)


def run_verify(s, out=None, **kw):
    B, D, V = s["sample"].numel(), s["drafted"].numel(), s["logits"].shape[1]
    if out is None:
        out = difr.DraftOut.allocate(B, D, s["K"], V)
        for x in (out.tokens, out.n_accepted, out.status):
            x.fill_(-77)
        out.p_draft.fill_(math.nan)
        out.workspace.fill_(0xAB)
    t = s["t"]
    one = float(t[0]) if B and torch.all(t == t[0]) else t.contiguous().cuda()
    c = lambda x: None if x is None else x.cuda()
    return difr.difr_verify_drafts(c(s["logits"]), c(s["drafted"]), c(s["offsets"]), c(s["accept"]), c(s["sample"]), one, out,
                                   draft_probs=c(s["probs"]), **kw)


def check_verify(s, out=None):
    out = run_verify(s) if out is None else out
    tokens, n, p, status = ref.verify(s["logits"], s["drafted"], s["offsets"], s["accept"], s["sample"], s["t"], s["K"], s["probs"])
    assert torch.equal(out.n_accepted.cpu(), n)
    assert torch.equal(out.tokens.cpu(), tokens)
    assert torch.equal(out.status.cpu(), status)
    got = out.p_draft.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(p))
    err = (got - p).abs()
    assert torch.all(torch.isnan(p) | (err <= 2.0 ** -16 * p + 2.0 ** -149))
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("temperature", [0.0, 0.7, 1.0, 8.0])
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("B,K,V", [(1, 0, 1), (1, 1, 2), (5, 3, 7), (9, 4, 33), (64, 5, 1000), (3, 4, 4096), (4, 2, 8193), (7, 8, 32003)])
def test_verification(B, K, V, probs, temperature, dtype):
    check_verify(make_drafts(B, K, V, dtype, probs, temperature, seed=B + V))


@pytest.mark.parametrize("B,K,V,dtype", [(2, 3, 151937, "bf16"), (1, 4, 128256, "f32"), (1, 1, 1000003, "f16")])
def test_verification_of_large_vocabularies(B, K, V, dtype):
    check_verify(make_drafts(B, K, V, dtype, True, 1.0, seed=V, ragged=False))


def test_many_requests_of_one_draft_each_and_the_longest_drafts():
    check_verify(make_drafts(3000, 1, 50, "f32", True, 1.0, seed=1))
    check_verify(make_drafts(2, 255, 40, "f32", True, 1.0, seed=2, ragged=False, near=0.01))


def test_a_temperature_per_request():
    """Zero, small and large ones in one batch, and values that are none."""
    t = torch.tensor([0.0, 0.1, 1.0, 30.0, -1.0, math.nan, math.inf, 1e-40, 1e30, 0.5])
    s = make_drafts(10, 4, 1003, "f32", True, t.nan_to_num(1.0, 1.0).clamp(min=0), seed=3)
    s["t"] = t
    out = check_verify(s)
    assert out.status.tolist() == [0, 0, 0, 0, 8, 8, 8, 0, 0, 0]


def test_acceptance_next_to_the_border():
    """Draft probabilities within 2^-22 of p / mu, on both sides: decided as in 64 bits."""
    B, V = 400, 5000
    s = make_drafts(B, 1, V, "f32", True, 1.0, seed=4, ragged=False)
    side = 0
    for b in range(B):
        p = ref.probabilities(s["logits"][2 * b], 1.0)
        x = int(s["drafted"][b])
        s["probs"][b, x] = float(p[x]) / ref.uniform(s["accept"][b]) * (1 + (-1) ** b * 2.0 ** -22)
    out = check_verify(s)
    assert 150 < int(out.n_accepted.sum()) < 250


def test_samples_next_to_the_borders_of_ids():
    """Equal logits: id i ends at (i + 1) / V.  Words one below and one above that border."""
    V = 4096
    at = torch.tensor([0, 1, 17, 511, 512, 513, 2047, 3000, 4094])
    word = ((at + 1) * (2 ** 32 // V)).repeat_interleave(2) - torch.tensor([1, 0]).repeat(at.numel())
    word = torch.where(word >= 2 ** 31, word - 2 ** 32, word).to(torch.int32)
    B = word.numel()
    s = dict(logits=torch.full((B, V), 3.25), drafted=torch.zeros(0, dtype=torch.int32), offsets=torch.zeros(B + 1, dtype=torch.int32),
             accept=torch.zeros(0, dtype=torch.int32), sample=word, t=torch.ones(B), K=0, probs=None)
    out = check_verify(s)
    assert out.tokens[:, 0].tolist() == [v for i in at.tolist() for v in (i, i + 1)]


def test_extreme_words():
    """The smallest and the largest word: first and last id with any probability left."""
    V = 3000
    logits = torch.full((4, V), -math.inf)
    logits[:, 100:2900] = randn(4, 2800, seed=6)
    s = dict(logits=logits, drafted=torch.zeros(0, dtype=torch.int32), offsets=torch.zeros(5, dtype=torch.int32),
             accept=torch.zeros(0, dtype=torch.int32), sample=torch.tensor([0, -1, 0, -1], dtype=torch.int32), t=torch.ones(4), K=0,
             probs=None)
    out = check_verify(s)
    assert out.tokens[:, 0].tolist() == [100, 2899, 100, 2899]


def test_masked_and_broken_rows():
    """Rows of masked ids, a single finite id, the type's lowest value as a mask; NaN, +infinity and nothing but -infinity stop a
    request where it reaches them, and only there."""
    B, K, V = 12, 2, 777
    s = make_drafts(B, K, V, "f32", True, 1.0, seed=7, ragged=False, near=0.05)
    l = s["logits"]
    for b in range(B):
        r = (K + 1) * b
        if b == 0:
            l[r, 5:] = -math.inf
        elif b == 1:
            l[r, :] = -math.inf
            l[r, 400] = -3e38
        elif b == 2:
            l[r, 1:] = torch.finfo(torch.float32).min
        elif b == 3:
            l[r, 9] = math.nan
        elif b == 4:
            l[r, 776] = math.inf
        elif b == 5:
            l[r, :] = -math.inf
        elif b == 6:
            l[r + 1, 3] = math.nan
        elif b == 7:
            l[r + 2, 3] = math.nan
        elif b == 8:
            l[r] = torch.finfo(torch.float32).min
        elif b == 9:
            l[r] = torch.finfo(torch.float32).max
    out = check_verify(s)
    assert out.status[3:6].tolist() == [2, 2, 2] and out.n_accepted[3:6].tolist() == [0, 0, 0]
    assert torch.all(out.tokens[3:6] == -1)
    s["probs"] = None
    check_verify(s)
    s["t"] = torch.zeros(B)
    check_verify(s)


def test_drafts_that_are_no_ids_and_probabilities_that_are_none():
    B, K, V = 40, 3, 300
    for probs in (True, False):
        s = make_drafts(B, K, V, "f32", probs, 1.0, seed=8, near=0.05)
        s["drafted"][::3] = V
        s["drafted"][1::5] = -1
        s["drafted"][2::7] = 2 ** 31 - 1
        if probs:
            s["probs"][::4, 11] = math.nan
            s["probs"][1::4] = math.nan
        out = check_verify(s)
        assert int((out.status == 1).sum()) > 5
        s["t"] = torch.zeros(B)
        check_verify(s)


def test_a_draft_that_leaves_nothing():
    """q at or above p everywhere (q = p counts as such in 64 bits only where p is a short number): p itself is sampled."""
    V = 64
    s = make_drafts(30, 1, V, "f32", True, 1.0, seed=9, ragged=False)
    s["logits"][:] = 1.0
    s["probs"][:] = 1.0  # no distribution: refuses nearly every draft and leaves nothing of p = 1 / 64
    out = check_verify(s)
    assert int((out.n_accepted == 0).sum()) >= 25 and int(out.tokens.max()) < V


def test_offsets_that_are_none():
    s = make_drafts(6, 4, 100, "f32", True, 1.0, seed=10, ragged=False)
    s["offsets"] = torch.tensor([0, 4, 2, 8, 30, -1, 3], dtype=torch.int32)
    out = check_verify_status(s)
    assert out.status.tolist() == [0, 4, 4, 4, 4, 4]
    assert torch.all(out.tokens[1:] == -1) and torch.all(out.n_accepted[1:] == 0)


def check_verify_status(s):
    out = run_verify(s)
    tokens, n, _, status = ref.verify(s["logits"], s["drafted"], s["offsets"], s["accept"], s["sample"], s["t"], s["K"], s["probs"])
    assert torch.equal(out.tokens.cpu(), tokens) and torch.equal(out.n_accepted.cpu(), n) and torch.equal(out.status.cpu(), status)
    return out


@pytest.mark.parametrize("dtype,ld,offset", [("f32", 1001, 0), ("f32", 1003, 1), ("bf16", 1001, 0), ("bf16", 1007, 3), ("f16", 1024, 5)])
def test_rows_at_every_alignment(dtype, ld, offset):
    V = 997
    s = make_drafts(6, 3, V, dtype, True, 1.0, seed=11)
    want = check_verify(s)
    rows, D = s["logits"].shape[0], s["drafted"].numel()
    buf = torch.full((rows * ld + 16,), math.nan, dtype=DTYPES[dtype], device="cuda")
    lg = torch.as_strided(buf, (rows, V), (ld, 1), offset).copy_(s["logits"].cuda())
    qbuf = torch.full((D * ld + 16,), math.nan, device="cuda")
    q = torch.as_strided(qbuf, (D, V), (ld, 1), offset).copy_(s["probs"].cuda())
    out = difr.DraftOut.allocate(6, D, 3, V)
    c = lambda x: s[x].cuda()
    difr.difr_verify_drafts(lg, c("drafted"), c("offsets"), c("accept"), c("sample"), 1.0, out, draft_probs=q)
    assert torch.equal(out.tokens, want.tokens) and torch.equal(out.n_accepted, want.n_accepted)


def test_verification_captured_replayed_and_on_another_stream():
    s = make_drafts(5, 4, 3001, "bf16", True, 0.9, seed=12)
    dev = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    D = s["drafted"].numel()
    out = difr.DraftOut.allocate(5, D, 4, 3001)
    args = (dev["logits"], dev["drafted"], dev["offsets"], dev["accept"], dev["sample"], 0.9, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        difr.difr_verify_drafts(*args, draft_probs=dev["probs"])
    for seed in (13, 14):
        new = torch.randint(-2 ** 31, 2 ** 31, (5,), generator=torch.Generator().manual_seed(seed), dtype=torch.int64).to(torch.int32)
        s["sample"] = new
        dev["sample"].copy_(new)
        graph.replay()
        check_verify(s, out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = difr.DraftOut.allocate(5, D, 4, 3001)
    difr.difr_verify_drafts(*args[:-1], other, draft_probs=dev["probs"], stream=side)
    side.synchronize()
    assert torch.equal(other.tokens, out.tokens)


def test_verified_tokens_have_the_targets_distribution():
    """Words of the library's own Philox; the next token after a draft of one, over 40000 requests, is distributed as p."""
    V, B = 12, 40000
    g = torch.Generator().manual_seed(15)
    target, draft = torch.randn(V, generator=g) * 1.5, torch.randn(V, generator=g) * 1.5
    q = torch.softmax(draft, 0)
    ctr = torch.zeros(2 * B, 4, dtype=torch.int32)
    ctr[:, 0] = torch.arange(2 * B)
    words = difr.difr_philox(ctr.cuda(), torch.full((2 * B, 2), 99, dtype=torch.int32).cuda(), torch.empty(2 * B, 4, dtype=torch.int32, device="cuda"))
    drafted = torch.multinomial(q, B, replacement=True, generator=g).to(torch.int32).cuda()
    out = difr.DraftOut.allocate(B, B, 1, V)
    difr.difr_verify_drafts(target.cuda().expand(2 * B, V).contiguous(), drafted, torch.arange(B + 1, dtype=torch.int32, device="cuda"),
                            words[:B, 0].contiguous(), words[B:, 0].contiguous(), 1.0, out, draft_probs=q.cuda().expand(B, V).contiguous())
    first = torch.bincount(out.tokens[:, 0].long().cpu(), minlength=V).double() / B
    p = torch.softmax(target.double(), 0)
    # five standard deviations of each frequency
    assert torch.all((first - p).abs() <= 5 * torch.sqrt(p * (1 - p) / B))
    assert abs(float(out.n_accepted.double().mean()) - float(torch.minimum(p, q.double()).sum())) <= 5 * 0.5 / math.sqrt(B)


def test_verification_refusals():
    s = make_drafts(3, 2, 50, "f32", True, 1.0, seed=16, ragged=False)
    d = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    out = difr.DraftOut.allocate(3, 6, 2, 50)

    def call(o=out, temperature=1.0, **kw):
        a = {**d, **kw}
        return difr.difr_verify_drafts(a["logits"], a["drafted"], a["offsets"], a["accept"], a["sample"], temperature, o,
                                       draft_probs=a["probs"])

    call()
    for bad in (dict(logits=d["logits"][:-1]), dict(logits=d["logits"].double()), dict(logits=d["logits"].T), dict(drafted=d["drafted"].long()),
                dict(drafted=d["drafted"][:-1]), dict(offsets=d["offsets"][:-1]), dict(accept=s["accept"]), dict(sample=d["sample"][:2]),
                dict(probs=d["probs"][:, :-1]), dict(probs=d["probs"].half()), dict(temperature=torch.ones(2, device="cuda"))):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in (dict(o=difr.DraftOut(out.tokens.long(), out.n_accepted, out.p_draft, out.status, out.workspace)),
                dict(o=difr.DraftOut(out.tokens, out.n_accepted[:2], out.p_draft, out.status, out.workspace)),
                dict(o=difr.DraftOut(out.tokens, out.n_accepted, out.p_draft[:2], out.status, out.workspace)),
                dict(o=difr.DraftOut(out.tokens, out.n_accepted, out.p_draft, out.status, out.workspace.float()))):
        with pytest.raises(TypeError):
            call(**bad)
    for status, bad in ((-4, dict(o=difr.DraftOut(out.tokens, out.n_accepted, out.p_draft, out.status, out.workspace[:16]))),
                        (-1, dict(temperature=-0.5)), (-1, dict(temperature=math.nan)), (-1, dict(temperature=math.inf)),
                        (-3, dict(o=difr.DraftOut(out.tokens, out.n_accepted, out.p_draft, out.status, out.workspace[8:])))):
        with pytest.raises(difr.DifrError) as e:
            call(**bad)
        assert e.value.status == status
    call(o=difr.DraftOut(out.tokens, out.n_accepted, None, None, out.workspace))
    e = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")
    difr.difr_verify_drafts(torch.empty(0, 50, device="cuda"), e(0), torch.zeros(1, dtype=torch.int32, device="cuda"), e(0), e(0), 1.0,
                            difr.DraftOut(e(0, 3), e(0), None, None, torch.empty(0, dtype=torch.uint8, device="cuda")))


# ------------------------------------------------------------------ 4-bit weights with group scales
def w4_of(rows, d, group):
    """A tensor whose buffers are full of a value that nothing writes."""
    w = difr.W4Tensor.allocate(rows, d, group)
    w.codes.fill_(0x5A)
    w.scales.fill_(math.nan)
    return w


def assert_w4_equal(w, x, group):
    codes, scales = ref.w4_pack(*ref.w4_quantize(x, group), x.shape[1], group)
    assert torch.equal(w.codes.cpu(), codes)
    assert torch.equal(torch.isnan(w.scales.cpu()), torch.isnan(scales))
    assert torch.equal(w.scales.cpu().nan_to_num(), scales.nan_to_num())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 32), (3, 31), (5, 33), (2, 100), (129, 128), (130, 1056), (257, 1749), (9, 70),
                                    (20, 1030), (7, 4096), (1, 8192)])
def test_w4_quantisation_is_bit_exact(rows, d, group, dtype):
    x = randn(rows, d, seed=rows + d).to(DTYPES[dtype])
    w = w4_of(rows, d, group)
    difr.difr_w4_quantize(x.cuda(), w)
    assert_w4_equal(w, x, group)


@pytest.mark.parametrize("group", [32, 128])
def test_w4_every_rounding_border(group):
    """All codes, all midpoints and their fp32 neighbours under scales that are no powers of two; largest magnitudes whose
    seventh is a bf16 midpoint, and their neighbours."""
    rows = []
    for mant in (128, 129, 173, 200, 255):
        for e in (-126, -60, -9, 0, 40, 110):
            s = math.ldexp(mant, e - 7)
            if s < 2.0 ** -126 or 7 * s > 3e38:
                continue
            pts = torch.tensor([s * k / 2 for k in range(-14, 15)], dtype=torch.float64).float()
            pts = torch.cat([pts, torch.nextafter(pts, torch.tensor(math.inf)), torch.nextafter(pts, torch.tensor(-math.inf))])
            pts = pts[pts.abs() <= 7 * s]
            for i in range(0, pts.numel(), group - 1):
                row = torch.zeros(group)
                row[:pts[i:i + group - 1].numel()] = pts[i:i + group - 1]
                row[-1] = 7 * s
                rows.append(row)
    for m in range(257, 512, 14):  # 7 * odd nine-bit numbers: a seventh lies between two bf16
        top = torch.tensor(7.0 * m)
        for v in (top, torch.nextafter(top, torch.tensor(math.inf)), torch.nextafter(top, torch.tensor(0.0))):
            row = v * torch.linspace(-1, 1, group)
            row[0] = v
            rows.append(row)
    x = torch.stack(rows)
    w = w4_of(x.shape[0], group, group)
    difr.difr_w4_quantize(x.cuda(), w)
    assert_w4_equal(w, x, group)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4_extreme_groups(group):
    x = randn(12, 3 * group - 5, seed=5)
    x[0] = 0.0
    x[1] = -0.0
    x[2] = torch.finfo(torch.float32).max
    x[3, :group] = 1e-45
    x[3, group:2 * group] = -3e-39
    x[4] = x[4] * 1e-42
    x[5, group + 3] = math.nan
    x[6, 0] = math.inf
    x[7, 3 * group - 6] = -math.inf
    x[8] = -torch.finfo(torch.float32).max
    x[9] = 7 * torch.finfo(torch.float32).tiny
    x[10] = 6.9 * torch.finfo(torch.float32).tiny
    x[11, group:] = 0.0
    w = w4_of(12, x.shape[1], group)
    difr.difr_w4_quantize(x.cuda(), w)
    assert_w4_equal(w, x, group)
    out = torch.empty_like(x, device="cuda")
    difr.difr_w4_dequantize(w, out)
    want = ref.w4_values(w.codes.cpu(), w.scales.cpu(), x.shape[1], group)
    assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want))
    assert torch.equal(out.cpu().double().nan_to_num(), want.nan_to_num())


def random_w4(rows, d, group, seed=0, std=None):
    """Codes over the whole range, -8 among them, scales of either sign over a few powers of two, eight bits each."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(-8, 8, (rows, d), generator=g)
    scales = torch.randint(128, 256, (rows, ref.w4_groups(d, group)), generator=g).double()
    scales *= 2.0 ** torch.randint(-10, -6, scales.shape, generator=g) * (std or d ** -0.5) / 8
    scales = scales.to(torch.bfloat16) * (1 - 2 * torch.randint(0, 2, scales.shape, generator=g))
    c, s = ref.w4_pack(codes, scales, d, group)
    return difr.W4Tensor(c.cuda(), s.cuda(), group, rows, d), ref.w4_values(c, s, d, group)


@pytest.mark.parametrize("out_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,d,ld", [(1, 1, 1), (3, 31, 40), (129, 256, 256), (70, 1749, 1749), (5, 4096, 4104), (9, 70, 70), (20, 1030, 1034)])
def test_w4_dequantisation(rows, d, ld, group, out_dtype):
    w, values = random_w4(rows, d, group, seed=d)
    buf = torch.full((rows, ld), -7.0, dtype=DTYPES[out_dtype], device="cuda")
    difr.difr_w4_dequantize(w, buf[:, :d])
    assert torch.equal(buf[:, :d].cpu(), values.to(DTYPES[out_dtype]))
    assert torch.all(buf[:, d:] == -7.0)


@pytest.mark.parametrize("offset,ld", [(0, 72), (1, 72), (0, 67), (8, 80)])
def test_w4_quantisation_of_strided_rows(offset, ld):
    buf = randn(40, ld + 8, seed=ld).to(torch.bfloat16)
    w = w4_of(40, 65, 64)
    difr.difr_w4_quantize(buf.cuda()[:, offset:offset + 65], w)
    assert_w4_equal(w, buf[:, offset:offset + 65], 64)


def w4_logits(h, W, dtype=torch.float32, ld=None, offset=0, status=True):
    T, V = h.shape[0], W.rows
    ld = ld or V
    buf = torch.full((T * ld + offset,), -7.0, dtype=dtype, device="cuda")
    logits = torch.as_strided(buf, (T, V), (ld, 1), offset)
    word = torch.zeros(1, dtype=torch.int32, device="cuda") if status else None
    ws = torch.full((difr.difr_w4_workspace_bytes(T, W.d),), 0xAB, dtype=torch.uint8, device="cuda")
    difr.difr_w4_logits(h.cuda() if not h.is_cuda else h, W, logits, ws, word)
    assert not status or int(word) == 0
    if ld > V:
        assert torch.all(torch.as_strided(buf, (T - 1, ld - V), (ld, 1), offset + V) == -7.0)
    return logits


def check_w4_logits(got, h, values):
    """The sum of ceil(d / 16) steps, each of which may drop what lies below the last bit of the largest number in it, and
    two roundings more: (steps + 2) 2^-23 of the sizes added up; bf16 rounds once more."""
    h, values = h.double().cpu(), values
    want, size = h @ values.T, h.abs() @ values.abs().T
    fp32 = ((h.shape[1] + 15) // 16 + 2) * 2.0 ** -23 * size
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
    err = (got.double().cpu() - want).abs()
    assert torch.all(err <= fp32 + half * (want.abs() + fp32) + 2.0 ** -134)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 128, 32), (1, 1000, 4096), (2, 129, 31), (3, 257, 33), (5, 300, 100), (16, 1000, 1749),
                                   (17, 1003, 2048), (33, 777, 130), (64, 2000, 1024), (65, 640, 70), (129, 1001, 513), (300, 515, 1030),
                                   (777, 400, 256), (1, 20000, 8191)])
def test_w4_logits(T, V, d, group, out):
    W, values = random_w4(V, d, group, seed=T + V + d)
    h = randn(T, d, seed=d).to(torch.bfloat16)
    check_w4_logits(w4_logits(h, W, DTYPES[out]), h, values)


@pytest.mark.parametrize("out,ld,offset", [("f32", 1008, 0), ("f32", 1001, 1), ("bf16", 1001, 0), ("bf16", 1002, 1), ("bf16", 1008, 3)])
@pytest.mark.parametrize("T", [1, 9, 130])
def test_w4_logits_of_strided_rows(T, out, ld, offset):
    d = 333
    W, values = random_w4(1001, d, 64, seed=1)
    h = randn(T, d + 11, seed=2).to(torch.bfloat16).cuda()[:, 3:3 + d]
    check_w4_logits(w4_logits(h, W, DTYPES[out], ld, offset), h, values)


def test_w4_logits_of_small_integers_are_exact():
    """Sums that fp32 holds: every product and every partial sum is an integer below 2^24."""
    g = torch.Generator().manual_seed(3)
    for T, V, d in ((1, 500, 4096), (40, 500, 2048), (200, 300, 999)):
        codes = torch.randint(-8, 8, (V, d), generator=g)
        scales = torch.tensor([1.0, 2.0, 3.0, 7.0])[torch.randint(0, 4, (V, ref.w4_groups(d, 32)), generator=g)]
        c, s = ref.w4_pack(codes, scales, d, 32)
        h = torch.randint(-16, 17, (T, d), generator=g).to(torch.bfloat16)
        want = h.double() @ ref.w4_values(c, s, d, 32).T
        assert torch.equal(w4_logits(h, difr.W4Tensor(c.cuda(), s.cuda(), 32, V, d)).double().cpu(), want)


def test_w4_logits_where_sizes_differ_by_a_lot():
    """Hidden states with outliers of 2^20, rows of weights whose scales are 2^-100 to 2^80 times the others', groups of one row
    that are up to 2^11 apart, ids of zero scales."""
    T, V, d = 20, 600, 640
    W, _ = random_w4(V, d, 64, seed=4)
    s = W.scales.cpu().float()
    s *= 2.0 ** torch.randint(-100, 81, (V, 1), generator=torch.Generator().manual_seed(5)).float()
    s[:, 3] *= 2.0 ** 11
    s[::7] = 0.0
    W.scales.copy_(s.to(torch.bfloat16))
    values = ref.w4_values(W.codes.cpu(), W.scales.cpu(), d, 64)
    h = randn(T, d, seed=6)
    h[::2, 5] *= 2.0 ** 20
    h[1] *= 2.0 ** -90
    h[3] = 0.0
    h[4] *= 2.0 ** 30
    h = h.to(torch.bfloat16)
    for t in (slice(0, T), slice(3, 4), slice(0, 1)):
        check_w4_logits(w4_logits(h[t], W), h[t], values)


def test_w4_logits_of_broken_rows_and_groups():
    """A NaN or an infinity in a row of h spoils that row, a NaN or infinite scale that id; nothing else."""
    T, V, d = 30, 400, 300
    W, _ = random_w4(V, d, 32, seed=7)
    W.scales[5, 2] = math.nan
    W.scales[399, 9] = math.inf
    W.scales[128, 0] = -math.inf
    h = randn(T, d, seed=8).to(torch.bfloat16)
    h[3, 7], h[11, 299], h[29, 0] = math.nan, math.inf, -math.inf
    got = w4_logits(h, W).cpu()
    bad = torch.zeros(T, V, dtype=torch.bool)
    bad[[3, 11, 29]] = True
    bad[:, [5, 399, 128]] = True
    assert torch.equal(torch.isnan(got), bad)
    values = ref.w4_values(W.codes.cpu(), W.scales.cpu(), d, 32)
    rows, ids = ~bad.all(1), ~bad.all(0)
    check_w4_logits(got[rows][:, ids], h[rows], values[ids])


@pytest.mark.parametrize("T", [1, 4, 60, 300])
def test_w4_logits_do_not_notice_their_batch(T):
    """A row alone, in the batch, and at another place of it: the same bits."""
    W, _ = random_w4(1111, 1024, 128, seed=9)
    h = randn(T, 1024, seed=10).to(torch.bfloat16)
    whole = w4_logits(h, W)
    for t in {0, T // 2, T - 1}:
        assert torch.equal(w4_logits(h[t:t + 1], W)[0], whole[t])
    assert torch.equal(w4_logits(h.flip(0), W).flip(0), whole)


def test_w4_logits_captured_and_on_another_stream():
    W, values = random_w4(3000, 512, 64, seed=11)
    for T in (1, 70):
        h = randn(T, 512, seed=12).to(torch.bfloat16).cuda()
        want = w4_logits(h, W)
        logits, ws = torch.empty_like(want), torch.empty(difr.difr_w4_workspace_bytes(T, 512), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            difr.difr_w4_logits(h, W, logits, ws)
        for seed in (13, 14):
            h.copy_(randn(T, 512, seed=seed).to(torch.bfloat16))
            graph.replay()
            check_w4_logits(logits, h, values)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        other = torch.empty_like(logits)
        difr.difr_w4_logits(h, W, other, torch.empty_like(ws), stream=side)
        side.synchronize()
        assert torch.equal(other, logits)


def test_w4_logits_of_a_head_beyond_32_bits_of_bytes():
    """Codes of more than 2^32 bytes, logits of more than 2^31 elements: ids at both ends."""
    V, d = 600_000, 16384  # 4.9e9 bytes of codes
    w = difr.W4Tensor(torch.randint(0, 256, (V, d // 2), dtype=torch.uint8, device="cuda"),
                      torch.rand(V, d // 128, device="cuda").to(torch.bfloat16), 128, V, d)
    h = randn(3600, d, seed=15).to(torch.bfloat16)
    h_all = h.cuda()
    logits = torch.empty(3600, V, dtype=torch.bfloat16, device="cuda")
    difr.difr_w4_logits(h_all, w, logits, torch.empty(difr.difr_w4_workspace_bytes(3600, d), dtype=torch.uint8, device="cuda"))
    for ids in (slice(0, 40), slice(V - 40, V)):
        values = ref.w4_values(w.codes[ids].cpu(), w.scales[ids].cpu(), d, 128)
        for rows in (slice(0, 3), slice(3597, 3600)):
            check_w4_logits(logits[rows, ids], h[rows], values)


def test_w4_refusals():
    W, _ = random_w4(40, 64, 32, seed=16)
    h = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    logits, ws = torch.empty(4, 40, device="cuda"), torch.empty(difr.difr_w4_workspace_bytes(4, 64), dtype=torch.uint8, device="cuda")
    difr.difr_w4_logits(h, W, logits, ws)
    for bad in ((h.half(), W, logits, ws), (h[:, :32], W, logits, ws), (h, W, logits[:, :39], ws), (h, W, logits.half(), ws),
                (h, W, logits, ws.float()), (h, W, logits, ws.cpu()), (h.T, W, logits, ws), (h, "W", logits, ws),
                (h, difr.W4Tensor(W.codes, W.scales, 48, 40, 64), logits, ws), (h, difr.W4Tensor(W.codes[:39], W.scales, 32, 40, 64), logits, ws)):
        with pytest.raises(TypeError):
            difr.difr_w4_logits(*bad)
    for status, args in ((-4, (h, W, logits, ws[:ws.numel() - 1])), (-3, (h, W, logits, torch.empty(ws.numel() + 8, dtype=torch.uint8, device="cuda")[8:])),
                         (-3, (h, difr.W4Tensor(torch.empty(40 * 32 + 8, dtype=torch.uint8, device="cuda")[8:], W.scales, 32, 40, 64), logits, ws))):
        with pytest.raises(difr.DifrError) as e:
            difr.difr_w4_logits(*args)
        assert e.value.status == status
    with pytest.raises(ValueError):
        difr.W4Tensor.allocate(4, 64, 48)
    with pytest.raises(TypeError):
        difr.difr_w4_dequantize(W, torch.empty(40, 64, dtype=torch.float16, device="cuda"))
    with pytest.raises(TypeError):
        difr.difr_w4_quantize(torch.zeros(39, 64, device="cuda"), W)
    difr.difr_w4_logits(h[:0], W, logits[:0], ws)
    difr.difr_w4_quantize(torch.empty(0, 64, device="cuda"), difr.W4Tensor.allocate(0, 64, 32))


# ------------------------------------------------------------------ together
def test_a_decoding_step_from_block_to_tokens():
    """The last block's output through norms and 4-bit head into the verification of drafts sampled near its logits: each step
    against its own statement on the step before it."""
    B, K, d, V = 9, 4, 512, 3000
    T = B * (K + 1)
    x, r, w, pw, g = block_inputs(T, d, "bf16", "token")
    out = run_block(x, r, w, 1e-6, pw, None, g, scale=0.5)
    check_stream(out.residual, x, r, "bf16", pw, 1e-6, g, scale=0.5)
    check_h(out.h, out.residual, w, 1e-6)
    W = w4_of(V, d, 64)
    head = randn(V, d, seed=20, std=2.5 * d ** -0.5)
    difr.difr_w4_quantize(head.cuda(), W)
    assert_w4_equal(W, head, 64)
    logits = w4_logits(out.h, W)
    check_w4_logits(logits, out.h.cpu(), ref.w4_values(W.codes.cpu(), W.scales.cpu(), d, 64))
    s = make_drafts(B, K, V, "f32", True, 0.8, seed=21, ragged=False)
    s["logits"] = logits.cpu()
    gen = torch.Generator().manual_seed(22)
    for b in range(B):
        for j in range(K):
            q = torch.softmax((s["logits"][b * (K + 1) + j] + 0.3 * torch.randn(V, generator=gen)) / 0.8, 0)
            s["probs"][b * K + j] = q
            s["drafted"][b * K + j] = int(torch.multinomial(q, 1, generator=gen))
    check_verify(s)
