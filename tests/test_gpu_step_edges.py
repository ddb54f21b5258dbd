"""Edges of a decoding step's operators on the GPU, against the plain 64-bit statements in step_reference.py."""
import math

import pytest
import torch

import paper_2511_02620_b200 as difr
import step_reference as ref
from test_gpu_step import (DTYPES, block_inputs, check_h, check_stream, check_verify, check_w4_logits, make_drafts, randn, random_w4,
                           run_block, run_verify, w4_logits)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ verification of drafted tokens
def outputs_that_held_something(s):
    B, D, V = s["sample"].numel(), s["drafted"].numel(), s["logits"].shape[1]
    out = difr.DraftOut.allocate(B, D, s["K"], V)
    for x in (out.tokens, out.n_accepted, out.status):
        x.fill_(-77)
    out.p_draft.fill_(0.25)  # an ordinary probability, such as an earlier call's
    return out


def test_probabilities_of_drafts_that_are_not_looked_at():
    """Requests with an unusable temperature or too many drafts, drafts of no request: NaN, whatever the buffer held."""
    s = make_drafts(6, 3, 100, "f32", True, 1.0, seed=30, ragged=False)
    s["t"] = torch.tensor([1.0, math.nan, -1.0, math.inf, 0.0, 2.0])
    out = check_verify(s, run_verify(s, outputs_that_held_something(s)))
    assert torch.equal(torch.isnan(out.p_draft).cpu(), torch.tensor([0, 1, 1, 1, 0, 0]).bool().repeat_interleave(3))
    s = make_drafts(6, 3, 100, "bf16", False, 1.0, seed=31, ragged=False)
    s["offsets"] = torch.tensor([2, 3, 3, 12, 13, 15, 17], dtype=torch.int32)
    out = check_verify(s, run_verify(s, outputs_that_held_something(s)))
    assert out.status.tolist() == [0, 0, 4, 0, 0, 0]
    nan = torch.tensor([i < 2 or 3 <= i < 12 or i >= 17 for i in range(18)])
    assert torch.equal(torch.isnan(out.p_draft).cpu(), nan)


def test_probabilities_of_drafts_where_offsets_descend():
    """No entry keeps what the buffer held."""
    s = make_drafts(6, 4, 100, "f32", True, 1.0, seed=10, ragged=False)
    s["offsets"] = torch.tensor([0, 4, 2, 8, 30, -1, 3], dtype=torch.int32)
    out = run_verify(s, outputs_that_held_something(s))
    assert not torch.any(out.p_draft == 0.25)


def test_a_nan_among_the_drafts_probabilities():
    """At the drafted token it refuses it, elsewhere in the refused draft's row its id is not sampled; an infinity does the same."""
    V = 8
    s = make_drafts(40, 1, V, "f32", True, 1.0, seed=38, ragged=False)
    s["logits"][:] = 0.0
    for bad in (math.nan, math.inf):
        s["probs"][:] = 1e-3  # (as no distribution: every draft is accepted, and 7/8 or more of p is left where not)
        s["probs"][:20, 3] = bad
        s["probs"][20:, 5] = bad
        s["drafted"][:20], s["drafted"][20:] = 3, 1
        s["accept"][:] = -1
        s["probs"][20:, 1] = 0.5  # refused by its probability
        out = check_verify(s, run_verify(s, outputs_that_held_something(s)))
        assert torch.all(out.n_accepted == 0)
        assert not torch.any(out.tokens[:20, 0] == 3) and not torch.any(out.tokens[20:, 0] == 5)


def test_more_requests_than_a_grid_holds():
    """70000 requests, looked at in one call and in two; the last ones against the definition."""
    B, K, V = 70000, 1, 9
    g = torch.Generator().manual_seed(32)
    n = torch.randint(0, K + 1, (B,), generator=g)
    off = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32)
    D = int(off[-1])
    words = lambda k: torch.randint(-2 ** 31, 2 ** 31, (k,), generator=g, dtype=torch.int64).to(torch.int32)
    logits, probs = 2 * torch.randn(D + B, V, generator=g), torch.softmax(2 * torch.randn(D, V, generator=g), 1)
    s = dict(logits=logits, drafted=torch.randint(0, V, (D,), generator=g).to(torch.int32), offsets=off, accept=words(D), sample=words(B),
             t=torch.ones(B), K=K, probs=probs)

    def part(b0, b1):
        o0, o1 = int(off[b0]), int(off[b1])
        return dict(logits=s["logits"][o0 + b0:o1 + b1], drafted=s["drafted"][o0:o1], offsets=off[b0:b1 + 1] - o0, accept=s["accept"][o0:o1],
                    sample=s["sample"][b0:b1], t=s["t"][b0:b1], K=K, probs=None if s["probs"] is None else s["probs"][o0:o1])

    for with_probs in (True, False):
        if not with_probs:
            s["probs"] = None
        whole = run_verify(s)
        for b0, b1 in ((0, 40000), (40000, B)):
            out = run_verify(part(b0, b1))
            assert torch.equal(out.tokens, whole.tokens[b0:b1]) and torch.equal(out.n_accepted, whole.n_accepted[b0:b1])
        assert int(whole.status.abs().max()) == 0
        check_verify(part(B - 300, B))
        check_verify(part(65400, 65700))


# ------------------------------------------------------------------ block norm
def test_block_norm_where_root_and_scale_leave_fp32_together():
    """1 / rms times the block's scale is beyond fp32 on either side, gate and scale are, and the result is an ordinary number."""
    d = 640
    x, r, w, pw, g = block_inputs(6, d, "f32", "token")
    x[:2] *= 1e-10
    out = run_block(x[:2], r[:2] * 1e30, w, 1e-6, pw, 1e-24, scale=1e30)
    check_stream(out.residual, x[:2], r[:2] * 1e30, "f32", pw, 1e-24, scale=1e30)
    check_h(out.h, out.residual, w, 1e-6)
    x[2:4] *= 1e30
    out = run_block(x[2:4], r[2:4] * 1e-28, w, 1e-45, pw, 1e-6, g[2:4], scale=1e-28)
    check_stream(out.residual, x[2:4], r[2:4] * 1e-28, "f32", pw, 1e-6, g[2:4], scale=1e-28)
    check_h(out.h, out.residual, w, 1e-45)
    x[4:] *= 1e20
    for gate in (g[4:] * 1e-30, g[4:5] * 1e-30):
        out = run_block(x[4:], r[4:] * 1e20, w, 1e-6, gate=gate, scale=1e30)
        check_stream(out.residual, x[4:], r[4:] * 1e20, "f32", gate=gate, scale=1e30)
        check_h(out.h, out.residual, w, 1e-6)


@pytest.mark.parametrize("dtype,d,ld", [("bf16", 1031, 1031), ("bf16", 1030, 1034), ("bf16", 1028, 1036), ("f16", 333, 341), ("f32", 1031, 1033),
                                        ("f32", 2050, 2050), ("bf16", 70, 71), ("bf16", 9001, 9003)])
@pytest.mark.parametrize("post", [True, False])
def test_block_norm_in_place_of_rows_off_16_bytes(dtype, d, ld, post):
    """The stream over the residual or over x, h over the other one (bf16), rows that go by way of shared memory."""
    T = 37
    x, r, w, pw, g = block_inputs(T, d, dtype, "token")
    kw = dict(post_weight=pw.cuda() if post else None, gate=g.cuda(), scale=0.5)
    place = lambda t: torch.as_strided(torch.full((T * ld + 8,), -3.0, dtype=t.dtype, device="cuda"), (T, d), (ld, 1)).copy_(t.cuda())
    def call(stream_over):
        xs, rs = place(x), place(r)
        stream = {"apart": torch.as_strided(torch.empty(T * ld, dtype=x.dtype, device="cuda"), (T, d), (ld, 1)), "x": xs, "residual": rs}[stream_over]
        h = torch.as_strided(torch.empty(T * ld, dtype=torch.bfloat16, device="cuda"), (T, d), (ld, 1))
        if dtype == "bf16" and stream_over != "apart":
            h = rs if stream_over == "x" else xs
        difr.difr_block_norm(xs, rs, w.cuda(), 1e-6, difr.NormOut(h=h, residual=stream), **kw)
        for t in (xs, rs):
            assert torch.all(torch.as_strided(t, (T - 1, ld - d), (ld, 1), d) == -3.0)
        return stream, h
    stream, h = call("apart")
    check_stream(stream.contiguous(), x, r, dtype, pw if post else None, 1e-6, g, scale=0.5)
    check_h(h.contiguous(), stream.contiguous(), w, 1e-6)
    for over in ("x", "residual"):
        got = call(over)
        assert torch.equal(got[0], stream) and torch.equal(got[1], h)


# ------------------------------------------------------------------ the product on 4-bit weights
@pytest.mark.parametrize("e", [-140, -130, -127, -126, -125, -123, -121, -120])
def test_w4_logits_below_the_normal_numbers_are_rounded_once(e):
    """Sums of integers N, exact in fp32, times 2^(e - 30): the nearest fp32 number, whatever takes the powers of two back."""
    V, d, group = 5000, 96, 32
    g = torch.Generator().manual_seed(33)
    eh, es = -40, e + 64  # exponents of the largest hidden state and of the largest scale: e = eh + es - 24
    codes = torch.randint(-8, 8, (V, d), generator=g)
    codes[:, :group] = 0
    scales = torch.full((V, 3), 2.0 ** (es - 20))
    scales[:, 0] = 2.0 ** es
    c, s = ref.w4_pack(codes, scales, d, group)
    W = difr.W4Tensor(c.cuda(), s.cuda(), group, V, d)
    h = torch.randint(-255, 256, (300, d), generator=g).double() * 2.0 ** (eh - 34)
    h[:, 0] = 2.0 ** eh
    h = h.to(torch.bfloat16)
    want = (h.double() @ ref.w4_values(c, s, d, group).T).float()
    assert e < -126 or 0 < int((want.abs() < 2.0 ** -126).sum())
    for T in (1, 16, 30, 60, 100, 300):
        got = w4_logits(h[:T], W).cpu()
        assert torch.equal(got, want[:T]), T


def test_w4_scales_below_the_normal_numbers():
    """Beside a larger scale of their id they count by their value, alone they count as zero."""
    T, V, d, group = 20, 200, 96, 32
    W, _ = random_w4(V, d, group, seed=36)
    scales = torch.full((V, 8), 0.0)
    scales[:, 0] = 1.5 * 2.0 ** -126
    scales[:, 1], scales[:, 2] = 2.0 ** -127, -3 * 2.0 ** -131
    scales[1::2, 0] = 2.0 ** -128
    W.scales.copy_(scales.to(torch.bfloat16))
    h = (randn(T, d, seed=37) * 2.0 ** 60).to(torch.bfloat16)
    values = ref.w4_values(W.codes.cpu(), W.scales.cpu(), d, group)
    for rows in (slice(0, T), slice(0, 3)):
        got = w4_logits(h[rows], W)
        check_w4_logits(got[:, ::2], h[rows], values[::2])
        assert torch.all(got[:, 1::2] == 0)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,d,group,ld", [(300, 10003, 513, 32, 10003), (300, 10003, 513, 64, 10004), (513, 10000, 1030, 128, 10000),
                                            (513, 10003, 1749, 32, 10008), (300, 10002, 1749, 64, 10003), (300, 10003, 130, 128, 10008),
                                            (700, 10003, 64, 32, 10008), (513, 10004, 2048, 64, 10008), (257, 10006, 1151, 32, 10008),
                                            (300, 10001, 4033, 64, 10004)])
def test_w4_logits_of_tiles_of_256_tokens(T, V, d, group, ld, out):
    """Enough tiles for every pair of CTAs, so that they are 256 tokens wide: both ways out (rows on 16 bytes or not, ids that
    end inside 16 bytes), even and odd numbers of steps, a last one of half the length."""
    W, values = random_w4(V, d, group, seed=V + d)
    h = randn(T, d, seed=d).to(torch.bfloat16)
    check_w4_logits(w4_logits(h, W, DTYPES[out], ld), h, values)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("d", [1, 70, 130, 513, 1100, 1749, 2048])
def test_w4_logits_are_the_same_bits_in_tiles_of_every_width(d, group):
    """Rows alone and in batches that go through mma.sync (up to 16) and through tiles of 32, 64, 128 and 256 tokens."""
    V = 10000
    W, _ = random_w4(V, d, group, seed=34)
    h = randn(300, d, seed=35).to(torch.bfloat16).cuda()
    whole = w4_logits(h, W)
    for t0, t1 in ((0, 1), (299, 300), (5, 13), (100, 116), (3, 23), (250, 282), (40, 100), (17, 145), (0, 299)):
        assert torch.equal(w4_logits(h[t0:t1], W), whole[t0:t1]), (t0, t1)


@pytest.mark.parametrize("out,ld", [("f32", 20009), ("f32", 20012), ("bf16", 20016)])
@pytest.mark.parametrize("d", [274, 384, 600, 1100])
def test_w4_logits_of_an_odd_number_of_steps(d, out, ld):
    """3, 3, 5 and 9 steps of 128 values in tiles of 256 tokens, three tiles and more a pair of CTAs: the steps of one tile follow
    those of another through two slots of converted weights.  Right, and the same bits every time."""
    T, V = 519, 20001
    W, values = random_w4(V, d, 32, seed=d)
    h = randn(T, d, seed=44).to(torch.bfloat16).cuda()
    got = w4_logits(h, W, DTYPES[out], ld)
    check_w4_logits(got[:, ::7], h, values[::7])
    for _ in range(25):
        assert torch.equal(w4_logits(h, W, DTYPES[out], ld), got)


@pytest.mark.parametrize("V,d,group", [(118775, 3730, 64), (110387, 2252, 64), (128256, 4096, 128), (60000, 8000, 32)])
def test_w4_logits_of_few_tokens_are_the_same_bits_in_every_call(V, d, group):
    """Hundreds of calls of 1 to 16 tokens, with weights from L2 and from memory and other work between: the bits of the tiles."""
    g = torch.Generator(device="cuda").manual_seed(45)
    W = difr.difr_w4_quantize(torch.randn(V, d, generator=g, device="cuda") * d ** -0.5, difr.W4Tensor.allocate(V, d, group))
    h = torch.randn(40, d, generator=g, device="cuda").to(torch.bfloat16)
    run = lambda x: difr.difr_w4_logits(x, W, torch.empty(x.shape[0], V, device="cuda"),
                                        torch.empty(difr.difr_w4_workspace_bytes(x.shape[0], d), dtype=torch.uint8, device="cuda"))
    whole = run(h)
    other = torch.zeros(64 << 20, device="cuda")
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for i in range(600):
        n = (1, 5, 8, 3, 16, 12)[i % 6]
        at = i * 7 % (41 - n)
        wrong += (run(h[at:at + n]) != whole[at:at + n]).sum()
        if i % 10 == 0:
            other += 1
        if i % 10 == 5:
            wrong += (run(h) != whole).sum()
    assert int(wrong) == 0


@pytest.mark.parametrize("T,V,d,ld,out", [(1, 5003, 96, 5003, "f32"), (16, 9800, 300, 9808, "bf16"), (20, 50000, 96, 50000, "bf16"),
                                          (40, 9800, 96, 9803, "bf16"), (300, 1100, 160, 1104, "f32"), (600, 9800, 160, 9800, "bf16"),
                                          (600, 9801, 160, 9801, "f32"), (2700, 9800, 40000, 9800, "bf16")])
def test_w4_logits_that_a_wait_keeps_from_being_computed_are_nan(T, V, d, ld, out):
    """The way out of either kernel after waits that ran out, at every tile width: all logits but those of the finished tiles are
    NaN, the status word says so, and the next call is as good as ever."""
    buf = torch.full((T + 1, ld), -7.0, dtype=DTYPES[out], device="cuda")
    part = buf[:T, :V]
    few = T <= 16
    width = 16 if few else 256 if T > 128 and (V + 255) // 256 * ((T + 255) // 256) > 37 else 128 if T > 64 else 64 if T > 32 else 32
    left = []
    for done in (0, 1, 2, 3, 1000):
        buf.fill_(-7.0)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        difr.difr_selftest_w4_wait(d, part, done, 1_000_000, status)
        nan = torch.isnan(part)
        assert int(status.item()) == (-7 if bool(nan.any()) else 0)
        assert torch.all(part[~nan] == -7.0)
        assert torch.all(buf[:T, V:] == -7.0) and torch.all(buf[T:] == -7.0)
        left.append(~nan)
        buf.fill_(-7.0)
        difr.difr_selftest_w4_wait(d, part, done, 1_000_000)  # no status word: the logits tell
        assert torch.equal(torch.isnan(part), nan)
    assert not left[0].any() and left[-1].all()
    for less, more in zip(left, left[1:]):
        new = more & ~less
        assert not (less & ~more).any()
        if few:
            assert more.all()
            continue
        # whole tiles, at most one for every pair of the 74
        pad = lambda x: torch.nn.functional.pad(x, (0, -V % 256, 0, -T % width)).view(-1, width, (V + 255) // 256, 256)
        tiles = pad(new).any(3).any(1)
        assert more.all() or int(tiles.sum()) <= 74
        assert torch.equal(pad(new), pad(torch.ones_like(new)) & tiles.view(-1, 1, tiles.shape[1], 1))
    W, values = random_w4(1000, 96, 32, seed=39)
    h = randn(T, 96, seed=40).to(torch.bfloat16)
    check_w4_logits(w4_logits(h, W), h, values)

# ------------------------------------------------------------------ calls at the same time
def test_calls_on_two_streams_at_once():
    """Each operator many times on two streams, outputs and workspaces apart, the other stream busy with the other ones: the same
    results as alone."""
    V, d, group = 20000, 1030, 64
    W, _ = random_w4(V, d, group, seed=41)
    h = randn(300, d, seed=42).to(torch.bfloat16).cuda()
    x, r, w, pw, g = (t.cuda() for t in block_inputs(300, d, "bf16", "token"))
    s = make_drafts(40, 4, 3001, "bf16", True, 0.9, seed=43)
    dev = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    D = s["drafted"].numel()

    def calls():
        """(a call on a stream, its outputs) of each operator, buffers of its own."""
        for T in (1, 16, 40, 100, 300):
            logits = torch.empty(T, V, device="cuda")
            ws = torch.empty(difr.difr_w4_workspace_bytes(T, d), dtype=torch.uint8, device="cuda")
            yield (lambda st, T=T, l=logits, ws=ws: difr.difr_w4_logits(h[:T], W, l, ws, stream=st)), [logits]
        o = difr.NormOut(h=torch.empty_like(x), residual=torch.empty_like(x))
        yield (lambda st: difr.difr_block_norm(x, r, w, 1e-6, o, post_weight=pw, gate=g, stream=st)), [o.h, o.residual]
        q = difr.W4Tensor.allocate(300, d, group)
        yield (lambda st: difr.difr_w4_quantize(x, q, stream=st)), [q.codes, q.scales]
        v = difr.DraftOut.allocate(40, D, 4, 3001)
        yield (lambda st: difr.difr_verify_drafts(dev["logits"], dev["drafted"], dev["offsets"], dev["accept"], dev["sample"], 0.9, v,
                                                  draft_probs=dev["probs"], stream=st)), [v.tokens, v.n_accepted, v.p_draft]

    alone = []
    for call, outs in calls():
        call(None)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in outs])
    sides = [list(calls()), list(calls())[::-1]]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for side in sides:
        for _, outs in side:
            for t in outs:
                t.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for k in range(len(sides[0])):
            for side, st in zip(sides, streams):
                side[k][0](st)
    torch.cuda.synchronize()
    for side, want in ((sides[0], alone), (sides[1], alone[::-1])):
        for (_, outs), expected in zip(side, want):
            for t, e in zip(outs, expected):
                assert torch.equal(t, e)
