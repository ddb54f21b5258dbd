"""Edges of a decoding step's operators on the GPU, against the plain 64-bit statements in step_reference.py."""
import math

import pytest
import torch

import paper_2511_02620_b200 as difr
import step_reference as ref
from test_gpu_step import (block_inputs, check_h, check_stream, check_verify, check_w4_logits, make_drafts, randn, random_w4, run_block,
                           run_verify, w4_logits)

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
