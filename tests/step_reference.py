"""Plain 64-bit statements of a decoding step's operators, for the tests.  Tensors are torch CPU tensors."""
import torch


def f32(x):
    """The double value of the float32 nearest to x (what the C ABI receives)."""
    return float(torch.tensor(x, dtype=torch.float32))


def rms(v, eps):
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + f32(eps))


def block_stream(x, residual, post_weight, post_eps, gate, scale, residual_scale, offset):
    """residual_scale * residual + scale * gate * norm(x), not rounded, and the size of what is added up."""
    n = x.double()
    if post_weight is not None:
        n = rms(n, post_eps) * (post_weight.double() + f32(offset))
    if gate is not None:
        n = n * gate.double()
    a, b = f32(residual_scale) * residual.double(), f32(scale) * n
    return a + b, a.abs() + b.abs()


def uniform(word):
    return ((int(word) % 2 ** 32) + 0.5) / 2 ** 32


def probabilities(row, temperature):
    """softmax of one row of logits in 64 bits; None where the row is broken."""
    row = row.double()
    if torch.isnan(row).any() or (row == float("inf")).any() or not torch.isfinite(row).any():
        return None
    if temperature == 0:
        p = torch.zeros_like(row)
        p[int((row == row.max()).nonzero()[0, 0])] = 1.0
        return p
    e = torch.exp((row - row.max()) / temperature)
    return e / e.sum()


def verify(logits, drafted, offsets, accept_words, sample_words, temperatures, max_drafts, probs=None):
    """(tokens, n_accepted, p_draft, status) request by request, as the header tells it; one temperature per request."""
    B, V = len(sample_words), logits.shape[1]
    D = len(drafted)
    tokens = torch.full((B, max_drafts + 1), -1, dtype=torch.int32)
    n_accepted = torch.zeros(B, dtype=torch.int32)
    status = torch.zeros(B, dtype=torch.int32)
    p_draft = torch.full((D,), float("nan"), dtype=torch.float64)
    for b in range(B):
        o0, o1, t = int(offsets[b]), int(offsets[b + 1]), f32(float(temperatures[b]))
        if o0 < 0 or o1 < o0 or o1 > D or o1 - o0 > max_drafts:
            status[b] |= 4
        if not (t >= 0) or t == float("inf"):
            status[b] |= 8
        if status[b]:
            continue
        P = [probabilities(logits[o0 + b + j], t) for j in range(o1 - o0 + 1)]
        known = [0 <= int(drafted[i]) < V for i in range(o0, o1)]
        if not all(known):
            status[b] |= 1
        for j in range(o1 - o0):
            if P[j] is not None:
                p_draft[o0 + j] = float(P[j][int(drafted[o0 + j])]) if known[j] else 0.0
        m, refused = 0, False
        while m < o1 - o0 and P[m] is not None:
            x = int(drafted[o0 + m])
            q = 1.0 if probs is None else float(probs[o0 + m, x]) if known[m] else 0.0
            refused = not (uniform(accept_words[o0 + m]) * q < float(p_draft[o0 + m]))
            if refused:
                break
            tokens[b, m] = x
            m += 1
        n_accepted[b] = m
        if P[m] is None:
            status[b] |= 2
            continue
        r = P[m].clone()
        if refused and probs is not None:
            r = (r - torch.nan_to_num(probs[o0 + m].double(), nan=float("inf"))).clamp(min=0)
        elif refused and known[m]:
            r[int(drafted[o0 + m])] = 0
        if float(r.sum()) <= 0:
            r = P[m]
        c = torch.cumsum(r, 0)
        tokens[b, m] = int(torch.searchsorted(c, c[-1:] * uniform(sample_words[b]), right=True).clamp(max=int(r.nonzero()[-1])))
    return tokens, n_accepted, p_draft, status


# ------------------------------------------------------------------ 4-bit weights with group scales
def w4_groups(d, group):
    return (d + group - 1) // group


def bf16_nearest(v):
    """Nearest bf16 to positive 64-bit values, ties to even, by comparison (no rounding instruction): normal numbers only."""
    m, e = torch.frexp(v)                      # v = m 2^e, 1/2 <= m < 1
    scaled = m * 256                           # eight bits
    low = torch.floor(scaled)
    over = scaled - low
    up = (over > 0.5) | ((over == 0.5) & (low % 2 == 1))
    return torch.ldexp(low + up.double(), e - 8)


def w4_quantize(x, group):
    """(codes [rows, groups * group], scales [rows, groups], both 64-bit) of rows of values."""
    rows, d = x.shape
    b = torch.nn.functional.pad(x.double(), (0, -d % group)).view(rows, -1, group)
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    seventh = torch.where(bad | (top == 0), 1.0, top) / 7  # (64 bits: 29 more than the values' own)
    s = torch.where((top == 0) | (bf16_nearest(seventh) < 2.0 ** -126), 0.0, bf16_nearest(seventh))
    ok = ~bad & (s > 0)
    q = torch.where(ok.unsqueeze(-1), b, 0.0) / torch.where(ok, s, 1.0).unsqueeze(-1)
    low = torch.floor(q)
    # the border above `low`, compared by products that 64 bits hold exactly
    over = torch.where(ok.unsqueeze(-1), b, 0.0) - (low + 0.5) * torch.where(ok, s, 1.0).unsqueeze(-1)
    code = low + ((over > 0) | ((over == 0) & (low % 2 != 0))).double()
    return torch.where(ok.unsqueeze(-1), code, 0.0).flatten(1), torch.where(bad, float("nan"), s)


def w4_pack(codes, scales, d, group):
    """Stored form of codes [rows, >= d] and scales [rows, groups]: uint8 and bf16, padded with zeros."""
    rows, groups = codes.shape[0], w4_groups(d, group)
    c = torch.zeros(rows, (d + 31) // 32 * 32, dtype=torch.int64)
    c[:, :d] = codes[:, :d].long() & 15
    s = torch.zeros(rows, (groups + 7) // 8 * 8, dtype=torch.bfloat16)
    s[:, :groups] = scales.to(torch.bfloat16)
    return (c[:, 0::2] | (c[:, 1::2] << 4)).to(torch.uint8), s


def w4_values(codes, scales, d, group):
    """64-bit values [rows, d] of codes and scales as they are stored."""
    c = codes.long()
    c = torch.stack((c & 15, c >> 4), -1).flatten(1)[:, :d]
    c = torch.where(c >= 8, c - 16, c).double()
    return c * scales.double()[:, :w4_groups(d, group)].repeat_interleave(group, 1)[:, :d]
