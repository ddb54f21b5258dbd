"""Cases that measure the operators of a decoding step with drafted tokens, from the last block's output to the tokens:
the norms before and after a block with its gate and residual scale (`difr_block_norm`), a head held as 4-bit integers
with group scales (`difr_w4_quantize`, `difr_w4_dequantize`) and the product with bf16 hidden states on it
(`difr_w4_logits`), and the verification of drafted tokens from given random words (`difr_verify_drafts`).

With `own` false `run` computes them in elementary torch operations, in 32 bits (64 where a border decides a whole
number), rounded once at the end; with `own` true it makes the library's calls.  `exact` gives the same from the
definitions in 64 bits.

A 4-bit weight is an integer code -8 .. 7 times the bf16 scale of its group of 32, 64 or 128 values along a row.  Codes lie
in two's complement, two to a byte (the even column in the low half), rows padded with zeros to whole 32 columns; scales
bf16 [rows, groups], rows padded to whole 8 scales.

Request b has the drafted tokens offsets[b] .. offsets[b + 1] - 1 and one row of target logits for each and one more: its
rows start at offsets[b] + b."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6

LISTED = [
    # the end of one decoding step of one token: norm after the last block, residual, final norm; latency
    dict(name="block norm one token", op="norm", T=1, d=4096, dtype="bf16", post=True, gate="none", alpha=1.0, beta=1.0,
         h=True, fmt=0),
    # a teacher-forced batch, the block's output scaled per channel
    dict(name="block norm prefill", op="norm", T=65536, d=2048, dtype="bf16", post=True, gate="channel", alpha=1.0, beta=1.0,
         h=True, fmt=0),
    # an odd hidden size in fp32, a gate per token, both scales, the result in 4 bits
    dict(name="block norm ragged 4 bits", op="norm", T=1531, d=1749, dtype="f32", post=True, gate="token", alpha=0.22,
         beta=1.5, h=False, fmt=4),
    # a whole LM head, as a server that quantises at load time holds it
    dict(name="quantise head", op="quantise", T=128256, d=4096, dtype="bf16", group=128),
    # a checkpoint in fp32, an odd vocabulary and hidden size, small groups
    dict(name="quantise ragged", op="quantise", T=32003, d=1749, dtype="f32", group=32),
    # one decoded token: the head's bytes are what counts
    dict(name="logits one token", op="logits", T=1, V=128256, d=4096, group=128, out="f32"),
    # a batch of requests with their drafted tokens
    dict(name="logits drafts", op="logits", T=60, V=151936, d=2048, group=64, out="bf16"),
    # a ragged re-scoring batch, an odd vocabulary and hidden size
    dict(name="logits ragged", op="logits", T=777, V=32003, d=1749, group=32, out="f32"),
    # teacher-forced re-scoring of 4096 positions
    dict(name="logits prefill", op="logits", T=4096, V=128256, d=4096, group=128, out="bf16"),
    # one request with four drafted tokens: latency
    dict(name="verify one request", op="verify", B=1, K=4, ragged=False, V=128256, dtype="f32", temperature=1.0, probs=True),
    # a serving batch, between none and eight drafted tokens each
    dict(name="verify batch", op="verify", B=192, K=8, ragged=True, V=151936, dtype="bf16", temperature=0.7, probs=True),
    # greedy requests whose drafts were looked up in the prompt (no draft probabilities), odd vocabulary
    dict(name="verify greedy lookups", op="verify", B=37, K=3, ragged=True, V=32003, dtype="f32", temperature=0.0, probs=False),
]


def listed():
    return [dict(c) for c in LISTED]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _hidden(rng):
    # hidden sizes are multiples of 64 as a rule; the operators take any
    return 64 * _log(rng, 2, 128) if rng.random() < 0.6 else _log(rng, 100, 8192)


def draw(rng):
    op = rng.choice(("norm", "quantise", "logits", "logits", "verify", "verify"))
    while True:
        d = _hidden(rng)
        if op == "norm":
            T, fmt = _log(rng, 1, 65536), rng.choice((0, 0, 8, 4))
            if T * d <= 65536 * 2048:
                return dict(op=op, T=T, d=d, dtype=rng.choice(("bf16", "bf16", "f16", "f32")), post=rng.random() < 0.8,
                            gate=rng.choice(("none", "channel", "token")), alpha=rng.choice((1.0, 0.22)),
                            beta=rng.choice((1.0, 1.5)), h=fmt == 0 or rng.random() < 0.3, fmt=fmt)
        elif op == "quantise":
            T = _log(rng, 1, 152064)
            if T * d <= 128256 * 4096:
                return dict(op=op, T=T, d=d, dtype=rng.choice(("bf16", "bf16", "f16", "f32")), group=rng.choice((32, 64, 128)))
        elif op == "logits":
            T, V = _log(rng, 1, 4096), _log(rng, 1000, 152064)
            if T * V * d <= 4096 * 128256 * 4096:
                return dict(op=op, T=T, V=V, d=d, group=rng.choice((32, 64, 128)), out=rng.choice(("f32", "bf16")))
        else:
            B, K, V = _log(rng, 1, 192), rng.randint(1, 8), _log(rng, 1000, 152064)
            return dict(op=op, B=B, K=K, ragged=rng.random() < 0.6, V=V, dtype=rng.choice(("bf16", "f32")),
                        temperature=rng.choice((1.0, 0.7, 0.0)), probs=rng.random() < 0.7)


# ------------------------------------------------------------------ the formats, plain
def _w4_pitches(d, group):
    return (d + 31) // 32 * 16, ((d + group - 1) // group + 7) // 8 * 8


def _w4_codes(y, group):
    """(codes [rows, d rounded up to groups], bf16 scales [rows, groups]) of rows of values."""
    rows, d = y.shape
    b = torch.nn.functional.pad(y, (0, -d % group)).view(rows, -1, group).double()
    s = (b.abs().amax(-1) / 7).float().to(torch.bfloat16)
    q = torch.round(b / torch.where(s > 0, s, 1).double().unsqueeze(-1)).clamp(-8, 7)
    return q.to(torch.int8).flatten(1), s


def _w4_pack(q, pitch):
    q = torch.nn.functional.pad(q, (0, max(0, 2 * pitch - q.shape[1])))[:, :2 * pitch]
    return (q[:, 0::2] & 15 | q[:, 1::2] << 4).view(torch.uint8)


def _w4_decode(codes, scales, group, rows, d):
    """fp32 [rows, d] values of codes and scales."""
    c = codes.view(torch.int8)
    q = torch.stack((c << 4 >> 4, c >> 4), -1).flatten(1)[:, :d]
    s = scales[:, :(d + group - 1) // group].float().repeat_interleave(group, 1)[:, :d]
    return q * s


EMAX = {8: 8, 4: 2}            # exponent of the microscaled formats' largest value: e4m3 448, e2m1 6


def _mx_values(y, fmt):
    """fp32 rows rounded to a microscaled format (blocks of 32, a power-of-two scale each), as bf16 values."""
    b = torch.nn.functional.pad(y, (0, -y.shape[1] % 32)).view(y.shape[0], -1, 32)
    top = b.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top).exponent - 1 - EMAX[fmt], 0).clamp(min=-126).unsqueeze(-1)
    q = torch.ldexp(b, -e)
    if fmt == 8:
        q = q.clamp(-448, 448).to(torch.float8_e4m3fn).float()
    else:
        step = torch.where(q.abs() < 2, 0.5, torch.where(q.abs() < 4, 1.0, 2.0))
        q = (torch.round(q / step) * step).clamp(-6, 6)
    return torch.ldexp(q, e).flatten(1)[:, :y.shape[1]].to(torch.bfloat16)


# ------------------------------------------------------------------ inputs
def _counts(case):
    """Drafted tokens of each request: all K, or between none and K."""
    B, K = case["B"], case["K"]
    return [(b * 5 + 3) % (K + 1) if case["ragged"] else K for b in range(B)]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "verify":
        return _prepare_verify(case, s, g, dev)
    T, d = case["T"], case["d"]
    if case["op"] == "logits":
        V, group = case["V"], case["group"]
        pitch, spitch = _w4_pitches(d, group)
        s["h"] = torch.randn(T, d, generator=g, device=dev).to(torch.bfloat16)
        s["codes"] = torch.empty(V, pitch, dtype=torch.uint8, device=dev)
        s["scales"] = torch.zeros(V, spitch, dtype=torch.bfloat16, device=dev)
        for r in range(0, V, 8192):
            q, scale = _w4_codes(torch.randn(min(8192, V - r), d, generator=g, device=dev) * d ** -0.5, group)
            s["codes"][r:r + 8192] = _w4_pack(q, pitch)
            s["scales"][r:r + 8192, :scale.shape[1]] = scale
        s["logits"] = torch.empty(T, V, dtype=DTYPES[case["out"]], device=dev)
        # what the product keeps of the hidden states for a call, at most: two bytes a value and a few more a row
        s["workspace"] = torch.empty(T * (2 * ((d + 63) // 64 * 64) + 64) + 1024, dtype=torch.uint8, device=dev)
        return s
    dt = DTYPES[case["dtype"]]
    s["x"] = torch.empty(T, d, dtype=dt, device=dev)
    std = 1.0 if case["op"] == "norm" else d ** -0.5
    for r in range(0, T, 16384):
        s["x"][r:r + 16384] = torch.randn(min(16384, T - r), d, generator=g, device=dev) * std
    if case["op"] == "quantise":
        pitch, spitch = _w4_pitches(d, case["group"])
        s["codes"] = torch.empty(T, pitch, dtype=torch.uint8, device=dev)
        s["scales"] = torch.empty(T, spitch, dtype=torch.bfloat16, device=dev)
        s["values"] = torch.empty(T, d, dtype=torch.bfloat16, device=dev)
        return s
    # a few channels of the residual stream are far larger than the others
    wide = torch.exp(torch.randn(d, generator=g, device=dev))
    s["residual"] = (torch.randn(T, d, generator=g, device=dev) * wide).to(dt)
    s["stream"] = torch.empty(T, d, dtype=dt, device=dev)
    s["weight"] = (1 + 0.2 * torch.randn(d, generator=g, device=dev)).to(dt)
    s["post_weight"] = (1 + 0.2 * torch.randn(d, generator=g, device=dev)).to(dt) if case["post"] else None
    gates = {"none": 0, "channel": 1, "token": T}[case["gate"]]
    s["gate"] = torch.tanh(torch.randn(gates, d, generator=g, device=dev)).to(dt) if gates else None
    if case["h"]:
        s["h"] = torch.empty(T, d, dtype=torch.bfloat16, device=dev)
    if case["fmt"]:
        nb = (d + 31) // 32
        s["mx"] = (torch.empty(T, nb * 4 * case["fmt"], dtype=torch.uint8, device=dev),
                   torch.empty((T + 127) // 128 * ((nb + 3) // 4) * 512, dtype=torch.uint8, device=dev))
        s["values"] = torch.empty(T, d, dtype=torch.bfloat16, device=dev)
    return s


def _prepare_verify(case, s, g, dev):
    B, V, K = case["B"], case["V"], case["K"]
    n = _counts(case)
    offsets = [0]
    for c in n:
        offsets.append(offsets[-1] + c)
    D = offsets[-1]
    s["D"] = D
    s["offsets"] = torch.tensor(offsets, dtype=torch.int32, device=dev)
    temperature = case["temperature"]
    s["logits"] = torch.empty(D + B, V, dtype=DTYPES[case["dtype"]], device=dev)
    s["tokens"] = torch.empty(D, dtype=torch.int32, device=dev)
    s["probs"] = torch.empty(D, V, device=dev) if case["probs"] else None
    for b in range(B):
        r = offsets[b] + b
        # a wide bulk and a few likely tokens
        l = 2.5 * torch.randn(n[b] + 1, V, generator=g, device=dev)
        at = torch.randint(0, V, (n[b] + 1, 4), generator=g, device=dev)
        l.scatter_(1, at, 9 + 2.5 * torch.randn(n[b] + 1, 4, generator=g, device=dev))
        s["logits"][r:r + n[b] + 1] = l
        if n[b]:
            # a draft model that is near the target: its tokens are sampled from its own probabilities
            q = (l[:-1] + 0.6 * torch.randn(n[b], V, generator=g, device=dev)) / (temperature or 0.5)
            noise = torch.rand(n[b], V, generator=g, device=dev).clamp_(1e-9, 1 - 1e-7)
            s["tokens"][offsets[b]:offsets[b + 1]] = (q - torch.log(-torch.log(noise))).argmax(-1)
            if case["probs"]:
                s["probs"][offsets[b]:offsets[b + 1]] = torch.softmax(q, -1)
    s["accept_words"] = torch.randint(-2 ** 31, 2 ** 31, (D,), generator=g, device=dev, dtype=torch.int32)
    s["sample_words"] = torch.randint(-2 ** 31, 2 ** 31, (B,), generator=g, device=dev, dtype=torch.int32)
    i = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=dev)
    # tokens, n_accepted, p_draft, status; and what a call keeps between its passes: at most 16 bytes per 2048 logits and a
    # few more a row
    s["out"] = (i(B, K + 1), i(B), torch.empty(D, device=dev), i(B),
                torch.empty((D + B) * ((V + 2047) // 2048 * 16 + 64) + 4096, dtype=torch.uint8, device=dev))
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "verify":
        return _plain_verify(s)
    if c["op"] == "logits":
        W = _w4_decode(s["codes"], s["scales"], c["group"], c["V"], c["d"])
        return {"logits": (s["h"].float() @ W.T).to(DTYPES[c["out"]])}
    if c["op"] == "quantise":
        q, scale = _w4_codes(s["x"], c["group"])
        v = (q.view(c["T"], -1, c["group"]) * scale.float().unsqueeze(-1)).flatten(1)[:, :c["d"]]
        return {"values": v.to(torch.bfloat16)}
    v = s["x"].float()
    if c["post"]:
        v = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * s["post_weight"].float()
    if s["gate"] is not None:
        v = v * s["gate"].float()
    r = (c["beta"] * s["residual"].float() + c["alpha"] * v).to(s["x"].dtype)
    v = r.float()
    y = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
    out = {"residual": r}
    if c["h"]:
        out["h"] = y.to(torch.bfloat16)
    if c["fmt"]:
        out["values"] = _mx_values(y, c["fmt"])
    return out


def _uniform(words):
    return ((words.long() & 0xFFFFFFFF).double() + 0.5) * 2.0 ** -32


def _plain_verify(s):
    """In 64 bits: a drafted token is accepted or not, and a sample falls into one token's interval or the next one's, at a
    border."""
    c = s["case"]
    B, V, K, D = c["B"], c["V"], c["K"], s["D"]
    dev = s["logits"].device
    off = s["offsets"].long()
    n = off[1:] - off[:-1]
    l = s["logits"].double()
    top = l.amax(-1, keepdim=True)
    if c["temperature"] > 0:
        p = torch.exp((l - top) / c["temperature"])
        p = p / p.sum(-1, keepdim=True)
    else:
        ids = torch.arange(V, device=dev)
        p = (ids == torch.where(l == top, ids, V).amin(-1, keepdim=True)).double()
    request = torch.repeat_interleave(torch.arange(B, device=dev), n, output_size=D)
    draft = torch.arange(D, device=dev)
    tok = s["tokens"].long()
    p_draft = p[draft + request, tok]
    q_draft = s["probs"][draft, tok].double() if c["probs"] else 1.0
    accepted = torch.zeros(B, K + 1, dtype=torch.bool, device=dev)
    accepted[request, draft - off[request]] = _uniform(s["accept_words"]) * q_draft < p_draft
    n_accepted = accepted.long().cumprod(1).sum(1)
    # the row that the last token is sampled from, and what the draft takes away from it
    r = p[off[:-1] + torch.arange(B, device=dev) + n_accepted]
    refused = (n_accepted < n).unsqueeze(1)
    at = (off[:-1] + n_accepted).clamp(max=max(D - 1, 0))
    if D > 0:
        if c["probs"]:
            less = (r - s["probs"][at].double()).clamp(min=0)
        else:
            less = torch.where(torch.arange(V, device=dev) == tok[at].unsqueeze(1), 0.0, r)
        r = torch.where(refused & (less.sum(1, keepdim=True) > 0), less, r)
    cum = r.cumsum(1)
    last = (cum <= _uniform(s["sample_words"]).unsqueeze(1) * cum[:, -1:]).sum(1)
    j = torch.arange(K + 1, device=dev)
    padded = torch.zeros(B, K + 1, dtype=torch.long, device=dev)
    padded[request, draft - off[request]] = tok
    tokens = torch.where(j < n_accepted.unsqueeze(1), padded, torch.where(j == n_accepted.unsqueeze(1), last.unsqueeze(1), -1))
    return {"tokens": tokens.to(torch.int32), "n_accepted": n_accepted.to(torch.int32), "p_draft": p_draft.float()}


def _run_own(s):
    import paper_2511_02620_b200 as difr

    c = s["case"]
    if c["op"] == "verify":
        o = difr.difr_verify_drafts(s["logits"], s["tokens"], s["offsets"], s["accept_words"], s["sample_words"],
                                    c["temperature"], difr.DraftOut(*s["out"]), draft_probs=s["probs"])
        return {"tokens": o.tokens, "n_accepted": o.n_accepted, "p_draft": o.p_draft}
    T, d = c["T"], c["d"]
    if c["op"] == "logits":
        W = difr.W4Tensor(s["codes"], s["scales"], c["group"], c["V"], d)
        return {"logits": difr.difr_w4_logits(s["h"], W, s["logits"], s["workspace"])}
    if c["op"] == "quantise":
        w = difr.W4Tensor(s["codes"], s["scales"], c["group"], T, d)
        difr.difr_w4_quantize(s["x"], w)
        return {"values": difr.difr_w4_dequantize(w, s["values"])}
    mx = difr.MxTensor(*s["mx"], c["fmt"], T, d) if c["fmt"] else None
    o = difr.NormOut(h=s.get("h"), residual=s["stream"], mx=mx)
    difr.difr_block_norm(s["x"], s["residual"], s["weight"], EPS, o, post_weight=s["post_weight"], gate=s["gate"],
                         scale=c["alpha"], residual_scale=c["beta"])
    out = {"residual": o.residual}
    if c["h"]:
        out["h"] = o.h
    if c["fmt"]:
        out["values"] = difr.difr_mx_dequantize(mx, s["values"])
    return out


# ------------------------------------------------------------------ what a pass cannot do without
def _w4_bytes(rows, d, group):
    return rows * d / 2 + rows * ((d + group - 1) // group) * 2


def work(case):
    if case["op"] == "verify":
        n = _counts(case)
        D, V, size = sum(n), case["V"], DTYPES[case["dtype"]].itemsize
        # the target's rows once, and one row of draft probabilities for a request whose draft is refused somewhere
        return {"bytes": (D + case["B"]) * V * size + (sum(c > 0 for c in n) * V * 4 if case["probs"] and case["temperature"] > 0 else 0),
                "flops": (D + case["B"]) * V * 4}
    T, d = case["T"], case["d"]
    if case["op"] == "logits":
        V, size = case["V"], DTYPES[case["out"]].itemsize
        return {"bytes": T * d * 2 + _w4_bytes(V, d, case["group"]) + T * V * size, "flops": 2 * T * V * d}
    size = DTYPES[case["dtype"]].itemsize
    if case["op"] == "quantise":
        # the codes are written and read again: the values are what a pass returns
        return {"bytes": T * d * (size + 2) + 2 * _w4_bytes(T, d, case["group"]), "flops": T * d * 4}
    b = T * d * size * 3 + d * size * (1 + case["post"])
    b += {"none": 0, "channel": 1, "token": T}[case["gate"]] * d * size + T * d * 2 * case["h"]
    if case["fmt"]:
        b += 2 * (T * d * case["fmt"] / 8 + T * ((d + 31) // 32)) + T * d * 2
    return {"bytes": b, "flops": T * d * 12}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_mx(y, fmt):
    """Nearest value of the format by its table, ties to the even code."""
    if fmt == 4:
        table = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    else:
        table = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)]
        table = table[:-1]  # the last pattern is NaN: 448 is the largest value
    t = torch.tensor(table, dtype=torch.float64, device=y.device)
    mid = (t[1:] + t[:-1]) / 2
    rows, d = y.shape
    b = torch.zeros(rows, (d + 31) // 32 * 32, dtype=torch.float64, device=y.device)
    b[:, :d] = y
    b = b.view(rows, -1, 32)
    top = b.abs().max(-1, keepdim=True).values
    scale = torch.where(top > 0, torch.exp2(torch.floor(torch.log2(top)) - EMAX[fmt]), 1.0)
    a = (b / scale).abs()
    low, high = torch.bucketize(a, mid, right=False), torch.bucketize(a, mid, right=True)
    return (torch.copysign(t[torch.where(low % 2 == 0, low, high)], b) * scale).reshape(rows, -1)[:, :d]


def _exact_group_values(x, group):
    """Values of one group of columns: scale the bf16 nearest to a seventh of the largest magnitude, integers by comparison
    with the borders between them."""
    x = x.double()
    top = x.abs().max(-1, keepdim=True).values
    s = (top / 7).to(torch.bfloat16).double()
    low = torch.floor(x / torch.where(s > 0, s, 1.0))
    over = x - (low + 0.5) * s
    q = torch.where((over > 0) | ((over == 0) & (low % 2 != 0)), low + 1, low)
    return torch.where(s > 0, q.clamp(-8, 7) * s, 0.0)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "verify":
        return _exact_verify(s)
    T, d = case["T"], case["d"]
    if case["op"] == "logits":
        group, V = case["group"], case["V"]
        W = torch.empty(V, d, dtype=torch.float64, device=s["h"].device)
        for k in range(d):
            nibble = (s["codes"][:, k // 2] >> (4 * (k % 2))) & 15
            W[:, k] = (nibble.double() - 16 * (nibble >= 8)) * s["scales"][:, k // group].double()
        return {"logits": torch.mm(s["h"].double(), W.t())}
    if case["op"] == "quantise":
        group = case["group"]
        out = torch.empty(T, d, dtype=torch.float64, device=s["x"].device)
        for k in range(0, d, group):
            out[:, k:k + group] = _exact_group_values(s["x"][:, k:k + group], group)
        return {"values": out}
    x = s["x"].double()
    if case["post"]:
        x = s["post_weight"].double() * (x / torch.sqrt((x * x).sum(1, keepdim=True) / d + EPS))
    if case["gate"] != "none":
        x = x * s["gate"].double()
    r = case["beta"] * s["residual"].double() + case["alpha"] * x
    out = {"residual": r}
    # the stream itself is held in the inputs' type, and the norm is taken of what is held
    held = r.float().to(s["x"].dtype).double()
    y = s["weight"].double() * (held / torch.sqrt((held * held).sum(1, keepdim=True) / d + EPS))
    if case["h"]:
        out["h"] = y
    if case["fmt"]:
        out["values"] = torch.cat([_exact_mx(part, case["fmt"]) for part in y.split(8192)])
    return out


def _exact_verify(s):
    """Request by request, as the procedure is told."""
    c = s["case"]
    B, V, K, temperature = c["B"], c["V"], c["K"], c["temperature"]
    off, drafted = s["offsets"].tolist(), s["tokens"].tolist()
    accept, sample = s["accept_words"].tolist(), s["sample_words"].tolist()
    tokens = torch.full((B, K + 1), -1, dtype=torch.int32)
    n_accepted = torch.zeros(B, dtype=torch.int32)
    p_draft = torch.zeros(s["D"], dtype=torch.float64)
    for b in range(B):
        n, refused = off[b + 1] - off[b], None
        rows = s["logits"][off[b] + b:off[b + 1] + b + 1].double()
        if temperature > 0:
            P = torch.exp(rows / temperature - torch.logsumexp(rows / temperature, 1, keepdim=True))
        else:
            P = torch.zeros_like(rows)
            for j in range(n + 1):
                P[j, int((rows[j] == rows[j].max()).nonzero()[0, 0])] = 1.0
        for j in range(n):
            i = off[b] + j
            p_draft[i] = P[j, drafted[i]]
            q = float(s["probs"][i, drafted[i]]) if c["probs"] else 1.0
            if refused is None and not ((accept[i] % 2 ** 32) + 0.5) / 2 ** 32 * q < float(p_draft[i]):
                refused = j
        m = n if refused is None else refused
        r = P[m].clone()
        if refused is not None:
            if c["probs"]:
                r -= s["probs"][off[b] + m].double()
                r[r < 0] = 0
            else:
                r[drafted[off[b] + m]] = 0
            if float(r.sum()) <= 0:
                r = P[m]
        cum = torch.cumsum(r, 0)
        at = torch.searchsorted(cum, cum[-1:] * (((sample[b] % 2 ** 32) + 0.5) / 2 ** 32), right=True)
        tokens[b, :m] = torch.tensor(drafted[off[b]:off[b] + m], dtype=torch.int32)
        tokens[b, m] = int(at)
        n_accepted[b] = m
    dev = s["logits"].device
    return {"tokens": tokens.to(dev), "n_accepted": n_accepted.to(dev), "p_draft": p_draft.to(dev)}
