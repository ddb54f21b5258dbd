"""Cases that measure the operators around the LM head: the final root-mean-square norm with the residual's addition
(`difr_rms_norm`), the microscaled formats with 8 and 4 bits (`difr_mx_quantize`, `difr_mx_dequantize`) and the LM-head
product on them (`difr_mx_logits`).

With `own` false `run` computes them in elementary torch operations, in 32 bits, rounded once at the end; with `own`
true it makes the library's calls.  `exact` gives the same from the definitions in 64 bits.

Microscaled tensors (blocks of 32 values along a row, one power-of-two scale each) are held as the library holds them:
`codes` uint8 [rows, pitch], a row padded with zero codes to whole blocks, one byte (e4m3) or half a byte (e2m1, the even
column in the low half) per value; `scales` uint8, exponent + 127, in blocks of 128 rows x 4 scales of 512 bytes: byte
16 (r % 32) + 4 (r % 128 // 32) + k % 4 of block (r // 128, k // 4), blocks of the same rows side by side.
What a format holds is returned as the values it stands for, in bf16 (which holds them exactly)."""
import math

import torch

own = False

EMAX = {8: 8, 4: 2}            # exponent of the formats' largest value: e4m3 448, e2m1 6
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6

LISTED = [
    # the final norm of one decoded token: latency
    dict(name="norm one token", op="norm", T=1, d=4096, dtype="bf16", residual=True, h=True, fmt=0),
    # the final norm of a teacher-forced batch, stored for the scoring calls, the residual stream updated as well
    dict(name="norm prefill", op="norm", T=65536, d=2048, dtype="bf16", residual=True, h=True, fmt=0),
    # the same for a head that multiplies in 8 bits
    dict(name="norm prefill 8 bits", op="norm", T=8192, d=5120, dtype="bf16", residual=True, h=False, fmt=8),
    # an odd hidden size, fp32 activations, no residual: rows end inside a block of 32
    dict(name="norm ragged 4 bits", op="norm", T=1531, d=1749, dtype="f32", residual=False, h=True, fmt=4),
    # the hidden states of a few decoded tokens on their way into the 4-bit product
    dict(name="quantise tokens 4 bits", op="quantise", T=61, d=4096, dtype="bf16", fmt=4),
    # a whole LM head, as a server that quantises at load time holds it
    dict(name="quantise head 4 bits", op="quantise", T=128256, d=4096, dtype="bf16", fmt=4),
    # a checkpoint in fp32, an odd vocabulary and hidden size
    dict(name="quantise ragged 8 bits", op="quantise", T=32003, d=1749, dtype="f32", fmt=8),
    # one decoded token: the head's bytes are what counts
    dict(name="logits one token 4 bits", op="logits", T=1, V=128256, d=4096, fmt=4, out="f32"),
    # a decoding batch
    dict(name="logits batch 8 bits", op="logits", T=48, V=151936, d=2048, fmt=8, out="bf16"),
    # a ragged re-scoring batch on an odd vocabulary
    dict(name="logits ragged 8 bits", op="logits", T=777, V=32003, d=1749, fmt=8, out="f32"),
    # teacher-forced re-scoring of 4096 positions
    dict(name="logits prefill 4 bits", op="logits", T=4096, V=128256, d=4096, fmt=4, out="bf16"),
    dict(name="logits prefill 8 bits", op="logits", T=4096, V=152064, d=5120, fmt=8, out="f32"),
]


def listed():
    return [dict(c) for c in LISTED]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _hidden(rng):
    # hidden sizes are multiples of 64 as a rule; the operators take any
    return 64 * _log(rng, 2, 128) if rng.random() < 0.6 else _log(rng, 100, 8192)


def draw(rng):
    op = rng.choice(("norm", "quantise", "logits"))
    while True:
        d = _hidden(rng)
        if op == "norm":
            T, dtype, fmt = _log(rng, 1, 65536), rng.choice(("bf16", "bf16", "f16", "f32")), rng.choice((0, 8, 4))
            if T * d <= 65536 * 2048:
                return dict(op=op, T=T, d=d, dtype=dtype, residual=rng.random() < 0.7, h=fmt == 0 or rng.random() < 0.3,
                            fmt=fmt)
        elif op == "quantise":
            T, dtype, fmt = _log(rng, 1, 152064), rng.choice(("bf16", "bf16", "f16", "f32")), rng.choice((8, 4))
            if T * d <= 128256 * 4096:
                return dict(op=op, T=T, d=d, dtype=dtype, fmt=fmt)
        else:
            T, V = _log(rng, 1, 4096), _log(rng, 1000, 152064)
            if T * V * d <= 4096 * 152064 * 5120:
                return dict(op=op, T=T, V=V, d=d, fmt=rng.choice((8, 4)), out=rng.choice(("f32", "bf16")))


# ------------------------------------------------------------------ the formats, plain
def _blocks(y):
    d = y.shape[1]
    return torch.nn.functional.pad(y, (0, -d % 32)).view(y.shape[0], -1, 32)


def _plain_round(y, fmt):
    """fp32 [rows, d] -> (quotients on the format's grid [rows, blocks, 32], exponents of the scales [rows, blocks])."""
    b = _blocks(y)
    amax = b.abs().amax(-1)
    e = torch.frexp(amax).exponent - 1 - EMAX[fmt]
    e = torch.where(amax > 0, e, 0).clamp(min=-126)
    q = torch.ldexp(b, -e.unsqueeze(-1))
    if fmt == 8:
        return q.clamp(-448, 448).to(torch.float8_e4m3fn).float(), e
    step = torch.where(q.abs() < 2, 0.5, torch.where(q.abs() < 4, 1.0, 2.0))
    return (torch.round(q / step) * step).clamp(-6, 6), e


def _plain_values(y, fmt):
    q, e = _plain_round(y, fmt)
    return torch.ldexp(q, e.unsqueeze(-1)).flatten(1)[:, :y.shape[1]].to(torch.bfloat16)


def _grid(device):
    return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float32, device=device)


def _encode(y, fmt):
    """(codes, exponents) of fp32 rows, as the library lays the codes out."""
    q, e = _plain_round(y, fmt)
    q = q.flatten(1)
    if fmt == 8:
        return q.to(torch.float8_e4m3fn).view(torch.uint8), e
    c = torch.bucketize(q.abs(), _grid(y.device)).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    return c[:, 0::2] | (c[:, 1::2] << 4), e


def _tile_scales(e):
    rows, nb = e.shape
    b = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -nb % 4, 0, -rows % 128))
    return b.view(b.shape[0] // 128, 4, 32, b.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _untile_scales(scales, rows, nb):
    b = scales.view(-1, (nb + 3) // 4, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, (nb + 3) // 4 * 4)
    return b[:rows, :nb].int() - 127


def _decode(codes, scales, fmt, rows, d):
    """fp32 [rows, d] values of codes and scales."""
    nb = (d + 31) // 32
    e = _untile_scales(scales, rows, nb)
    if fmt == 8:
        q = codes.view(torch.float8_e4m3fn).float()
    else:
        c = torch.stack((codes & 15, codes >> 4), -1).flatten(1)
        q = _grid(codes.device)[(c & 7).long()] * (1 - 2 * (c >> 3).float())
    return torch.ldexp(q.view(rows, nb, 32), e.unsqueeze(-1)).flatten(1)[:, :d]


# ------------------------------------------------------------------ inputs
def _mx_empty(rows, d, fmt, device):
    nb = (d + 31) // 32
    codes = torch.empty(rows, nb * 32 * fmt // 8, dtype=torch.uint8, device=device)
    return codes, torch.empty((rows + 127) // 128 * ((nb + 3) // 4) * 512, dtype=torch.uint8, device=device)


def _mx_normal(rows, d, fmt, std, g, device):
    """A microscaled tensor whose values were N(0, std^2) before they were rounded, made a part of the rows at a time."""
    codes, scales = _mx_empty(rows, d, fmt, device)
    at = 0
    for r in range(0, rows, 16384):
        n = min(16384, rows - r)
        codes[r:r + n], e = _encode(torch.randn(n, d, generator=g, device=device) * std, fmt)
        s = _tile_scales(e)
        scales[at:at + s.numel()] = s
        at += s.numel()
    return codes, scales


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    T, d = case["T"], case["d"]
    s = {"case": case}
    if case["op"] == "logits":
        V = case["V"]
        s["h"] = _mx_normal(T, d, case["fmt"], 1.0, g, dev)
        s["W"] = _mx_normal(V, d, case["fmt"], d ** -0.5, g, dev)
        s["logits"] = torch.empty(T, V, dtype=DTYPES[case["out"]], device=dev)
        return s
    dt = DTYPES[case["dtype"]]
    s["x"] = torch.empty(T, d, dtype=dt, device=dev)
    std = 1.0 if case["op"] == "norm" else d ** -0.5
    for r in range(0, T, 16384):
        s["x"][r:r + 16384] = torch.randn(min(16384, T - r), d, generator=g, device=dev) * std
    if case["op"] == "norm":
        # a few channels of the residual stream are far larger than the others
        wide = torch.exp(torch.randn(d, generator=g, device=dev))
        s["weight"] = (1 + 0.2 * torch.randn(d, generator=g, device=dev)).to(dt)
        if case["residual"]:
            s["residual"] = (torch.randn(T, d, generator=g, device=dev) * wide).to(dt)
            s["stream"] = torch.empty(T, d, dtype=dt, device=dev)
        if case["h"]:
            s["h"] = torch.empty(T, d, dtype=torch.bfloat16, device=dev)
    if case["fmt"]:
        s["mx"] = _mx_empty(T, d, case["fmt"], dev)
        s["values"] = torch.empty(T, d, dtype=torch.bfloat16, device=dev)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "logits":
        h = _decode(*s["h"], c["fmt"], c["T"], c["d"])
        W = _decode(*s["W"], c["fmt"], c["V"], c["d"])
        return {"logits": (h @ W.T).to(DTYPES[c["out"]])}
    if c["op"] == "quantise":
        return {"values": _plain_values(s["x"].float(), c["fmt"])}
    out = {}
    v = s["x"].float()
    if c["residual"]:
        out["residual"] = (v + s["residual"].float()).to(s["x"].dtype)
        v = out["residual"].float()
    y = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
    if c["h"]:
        out["h"] = y.to(torch.bfloat16)
    if c["fmt"]:
        out["values"] = _plain_values(y, c["fmt"])
    return out


def _run_own(s):
    import paper_2511_02620_b200 as difr

    c = s["case"]
    T, d = c["T"], c["d"]
    if c["op"] == "logits":
        difr.difr_mx_logits(difr.MxTensor(*s["h"], c["fmt"], T, d), difr.MxTensor(*s["W"], c["fmt"], c["V"], d), s["logits"])
        return {"logits": s["logits"]}
    mx = difr.MxTensor(*s["mx"], c["fmt"], T, d) if c["fmt"] else None
    out = {}
    if c["op"] == "quantise":
        difr.difr_mx_quantize(s["x"], mx)
    else:
        o = difr.NormOut(h=s.get("h"), residual=s.get("stream"), mx=mx)
        difr.difr_rms_norm(s["x"], s["weight"], EPS, o, residual=s.get("residual"))
        if c["residual"]:
            out["residual"] = o.residual
        if c["h"]:
            out["h"] = o.h
    if c["fmt"]:
        out["values"] = difr.difr_mx_dequantize(mx, s["values"])
    return out


# ------------------------------------------------------------------ what a pass cannot do without
def _mx_bytes(rows, d, fmt):
    return rows * d * fmt / 8 + rows * ((d + 31) // 32)


def work(case):
    T, d = case["T"], case["d"]
    if case["op"] == "logits":
        V, size = case["V"], DTYPES[case["out"]].itemsize
        return {"bytes": _mx_bytes(T, d, case["fmt"]) + _mx_bytes(V, d, case["fmt"]) + T * V * size,
                "flops": 2 * T * V * d}
    size = DTYPES[case["dtype"]].itemsize
    n = T * d * size
    if case["fmt"]:
        n += _mx_bytes(T, d, case["fmt"]) + T * d * 2
    if case["op"] == "norm":
        n += d * size + 2 * T * d * size * case["residual"] + T * d * 2 * case["h"]
    return {"bytes": n, "flops": T * d * (6 if case["op"] == "norm" else 3)}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_nearest(q, fmt):
    """Nearest value of the format, ties to the even code, by its table: no rounding instruction of any kind."""
    if fmt == 4:
        table = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    else:
        table = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)]
        table = table[:-1]  # the last pattern is NaN: 448 is the largest value
    t = torch.tensor(table, dtype=torch.float64, device=q.device)
    mid = (t[1:] + t[:-1]) / 2
    a = q.abs()
    low = torch.bucketize(a, mid, right=False)   # a tie goes to the lower code ...
    high = torch.bucketize(a, mid, right=True)   # ... or to the upper one
    return torch.copysign(t[torch.where(low % 2 == 0, low, high)], q)


def _exact_values(y, fmt):
    y = y.double()
    rows, d = y.shape
    out = torch.zeros(rows, (d + 31) // 32 * 32, dtype=torch.float64, device=y.device)
    out[:, :d] = y
    out = out.view(rows, -1, 32)
    top = out.abs().max(-1, keepdim=True).values
    s = torch.where(top > 0, torch.exp2(torch.floor(torch.log2(top)) - EMAX[fmt]), 1.0)
    return (_exact_nearest(out / s, fmt) * s).reshape(rows, -1)[:, :d]


def _exact_decode(codes, scales, fmt, rows, d):
    nb = (d + 31) // 32
    r = torch.arange(rows, device=codes.device).view(-1, 1)
    k = torch.arange(nb, device=codes.device).view(1, -1)
    at = (r // 128 * ((nb + 3) // 4) + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4
    s = torch.exp2(scales[at].double() - 127)
    col = torch.arange(nb * 32, device=codes.device)
    if fmt == 4:
        code = (codes[:, col // 2] >> (col % 2 * 4).to(torch.uint8)) & 15
        sign, exp, man = code >> 3, (code >> 1) & 3, code & 1
        q = torch.where(exp == 0, man * 0.5, (1 + man * 0.5) * torch.exp2(exp.double() - 1))
    else:
        sign, exp, man = codes >> 7, (codes >> 3) & 15, codes & 7
        q = torch.where(exp == 0, man / 8 * 2.0 ** -6, (1 + man.double() / 8) * torch.exp2(exp.double() - 7))
    q = torch.where(sign == 1, -q, q).double()
    return (q.view(rows, nb, 32) * s.view(rows, nb, 1)).view(rows, -1)[:, :d]


def exact(case, seed):
    s = prepare(case, seed)
    T, d, fmt = case["T"], case["d"], case["fmt"]
    if case["op"] == "logits":
        h = _exact_decode(*s["h"], fmt, T, d)
        W = torch.empty(case["V"], d, dtype=torch.float64, device=h.device)
        codes, scales = s["W"]
        per = scales.numel() // ((case["V"] + 127) // 128)
        for r in range(0, case["V"], 16384):
            n = min(16384, case["V"] - r)
            W[r:r + n] = _exact_decode(codes[r:r + n], scales[r // 128 * per:(r + n + 127) // 128 * per], fmt, n, d)
        return {"logits": torch.mm(h, W.t())}
    if case["op"] == "quantise":
        out = torch.empty(T, d, dtype=torch.float64, device=s["x"].device)
        for r in range(0, T, 16384):
            out[r:r + 16384] = _exact_values(s["x"][r:r + 16384], fmt)
        return {"values": out}
    out = {}
    v = s["x"].double()
    if case["residual"]:
        # the stream itself is held in the inputs' type, and the norm is taken of what is held
        v = (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()
        out["residual"] = v
    y = s["weight"].double() * (v / torch.sqrt((v * v).sum(1, keepdim=True) / d + EPS))
    if case["h"]:
        out["h"] = y
    if fmt:
        out["values"] = torch.cat([_exact_values(p, fmt) for p in y.split(8192)])
    return out
