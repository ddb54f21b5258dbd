"""Plain 64-bit statements of the microscaled formats and the final norm, for the tests: by table and comparison, no
rounding instruction of the formats is used.  Tensors are torch CPU tensors."""
import torch

EMAX = {8: 8, 4: 2}


def table(fmt):
    """Magnitudes of the format in the order of their codes."""
    if fmt == 4:
        return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    t = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)]
    return torch.tensor(t[:-1], dtype=torch.float64)  # the last pattern is NaN


def blocks(y):
    d = y.shape[1]
    return torch.nn.functional.pad(y.double(), (0, -d % 32)).view(y.shape[0], -1, 32)


def scale_exponents(b, fmt):
    """Exponents of the blocks' scales, 128 for blocks that hold a NaN or an infinity."""
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    m, e = torch.frexp(torch.where(bad | (top == 0), 1.0, top))
    e = (e - 1 - EMAX[fmt]).clamp(min=-127)
    e = torch.where(top == 0, -127, e)
    return torch.where(bad, 128, e)


def quantize(y, fmt):
    """(codes [rows, padded d] one per value, scale bytes [rows, blocks])."""
    b = blocks(y)
    e = scale_exponents(b, fmt)
    bad = e == 128
    q = torch.where(bad.unsqueeze(-1), 0.0, b) * torch.exp2(-torch.where(bad, 0, e).double()).unsqueeze(-1)
    t = table(fmt)
    mid = (t[1:] + t[:-1]) / 2
    a = q.abs()
    low, high = torch.bucketize(a, mid, right=False), torch.bucketize(a, mid, right=True)
    c = torch.where(low % 2 == 0, low, high)  # a tie goes to the even code
    c = c | (torch.signbit(q).long() << (fmt - 1))
    return c.flatten(1), (e + 127)


def pack(c, fmt):
    c = c.to(torch.uint8)
    return c if fmt == 8 else c[:, 0::2] | (c[:, 1::2] << 4)


def tile_scales(byte, fill=0):
    """Scale bytes [rows, blocks] in the stored layout, one at a time as the header states it."""
    rows, nb = byte.shape
    words = (nb + 3) // 4
    out = torch.full(((rows + 127) // 128 * words * 512,), fill, dtype=torch.uint8)
    r = torch.arange(rows).view(-1, 1)
    k = torch.arange(words * 4).view(1, -1)
    full = torch.zeros(rows, words * 4, dtype=torch.uint8)
    full[:, :nb] = byte.to(torch.uint8)
    out[512 * (r // 128 * words + k // 4) + 16 * (r % 32) + 4 * (r % 128 // 32) + k % 4] = full
    return out


def values(c, byte, fmt, d):
    """64-bit values of codes (one per value) and scale bytes."""
    mag = table(fmt)[(c & (2 ** (fmt - 1) - 1))]
    v = torch.where((c >> (fmt - 1)) == 1, -mag, mag).view(c.shape[0], -1, 32)
    s = torch.where(byte == 255, float("nan"), torch.exp2(byte.double() - 127))
    return (v * s.unsqueeze(-1)).flatten(1)[:, :d]


def unpack(codes, fmt):
    codes = codes.long()
    return codes if fmt == 8 else torch.stack((codes & 15, codes >> 4), -1).flatten(1)


def untile_scales(scales, rows, nb):
    words = (nb + 3) // 4
    r = torch.arange(rows).view(-1, 1)
    k = torch.arange(nb).view(1, -1)
    return scales[512 * (r // 128 * words + k // 4) + 16 * (r % 32) + 4 * (r % 128 // 32) + k % 4].long()


def rms_norm(x, residual, weight, eps):
    """(residual stream in x's type, y in 64 bits)."""
    r = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    v = r.double()
    return r, v / torch.sqrt((v * v).mean(-1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32))) * weight.double()
