"""Host side of the operators around the LM head: sizes, refusals before the device is touched, and the test reference's
own pins (CPU)."""
import ctypes

import pytest
import torch

import mx_reference as ref
import paper_2511_02620_b200 as difr
from paper_2511_02620_b200.build import build

INVALID, SHAPE, ALIGN, OK = -1, -2, -3, 0


def test_sizes():
    build()
    assert difr.difr_mx_codes_bytes(8, 3, 33) == 3 * 64
    assert difr.difr_mx_codes_bytes(4, 3, 33) == 3 * 32
    assert difr.difr_mx_codes_bytes(4, 128256, 4096) == 128256 * 2048
    assert difr.difr_mx_scales_bytes(1, 1) == 512
    assert difr.difr_mx_scales_bytes(129, 129) == 2 * 2 * 512
    for fmt, rows, d in ((6, 1, 1), (8, 0, 1), (8, 1, 0), (4, -1, 5), (4, (1 << 30) + 1, 1), (4, 1, (1 << 20) + 1)):
        assert difr.difr_mx_codes_bytes(fmt, rows, d) == 0
    assert difr.difr_mx_scales_bytes(0, 5) == 0 and difr.difr_mx_scales_bytes(5, 0) == 0
    with pytest.raises(ValueError):
        difr.MxTensor.allocate(4, 64, 6, device="cpu")


def test_refusals_on_the_host():
    """These calls run without a GPU and never dereference the (fake) pointers."""
    if torch.cuda.is_available():
        pytest.skip("host-only check: run it where no CUDA device is visible")
    L = difr.lib()
    p, odd = 0x10000, 0x10008

    def q(x=p, dtype=0, rows=8, d=64, ld=64, fmt=4, codes=p, scales=p):
        return L.difr_mx_quantize(x, dtype, rows, d, ld, fmt, codes, scales, None)

    assert q(x=None) == INVALID and q(codes=None) == INVALID and q(scales=None) == INVALID
    assert q(dtype=3) == INVALID and q(dtype=-1) == INVALID and q(fmt=0) == INVALID and q(fmt=6) == INVALID
    assert q(rows=-1) == INVALID and q(d=0) == INVALID and q(ld=63) == INVALID
    assert q(rows=(1 << 30) + 1) == SHAPE and q(d=(1 << 20) + 1, ld=1 << 21) == SHAPE
    assert q(codes=odd) == ALIGN and q(scales=odd) == ALIGN and q(x=p + 1) == ALIGN and q(x=p + 2, dtype=2) == ALIGN
    assert q(rows=0, x=None, codes=None, scales=None) == OK

    def dq(codes=p, scales=p, fmt=8, rows=8, d=64, out=p, dtype=0, ld=64):
        return L.difr_mx_dequantize(codes, scales, fmt, rows, d, out, dtype, ld, None)

    assert dq(out=None) == INVALID and dq(codes=None) == INVALID and dq(fmt=5) == INVALID and dq(ld=10) == INVALID
    assert dq(dtype=1) == INVALID  # fp16 cannot hold the formats' range
    assert dq(rows=0, out=None) == OK

    def norm(x=p, ldx=64, res=None, ldr=0, w=p, dtype=0, T=8, d=64, eps=1e-6, **kw):
        o = difr._CNormOut()
        o.h, o.ldh = p, 64
        for k, v in kw.items():
            setattr(o, k, v)
        return L.difr_rms_norm(x, ldx, res, ldr, w, dtype, T, d, eps, ctypes.byref(o), None)

    assert norm(x=None) == INVALID and norm(w=None) == INVALID and norm(dtype=4) == INVALID
    assert norm(T=-1) == INVALID and norm(d=0) == INVALID and norm(ldx=63) == INVALID and norm(ldh=63) == INVALID
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert norm(eps=eps) == INVALID
    assert norm(h=None) == INVALID                              # no output
    assert norm(mx_format=4) == INVALID                         # a format without buffers
    assert norm(codes=p, scales=p) == INVALID                   # buffers without a format
    assert norm(mx_format=5, codes=p, scales=p) == INVALID
    assert norm(residual=p, ld_residual=64) == INVALID          # a stream without a residual
    assert norm(res=p, ldr=63) == INVALID and norm(res=p, ldr=64, residual=p, ld_residual=1) == INVALID
    assert norm(d=32769, ldx=40000, ldh=40000) == SHAPE
    assert norm(x=p + 1) == ALIGN and norm(h=p + 1) == ALIGN and norm(mx_format=8, codes=odd, scales=p) == ALIGN
    assert norm(T=0, x=None) == OK

    def logits(hc=p, hs=p, wc=p, ws=p, fmt=4, T=8, d=64, V=100, out=p, dtype=2, ld=100):
        return L.difr_mx_logits(hc, hs, wc, ws, fmt, T, d, V, out, dtype, ld, None, None)

    for name in ("hc", "hs", "wc", "ws", "out"):
        assert logits(**{name: None}) == INVALID
    for name in ("hc", "hs", "wc", "ws"):
        assert logits(**{name: odd}) == ALIGN
    assert logits(out=p + 2) == ALIGN and logits(out=p + 1, dtype=0) == ALIGN
    assert logits(fmt=1) == INVALID and logits(dtype=1) == INVALID and logits(ld=99) == INVALID
    assert logits(T=-1) == INVALID and logits(V=0) == INVALID and logits(d=0) == INVALID
    assert logits(T=1 << 30, V=1 << 30, ld=1 << 30) == SHAPE   # more tiles than 32-bit numbers
    assert logits(T=0, hc=None, hs=None) == OK


def test_refusals_of_the_wait_self_test():
    if torch.cuda.is_available():
        pytest.skip("host-only check")
    L, p = difr.lib(), 0x10000

    def call(done=0, limit=1000, fmt=4, T=8, ld=100, out=p):
        return L.difr_selftest_mx_wait(fmt, T, 64, 100, out, 2, ld, done, limit, None, None)

    for limit in (0, -1, 1_000_000_001):
        assert call(limit=limit) == INVALID
    assert call(done=-1) == INVALID
    assert call(fmt=1) == INVALID and call(ld=99) == INVALID and call(out=None) == INVALID and call(out=p + 2) == ALIGN
    assert call(T=0, out=None) == OK


def test_a_well_formed_call_without_a_device_reports_a_cuda_error():
    if torch.cuda.is_available():
        pytest.skip("host-only check")
    L = difr.lib()
    p = 0x10000
    assert L.difr_mx_quantize(p, 0, 8, 64, 64, 4, p, p, None) == -5
    assert L.difr_mx_logits(p, p, p, p, 8, 8, 64, 100, p, 0, 100, None, None) == -5


def test_norm_struct_has_the_headers_layout():
    import os
    import subprocess
    import tempfile

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = ['printf("%zu\\n", sizeof(difr_norm_out));']
    lines += [f'printf("%zu\\n", offsetof(difr_norm_out, {f}));' for f, _ in difr._CNormOut._fields_]
    lines += ['printf("%d %d %d %d %d\\n", DIFR_BF16, DIFR_F16, DIFR_F32, DIFR_MX8, DIFR_MX4);']
    src = '#include <stddef.h>\n#include <stdio.h>\n#include "difr.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n"
    with tempfile.TemporaryDirectory() as tmp:
        c, exe = os.path.join(tmp, "l.c"), os.path.join(tmp, "l")
        open(c, "w").write(src)
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(root, "include"), "-o", exe, c])
        got = subprocess.check_output([exe], text=True).split("\n")
    assert int(got[0]) == ctypes.sizeof(difr._CNormOut)
    for (f, _), v in zip(difr._CNormOut._fields_, got[1:]):
        assert int(v) == getattr(difr._CNormOut, f).offset, f
    assert got[1 + len(difr._CNormOut._fields_)] == f"{difr.DIFR_BF16} {difr.DIFR_F16} {difr.DIFR_F32} {difr.DIFR_MX8} {difr.DIFR_MX4}"


# ------------------------------------------------------------------ pins of the reference the GPU tests compare with
def test_reference_tables_match_the_formats():
    assert ref.table(4).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    codes = torch.arange(127, dtype=torch.uint8)
    assert torch.equal(codes.view(torch.float8_e4m3fn).double(), ref.table(8))


def test_reference_quantisation_by_hand():
    # largest 7 -> scale 2^0 (floor(log2 7) = 2 = emax of e2m1): 7 saturates to 6, ties go to the even code
    x = torch.zeros(1, 32)
    x[0, :10] = torch.tensor([7.0, -7.0, 0.25, 0.75, 1.25, 2.5, 3.5, 5.0, -0.2, 5.01])
    c, byte = ref.quantize(x, 4)
    assert byte.item() == 127
    assert ref.values(c, byte, 4, 10)[0].tolist() == [6, -6, 0, 1, 1, 2, 4, 4, -0.0, 6]
    # e4m3: largest 500 -> 2^0, saturates to 448; 17 lies between 16 and 18: the even mantissa
    x[0, :4] = torch.tensor([500.0, 17.0, 19.0, 2.0 ** -10])
    x[0, 4:] = 0
    c, byte = ref.quantize(x, 8)
    assert byte.item() == 127 and ref.values(c, byte, 8, 4)[0].tolist() == [448, 16, 20, 0]


def test_reference_layout_by_hand():
    e = torch.arange(130 * 5).view(130, 5) % 200
    s = ref.tile_scales(e, fill=255)
    assert s.numel() == 2 * 2 * 512
    assert s[512 * (0 * 2 + 1) + 16 * 3 + 4 * 2 + 0] == e[67, 4]   # row 67 = 2 * 32 + 3, block 4 = word 1, byte 0
    assert s[512 * (1 * 2 + 0) + 16 * 1 + 0 + 3] == e[129, 3]
    assert s[512 * 1 + 16 * 3 + 4 * 2 + 1] == 0                    # blocks behind the last
    assert s[512 * 2 + 16 * 2] == 255                              # rows behind the last
    assert torch.equal(ref.untile_scales(s, 130, 5), e)
