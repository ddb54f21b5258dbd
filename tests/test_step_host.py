"""Host side of a decoding step's operators: sizes, refusals before the device is touched, struct layouts (CPU)."""
import ctypes

import pytest
import torch

import paper_2511_02620_b200 as difr

INVALID, SHAPE, ALIGN, WORKSPACE, CUDA, OK = -1, -2, -3, -4, -5, 0
P, ODD = 0x10000, 0x10008
host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="host-only check: fake pointers")


@host_only
def test_refusals_of_the_block_norm():
    def norm(x=P, ldx=64, res=P, ldr=64, w=P, dtype=0, T=8, d=64, eps=1e-6, no_block=False, block=None, **kw):
        o, b = difr._CNormOut(), difr._CBlock(None, None, 0, 0.0, 1.0, 1.0, 0.0)
        o.h, o.ldh = P, 64
        for k, v in (block or {}).items():
            setattr(b, k, v)
        for k, v in kw.items():
            setattr(o, k, v)
        return difr.lib().difr_block_norm(x, ldx, res, ldr, None if no_block else ctypes.byref(b), w, dtype, T, d, eps,
                                          ctypes.byref(o), None)

    assert norm(x=None) == INVALID and norm(res=None) == INVALID and norm(w=None) == INVALID and norm(no_block=True) == INVALID
    assert norm(dtype=3) == INVALID and norm(T=-1) == INVALID and norm(d=0) == INVALID
    assert norm(ldx=63) == INVALID and norm(ldr=63) == INVALID and norm(ldh=63) == INVALID
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert norm(eps=eps) == INVALID
        assert norm(block=dict(post_weight=P, post_eps=eps)) == INVALID
    for name in ("scale", "residual_scale", "weight_offset"):
        assert norm(block={name: float("nan")}) == INVALID and norm(block={name: float("inf")}) == INVALID
    assert norm(block=dict(gate=P, ld_gate=63)) == INVALID
    assert norm(h=None) == INVALID                                    # weights without an output
    assert norm(h=None, w=None) == INVALID                            # no output at all
    assert norm(mx_format=4) == INVALID and norm(codes=P, scales=P) == INVALID
    assert norm(residual=P, ld_residual=63) == INVALID
    assert norm(d=32769, ldx=40000, ldr=40000, ldh=40000) == SHAPE and norm(T=(1 << 30) + 1) == SHAPE
    assert norm(x=P + 1) == ALIGN and norm(h=P + 1) == ALIGN and norm(block=dict(gate=P + 1)) == ALIGN
    assert norm(w=P + 1) == ALIGN and norm(block=dict(post_weight=P + 1, post_eps=1e-6)) == ALIGN
    assert norm(mx_format=8, codes=ODD, scales=P) == ALIGN
    assert norm(T=0, x=None, res=None) == OK
    assert norm() == CUDA and norm(h=None, w=None, residual=P, ld_residual=64) == CUDA


def struct_layouts(structs):
    """sizeof and offsetof of each member as a C compiler has them."""
    import os
    import subprocess
    import tempfile

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = []
    for name, cls in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src = '#include <stddef.h>\n#include <stdio.h>\n#include "difr.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n"
    with tempfile.TemporaryDirectory() as tmp:
        c, exe = os.path.join(tmp, "l.c"), os.path.join(tmp, "l")
        open(c, "w").write(src)
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(root, "include"), "-o", exe, c])
        return dict(line.split() for line in subprocess.check_output([exe], text=True).splitlines())


def test_structs_have_the_headers_layout():
    structs = {"difr_block": difr._CBlock, "difr_drafts": difr._CDrafts, "difr_drafts_out": difr._CDraftsOut}
    got = struct_layouts(structs)
    for name, cls in structs.items():
        assert int(got[name]) == ctypes.sizeof(cls), name
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)


def test_sizes_of_the_verification():
    size = difr.difr_verify_workspace_bytes
    assert size(1, 0, 1) == 2 * 16 and size(2, 3, 4096) == (5 * 2 + 2) * 16 and size(2, 3, 4090) == (5 + 2) * 16
    for bad in ((0, 0, 10), (1, -1, 10), (1, 0, 0), (1, 0, (1 << 27) + 1), (1, 1 << 30, 10), ((1 << 27) + 1, 0, 10)):
        assert size(*bad) == 0


@host_only
def test_refusals_of_the_verification():
    fields = dict(logits=P, ld=100, dtype=2, max_drafts=4, draft_probs=P, ld_draft=100, draft_tokens=P, offsets=P, accept_words=P,
                  sample_words=P, temperature=1.0, temperatures=None)
    outs = dict(tokens=P, n_accepted=P, p_draft=P, status=P, workspace=P, workspace_bytes=1 << 20)

    def verify(B=3, D=6, V=100, **kw):
        i, o = difr._CDrafts(), difr._CDraftsOut()
        for k, v in {**fields, **kw}.items():
            if k in fields:
                setattr(i, k, v)
        for k, v in {**outs, **kw}.items():
            if k in outs:
                setattr(o, k, v)
        return difr.lib().difr_verify_drafts(ctypes.byref(i), B, D, V, ctypes.byref(o), None)

    assert verify() == CUDA and verify(p_draft=None, status=None, draft_probs=None) == CUDA
    for name in ("logits", "draft_tokens", "offsets", "accept_words", "sample_words", "tokens", "n_accepted"):
        assert verify(**{name: None}) == INVALID, name
    assert verify(D=0, draft_tokens=None, accept_words=None) == CUDA
    for name in ("draft_probs", "draft_tokens", "offsets", "accept_words", "sample_words", "temperatures", "tokens", "n_accepted",
                 "p_draft", "status"):
        assert verify(**{name: P + 2}) == ALIGN, name
    assert verify(logits=P + 1, dtype=0) == ALIGN and verify(workspace=ODD) == ALIGN
    assert verify(dtype=3) == INVALID and verify(max_drafts=-1) == INVALID and verify(max_drafts=256) == INVALID
    assert verify(B=-1) == INVALID and verify(D=-1) == INVALID and verify(V=0) == INVALID
    assert verify(ld=99) == INVALID and verify(ld_draft=99) == INVALID and verify(ld_draft=99, draft_probs=None) == CUDA
    for t in (-1.0, float("nan"), float("inf")):
        assert verify(temperature=t) == INVALID and verify(temperature=t, temperatures=P) == CUDA
    assert verify(V=(1 << 27) + 1, ld=1 << 29, ld_draft=1 << 29) == SHAPE and verify(B=1 << 28) == SHAPE
    assert verify(workspace=None) == WORKSPACE and verify(workspace_bytes=difr.difr_verify_workspace_bytes(3, 6, 100) - 1) == WORKSPACE
    assert verify(B=0, logits=None, offsets=None) == OK


def test_sizes_of_4_bit_tensors():
    assert difr.difr_w4_codes_bytes(3, 33) == 3 * 32 and difr.difr_w4_codes_bytes(128256, 4096) == 128256 * 2048
    assert difr.difr_w4_scales_bytes(3, 33, 32) == 3 * 16 and difr.difr_w4_scales_bytes(2, 1025, 128) == 2 * 32
    for rows, d in ((0, 1), (1, 0), (-1, 5), ((1 << 30) + 1, 1), (1, (1 << 20) + 1)):
        assert difr.difr_w4_codes_bytes(rows, d) == 0 and difr.difr_w4_scales_bytes(rows, d, 32) == 0
        assert difr.difr_w4_workspace_bytes(rows, d) == 0
    assert difr.difr_w4_scales_bytes(4, 64, 48) == 0
    w = difr.W4Tensor.allocate(5, 300, 64, device="cpu")
    assert w.codes.numel() == difr.difr_w4_codes_bytes(5, 300) and 2 * w.scales.numel() == difr.difr_w4_scales_bytes(5, 300, 64)


@host_only
def test_refusals_of_4_bit_tensors():
    L = difr.lib()

    def q(x=P, dtype=0, rows=8, d=64, ld=64, group=32, codes=P, scales=P):
        return L.difr_w4_quantize(x, dtype, rows, d, ld, group, codes, scales, None)

    assert q(x=None) == INVALID and q(codes=None) == INVALID and q(scales=None) == INVALID
    assert q(dtype=3) == INVALID and q(group=16) == INVALID and q(group=0) == INVALID and q(group=96) == INVALID
    assert q(rows=-1) == INVALID and q(d=0) == INVALID and q(ld=63) == INVALID
    assert q(rows=(1 << 30) + 1) == SHAPE and q(d=(1 << 20) + 1, ld=1 << 21) == SHAPE
    assert q(codes=ODD) == ALIGN and q(scales=ODD) == ALIGN and q(x=P + 1) == ALIGN and q(x=P + 2, dtype=2) == ALIGN
    assert q(rows=0, x=None, codes=None, scales=None) == OK and q() == CUDA

    def dq(codes=P, scales=P, group=64, rows=8, d=64, out=P, dtype=0, ld=64):
        return L.difr_w4_dequantize(codes, scales, group, rows, d, out, dtype, ld, None)

    assert dq(out=None) == INVALID and dq(codes=None) == INVALID and dq(group=5) == INVALID and dq(ld=10) == INVALID
    assert dq(dtype=1) == INVALID and dq(rows=0, out=None) == OK and dq() == CUDA

    def logits(h=P, ldh=64, wc=P, ws=P, group=32, T=8, d=64, V=100, out=P, dtype=2, ld=100, work=P, nbytes=1 << 20, status=None):
        return L.difr_w4_logits(h, ldh, wc, ws, group, T, d, V, out, dtype, ld, work, nbytes, status, None)

    for name in ("h", "wc", "ws", "out"):
        assert logits(**{name: None}) == INVALID
    for name in ("wc", "ws", "work"):
        assert logits(**{name: ODD}) == ALIGN
    assert logits(h=P + 1) == ALIGN and logits(out=P + 2) == ALIGN and logits(out=P + 1, dtype=0) == ALIGN and logits(status=P + 2) == ALIGN
    assert logits(group=48) == INVALID and logits(dtype=1) == INVALID and logits(ld=99) == INVALID and logits(ldh=63) == INVALID
    assert logits(T=-1) == INVALID and logits(V=0) == INVALID and logits(d=0) == INVALID
    assert logits(T=(1 << 30) + 1) == SHAPE and logits(V=(1 << 30) + 1, ld=1 << 31) == SHAPE
    assert logits(work=None) == WORKSPACE and logits(nbytes=difr.difr_w4_workspace_bytes(8, 64) - 1) == WORKSPACE
    assert logits(T=0, h=None, wc=None) == OK and logits() == CUDA
