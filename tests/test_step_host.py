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
    assert size(1, 0, 1) == 16 and size(2, 3, 4096) == 5 * 2 * 16 and size(2, 3, 4090) == 5 * 16
    for bad in ((0, 0, 10), (1, -1, 10), (1, 0, 0), (1, 0, (1 << 28) + 1), (1, 1 << 30, 10), ((1 << 27) + 1, 0, 10)):
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
    assert verify(V=(1 << 28) + 1, ld=1 << 29, ld_draft=1 << 29) == SHAPE and verify(B=1 << 28) == SHAPE
    assert verify(workspace=None) == WORKSPACE and verify(workspace_bytes=difr.difr_verify_workspace_bytes(3, 6, 100) - 1) == WORKSPACE
    assert verify(B=0, logits=None, offsets=None) == OK
