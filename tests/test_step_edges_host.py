"""Refusals of the self-test of the waits of the product on 4-bit weights, before the device is touched (CPU)."""
import pytest
import torch

import paper_2511_02620_b200 as difr

INVALID, SHAPE, ALIGN, CUDA, OK = -1, -2, -3, -5, 0
P = 0x10000


@pytest.mark.skipif(torch.cuda.is_available(), reason="host-only check: fake pointers")
def test_refusals_of_the_wait_self_test():
    def wait(T=8, d=64, V=100, logits=P, dtype=2, ld=100, done=0, limit=1000, status=None):
        return difr.lib().difr_selftest_w4_wait(T, d, V, logits, dtype, ld, done, limit, status, None)

    assert wait(done=-1) == INVALID and wait(limit=0) == INVALID and wait(limit=1_000_000_001) == INVALID
    assert wait(dtype=1) == INVALID and wait(T=-1) == INVALID and wait(d=0) == INVALID and wait(V=0) == INVALID and wait(ld=99) == INVALID
    assert wait(logits=None) == INVALID and wait(logits=P + 2) == ALIGN and wait(status=P + 2) == ALIGN
    assert wait(T=(1 << 30) + 1) == SHAPE and wait(d=(1 << 20) + 1) == SHAPE and wait(V=(1 << 30) + 1, ld=1 << 31) == SHAPE
    assert wait(T=0, logits=None) == OK and wait() == CUDA
