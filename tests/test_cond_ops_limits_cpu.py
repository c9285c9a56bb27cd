"""Sizes of cross attention far past its limits, whose products do not fit 64 bits either, are refused like those just past them.  Host only."""
import ctypes as C
import os

import pytest

from paper_2511_20390_amd import binding as b


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return b.load()


def _sizes():
    """(B, Nq, Nk, heads, kv_heads): samples times key heads times blocks of 32 rows or keys is a power of two, up to 2^66."""
    for B in range(0, 31, 3):
        for n in range(0, 31, 3):
            for kv in (0, 5, 10, 21):
                for group in (0, 1):
                    if kv + group <= 22 and n + group <= 30:
                        yield 1 << B, 1 << n, 1, 1 << (kv + group), 1 << kv
                        yield 1 << B, 1, 1 << n, 1 << (kv + group), 1 << kv
    yield 1 << 30, 1 << 29, 1, 1 << 10, 1 << 10              # 2^64
    yield 2**31 - 1, 2**31 - 129, 2**31 - 129, 1 << 22, 1 << 22


def test_limit_of_workgroups(lib):
    """Samples x key heads x blocks of 32 rows (or keys) below 2^23."""
    fake = C.c_void_p(4096)              # never dereferenced: the checks fail first
    refused = 0
    for B, Nq, Nk, heads, kv in _sizes():
        blocks = -(-max(Nq * (heads // kv), Nk, 1) // 32)
        fits = B * kv * blocks < 1 << 23
        for back in (0, 1):
            size = lib.free_cross_attention_workspace_bytes(B, Nq, Nk, heads, kv, 1, 1, back)
            assert (size > 0) == fits, (B, Nq, Nk, heads, kv, size)
        if fits:
            continue
        refused += 1
        assert lib.free_op_cross_attention(fake, heads, fake, kv, fake, kv, None, None, B, Nq, Nk, heads, kv, 1, 1.0, 1, fake, heads, None, fake, 1 << 62,
                                           None) == b.FREE_ERR_LIMIT
        assert lib.free_op_cross_attention_backward(fake, heads, fake, heads, fake, kv, fake, kv, fake, heads, fake, None, None, B, Nq, Nk, heads, kv, 1, 1.0, 1, fake,
                                                    heads, fake, kv, fake, kv, fake, 1 << 62, None) == b.FREE_ERR_LIMIT
    assert refused > 100
