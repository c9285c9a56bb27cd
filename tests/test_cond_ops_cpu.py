"""What cross attention and the projection with adapters refuse, before any device call, and the sizes of their workspaces.  Host only."""
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


ONE = C.c_void_p(4096)               # never dereferenced: the checks fail first
ODD = C.c_void_p(4097)
BIG = 1 << 50


def _cross(lib, q=ONE, qs=64, k=ONE, ks=64, v=ONE, vs=64, n=None, mask=None, B=2, Nq=4, Nk=4, heads=2, kv=2, dh=32, scale=1.0, t=1, out=ONE, os_=64,
           lse=None, ws=ONE, bytes_=BIG):
    return lib.free_op_cross_attention(q, qs, k, ks, v, vs, n, mask, B, Nq, Nk, heads, kv, dh, scale, t, out, os_, lse, ws, bytes_, None)


def _cross_back(lib, q=ONE, qs=64, k=ONE, ks=64, v=ONE, vs=64, n=None, mask=None, B=2, Nq=4, Nk=4, heads=2, kv=2, dh=32, scale=1.0, t=1, out=ONE, os_=64,
                lse=ONE, ws=ONE, bytes_=BIG, g=ONE, gs=64, dq=ONE, dqs=64, dk=ONE, dks=64, dv=ONE, dvs=64):
    return lib.free_op_cross_attention_backward(g, gs, q, qs, k, ks, v, vs, out, os_, lse, n, mask, B, Nq, Nk, heads, kv, dh, scale, t, dq, dqs, dk, dks, dv,
                                                dvs, ws, bytes_, None)


@pytest.mark.parametrize("call", [_cross, _cross_back])
def test_cross_attention_refusals(lib, call):
    for name in ("q", "k", "v", "out") + (("g", "dq", "dk", "dv", "lse") if call is _cross_back else ()):
        assert call(lib, **{name: None}) == b.FREE_ERR_NULL, name
        assert call(lib, **{name: ODD}) == b.FREE_ERR_SHAPE, name
    for name in ("qs", "ks", "vs", "os_") + (("gs", "dqs", "dks", "dvs") if call is _cross_back else ()):
        assert call(lib, **{name: 63}) == b.FREE_ERR_SHAPE, name
        assert call(lib, **{name: (1 << 22) + 1}) == b.FREE_ERR_LIMIT, name
    assert call(lib, t=2) == call(lib, t=-1) == b.FREE_ERR_DTYPE
    assert call(lib, B=-1) == call(lib, Nq=-1) == call(lib, Nk=-1) == call(lib, heads=0) == call(lib, kv=0) == call(lib, dh=0) == b.FREE_ERR_SHAPE
    assert call(lib, heads=3) == call(lib, kv=4) == b.FREE_ERR_SHAPE
    assert call(lib, n=ODD) == b.FREE_ERR_SHAPE
    for scale in (0.0, -1.0, 2.0 ** -65, 2.0 ** 65, float("nan"), float("inf")):
        assert call(lib, scale=scale) == b.FREE_ERR_RANGE
    assert call(lib, dh=129) == call(lib, B=1 << 24) == call(lib, Nq=2**31 - 1) == call(lib, Nk=2**31 - 1) == b.FREE_ERR_LIMIT
    assert call(lib, B=1 << 23, kv=1, Nq=1 << 20) == call(lib, heads=1 << 18, kv=1 << 18) == b.FREE_ERR_LIMIT
    assert call(lib, ws=None) == call(lib, ws=C.c_void_p(4100)) == call(lib, bytes_=0) == b.FREE_ERR_WORKSPACE
    # nothing to do
    assert call(lib, B=0, q=None, k=None, v=None, out=None, ws=None, bytes_=0) == b.FREE_OK
    # a single row's distance to the next does not count
    assert call(lib, B=1, Nq=1, Nk=1, qs=0, ks=0, vs=0, os_=0, bytes_=0) == b.FREE_ERR_WORKSPACE


def test_cross_attention_workspaces(lib):
    size = lambda *a: lib.free_cross_attention_workspace_bytes(*a)
    assert size(2, 4, 4, 3, 2, 64, 1, 0) == size(-1, 4, 4, 2, 2, 64, 1, 0) == size(2, 4, 4, 2, 2, 200, 1, 1) == size(2, 4, 4, 2, 2, 64, 5, 1) == 0
    for t in (0, 1):
        for back in (0, 1):
            for B, Nq, Nk, heads, kv, dh in [(1, 1, 1, 1, 1, 1), (4, 1, 16384, 32, 8, 128), (2, 6144, 300, 16, 16, 72), (0, 5, 5, 1, 1, 8), (1, 0, 5, 1, 1, 8),
                                             (1, 5, 0, 1, 1, 8), (1, 1 << 24, 1 << 10, 2, 2, 64)]:
                n = size(B, Nq, Nk, heads, kv, dh, t, back)
                assert n > 0 and n % 256 == 0
                # parts are bounded: a workspace is not larger than 64 fp32 results
                assert n <= 4096 + 4 * B * (64 * (Nq * heads + 2 * Nk * kv) * (dh + 2) + 8192 * dh)
    with pytest.raises(b.FreeError):
        b.cross_attention_workspace_bytes(1 << 32, 1, 1, 1, 1, 8, "bf16")


def _adapt(lib, x=ONE, w=ONE, bias=ONE, a=ONE, bb=ONE, scale=ONE, which=ONE, rows=4, M=8, K=64, N=64, r=8, n=2, t=1, out=ONE, saved=None, sb=0, ws=ONE, bytes_=BIG):
    return lib.free_op_linear_adapters(x, w, bias, a, bb, scale, which, rows, M, K, N, r, n, t, out, saved, sb, ws, bytes_, None)


def _adapt_back(lib, g=ONE, x=ONE, w=ONE, a=ONE, bb=ONE, scale=ONE, which=ONE, rows=4, M=8, K=64, N=64, r=8, n=2, t=1, dx=ONE, da=ONE, db=ONE, saved=ONE, sb=BIG,
                ws=ONE, bytes_=BIG):
    return lib.free_op_linear_adapters_backward(g, x, w, a, bb, scale, which, rows, saved, sb, M, K, N, r, n, t, dx, da, db, ws, bytes_, None)


@pytest.mark.parametrize("call", [_adapt, _adapt_back])
def test_linear_adapters_refusals(lib, call):
    back = call is _adapt_back
    for name in ("x", "w", "a", "bb", "which") + (("g", "dx", "da", "db") if back else ("out",)):
        assert call(lib, **{name: None}) == b.FREE_ERR_NULL, name
        assert call(lib, **{name: ODD}) == b.FREE_ERR_SHAPE, name
    for name in ("x", "w") + (("g", "dx") if back else ("out",)):
        assert call(lib, **{name: C.c_void_p(4104)}) == b.FREE_ERR_SHAPE, name
    assert call(lib, scale=ODD) == b.FREE_ERR_SHAPE
    if not back:
        assert call(lib, bias=ODD) == b.FREE_ERR_SHAPE
    assert call(lib, t=2) == call(lib, t=-1) == b.FREE_ERR_DTYPE
    assert call(lib, M=-1) == call(lib, K=0) == call(lib, N=0) == call(lib, r=0) == call(lib, n=0) == call(lib, rows=0) == b.FREE_ERR_SHAPE
    assert call(lib, r=129) == call(lib, n=16385) == call(lib, K=(1 << 20) + 1) == call(lib, N=(1 << 20) + 1) == b.FREE_ERR_LIMIT
    assert call(lib, M=2**31 - 1, K=1 << 20) == call(lib, M=2**31 - 1, N=1 << 20) == call(lib, K=1 << 20, N=1 << 20, r=128, n=16384) == b.FREE_ERR_LIMIT
    # grids of the launches: copies of W in tiles, and of A and B, and rows
    assert call(lib, M=(1 << 27) + 1, K=1, N=1) == b.FREE_ERR_LIMIT
    assert call(lib, M=1, K=1 << 20, N=1 << 15) == call(lib, M=1, K=1 << 18, N=1, r=1, n=2048) == b.FREE_ERR_LIMIT
    assert call(lib, ws=None) == call(lib, ws=C.c_void_p(4100)) == call(lib, bytes_=0) == b.FREE_ERR_WORKSPACE
    assert call(lib, saved=C.c_void_p(4100), sb=BIG) == call(lib, saved=ONE, sb=100) == b.FREE_ERR_WORKSPACE
    if back:
        assert call(lib, saved=None) == b.FREE_ERR_WORKSPACE
    else:
        assert call(lib, M=0, x=None, w=None, out=None, ws=None) == b.FREE_OK


def test_linear_adapters_workspaces(lib):
    size = lib.free_linear_adapters_workspace_bytes
    assert size(8, 64, 64, 129, 2, 1, 0) == size(-1, 64, 64, 8, 2, 1, 0) == size(8, 0, 64, 8, 2, 1, 1) == size(8, 64, 64, 8, 2, 7, 1) == 0
    assert lib.free_linear_adapters_saved_bytes(8, 129, 1) == lib.free_linear_adapters_saved_bytes(-1, 8, 1) == 0
    for t in (0, 1):
        for back in (0, 1):
            for M, K, N, r, n in [(0, 64, 64, 8, 2), (1, 1, 1, 1, 1), (8, 4096, 4096, 16, 8), (12288, 1152, 1152, 16, 4), (1000, 1001, 77, 33, 2)]:
                got = size(M, K, N, r, n, t, back)
                assert got > 0 and got % 256 == 0
    with pytest.raises(b.FreeError):
        b.linear_adapters_workspace_bytes(1 << 32, 64, 64, 8, 2, "bf16")
