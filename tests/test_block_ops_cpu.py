"""What layer norm, rotary positions and the gated feed-forward block refuse, before any device call, and the sizes of their
workspaces.  Host only."""
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
BIG = 1 << 40


def test_layer_norm_refusals(lib):
    call = lambda x=ONE, xt=0, w=ONE, bias=ONE, stride=64, eps=1e-6, M=8, D=64, rows=8, t=0, out=ONE: lib.free_op_layer_norm(
        x, xt, w, bias, stride, 0, eps, M, D, rows, t, out, None)
    assert call(x=None) == call(out=None) == b.FREE_ERR_NULL
    assert call(xt=2) == call(t=-1) == b.FREE_ERR_DTYPE
    assert call(M=-1) == call(D=0) == call(rows=0) == call(rows=4, stride=63) == b.FREE_ERR_SHAPE
    assert call(rows=4, stride=63, w=None) == b.FREE_ERR_SHAPE
    assert call(eps=-1.0) == call(eps=float("nan")) == call(eps=float("inf")) == b.FREE_ERR_RANGE
    assert call(D=16385) == b.FREE_ERR_LIMIT
    assert call(M=0, x=None, out=None) == b.FREE_OK


def test_layer_norm_gradient_refusals(lib):
    def call(dy=ONE, t=0, x=ONE, xt=0, w=ONE, stride=64, eps=1e-6, M=8, D=64, rows=8, dx=ONE, dw=ONE, db=ONE, gs=64, ws=ONE, n=BIG):
        return lib.free_op_layer_norm_backward(dy, t, x, xt, w, stride, 0, eps, M, D, rows, dx, dw, db, gs, ws, n, None)
    assert call(dy=None) == call(x=None) == call(dx=None) == call(dw=None) == call(db=None) == b.FREE_ERR_NULL
    assert call(xt=2) == call(t=7) == b.FREE_ERR_DTYPE
    assert call(M=-1) == call(D=0) == call(rows=0) == call(rows=4, stride=63) == call(rows=4, gs=63) == b.FREE_ERR_SHAPE
    assert call(eps=-1.0) == call(eps=float("nan")) == b.FREE_ERR_RANGE
    assert call(D=16385) == call(M=(1 << 22) + 1, rows=1) == b.FREE_ERR_LIMIT
    assert call(ws=None) == call(ws=C.c_void_p(4100)) == call(n=16) == b.FREE_ERR_WORKSPACE
    assert lib.free_op_layer_norm_backward(None, 0, None, 0, None, 0, 0, 1e-6, 0, 64, 1, None, None, None, 0, None, 0, None) == b.FREE_OK
    for M, D, rows in [(-1, 64, 1), (8, 0, 1), (8, 64, 0), (8, 16385, 8)]:
        assert lib.free_layer_norm_backward_workspace_bytes(M, D, rows) == 0
    for D in (1, 77, 1152, 16384):
        sizes = [lib.free_layer_norm_backward_workspace_bytes(M, D, M) for M in (1, 100, 10000, 1 << 20, 2**31 - 1)]
        assert sizes == sorted(sizes) and all(s % 256 == 0 and s > 0 for s in sizes)
        assert sizes[-1] <= 1100 * 2 * D * 4


def test_rope_refusals(lib):
    def call(x=ONE, xs=128, pos=ONE, pr=1, rows=8, heads=2, dh=64, dims=(32, 32), theta=1e4, pairing=0, t=0, out=ONE, os_=128):
        arr = (C.c_int32 * max(1, len(dims)))(*dims) if dims is not None else None
        return lib.free_op_rope_axes(x, xs, pos, pr, rows, heads, dh, len(dims or ()), arr, theta, pairing, 0, t, out, os_, None)
    assert call(x=None) == call(pos=None) == call(out=None) == call(dims=None) == b.FREE_ERR_NULL
    assert call(t=2) == b.FREE_ERR_DTYPE
    assert call(pairing=2) == call(theta=0.5) == call(theta=float("nan")) == call(theta=float("inf")) == b.FREE_ERR_RANGE
    assert call(rows=-1) == call(heads=0) == call(dh=63) == call(dh=258) == call(dh=0) == call(pr=0) == b.FREE_ERR_SHAPE
    assert call(dims=()) == call(dims=(8,) * 5) == call(dims=(31, 33)) == call(dims=(64, 2)) == call(dims=(-2, 4)) == b.FREE_ERR_SHAPE
    assert call(xs=127) == call(os_=127) == b.FREE_ERR_SHAPE
    assert call(xs=256) == b.FREE_ERR_SHAPE                        # in place with another stride
    assert call(rows=2**31 - 1, heads=1 << 10, xs=1 << 20, os_=1 << 20) == b.FREE_ERR_LIMIT
    assert call(rows=1, heads=2**31 - 1) == b.FREE_ERR_LIMIT
    assert call(rows=0, x=None, pos=None, out=None) == b.FREE_OK


def test_ffn_refusals(lib):
    def fwd(x=ONE, wi=ONE, wo=ONE, M=8, D=64, F=64, t=1, act=0, out=ONE, saved=None, sb=0, ws=ONE, n=BIG):
        return lib.free_op_gated_ffn(x, wi, wo, M, D, F, t, act, out, saved, sb, ws, n, None)

    def bwd(dy=ONE, x=ONE, wi=ONE, wo=ONE, saved=ONE, sb=BIG, M=8, D=64, F=64, t=1, act=0, dx=ONE, dwi=ONE, dwo=ONE, ws=ONE, n=BIG):
        return lib.free_op_gated_ffn_backward(dy, x, wi, wo, saved, sb, M, D, F, t, act, dx, dwi, dwo, ws, n, None)
    assert fwd(x=None) == fwd(wi=None) == fwd(wo=None) == fwd(out=None) == b.FREE_ERR_NULL
    for name in ("dy", "x", "wi", "wo", "dx", "dwi", "dwo"):
        assert bwd(**{name: None}) == b.FREE_ERR_NULL
        assert bwd(**{name: C.c_void_p(4104)}) == b.FREE_ERR_SHAPE
    for call in (fwd, bwd):
        assert call(t=3) == b.FREE_ERR_DTYPE
        assert call(act=2) == b.FREE_ERR_RANGE
        assert call(M=-1) == call(D=0) == call(F=0) == b.FREE_ERR_SHAPE
        assert call(ws=None) == call(ws=C.c_void_p(4112)) == call(n=64) == b.FREE_ERR_WORKSPACE
        assert call(F=2**31 - 1) == call(D=2**31 - 1) == call(M=2**31 - 1, F=1 << 15) == b.FREE_ERR_LIMIT
        assert call(M=1 << 20, F=1 << 14, t=0) == b.FREE_ERR_LIMIT
    assert fwd(x=C.c_void_p(4104)) == fwd(out=C.c_void_p(4104)) == b.FREE_ERR_SHAPE
    assert fwd(saved=ONE, sb=64) == fwd(saved=C.c_void_p(4112), sb=BIG) == b.FREE_ERR_WORKSPACE
    assert bwd(saved=None) == bwd(sb=64) == bwd(saved=C.c_void_p(4112)) == b.FREE_ERR_WORKSPACE
    assert fwd(M=0, x=None, out=None, ws=None) == b.FREE_OK
    assert lib.free_gated_ffn_saved_bytes(8, 0, 64, 1) == lib.free_gated_ffn_workspace_bytes(8, 64, 64, 5, 0) == 0
    for M in (0, 1, 33, 5000):
        for t in (0, 1):
            assert lib.free_gated_ffn_saved_bytes(M, 384, 1536, t) >= M * 1536 * (8 + (2 if t else 4))
            assert 0 < lib.free_gated_ffn_workspace_bytes(M, 384, 1536, t, 0) <= lib.free_gated_ffn_workspace_bytes(M, 384, 1536, t, 1)


def test_binding_refusals():
    """Tensors that the library would misread raise before any call: on the host, of another type or shape."""
    import torch
    b.load()
    f = lambda *s: torch.zeros(*s)
    h = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    u8 = torch.zeros(1 << 20, dtype=torch.uint8)
    calls = [
        (lambda: b.op_layer_norm(f(4, 8)), b.FREE_ERR_NULL),
        (lambda: b.op_layer_norm(f(8)), b.FREE_ERR_SHAPE),
        (lambda: b.op_layer_norm(f(4, 8).double()), b.FREE_ERR_DTYPE),
        (lambda: b.op_layer_norm(f(4, 8), rows_per_sample=0), b.FREE_ERR_SHAPE),
        (lambda: b.op_layer_norm(f(4, 8), f(8)), b.FREE_ERR_NULL),
        (lambda: b.op_layer_norm_backward(f(4, 8), f(4, 8), workspace=u8), b.FREE_ERR_NULL),
        (lambda: b.op_rope_axes(f(4, 8), f(4), 1, 8, [8]), b.FREE_ERR_SHAPE),
        (lambda: b.op_rope_axes(f(4, 9), torch.zeros(4, 1, dtype=torch.int32), 1, 8, [8]), b.FREE_ERR_SHAPE),
        (lambda: b.op_rope_axes(f(4, 8), torch.zeros(4, 2, dtype=torch.int32), 1, 8, [8]), b.FREE_ERR_SHAPE),
        (lambda: b.op_rope_axes(f(4, 8), torch.zeros(4, 1, dtype=torch.int32), 1, 8, [8]), b.FREE_ERR_NULL),
        (lambda: b.op_rope_axes(f(4, 8), torch.zeros(4, 1, dtype=torch.int32), 1, 8, [8], out=h(4, 8)), b.FREE_ERR_DTYPE),
        (lambda: b.op_gated_ffn(f(4), f(8, 4), f(4, 4)), b.FREE_ERR_SHAPE),
        (lambda: b.op_gated_ffn(f(2, 4).half(), f(8, 4), f(4, 4)), b.FREE_ERR_DTYPE),
        (lambda: b.op_gated_ffn(f(2, 4), f(8, 4), f(4, 4), workspace=u8), b.FREE_ERR_NULL),
        (lambda: b.op_gated_ffn_backward(f(2, 4), f(2, 4), f(8, 4), f(4, 4), u8, workspace=u8), b.FREE_ERR_NULL),
    ]
    for k, (call, status) in enumerate(calls):
        with pytest.raises(b.FreeError) as e:
            call()
        assert e.value.status == status, k


def test_calls_go_to_the_device_of_their_tensors(monkeypatch):
    """The device and the stream of a call are its tensors', whichever device is current; tensors on two devices are refused."""
    import contextlib
    import types
    torch = pytest.importorskip("torch")
    seen = []
    current = [0]

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 40 + dev, raising=False)
    fn = lambda *a: seen.append((current[0], a)) or 0
    b._enqueue(fn, "call", 0, 1, 2)
    b._enqueue(fn, "call", 3, 1, 2)
    assert seen == [(0, (1, 2, 40)), (3, (1, 2, 43))] and current[0] == 0
    on = lambda index: types.SimpleNamespace(get_device=lambda: index, device=f"cuda:{index}")
    assert b._same_device(on(2), None, on(2)) == 2
    with pytest.raises(b.FreeError) as e:
        b._same_device(on(2), on(0))
    assert e.value.status == b.FREE_ERR_SHAPE
    with pytest.raises(b.FreeError):
        b._enqueue(lambda *a: b.FREE_ERR_SHAPE, "call", 0)
