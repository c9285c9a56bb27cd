"""The projection with the adapters of many requests and its gradient against the formulas in 64 bits, with bounds from the roundings alone
(cond_ops_util.py)."""
import math

import pytest
import torch

from paper_2511_20390_amd import binding as b
from tests.block_ops_util import check
from tests.cond_ops_util import adapters_reference

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.bfloat16, torch.float32]
MODE = {torch.bfloat16: "bf16", torch.float32: "fp32"}


def normal(gen, shape, std, dtype):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0, std, generator=gen).to(dtype)


def problem(seed, M, K, N, r, n, rows, dtype):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    x, w, g = normal(gen, (M, K), 1.0, dtype), normal(gen, (N, K), K ** -0.5, dtype), normal(gen, (M, N), 1.0, dtype)
    a, bb = normal(gen, (n, r, K), K ** -0.5, dtype), normal(gen, (n, N, r), r ** -0.5, dtype)
    bias, scale = normal(gen, (N,), 1.0, torch.float32), 0.5 + torch.rand(n, device=DEV, generator=gen)
    # n stands for none too
    adapter = torch.randint(-1, n + 1, (-(-M // rows),), device=DEV, dtype=torch.int32, generator=gen)
    return x, w, bias, a, bb, adapter, scale, g


def both_passes(x, w, bias, a, bb, adapter, scale, g, rows):
    saved = torch.empty(b.linear_adapters_saved_bytes(x.shape[0], a.shape[1], MODE[x.dtype]), dtype=torch.uint8, device=DEV)
    how = dict(scale=scale, rows_per_sample=rows)
    out = b.op_linear_adapters(x, w, bias, a, bb, adapter, saved=saved, **how)
    return out, *b.op_linear_adapters_backward(g, x, w, a, bb, adapter, saved, **how)


def compare(x, w, bias, a, bb, adapter, scale, g, rows):
    ref = adapters_reference(x, w, bias, a, bb, adapter, scale, rows, g)
    got = both_passes(x, w, bias, a, bb, adapter, scale, g, rows)
    for t, r, what in zip(got, ref, ("out", "dx", "dA", "dB")):
        check(t, r, what)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N,r,n,rows", [
    (1, 64, 64, 4, 1, 1), (8, 128, 192, 16, 8, 1), (17, 64, 320, 8, 3, 5), (33, 192, 64, 16, 2, 7), (20, 2112, 2112, 24, 3, 6), (12, 1024, 512, 64, 4, 3), (1100, 64, 192, 40, 3, 300), (100, 64, 128, 32, 3, 100), (130, 320, 192, 64, 4, 33),
    (257, 128, 256, 100, 2, 64), (300, 64, 64, 128, 5, 1), (512, 384, 640, 16, 3, 256),
])
def test_whole_widths(dtype, M, K, N, r, n, rows):
    compare(*problem(1, M, K, N, r, n, rows, dtype), rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N,r,n,rows", [
    (1, 1, 1, 1, 1, 1), (5, 3, 7, 2, 2, 2), (40, 24, 40, 3, 2, 9), (64, 72, 1000, 5, 3, 16), (65, 1001, 77, 33, 2, 10), (200, 129, 63, 17, 4, 13), (90, 8, 8, 1, 1, 90),
    (150, 56, 120, 48, 3, 64),
])
def test_ragged_widths(dtype, M, K, N, r, n, rows):
    compare(*problem(2, M, K, N, r, n, rows, dtype), rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N,r,n,rows", [
    (4200, 128, 192, 24, 3, 512), (6000, 256, 128, 16, 12, 60), (200, 2048, 384, 16, 2, 50), (5000, 64, 64, 64, 2, 5000), (2100, 4160, 2304, 40, 3, 700), (40, 5000, 5008, 16, 3, 7), (700, 1152, 2304, 16, 4, 350),
])
def test_sums_in_parts_and_large_tiles(dtype, M, K, N, r, n, rows):
    compare(*problem(3, M, K, N, r, n, rows, dtype), rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N,r,n,rows", [(9, 72, 130, 5, 2, 4), (33, 128, 192, 16, 3, 8), (700, 128, 192, 16, 3, 50), (70, 33, 50, 3, 2, 9)])
def test_without_bias_scale_and_adapters(dtype, M, K, N, r, n, rows):
    x, w, bias, a, bb, adapter, scale, g = problem(4, M, K, N, r, n, rows, dtype)
    compare(x, w, None, a, bb, adapter, None, g, rows)
    compare(x, w, bias, a, bb, adapter, None, g, rows)
    # one sample of all rows, and more rows to a sample than there are
    one = adapter[:1].clamp(0, n - 1)
    compare(x, w, None, a, bb, one, scale, g, M)
    assert torch.equal(b.op_linear_adapters(x, w, None, a, bb, one), b.op_linear_adapters(x, w, None, a, bb, one, rows_per_sample=M + 100))
    # nobody has an adapter
    out, dx, da, db = both_passes(x, w, bias, a, bb, torch.full_like(adapter, -1), scale, g, rows)
    assert torch.equal(da, torch.zeros_like(a)) and torch.equal(db, torch.zeros_like(bb))
    ref = adapters_reference(x, w, bias, a, bb, torch.full_like(adapter, -1), scale, rows, g)
    check(out, ref[0], "out")
    check(dx, ref[1], "dx")


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(dtype):
    x, w, bias, a, bb, adapter, scale, g = problem(5, 4, 64, 96, 8, 2, 2, dtype)
    saved = torch.empty(b.linear_adapters_saved_bytes(0, 8, MODE[dtype]), dtype=torch.uint8, device=DEV)
    assert b.op_linear_adapters(x[:0], w, bias, a, bb, adapter[:0], scale=scale, rows_per_sample=2, saved=saved).shape == (0, 96)
    dx, da, db = b.op_linear_adapters_backward(g[:0], x[:0], w, a, bb, adapter[:0], saved, scale=scale, rows_per_sample=2)
    assert dx.shape == (0, 64) and torch.equal(da, torch.zeros_like(a)) and torch.equal(db, torch.zeros_like(bb))


def unhit(t, ref, hit):
    """t, with the reference's values where `hit`, which have to be infinite or NaN."""
    assert not t[hit].isfinite().any()
    return torch.where(hit, ref[0].to(t.dtype), t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N,r,n,rows", [(8, 64, 128, 16, 8, 1), (30, 128, 192, 16, 3, 8), (100, 128, 192, 5, 4, 9), (700, 128, 192, 16, 3, 50), (4200, 256, 640, 32, 4, 300),
                                            (4200, 256, 640, 32, 4, 33), (90, 33, 50, 3, 3, 7)])
def test_nan_stays_with_its_request(dtype, M, K, N, r, n, rows):
    x, w, bias, a, bb, adapter, scale, g = problem(6, M, K, N, r, n, rows, dtype)
    adapter[:3] = torch.tensor([0, 1, 0], device=DEV, dtype=torch.int32)
    ref = adapters_reference(x, w, bias, a, bb, adapter, scale, rows, g)
    which = adapter.long()[torch.arange(M, device=DEV) // rows]
    theirs = (which == 1)[:, None]
    names = ("out", "dx", "dA", "dB")
    # an adapter: its requests' rows, and of the gradients those that read it
    for place, value in ((0, math.nan), (1, math.inf), (1, math.nan)):
        a1, b1 = a.clone(), bb.clone()
        (a1 if place == 0 else b1)[1, (r - 1 if place == 0 else 3)] = value
        got = both_passes(x, w, bias, a1, b1, adapter, scale, g, rows)
        none = lambda t: torch.zeros_like(t, dtype=torch.bool)
        hit = [none(t) for t in got]
        if place == 0:               # one rank's row of A: t of that rank
            hit[0][:], hit[1][:] = theirs, theirs
            hit[3][1, :, r - 1] = True
        else:                        # row 3 of B: column 3 of out, and u
            hit[0][:, 3:4] = theirs
            hit[1][:] = theirs
            hit[2][1] = True
        for t, e, h, what in zip(got, ref, hit, names):
            check(unhit(t, e, h), e, what)
    # a row of x, a row of dout
    x1, g1 = x.clone(), g.clone()
    x1[0, 1], g1[0, 2] = math.nan, math.nan
    got = both_passes(x1, w, bias, a, bb, adapter, scale, g1, rows)
    hit = [torch.zeros_like(t, dtype=torch.bool) for t in got]
    hit[0][0], hit[1][0] = True, True
    hit[2][0], hit[3][0] = True, True
    for t, e, h, what in zip(got, ref, hit, names):
        check(unhit(t, e, h), e, what)


@pytest.mark.parametrize("dtype", TYPES)
def test_outputs_given_and_equal_bits(dtype):
    M, K, N, r, n, rows = 700, 136, 200, 12, 3, 64
    x, w, bias, a, bb, adapter, scale, g = problem(7, M, K, N, r, n, rows, dtype)
    mode, new = MODE[dtype], lambda *s: torch.full(s, math.nan, dtype=dtype, device=DEV)
    byte = lambda k: torch.full((k,), 0xff, dtype=torch.uint8, device=DEV)
    runs = []
    for _ in range(3):
        saved, ws = byte(b.linear_adapters_saved_bytes(M, r, mode)), byte(b.linear_adapters_workspace_bytes(M, K, N, r, n, mode, backward=True))
        how = dict(scale=scale, rows_per_sample=rows, workspace=ws)
        out, grads = new(M, N), (new(M, K), new(n, r, K), new(n, N, r))
        assert b.op_linear_adapters(x, w, bias, a, bb, adapter, saved=saved, out=out, **how) is out
        assert b.op_linear_adapters_backward(g, x, w, a, bb, adapter, saved, out=grads, **how) is grads
        runs.append((out, *grads))
    for t, e, what in zip(runs[0], adapters_reference(x, w, bias, a, bb, adapter, scale, rows, g), ("out", "dx", "dA", "dB")):
        check(t, e, what)
    assert all(torch.equal(s, t) for run in runs[1:] for s, t in zip(runs[0], run))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N,r,n,rows", [(9, 64, 96, 8, 3, 2), (300, 128, 192, 16, 3, 50), (300, 128, 192, 6, 3, 50), (70, 33, 50, 3, 2, 9)])
def test_adapters_of_any_alignment(dtype, M, K, N, r, n, rows):
    """A, B, their gradients, bias and scale one value behind an aligned address, with NaN around what is read."""
    x, w, bias, a, bb, adapter, scale, g = problem(13, M, K, N, r, n, rows, dtype)
    behind = lambda t: torch.cat([torch.full((1,), math.nan, device=DEV), t, torch.full((1,), math.nan, device=DEV)])[1:-1]
    bias, scale = behind(bias), behind(scale)

    def shift(t, guard):
        whole = torch.full((t.numel() + 2,), guard, dtype=dtype, device=DEV)
        whole[1:-1] = t.reshape(-1)
        return whole, whole[1:-1].view(t.shape)

    (_, a1), (_, b1) = shift(a, math.nan), shift(bb, math.nan)
    (wa, da), (wb, db) = shift(a, 7.0), shift(bb, 7.0)
    saved = torch.empty(b.linear_adapters_saved_bytes(M, r, MODE[dtype]), dtype=torch.uint8, device=DEV)
    how = dict(scale=scale, rows_per_sample=rows)
    out = b.op_linear_adapters(x, w, bias, a1, b1, adapter, saved=saved, **how)
    dx = torch.empty_like(x)
    b.op_linear_adapters_backward(g, x, w, a1, b1, adapter, saved, out=(dx, da, db), **how)
    for t, e, what in zip((out, dx, da, db), adapters_reference(x, w, bias, a, bb, adapter, scale, rows, g), ("out", "dx", "dA", "dB")):
        check(t, e, what)
    assert wa[0] == wa[-1] == wb[0] == wb[-1] == 7.0


def test_gradient_against_differences():
    """Along a direction; the formula is a polynomial of the second degree in A and B together and of the first in x, so that the central difference in 64
    bits has no error but its roundings."""
    M, K, N, r, n, rows = 37, 24, 40, 3, 3, 5
    x, w, bias, a, bb, adapter, scale, g = problem(8, M, K, N, r, n, rows, torch.float32)
    ref = adapters_reference(x, w, bias, a, bb, adapter, scale, rows, g)
    grads = both_passes(x, w, bias, a, bb, adapter, scale, g, rows)[1:]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)
    for i, (grad, (v, e)) in enumerate(zip(grads, ref[1:])):
        along = torch.randn(grad.shape, device=DEV, dtype=torch.float64, generator=gen)

        def loss(step):
            at = [t.double() for t in (x, a, bb)]
            at[i] = at[i] + step * along
            return (adapters_reference(at[0], w, bias, at[1], at[2], adapter, scale, rows)[0][0] * g.double()).sum().item()

        limit = ((e + 2.0 ** -24 * v.abs()) * along.abs()).sum().item() + 1e-9
        assert abs((grad.double() * along).sum().item() - (loss(0.5) - loss(-0.5))) <= limit


def test_rows_past_32_bits():
    """More than 2^31 values of x and of out: the first and last rows, and the adapter's gradient where the last rows alone have one."""
    M, K, N, r, n, rows = (1 << 21) + 130, 1024, 1152, 8, 2, 1 << 20
    gen = torch.Generator(device=DEV)
    gen.manual_seed(10)
    x = torch.empty(M, K, device=DEV, dtype=torch.bfloat16).normal_(0, 1, generator=gen)
    _, w, bias, a, bb, _, scale, _ = problem(11, 1, K, N, r, n, 1, torch.bfloat16)
    adapter = torch.tensor([0, -1, 1], device=DEV, dtype=torch.int32)
    g = torch.zeros(M, N, device=DEV, dtype=torch.bfloat16)
    last = slice(M - 130, M)
    g[last] = normal(gen, (130, N), 1.0, torch.bfloat16)
    out, dx, da, db = both_passes(x, w, bias, a, bb, adapter, scale, g, rows)
    ref = adapters_reference(x[last], w, bias, a, bb, adapter[2:], scale, 130, g[last])
    for t, e, what in ((out[last], ref[0], "out"), (dx[last], ref[1], "dx"), (da, ref[2], "dA"), (db, ref[3], "dB")):
        check(t, e, what)
    check(out[:300], adapters_reference(x[:300], w, bias, a, bb, adapter[:1], scale, 300)[0], "out")
    assert not dx[:M - 130].any()


def test_refused_tensors():
    x, w, bias, a, bb, adapter, scale, g = problem(12, 12, 64, 96, 8, 2, 4, torch.bfloat16)
    saved = torch.empty(b.linear_adapters_saved_bytes(12, 8, "bf16"), dtype=torch.uint8, device=DEV)
    call = lambda x=x, w=w, bias=bias, a=a, bb=bb, adapter=adapter, **more: b.op_linear_adapters(x, w, bias, a, bb, adapter, **{"rows_per_sample": 4, **more})
    back = lambda g=g, saved=saved, **more: b.op_linear_adapters_backward(g, x, w, a, bb, adapter, saved, **{"rows_per_sample": 4, **more})
    call(saved=saved)
    for code, f in ((b.FREE_ERR_DTYPE, lambda: call(x=x.half())), (b.FREE_ERR_DTYPE, lambda: call(w=w.float())), (b.FREE_ERR_DTYPE, lambda: call(bb=bb.float())),
                    (b.FREE_ERR_DTYPE, lambda: call(bias=bias.bfloat16())), (b.FREE_ERR_DTYPE, lambda: call(adapter=adapter.long())),
                    (b.FREE_ERR_SHAPE, lambda: call(x=x[:, :-1])), (b.FREE_ERR_SHAPE, lambda: call(a=a[:, :-1])), (b.FREE_ERR_SHAPE, lambda: call(bb=bb[:1])),
                    (b.FREE_ERR_SHAPE, lambda: call(adapter=adapter[:-1])), (b.FREE_ERR_SHAPE, lambda: call(rows_per_sample=0)),
                    (b.FREE_ERR_SHAPE, lambda: call(scale=scale[:1])), (b.FREE_ERR_SHAPE, lambda: call(w=w[0])), (b.FREE_ERR_NULL, lambda: call(a=a.cpu())),
                    (b.FREE_ERR_WORKSPACE, lambda: call(saved=saved[:64])), (b.FREE_ERR_WORKSPACE, lambda: call(workspace=saved[:0])),
                    (b.FREE_ERR_NULL, lambda: back(saved=None)), (b.FREE_ERR_SHAPE, lambda: back(g=g[:, :-1])), (b.FREE_ERR_DTYPE, lambda: back(g=g.float())),
                    (b.FREE_ERR_WORKSPACE, lambda: back(saved=saved[:64]))):
        with pytest.raises(b.FreeError) as e:
            f()
        assert e.value.status == code, (code, e.value)
