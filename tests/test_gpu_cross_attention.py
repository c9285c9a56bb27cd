"""Cross attention and its gradient against the formulas in 64 bits, with bounds from the roundings alone (cond_ops_util.py)."""
import math

import pytest
import torch

from paper_2511_20390_amd import binding as b
from tests.block_ops_util import check
from tests.cond_ops_util import cross_reference, keys_that_count

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.bfloat16, torch.float32]


def normal(gen, shape, std, dtype):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0, std, generator=gen).to(dtype)


def problem(seed, B, Nq, Nk, heads, kv, dh, dtype, keys):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    q, g = normal(gen, (B * Nq, heads * dh), 1.5, dtype), normal(gen, (B * Nq, heads * dh), 1.0, dtype)
    k, v = normal(gen, (B * Nk, kv * dh), 1.0, dtype), normal(gen, (B * Nk, kv * dh), 1.0, dtype)
    key_len = key_mask = None
    if keys != "all":
        key_len = torch.randint(0, Nk + 1, (B,), device=DEV, dtype=torch.int32, generator=gen)
        key_len[0] = Nk
        if B > 1:
            key_len[1] = 0
    if keys == "holes":
        key_mask = (torch.rand(B, Nk, device=DEV, generator=gen) < 0.6).to(torch.uint8)
    return q, k, v, g, key_len, key_mask


def spoil(t, keys):
    """NaN in the rows of keys that do not count."""
    t = t.clone()
    t[~keys.reshape(-1)] = math.nan
    return t


def both_passes(q, k, v, g, key_len, key_mask, B, heads, kv, dh, scale=None, **more):
    lse = torch.full((B, heads, q.shape[0] // B), 7.0, device=DEV)
    how = dict(B=B, heads=heads, dh=dh, kv_heads=kv, key_len=key_len, key_mask=key_mask, scale=scale)
    out = b.op_cross_attention(q, k, v, lse=lse, **how)
    return out, lse, *b.op_cross_attention_backward(g, q, k, v, out, lse, **how, **more)


def compare(q, k, v, g, key_len, key_mask, B, heads, kv, dh, scale=None):
    Nk = k.shape[0] // B
    keys = keys_that_count(B, Nk, key_len, key_mask, DEV)
    ref = cross_reference(q, k, v, B, heads, kv, dh, dh ** -0.5 if scale is None else scale, keys, g)
    got = both_passes(q, spoil(k, keys), spoil(v, keys), g, key_len, key_mask, B, heads, kv, dh, scale)
    for t, r, what in zip(got, ref, ("out", "lse", "dq", "dk", "dv")):
        check(t, r, what)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("keys", ["all", "len", "holes"])
@pytest.mark.parametrize("B,Nq,Nk,heads,kv,dh", [
    (1, 1, 1, 1, 1, 8), (2, 1, 1, 2, 2, 72), (3, 5, 7, 2, 1, 16), (2, 33, 65, 3, 3, 64), (3, 64, 64, 2, 2, 32), (2, 129, 77, 4, 4, 72),
    (3, 200, 130, 4, 2, 80), (2, 50, 300, 3, 1, 96), (3, 70, 129, 2, 2, 128), (1, 300, 31, 2, 2, 72), (2, 17, 33, 6, 2, 128),
])
def test_sizes_and_masks(dtype, keys, B, Nq, Nk, heads, kv, dh):
    compare(*problem(1, B, Nq, Nk, heads, kv, dh, dtype, keys), B, heads, kv, dh)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh", [1, 2, 3, 7, 12, 20, 31, 33, 40, 63, 65, 71, 90, 97, 127])
def test_odd_head_dimensions(dtype, dh):
    compare(*problem(2, 3, 45, 70, 3, 3, dh, dtype, "holes"), 3, 3, 3, dh)
    compare(*problem(3, 3, 3, 70, 4, 2, dh, dtype, "len"), 3, 4, 2, dh)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,Nq,Nk,heads,kv,dh", [
    (2, 1, 3000, 8, 2, 128),             # keys in parts, few rows
    (1, 4, 1025, 8, 1, 72),
    (2, 7, 999, 4, 4, 64),
    (1, 150, 2050, 2, 2, 72),            # keys in parts, many rows
    (2, 1100, 40, 2, 2, 72),             # queries in parts
    (1, 700, 200, 4, 1, 128),
    (1, 2000, 130, 8, 8, 64),
    (2, 2500, 4, 8, 1, 72),              # queries in parts and shared out among the wavefronts
    (1, 3000, 1, 2, 2, 128),
    (2, 1700, 64, 3, 3, 96),
])
def test_sums_in_parts(dtype, B, Nq, Nk, heads, kv, dh):
    for keys in ("all", "holes"):
        compare(*problem(4, B, Nq, Nk, heads, kv, dh, dtype, keys), B, heads, kv, dh)


@pytest.mark.parametrize("keys", ["all", "len", "holes"])
@pytest.mark.parametrize("B,Nq,Nk,heads,kv,dh", [
    (2, 2100, 130, 16, 16, 72),          # keys stay in LDS
    (3, 1500, 383, 16, 16, 80), (1, 4100, 77, 32, 16, 64), (2, 1100, 250, 32, 32, 128), (4, 1030, 1000, 16, 16, 32), (2, 2100, 340, 16, 16, 96),
    (1, 4200, 65, 16, 16, 40),
    (1, 2100, 700, 32, 32, 64),          # keys pass through it
    (2, 2049, 450, 16, 16, 72), (1, 1100, 513, 64, 8, 128), (2, 2100, 520, 16, 16, 96),
])
def test_many_queries(keys, B, Nq, Nk, heads, kv, dh):
    compare(*problem(5, B, Nq, Nk, heads, kv, dh, torch.bfloat16, keys), B, heads, kv, dh)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_queries_and_no_keys(dtype):
    q, k, v, g, _, _ = problem(6, 2, 5, 9, 4, 2, 24, dtype, "all")
    how = dict(B=2, heads=4, dh=24, kv_heads=2)
    none = q[:0]
    lse = torch.empty(2, 4, 0, device=DEV)
    assert b.op_cross_attention(none, k, v, lse=lse, **how).shape == (0, 96)
    dq, dk, dv = b.op_cross_attention_backward(none, none, k, v, none, lse, **how)
    assert dq.shape == (0, 96) and torch.equal(dk, torch.zeros_like(k)) and torch.equal(dv, torch.zeros_like(v))
    lse = torch.empty(2, 4, 5, device=DEV)
    out = b.op_cross_attention(q, k[:0], v[:0], lse=lse, **how)
    assert torch.equal(out, torch.zeros_like(q)) and torch.equal(lse, torch.full_like(lse, -math.inf))
    dq, dk, dv = b.op_cross_attention_backward(g, q, k[:0], v[:0], out, lse, **how)
    assert torch.equal(dq, torch.zeros_like(q)) and dk.shape == dv.shape == (0, 48)


def within(rows, width, before, extra, dtype, guard):
    """(the whole buffer, rows of `width` values in it that begin `before` values into each of its rows), the buffer full of `guard`."""
    whole = torch.full((rows + 2, width + extra), guard, dtype=dtype, device=DEV)
    return whole, whole[1:-1, before:before + width]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("before,extra", [(0, 16), (8, 24), (1, 3), (5, 8)])
@pytest.mark.parametrize("B,Nq,Nk,heads,kv,dh", [(2, 3, 45, 4, 2, 72), (2, 130, 70, 4, 4, 72), (1, 200, 90, 2, 1, 33), (2, 2100, 130, 16, 16, 72), (1, 1100, 513, 64, 16, 128)])
def test_rows_any_distance_apart(dtype, before, extra, B, Nq, Nk, heads, kv, dh):
    if dtype == torch.float32 and Nq > 1000:
        Nq = 150
    q, k, v, g, key_len, key_mask = problem(7, B, Nq, Nk, heads, kv, dh, dtype, "len")
    keys = keys_that_count(B, Nk, key_len, key_mask, DEV)
    ref = cross_reference(q, k, v, B, heads, kv, dh, dh ** -0.5, keys, g)

    def place(t, guard):
        whole, rows = within(*t.shape, before, extra, dtype, guard)
        rows.copy_(t)
        return whole, rows

    # what stands between the rows that are read is NaN, and between those that are written stays
    (_, qs), (_, gs) = place(q, math.nan), place(g, math.nan)
    packed = torch.full((B * Nk, 2 * kv * dh + extra), math.nan, dtype=dtype, device=DEV)
    ks, vs = packed[:, before:before + kv * dh], packed[:, extra + kv * dh:]
    ks.copy_(k)
    vs.copy_(v)
    bufs = [within(*t.shape, before, extra, dtype, 7.0) for t in (q, q, k, v)]
    lse = torch.empty(B, heads, Nq, device=DEV)
    how = dict(B=B, heads=heads, dh=dh, kv_heads=kv, key_len=key_len)
    b.op_cross_attention(qs, ks, vs, lse=lse, out=bufs[0][1], **how)
    b.op_cross_attention_backward(gs, qs, ks, vs, bufs[0][1], lse, grads=tuple(rows for _, rows in bufs[1:]), **how)
    for (_, rows), (r, what) in zip(bufs, ((ref[0], "out"), (ref[2], "dq"), (ref[3], "dk"), (ref[4], "dv"))):
        check(rows, r, what)
    check(lse, ref[1], "lse")
    for whole, rows in bufs:
        rows.fill_(7.0)
        assert torch.equal(whole, torch.full_like(whole, 7.0))


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_out_of_range_and_bool_masks(dtype):
    q, k, v, g, _, mask = problem(8, 4, 40, 70, 2, 2, 64, dtype, "holes")
    far = torch.tensor([70, -3, 1000, 33], device=DEV, dtype=torch.int32)
    near = far.clamp(0, 70)
    a = both_passes(q, k, v, g, far, mask.bool(), 4, 2, 2, 64)
    c = both_passes(q, k, v, g, near, 3 * mask, 4, 2, 2, 64)
    assert all(torch.equal(x, y) for x, y in zip(a, c))
    compare(q, k, v, g, near, mask, 4, 2, 2, 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("factor,scale", [(40.0, None), (1.0, 2.0 ** -20), (2.0 ** -20, 2.0 ** 18)])
def test_large_and_small_scores(dtype, factor, scale):
    """Rows that one key decides, rows all of whose keys count alike, and a scale far from the usual ones."""
    q, k, v, g, n, mask = problem(9, 2, 100, 140, 2, 2, 64, dtype, "holes")
    compare(q * factor, k, v, g, n, mask, 2, 2, 2, 64, scale)
    compare(q[:8] * factor, k, v, g[:8], n, mask, 2, 2, 2, 64, scale)


@pytest.mark.parametrize("B,Nq,Nk,heads,dh,dtype", [(2, 4, 300, 4, 64, torch.bfloat16), (2, 100, 130, 4, 72, torch.bfloat16), (2, 1100, 130, 32, 72, torch.bfloat16),
                                                     (2, 1100, 700, 32, 64, torch.bfloat16), (2, 100, 130, 4, 72, torch.float32)])
def test_nan_stays_with_its_row(B, Nq, Nk, heads, dh, dtype):
    q, k, v, g, _, _ = problem(10, B, Nq, Nk, heads, heads, dh, dtype, "all")
    keys = keys_that_count(B, Nk, None, None, DEV)
    ref = cross_reference(q, k, v, B, heads, heads, dh, dh ** -0.5, keys, g)
    bad = Nq + 1                         # a row of the second sample, in its second head
    spoiled = q.clone()
    spoiled[bad, dh + 3] = math.nan
    out, lse, dq, dk, dv = both_passes(spoiled, k, v, g, None, None, B, heads, heads, dh)
    hit = torch.zeros_like(q, dtype=torch.bool)
    hit[bad, dh:2 * dh] = True
    assert out[hit].isnan().all() and dq[hit].isnan().all() and lse[1, 1, 1].isnan()
    lse[1, 1, 1] = ref[1][0][1, 1, 1]
    for t, (r, e), what in ((out, ref[0], "out"), (dq, ref[2], "dq")):
        check(torch.where(hit, r.to(dtype), t), (r, e), what)
    check(lse, ref[1], "lse")
    # keys of the second sample's second head depend on it
    hit = torch.zeros_like(k, dtype=torch.bool)
    hit[Nk:, dh:2 * dh] = True
    for t, (r, e), what in ((dk, ref[3], "dk"), (dv, ref[4], "dv")):
        assert t[hit].isnan().all()
        check(torch.where(hit, r.to(dtype), t), (r, e), what)


@pytest.mark.parametrize("B,Nq,Nk,heads,kv,dh,dtype", [(2, 1, 900, 8, 2, 64, torch.bfloat16), (1, 2100, 130, 16, 16, 72, torch.bfloat16),
                                                       (1, 700, 200, 4, 1, 128, torch.bfloat16), (2, 70, 150, 4, 2, 72, torch.float32)])
def test_equal_bits(B, Nq, Nk, heads, kv, dh, dtype):
    p = problem(11, B, Nq, Nk, heads, kv, dh, dtype, "holes")
    first = both_passes(*p, B, heads, kv, dh)
    assert all(t.isfinite().all() for t in first[2:])
    for fill in (0xff, 0, 0x7f):         # whatever the workspace held
        ws = torch.full((b.cross_attention_workspace_bytes(B, Nq, Nk, heads, kv, dh, "bf16" if dtype == torch.bfloat16 else "fp32", backward=True),), fill,
                        dtype=torch.uint8, device=DEV)
        assert all(torch.equal(x, y) for x, y in zip(first, both_passes(*p, B, heads, kv, dh, workspace=ws)))


@pytest.mark.parametrize("heads,kv", [(3, 3), (4, 2), (4, 1)])
def test_gradient_against_differences(heads, kv):
    """Along a direction: the central difference of the formula in 64 bits, whose own error is below a third of what it changes by when its step is
    doubled (its next term grows with the square of the step), against the gradient, which may be off by its bounds."""
    B, Nq, Nk, dh = 2, 9, 13, 20
    q, k, v, g, _, mask = problem(12, B, Nq, Nk, heads, kv, dh, torch.float32, "holes")
    mask[:, 0] = 1
    keys = keys_that_count(B, Nk, None, mask, DEV)
    how = (B, heads, kv, dh, dh ** -0.5, keys)
    ref = cross_reference(q, k, v, *how, g)
    grads = both_passes(q, k, v, g, None, mask, B, heads, kv, dh)[2:]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(13)
    for i, (grad, (r, e)) in enumerate(zip(grads, ref[2:])):
        along = torch.randn(grad.shape, device=DEV, dtype=torch.float64, generator=gen)

        def loss(step):
            x = [t.double() for t in (q, k, v)]
            x[i] = x[i] + step * along
            return (cross_reference(*x, *how)[0][0] * g.double()).sum().item()

        h = 1e-3
        d1, d2 = (loss(h) - loss(-h)) / (2 * h), (loss(2 * h) - loss(-2 * h)) / (4 * h)
        # (the losses' own roundings: 64 bits of sums of a few hundred values of order one, over the step)
        limit = ((e + 2.0 ** -24 * r.abs()) * along.abs()).sum().item() + abs(d1 - d2) + 1e-9
        assert abs((grad.double() * along).sum().item() - d1) <= limit


def test_keys_past_32_bits():
    """One query of each of two samples, whose keys are 2^31 values and more."""
    B, Nk, kv, dh = 2, (1 << 20) + 37, 8, 128
    gen = torch.Generator(device=DEV)
    gen.manual_seed(14)
    k = torch.empty(B * Nk, kv * dh, device=DEV, dtype=torch.bfloat16).normal_(0, 1, generator=gen)
    v = torch.empty(B * Nk, kv * dh, device=DEV, dtype=torch.bfloat16).normal_(0, 1, generator=gen)
    assert k.numel() > 2 ** 31
    q = normal(gen, (B, kv * dh), 2.0, torch.bfloat16)
    mask = torch.zeros(B, Nk, dtype=torch.uint8, device=DEV)
    mask[:, ::4097] = 1                  # spread over all of them, the last one too
    mask[:, -1] = 1
    out = b.op_cross_attention(q, k, v, B, kv, dh, key_mask=mask)
    for s in range(B):
        at = s * Nk + mask[s].nonzero()[:, 0]
        keys = torch.ones(1, at.numel(), dtype=torch.bool, device=DEV)
        check(out[s:s + 1], cross_reference(q[s:s + 1], k[at], v[at], 1, kv, kv, dh, dh ** -0.5, keys)[0], "out")


def test_queries_past_32_bits():
    """More than 2^31 values of queries: the first and last rows, and the keys' gradient where the last rows alone have one."""
    Nq, Nk, heads, dh = (1 << 21) + 70, 77, 8, 128
    gen = torch.Generator(device=DEV)
    gen.manual_seed(15)
    q = torch.empty(Nq, heads * dh, device=DEV, dtype=torch.bfloat16).normal_(0, 1, generator=gen)
    k, v = normal(gen, (Nk, heads * dh), 1.0, torch.bfloat16), normal(gen, (Nk, heads * dh), 1.0, torch.bfloat16)
    assert q.numel() > 2 ** 31
    last = slice(Nq - 100, Nq)
    g = torch.zeros_like(q)
    g[last] = normal(gen, (100, heads * dh), 1.0, torch.bfloat16)
    out, lse, dq, dk, dv = both_passes(q, k, v, g, None, None, 1, heads, heads, dh)
    keys = torch.ones(1, Nk, dtype=torch.bool, device=DEV)
    ref = cross_reference(q[last], k, v, 1, heads, heads, dh, dh ** -0.5, keys, g[last])
    for t, r, what in ((out[last], ref[0], "out"), (lse[:, :, last], ref[1], "lse"), (dq[last], ref[2], "dq"), (dk, ref[3], "dk"), (dv, ref[4], "dv")):
        check(t, r, what)
    check(out[:100], cross_reference(q[:100], k, v, 1, heads, heads, dh, dh ** -0.5, keys)[0], "out")
    assert not dq[:Nq - 100].any()


def test_refused_tensors():
    q, k, v, g, n, mask = problem(16, 2, 6, 8, 4, 2, 16, torch.bfloat16, "holes")
    lse = torch.empty(2, 4, 6, device=DEV)
    ok = dict(B=2, heads=4, dh=16, kv_heads=2)
    call = lambda q=q, k=k, v=v, **more: b.op_cross_attention(q, k, v, **{**ok, **more})
    out = call(lse=lse)
    back = lambda g=g, out=out, lse=lse, **more: b.op_cross_attention_backward(g, q, k, v, out, lse, **{**ok, **more})
    for code, f in ((b.FREE_ERR_DTYPE, lambda: call(q=q.half())), (b.FREE_ERR_DTYPE, lambda: call(k=k.float())), (b.FREE_ERR_DTYPE, lambda: call(out=q.float())),
                    (b.FREE_ERR_DTYPE, lambda: call(key_len=n.long())), (b.FREE_ERR_DTYPE, lambda: call(key_mask=mask.float())),
                    (b.FREE_ERR_DTYPE, lambda: call(lse=lse.double())), (b.FREE_ERR_SHAPE, lambda: call(k=k[:-1])), (b.FREE_ERR_SHAPE, lambda: call(v=v[:-2])),
                    (b.FREE_ERR_SHAPE, lambda: call(heads=3)), (b.FREE_ERR_SHAPE, lambda: call(B=5)), (b.FREE_ERR_SHAPE, lambda: call(B=0)),
                    (b.FREE_ERR_SHAPE, lambda: call(q=q.t().contiguous().t())), (b.FREE_ERR_SHAPE, lambda: call(key_mask=mask[:, :-1])),
                    (b.FREE_ERR_SHAPE, lambda: call(q=q[:1].expand(12, 64))), (b.FREE_ERR_NULL, lambda: call(k=k.cpu())),
                    (b.FREE_ERR_NULL, lambda: call(key_len=n.cpu())), (b.FREE_ERR_WORKSPACE, lambda: call(workspace=torch.empty(0, dtype=torch.uint8, device=DEV))),
                    (b.FREE_ERR_NULL, lambda: back(lse=None)), (b.FREE_ERR_SHAPE, lambda: back(lse=lse[:, :2])), (b.FREE_ERR_SHAPE, lambda: back(g=g[:, :-1])),
                    (b.FREE_ERR_DTYPE, lambda: back(out=out.float()))):
        with pytest.raises(b.FreeError) as e:
            f()
        assert e.value.status == code, (code, e.value)
