"""Cross attention at the edges of what its calls allow, against the formulas in 64 bits (cond_ops_util.py)."""
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


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


@pytest.mark.parametrize("Nq,heads", [((1 << 26) + 33, 1), ((1 << 20) + 1, 64), ((1 << 27) + 33, 1)])
def test_rows_past_26_bits(Nq, heads):
    """More rows of a (sample, key head) than 32 bits have room for 32 times as many, more keys than stay in LDS, and a last workgroup of which wavefronts
    have no row: the first rows, the last ones and some between."""
    Nk, dh, gen = 1100, 8, generator(1)
    q = torch.empty(Nq, heads * dh, device=DEV, dtype=torch.bfloat16).normal_(0, 1.5, generator=gen)
    k, v = normal(gen, (Nk, dh), 1.0, torch.bfloat16), normal(gen, (Nk, dh), 1.0, torch.bfloat16)
    assert (Nq * heads + 31) // 32 % 4 != 0
    lse = torch.full((1, heads, Nq), 7.0, device=DEV)
    out = b.op_cross_attention(q, k, v, 1, heads, dh, kv_heads=1, lse=lse, out=torch.full_like(q, 7.0))
    keys = torch.ones(1, Nk, dtype=torch.bool, device=DEV)
    few = 3000 // heads
    for first in (0, Nq // 2, Nq - few):
        at = slice(first, first + few)
        ref = cross_reference(q[at], k, v, 1, heads, 1, dh, dh ** -0.5, keys)
        check(out[at], ref[0], f"out of rows from {first} on")
        check(lse[:, :, at], ref[1], f"lse of rows from {first} on")


@pytest.mark.parametrize("B,Nq,Nk,heads,kv,dh,dtype", [
    (1, 1, 4096, 4, 2, 64, torch.bfloat16), (2, 3, 3000, 4, 4, 72, torch.bfloat16), (1, 150, 2050, 2, 2, 72, torch.bfloat16), (2, 40, 3000, 2, 2, 33, torch.bfloat16),
    (1, 1, 3000, 4, 2, 64, torch.float32), (1, 150, 2050, 2, 2, 72, torch.float32), (2, 9, 100, 4, 2, 64, torch.bfloat16), (2, 2100, 130, 16, 16, 72, torch.bfloat16),
    (2, 1100, 700, 32, 32, 64, torch.bfloat16),
])
@pytest.mark.parametrize("what", ["key alone", "key beside a small score", "value of a small weight"])
def test_nan_in_a_key_that_counts(B, Nq, Nk, heads, kv, dh, dtype, what):
    """NaN in one key (or value) of the last sample's second key head: everything that depends on it is NaN, however the keys are cut and whatever the
    weight of the part that it is in, and nothing else."""
    gen = generator(2)
    q, g = normal(gen, (B * Nq, heads * dh), 1.0, dtype).abs() + 1, normal(gen, (B * Nq, heads * dh), 1.0, dtype)
    k, v = normal(gen, (B * Nk, kv * dh), 1.0, dtype), normal(gen, (B * Nk, kv * dh), 1.0, dtype)
    group = heads // kv
    mask = torch.zeros(B, Nk, dtype=torch.uint8, device=DEV)
    mask[:, :Nk // 4] = 1
    # of the other keys, in parts of their own where there are parts: one or two
    at = Nk * 4 // 5 // 64 * 64
    mask[:, at] = 1
    row = (B - 1) * Nk + at
    head = slice(dh, 2 * dh)
    if what == "key alone":
        k[row, dh + 3] = math.nan
    else:
        k[row, head] = -80.0             # a score of -80 sqrt(dh) and less, 300 binary orders under the others where dh is 33 and more
        if what == "value of a small weight":
            v[row, dh + 3] = math.nan
        else:
            mask[:, at + 1] = 1
            k[row + 1, dh + 3] = math.nan
    keys = keys_that_count(B, Nk, None, mask, DEV)
    lse = torch.empty(B, heads, Nq, device=DEV)
    how = dict(B=B, heads=heads, dh=dh, kv_heads=kv, key_mask=mask)
    out = b.op_cross_attention(q, k, v, lse=lse, **how)
    ref = cross_reference(q, k, v, B, heads, kv, dh, dh ** -0.5, keys, g)
    assert ref[0][0].isnan().any()
    check(out, ref[0], "out")
    check(lse, ref[1], "lse")
    dq, dk, dv = b.op_cross_attention_backward(g, q, k, v, out, lse, **how)
    hit = torch.zeros_like(q, dtype=torch.bool)
    hit[(B - 1) * Nq:, group * dh:2 * group * dh] = True
    assert dq[hit].isnan().all()
    check(torch.where(hit, ref[2][0].to(dtype), dq), ref[2], "dq")
    theirs = torch.zeros_like(k, dtype=torch.bool)
    theirs[(B - 1) * Nk:, head] = True
    hit = theirs & keys.reshape(-1, 1)
    unkeyed = ~keys.reshape(-1)
    for t, r, name in ((dk, ref[3], "dk"), (dv, ref[4], "dv")):
        assert not t[unkeyed].any(), name
        if name == "dv" and what == "value of a small weight":
            check(t, r, name)            # (depends on keys and queries alone)
            continue
        assert t[hit].isnan().all(), name
        check(torch.where(theirs, r[0].to(dtype), t), r, name)


def ragged(seed, lens, Nq, Nk, heads, kv, dh, dtype, masked):
    """Both passes on samples whose keys end anywhere, NaN in those that do not count."""
    B, gen = len(lens), generator(seed)
    q, g = normal(gen, (B * Nq, heads * dh), 1.5, dtype), normal(gen, (B * Nq, heads * dh), 1.0, dtype)
    k, v = normal(gen, (B * Nk, kv * dh), 1.0, dtype), normal(gen, (B * Nk, kv * dh), 1.0, dtype)
    key_len = torch.tensor(lens, device=DEV, dtype=torch.int32)
    mask = (torch.rand(B, Nk, device=DEV, generator=gen) < 0.6).to(torch.uint8) if masked else None
    keys = keys_that_count(B, Nk, key_len, mask, DEV)
    ref = cross_reference(q, k, v, B, heads, kv, dh, dh ** -0.5, keys, g)
    for t in (k, v):
        t[~keys.reshape(-1)] = math.nan
    lse = torch.full((B, heads, Nq), 7.0, device=DEV)
    how = dict(B=B, heads=heads, dh=dh, kv_heads=kv, key_len=key_len, key_mask=mask)
    out = b.op_cross_attention(q, k, v, lse=lse, **how)
    got = (out, lse, *b.op_cross_attention_backward(g, q, k, v, out, lse, **how))
    for t, r, what in zip(got, ref, ("out", "lse", "dq", "dk", "dv")):
        check(t, r, what)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Nq,Nk,heads,kv,dh,lens", [
    (1, 3000, 4, 2, 64, [3000, 0, 1, 287, 288, 289, 1500, 2999]),            # few rows: parts of 288 keys
    (3, 3000, 8, 2, 72, [3000, 0, 1, 31, 33, 288, 577, 2999]),
    (5, 1100, 3, 3, 33, [1100, 0, 1, 256, 512, 513, 7]),
    (150, 2050, 4, 2, 72, [2050, 0, 1, 100, 255, 256, 257, 320, 321, 1999]), # many rows: parts of 320 keys, delta by one pass and by two
    (150, 2050, 2, 2, 128, [2050, 0, 1, 64, 256, 257]),
    (40, 700, 6, 2, 40, [700, 1, 100, 256, 257, 640]),
])
def test_lengths_that_end_in_any_part(Nq, Nk, heads, kv, dh, lens, dtype, masked):
    ragged(3, lens, Nq, Nk, heads, kv, dh, dtype, masked)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("Nq,Nk,heads,kv,dh", [
    (1500, 700, 16, 16, 72), (1500, 700, 16, 16, 96), (1500, 700, 16, 16, 128), (1500, 900, 16, 16, 64),      # keys pass through LDS
    (1500, 250, 16, 16, 72), (1500, 200, 16, 16, 40),                                                         # keys stay in it
    (500, 700, 48, 16, 72), (500, 130, 48, 16, 64), (250, 700, 96, 16, 128), (250, 300, 112, 16, 96),         # groups that no tile of rows is a multiple of
])
@pytest.mark.parametrize("lens", [[1.0, 100, 256], [257, 0, 1], [1.0, 63, 64]])
def test_many_queries_of_ragged_samples(Nq, Nk, heads, kv, dh, lens, masked):
    ragged(4, [int(n * Nk) if isinstance(n, float) else min(n, Nk) for n in lens], Nq, Nk, heads, kv, dh, torch.bfloat16, masked)


@pytest.mark.parametrize("Nq,heads,Nk,dtype", [((1 << 20) + 1, 64, 1100, torch.bfloat16), ((1 << 26) + 33, 1, 1100, torch.bfloat16), ((1 << 20) + 1, 65, 77, torch.float32)])
def test_gradient_of_rows_past_26_bits(Nq, heads, Nk, dtype):
    """The last rows alone have a gradient."""
    dh, gen, few = 8, generator(5), 3000 // heads
    q = torch.empty(Nq, heads * dh, device=DEV, dtype=dtype).normal_(0, 1.5, generator=gen)
    k, v = normal(gen, (Nk, dh), 1.0, dtype), normal(gen, (Nk, dh), 1.0, dtype)
    last = slice(Nq - few, Nq)
    g = torch.zeros_like(q)
    g[last] = normal(gen, (few, heads * dh), 1.0, dtype)
    lse = torch.empty(1, heads, Nq, device=DEV)
    how = dict(B=1, heads=heads, dh=dh, kv_heads=1)
    out = b.op_cross_attention(q, k, v, lse=lse, **how)
    dq, dk, dv = b.op_cross_attention_backward(g, q, k, v, out, lse, **how)
    ref = cross_reference(q[last], k, v, 1, heads, 1, dh, dh ** -0.5, torch.ones(1, Nk, dtype=torch.bool, device=DEV), g[last])
    for t, r, what in ((out[last], ref[0], "out"), (lse[:, :, last], ref[1], "lse"), (dq[last], ref[2], "dq"), (dk, ref[3], "dk"), (dv, ref[4], "dv")):
        check(t, r, what)
    assert not dq[:Nq - few].any()
