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
