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
