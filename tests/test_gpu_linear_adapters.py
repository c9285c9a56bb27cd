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
    (1, 64, 64, 4, 1, 1), (8, 128, 192, 16, 8, 1), (17, 64, 320, 8, 3, 5), (33, 192, 64, 16, 2, 7), (100, 64, 128, 32, 3, 100), (130, 320, 192, 64, 4, 33),
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
    (4200, 128, 192, 24, 3, 512), (6000, 256, 128, 16, 12, 60), (200, 2048, 384, 16, 2, 50), (5000, 64, 64, 64, 2, 5000), (700, 1152, 2304, 16, 4, 350),
])
def test_sums_in_parts_and_large_tiles(dtype, M, K, N, r, n, rows):
    compare(*problem(3, M, K, N, r, n, rows, dtype), rows)
