"""The projection with adapters at the edges of what its calls allow, against the formulas in 64 bits (cond_ops_util.py)."""
import pytest
import torch

from paper_2511_20390_amd import binding as b
from tests.block_ops_util import check
from tests.cond_ops_util import adapters_reference

pytestmark = pytest.mark.gpu

DEV = "cuda"


def normal(gen, shape, std, dtype):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0, std, generator=gen)


@pytest.mark.parametrize("dtype,K,N", [(torch.bfloat16, 64, 64), (torch.float32, 32, 32)])
def test_most_rows(dtype, K, N):
    """As many rows as there may be, without a bias: the first and last rows, and the adapters' gradient where the last rows alone have one."""
    M, r, n, rows = 1 << 27, 4, 2, 1 << 26
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x, w = normal(gen, (M, K), 1.0, dtype), normal(gen, (N, K), K ** -0.5, dtype)
    a, bb = normal(gen, (n, r, K), K ** -0.5, dtype), normal(gen, (n, N, r), r ** -0.5, dtype)
    scale = 0.5 + torch.rand(n, device=DEV, generator=gen)
    adapter = torch.arange(n, device=DEV, dtype=torch.int32)
    g = torch.zeros(M, N, device=DEV, dtype=dtype)
    last = slice(M - 130, M)
    g[last] = normal(gen, (130, N), 1.0, dtype)
    saved = torch.empty(b.linear_adapters_saved_bytes(M, r, "bf16" if dtype == torch.bfloat16 else "fp32"), dtype=torch.uint8, device=DEV)
    how = dict(scale=scale, rows_per_sample=rows)
    out = b.op_linear_adapters(x, w, None, a, bb, adapter, saved=saved, **how)
    dx, da, db = b.op_linear_adapters_backward(g, x, w, a, bb, adapter, saved, **how)
    first = slice(0, 300)
    check(out[first], adapters_reference(x[first], w, None, a, bb, adapter[:1], scale, 300)[0], "out of the first rows")
    ref = adapters_reference(x[last], w, None, a, bb, adapter[1:], scale, 130, g[last])
    for t, e, what in ((out[last], ref[0], "out"), (dx[last], ref[1], "dx"), (da, ref[2], "dA"), (db, ref[3], "dB")):
        check(t, e, what)
    assert not dx[:M - 130].any()
