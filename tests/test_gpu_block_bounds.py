"""What the operators of rotary, gated blocks read and keep at the ends of their tensors, at the largest sums and at the farthest
positions."""
import pytest

pytestmark = pytest.mark.gpu


def _gen(*seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(sum((i + 1) * s for i, s in enumerate(seed)) + 41)


def _rnd(g, *shape, std=1.0, dtype=None):
    import torch
    v = torch.randn(*shape, generator=g, device="cuda") * std
    return v if dtype is None else v.to(dtype)


def _fenced(t, rows, fill):
    """t as a view into a larger buffer, `rows` rows of `fill` behind it."""
    import torch
    room = torch.full((t.shape[0] + rows, t.shape[1]), fill, dtype=t.dtype, device=t.device)
    room[:t.shape[0]] = t
    return room[:t.shape[0]]


def _kept(saved, M, F):
    """g and u of the kept state [M, H] each, H = F rounded up to 64: blocks of 32 x 32, [M / 32][2 H / 32][4][lane][4], lane l's values being
    row l % 32, columns 8 q + 4 (l / 32) + 0 .. 3 of a block."""
    import torch
    H, blocks_m = -(-F // 64) * 64, -(-M // 32)
    n = blocks_m * 32 * 2 * H
    v = saved[:4 * n].view(torch.float32).view(blocks_m, 2 * H // 32, 4, 2, 32, 4)          # mb, nb, q, lane / 32, lane % 32, c
    v = v.permute(0, 4, 1, 2, 3, 5).reshape(blocks_m * 32, 2 * H)[:M]
    return v[:, :H], v[:, H:]


# hidden values of which the last tile has 8, 16, 24 or 40, and fewer in all than one tile; the three tiles, K whole; K in parts (33, 40 rows);
# fp32, whose other widths go through padded copies
@pytest.mark.parametrize("M,D,F,dtype", [(100, 8, 8, "bf16"), (100, 8, 16, "bf16"), (50, 72, 136, "bf16"), (50, 72, 144, "bf16"), (50, 72, 152, "bf16"),
                                         (2100, 1144, 4616, "bf16"), (2100, 1144, 4624, "bf16"), (6000, 328, 1544, "bf16"), (6000, 328, 1552, "bf16"),
                                         (9000, 264, 1032, "bf16"), (9000, 264, 1040, "bf16"), (9000, 256, 1064, "bf16"), (33, 2048, 1032, "bf16"),
                                         (40, 1096, 4104, "bf16"), (70, 96, 136, "fp32"), (12, 72, 136, "bf16"), (3, 75, 133, "bf16"), (12, 64, 136, "fp32")])
def test_ffn_reads_nothing_behind_its_operands(M, D, F, dtype):
    """Memory behind every operand NaN or one: the same results to the bit, and what is kept past the hidden values zero."""
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(M, D, F)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, w_in, w_out, dy = _rnd(g, M, D, dtype=dt), _rnd(g, 2 * F, D, std=D ** -0.5, dtype=dt), _rnd(g, D, F, std=F ** -0.5, dtype=dt), _rnd(g, M, D, dtype=dt)
    results = []
    for fill in (1.0, float("nan")):
        fx, fi, fo, fy = (_fenced(t, 512, fill) for t in (x, w_in, w_out, dy))
        saved = torch.full((b.gated_ffn_saved_bytes(M, D, F, dtype),), 255, dtype=torch.uint8, device="cuda")
        plain = b.op_gated_ffn(fx, fi, fo)
        out = b.op_gated_ffn(fx, fi, fo, saved=saved)
        results.append((plain, out, *b.op_gated_ffn_backward(fy, fx, fi, fo, saved)))
        kept = _kept(saved, M, F)
        for t, w, name in zip(kept, (w_in[:F], w_in[F:]), "gu"):
            assert not t[:, F:].any(), f"{name} past the hidden values"
            ref = x.double() @ w.double().T
            # a sum of D products, a rounding each; fp32 operands: cut into three parts, 2^-24 of a product more
            assert ((t[:, :F] - ref).abs() <= (D + 16) * 2.0 ** -24 * (x.double().abs() @ w.double().abs().T)).all(), name
    for a, e in zip(*results):
        assert torch.isfinite(a).all() and torch.equal(a, e)


@pytest.mark.parametrize("theta,d", [(1.0, 8), (1.5, 256), (2.0, 64), (100.0, 36), (1e4, 128), (5e5, 64), (1e9, 20)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_angles(theta, d, inverse):
    """The pair (1, 0) becomes (cos, sin) of its angle, here against angles of 60 digits: off by less than 2^-25 turns at any position, where
    64-bit products of position and frequency would be off by more themselves."""
    import math
    from decimal import Decimal, getcontext

    import torch
    from paper_2511_20390_amd import binding as b
    getcontext().prec = 60
    turn = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
    g = _gen(int(theta), d)
    pos = [0, 1, -1, 5000, 2**24 + 1, -2**30 - 7, 2**31 - 1, -2**31] + torch.randint(-2**31, 2**31 - 1, (40,), generator=g, device="cuda").tolist()
    want = torch.empty(len(pos), d, dtype=torch.float64)
    for i in range(d // 2):
        f = Decimal(theta) ** (Decimal(-2 * i) / Decimal(d)) / turn
        for m, p in enumerate(pos):
            t = p * f
            a = float(t - t.to_integral_value()) * 2 * math.pi * (-1 if inverse else 1)
            want[m, 2 * i], want[m, 2 * i + 1] = math.cos(a), math.sin(a)
    x = torch.zeros(len(pos), d, device="cuda")
    x[:, 0::2] = 1.0
    got = b.op_rope_axes(x, torch.tensor(pos, dtype=torch.int32, device="cuda")[:, None].contiguous(), 1, d, [d], theta=theta, inverse=inverse)
    # the angle, and sine and cosine themselves: two steps of fp32 at one
    bound = 2 * math.pi * 2.0 ** -25 + 2 * 2.0 ** -23
    assert (got.double().cpu() - want).abs().max().item() <= bound


@pytest.mark.parametrize("M,D,x_dtype,out_dtype", [(3_000_001, 24, "bfloat16", "bfloat16"), (4_000_003, 3, "float32", "float32"),
                                                   (1_500_000, 130, "bfloat16", "bfloat16"), (250_001, 1152, "float32", "bfloat16")])
def test_norm_long_column_sums(M, D, x_dtype, out_dtype):
    """The weight's gradient over millions of rows, all of them in it, and with a mean, so that the sums grow."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    g = _gen(M, D)
    x = (_rnd(g, M, D) + 0.3).to(getattr(torch, x_dtype))
    dy = (_rnd(g, M, D) * 0.5 + 0.5 + 0.25 * x.float().sign()).to(getattr(torch, out_dtype))
    w = _rnd(g, D)
    dx, dw, db = b.op_layer_norm_backward(dy, x, w)
    # the definition in plain sums (the general reference adds every row to its sample's with atomics: minutes for so many)
    x, dy, w = x.double(), dy.double(), w.double()
    xc = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((xc * xc).mean(1, keepdim=True) + 1e-6)
    xh = xc * r
    gw = dy * w
    ref_dx = r * (gw - gw.mean(1, keepdim=True) - xh * (gw * xh).mean(1, keepdim=True))
    ref_dw, ref_db, size_w, size_b = (dy * xh).sum(0), dy.sum(0), (dy * xh).abs().sum(0), dy.abs().sum(0)
    # of a row: 64 roundings in a chain at most, in its mean, its deviation and the two means of the gradient
    e_xh = 64 * u.U * ((x.abs().mean(1, keepdim=True) + x.abs()) * r + xh.abs())
    e_dx = r * (64 * u.U * 2 * (gw.abs() + gw.abs().mean(1, keepdim=True) + xh.abs() * (gw * xh).abs().mean(1, keepdim=True)) +
                xh.abs() * (gw.abs() * e_xh).mean(1, keepdim=True) + e_xh * (gw * xh).mean(1, keepdim=True).abs())
    u.check(dx, (ref_dx, e_dx), "dx")
    # The chain of additions of a column: the rows of a group (a workgroup has 16 of 16 lanes, or four wavefronts, two where 8-value pieces
    # leave no more: 2 at least), the groups of a workgroup, the partial rows of a thread of the second launch, four of these, sixteen.
    # Workgroups: by the workspace, a partial row of 2 D values each.
    chunks = (b.layer_norm_backward_workspace_bytes(M, D) - 256) // (8 * D)
    groups = 16 if D <= 256 else 2
    chain = -(-M // (chunks * groups)) + 16 + -(-chunks // 64) + 4 + 16
    u.check(dw[0], (ref_dw, chain * u.U * size_w + (dy.abs() * e_xh).sum(0)), "dweight")
    u.check(db[0], (ref_db, chain * u.U * size_b), "dbias")
    # Roundings of both signs: a partial sum is off by U / sqrt(3) of itself at every addition, n of them that grow evenly to a column's sum
    # S add to U S sqrt(n) / 3; those of the groups and columns are independent.  xh's own errors average out over the rows likewise.  All
    # columns together stay below eight times that.
    for got, ref, size in ((dw[0], ref_dw, size_w), (db[0], ref_db, size_b)):
        assert (got.double() - ref).norm() <= 8 * u.U * (1 + chain ** 0.5 / 3) * size.norm()
