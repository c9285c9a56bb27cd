"""Layer norm, rotary positions over several axes and the gated feed-forward block, forward and backward, against the definitions in 64
bits, at the sizes, types, strides and layouts where a kernel changes its way."""
import pytest

pytestmark = pytest.mark.gpu

TYPES = {"bf16": "bfloat16", "fp32": "float32"}


def _t(name):
    import torch
    return getattr(torch, TYPES[name])


def _gen(*seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(sum((i + 1) * s for i, s in enumerate(seed)) + 17)


def _rnd(g, *shape, std=1.0, dtype=None):
    import torch
    v = torch.randn(*shape, generator=g, device="cuda") * std
    return v if dtype is None else v.to(dtype)


# ---- layer norm ----------------------------------------------------------------------------------------------------
# widths at both sides of every row layout (16-byte chunks: 256, 512, 1280, 2560, 5120, 8192 values; one value at a time: 512, 2048,
# 4096, 8192), one value, the largest; row counts from one over less than a workgroup's to several partial rows per sample
NORM_WIDTHS = [1, 2, 3, 8, 77, 256, 260, 511, 512, 513, 516, 1152, 1279, 1280, 1284, 2047, 2049, 2560, 2564, 4096, 4097, 5120, 5124, 8192,
               8193, 8196, 16381, 16384]


def _norm_case(M, D, rows, x_dtype, out_dtype, affine=True, modulate=False, offset=0.5, seed=0):
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    g = _gen(M, D, seed)
    n = max(1, -(-M // rows))
    x = (_rnd(g, M, D) * torch.exp(_rnd(g, 1, D, std=0.5)) + offset).to(_t(x_dtype))
    w = _rnd(g, n, D, std=0.3) + (0.0 if modulate else 1.0) if affine else None
    bias = _rnd(g, n, D, std=0.3) if affine else None
    dy = _rnd(g, M, D, dtype=_t(out_dtype))
    what = f"layer norm {M} x {D}, {rows} rows per sample, {x_dtype} -> {out_dtype}"
    ref = u.norm_reference(x, w, bias, rows, modulate, 1e-6, dy)
    got = b.op_layer_norm(x, w, bias, out_dtype, rows_per_sample=rows, modulate=modulate)
    u.check(got, ref[0], what)
    grads = b.op_layer_norm_backward(dy, x, w, rows_per_sample=rows, modulate=modulate)
    for k, name in enumerate(("dx", "dweight", "dbias")):
        u.check(grads[k], ref[1 + k], what + " " + name)
    alone = b.op_layer_norm_backward(dy, x, w, rows_per_sample=rows, modulate=modulate, want_weight=False)
    assert torch.equal(alone[0], grads[0]) and alone[1] is None


@pytest.mark.parametrize("D", NORM_WIDTHS)
def test_norm_widths(D):
    _norm_case(5, D, 5, "fp32", "bf16")
    _norm_case(37, D, 37, "bf16", "bf16")


@pytest.mark.parametrize("M", [1, 2, 3, 4, 7, 8, 31, 32, 33, 65, 129, 1000, 4097])
def test_norm_rows(M):
    _norm_case(M, 1152, M, "fp32", "fp32")
    _norm_case(M, 130, max(1, M // 3), "bf16", "fp32", modulate=True)


@pytest.mark.parametrize("x,out", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,D,rows", [(64, 1152, 16), (70, 768, 32), (5, 384, 1), (40, 4096, 7), (513, 99, 512), (3000, 64, 1024)])
def test_norm_samples(x, out, M, D, rows):
    """Every sample its own weight; the last one has fewer rows; samples of one row."""
    _norm_case(M, D, rows, x, out, modulate=True)
    _norm_case(M, D, rows, x, out, modulate=False, seed=1)
    _norm_case(M, D, rows, x, out, affine=False, seed=2)


def test_norm_large_mean():
    """The mean taken off first: a row whose offset is 3000 standard deviations keeps what its fp32 values carry."""
    _norm_case(33, 1152, 33, "fp32", "fp32", offset=3000.0)
    _norm_case(6, 1001, 6, "fp32", "fp32", offset=3000.0)


def test_norm_constant_rows():
    """Rows without variance: the result is the bias, and finite gradients."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    x = torch.full((9, 640), 2.5, device="cuda")
    x[3] = 0.0
    w, bias = torch.rand(640, device="cuda"), torch.rand(640, device="cuda")
    dy = _rnd(_gen(1), 9, 640)
    ref = u.norm_reference(x, w, bias, 9, False, 1e-6, dy)
    assert torch.equal(b.op_layer_norm(x, w, bias), bias.expand(9, 640))
    for got, r in zip(b.op_layer_norm_backward(dy, x, w), ref[1:]):
        u.check(got, r, "constant rows")


def test_norm_not_finite_rows_stay_alone():
    import torch
    from paper_2511_20390_amd import binding as b
    x = _rnd(_gen(2), 12, 1152)
    clean = b.op_layer_norm(x)
    x[2, 7], x[5, 0], x[11, 1151] = float("nan"), float("inf"), -float("inf")
    got = b.op_layer_norm(x)
    bad = torch.zeros(12, dtype=torch.bool, device="cuda")
    bad[[2, 5, 11]] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], clean[~bad])


def test_norm_strided_vectors_and_odd_addresses():
    """Weights that are columns of a wider modulation tensor, and tensors that start at an odd value."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    g = _gen(3)
    for wide, at in ((3000, 0), (3000, 1152), (3001, 5)):
        mod = _rnd(g, 4, wide, std=0.3)
        shift, scale = mod[:, at:at + 640], mod[:, at + 640:at + 1280]
        for skip in (0, 1, 2):
            x = _rnd(g, 50 * 640 + 4)[skip:skip + 50 * 640].view(50, 640)
            dy = _rnd(g, 50 * 640 + 4)[skip:skip + 50 * 640].view(50, 640)
            ref = u.norm_reference(x, scale, shift, 13, True, 1e-6, dy)
            u.check(b.op_layer_norm(x, scale, shift, rows_per_sample=13, modulate=True), ref[0], "strided")
            grads = torch.empty(4, wide, device="cuda").fill_(7.0)
            out = (torch.empty_like(x), grads[:, at + 640:at + 1280], grads[:, at:at + 640])
            got = b.op_layer_norm_backward(dy, x, scale, rows_per_sample=13, modulate=True, out=out)
            for k in range(3):
                u.check(got[k], ref[1 + k], "strided gradients")
            rest = torch.ones(wide, dtype=torch.bool, device="cuda")
            rest[at:at + 1280] = False
            assert (grads[:, rest] == 7.0).all()


@pytest.mark.parametrize("M,D,rows", [(1, 5, 1), (300, 130, 300), (300, 1152, 25), (67, 1001, 67), (90, 4100, 90)])
def test_norm_what_buffers_held(M, D, rows):
    """A workspace that starts as NaN, and memory behind every output left as it was."""
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(19, M, D)
    n = -(-M // rows)
    for dt in (torch.float32, torch.bfloat16):
        x, dy, w, bias = _rnd(g, M, D, dtype=dt), _rnd(g, M, D, dtype=dt), _rnd(g, n, D), _rnd(g, n, D)
        results = []
        for fill in (0, 255):
            ws = torch.full((b.layer_norm_backward_workspace_bytes(M, D, rows),), fill, dtype=torch.uint8, device="cuda")
            room = [torch.full((k * D + 64,), 7.0, dtype=t, device="cuda") for k, t in ((M, dt), (M, dt), (n, torch.float32), (n, torch.float32))]
            outs = [r[:-64].view(-1, D) for r in room]
            b.op_layer_norm(x, w, bias, rows_per_sample=rows, out=outs[0])
            b.op_layer_norm_backward(dy, x, w, rows_per_sample=rows, out=outs[1:], workspace=ws)
            for r in room:
                assert (r[-64:] == 7.0).all()
            results.append(outs)
        for a, e in zip(*results):
            assert torch.equal(a, e) and torch.isfinite(a).all()


def test_norm_gradient_in_place():
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(4)
    x, dy, w = _rnd(g, 300, 1152), _rnd(g, 300, 1152), _rnd(g, 1152)
    ref = b.op_layer_norm_backward(dy, x, w)
    for target in (0, 1):
        args = [dy.clone(), x.clone()]
        got = b.op_layer_norm_backward(*args, w, out=(args[target], torch.empty(1152, device="cuda"), torch.empty(1152, device="cuda")))
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1][0]) and torch.equal(got[2], ref[2][0])


def test_norm_gradient_against_differences():
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(5)
    x, dy, w, bias = _rnd(g, 6, 40), _rnd(g, 6, 40), _rnd(g, 40), _rnd(g, 40)
    dx, dw, db = b.op_layer_norm_backward(dy, x, w)
    loss = lambda *a: (b.op_layer_norm(*a).double() * dy.double()).sum().item()
    # central difference over 2 h: each result off by some 8 U of its size (240 products of about one in the loss: 1e-5), the third
    # derivative times h^2 below 2e-3 of the gradient's size
    h = 2.0 ** -6
    for t, grad, args in ((x, dx, lambda t: (t, w, bias)), (w, dw[0], lambda t: (x, t, bias)), (bias, db[0], lambda t: (x, w, t))):
        for k in range(0, t.numel(), 13):
            up, down = t.clone().flatten(), t.clone().flatten()
            up[k] += h
            down[k] -= h
            diff = (loss(*args(up.view_as(t))) - loss(*args(down.view_as(t)))) / (2 * h)
            assert abs(diff - grad.flatten()[k].item()) < 2e-2 * max(1.0, grad.abs().max().item())


def test_norm_far_rows():
    """Offsets past 2^31 values and 2^32 bytes."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    M, D = 1_050_001, 2052
    x = torch.zeros(M, D, dtype=torch.bfloat16, device="cuda")
    g = _gen(6)
    tail = _rnd(g, 7, D, dtype=torch.bfloat16)
    x[-7:] = tail
    w, bias = _rnd(g, D), _rnd(g, D)
    out = b.op_layer_norm(x, w, bias)
    u.check(out[-7:], u.norm_reference(tail, w, bias, 7, False, 1e-6), "far rows")
    assert torch.equal(out[:3], bias.to(torch.bfloat16).expand(3, D))
    dy = torch.zeros_like(x)
    dy[-7:] = _rnd(g, 7, D, dtype=torch.bfloat16)
    dx, dw, db = b.op_layer_norm_backward(dy, x, w, out=(out, torch.empty(D, device="cuda"), torch.empty(D, device="cuda")))
    ref = u.norm_reference(tail, w, bias, 7, False, 1e-6, dy[-7:])
    u.check(dx[-7:], ref[1], "far dx")
    u.check(dw[None], ref[2], "far dweight")
    u.check(db[None], ref[3], "far dbias")


def test_norm_many_rows():
    """More rows than a grid's workgroups take at once."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    M, D = 70_000_003, 3
    g = _gen(22)
    x = torch.zeros(M, D, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, 67_108_863, 67_108_864, 67_108_865, M - 1], device="cuda")
    x[at] = _rnd(g, 6, D, dtype=torch.bfloat16)
    w, bias = _rnd(g, D), _rnd(g, D)
    out = b.op_layer_norm(x, w, bias)
    ref = u.norm_reference(x[at], w, bias, 6, False, 1e-6, x[at])
    u.check(out[at], ref[0], "many rows")
    rest = torch.ones(M, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert (out[rest] == bias.to(torch.bfloat16)).all()
    dx, dw, db = b.op_layer_norm_backward(x, x, w)
    u.check(dx[at], ref[1], "many rows dx")
    u.check(dw, ref[2], "many rows dweight")
    u.check(db, ref[3], "many rows dbias")


# ---- rotary positions ------------------------------------------------------------------------------------------------
ROPE = [(72, [36, 36]), (128, [16, 56, 56]), (128, [128]), (64, [8, 24, 24]), (2, [2]), (6, [2, 2, 2]), (40, [4, 6, 8, 10]), (16, [0, 8]),
        (256, [64, 96, 96]), (34, [16, 16]), (20, [10])]


def _rope_case(rows, heads, dh, dims, pairs, inverse, dtype, pos_rows=None, theta=10000.0, low=-50, high=5000, extra=0, skip=0):
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    g = _gen(rows, heads, dh, len(dims))
    width = heads * dh
    flat = _rnd(g, rows * (width + extra) + skip, dtype=_t(dtype))[skip:]
    x = flat.view(rows, width + extra)[:, :width]
    pos = torch.randint(low, high, (pos_rows or rows, len(dims)), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    kw = dict(theta=theta, pairing=b.ROPE_PAIRS if pairs else b.ROPE_HALVES, inverse=inverse)
    got = b.op_rope_axes(x, pos, heads, dh, dims, **kw)
    ref, bound = u.rope_reference(x, pos, heads, dh, dims, theta, pairs, inverse)
    what = f"rotary {rows} x {heads} x {dh} {dims} {'pairs' if pairs else 'halves'} {dtype}"
    u.check(got, (ref, bound), what)
    done = sum(dims)
    assert torch.equal(got.view(rows, heads, dh)[:, :, done:], x.reshape(rows, heads, dh)[:, :, done:]), what
    before = flat.clone()
    same = b.op_rope_axes(x, pos, heads, dh, dims, out=x, **kw)
    assert same is x and torch.equal(x, got)
    flat.view(rows, width + extra)[:, :width] = before.view(rows, width + extra)[:, :width]
    assert torch.equal(flat, before), what + ": values between the rows"


@pytest.mark.parametrize("dh,dims", ROPE)
@pytest.mark.parametrize("pairs", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rope_layouts(dh, dims, pairs, dtype):
    _rope_case(33, 5, dh, dims, pairs, False, dtype)
    _rope_case(20, 8, dh, dims, pairs, True, dtype, pos_rows=7)
    for extra, skip in ((1, 0), (2, 2), (4, 4), (3, 1), (8, 8), (0, 1)):      # strides and first addresses of every alignment
        _rope_case(9, 3, dh, dims, pairs, False, dtype, extra=extra, skip=skip)


@pytest.mark.parametrize("rows,heads", [(1, 1), (1, 64), (2, 4), (255, 1), (257, 9), (1000, 32)])
def test_rope_counts(rows, heads):
    _rope_case(rows, heads, 72, [36, 36], True, False, "bf16")
    _rope_case(rows, heads, 64, [64], False, False, "fp32", pos_rows=1)


@pytest.mark.parametrize("theta", [1.0, 100.0, 1e4, 5e5, 1e9])
def test_rope_far_positions(theta):
    """Any int32 is a position (the 64-bit reference's own angle is off by 2^-53 of it: the bound says so)."""
    _rope_case(64, 2, 64, [32, 32], True, False, "fp32", theta=theta, low=-2**31, high=2**31 - 1)
    _rope_case(64, 2, 64, [32, 32], False, True, "fp32", theta=theta, low=2**23, high=2**25)


def test_rope_inverse_undoes():
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(8)
    x = _rnd(g, 500, 12 * 72)
    pos = torch.randint(0, 4000, (500, 2), generator=g, device="cuda", dtype=torch.int32)
    y = b.op_rope_axes(x, pos, 12, 72, [36, 36])
    back = b.op_rope_axes(y, pos, 12, 72, [36, 36], inverse=True)
    assert ((back - x).abs() <= 32 * 2.0 ** -24 * (1 + x.abs().max())).all()
    # the turn keeps lengths, and the gradient of <dy, turned x> is dy turned back
    dy = _rnd(g, 500, 12 * 72)
    lhs = (y.double() * dy.double()).sum()
    rhs = (x.double() * b.op_rope_axes(dy, pos, 12, 72, [36, 36], inverse=True).double()).sum()
    assert abs(lhs - rhs) < 1e-6 * x.double().norm() * dy.double().norm()


def test_rope_not_finite_values_stay_in_their_pair():
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(9)
    x = _rnd(g, 10, 2 * 72)
    pos = torch.randint(0, 4000, (10, 2), generator=g, device="cuda", dtype=torch.int32)
    clean = b.op_rope_axes(x, pos, 2, 72, [32, 32])
    x[4, 10], x[6, 70], x[7, 72 + 71] = float("inf"), float("nan"), float("inf")
    got = b.op_rope_axes(x, pos, 2, 72, [32, 32])
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[4, 10:12] = bad[6, 70] = bad[7, 143] = True
    assert torch.equal(got[~bad], clean[~bad]) and not torch.isfinite(got[bad]).any() and got[7, 143] == float("inf")


def test_rope_queries_and_keys_of_packed_rows():
    """The q | k part of q | k | v rows turned in place, v untouched: what free_op_attention reads next."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    g = _gen(10)
    B, N, heads, dh = 3, 64, 4, 72
    qkv = _rnd(g, B * N, 3 * heads * dh, dtype=torch.bfloat16)
    pos = torch.stack(torch.meshgrid(torch.arange(8, device="cuda"), torch.arange(8, device="cuda"), indexing="ij"), -1).view(64, 2).int()
    before = qkv.clone()
    width = 2 * heads * dh
    b.op_rope_axes(qkv[:, :width], pos, 2 * heads, dh, [36, 36], out=qkv[:, :width])
    u.check(qkv[:, :width], u.rope_reference(before[:, :width], pos, 2 * heads, dh, [36, 36], 1e4, True, False), "packed rows")
    assert torch.equal(qkv[:, width:], before[:, width:])


def test_rope_far_rows():
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    rows, heads, dh = 600_001, 56, 64
    x = torch.zeros(rows, heads * dh, dtype=torch.bfloat16, device="cuda")
    g = _gen(11)
    tail = _rnd(g, 5, heads * dh, dtype=torch.bfloat16)
    x[-5:] = tail
    pos = torch.arange(rows, device="cuda", dtype=torch.int32)[:, None].contiguous()
    b.op_rope_axes(x, pos, heads, dh, [64], out=x)
    u.check(x[-5:], u.rope_reference(tail, pos[-5:], heads, dh, [64], 1e4, True, False), "far rows")
    assert not x[:-5].any()


# ---- gated feed-forward block -----------------------------------------------------------------------------------------
def _ffn_case(M, D, F, act, dtype, seed=0, norms=True):
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    g = _gen(M, D, F, seed)
    dt = _t(dtype)
    x = _rnd(g, M, D, dtype=dt)
    w_in, w_out = _rnd(g, 2 * F, D, std=D ** -0.5, dtype=dt), _rnd(g, D, F, std=F ** -0.5, dtype=dt)
    dy = _rnd(g, M, D, dtype=dt)
    what = f"ffn {M} x {D} x {F} {act} {dtype}"
    ref = u.ffn_reference(x, w_in, w_out, act, dy)
    saved = torch.empty(b.gated_ffn_saved_bytes(M, D, F, dtype), dtype=torch.uint8, device="cuda")
    plain = b.op_gated_ffn(x, w_in, w_out, act)
    out = b.op_gated_ffn(x, w_in, w_out, act, saved=saved)
    grads = b.op_gated_ffn_backward(dy, x, w_in, w_out, saved, act)
    u.check(plain, ref[0], what)
    for got, r, name in zip((out, *grads), ref, ("out", "dx", "dw_in", "dw_out")):
        u.check(got, r, what + " " + name)
        if norms and got.numel() >= 1024 and min(M, F) >= 32:
            # two independent roundings (of a factor, of the result), uniform within half a step: 2/3 of its square together; fp32: sums
            # of up to K roundings that average out, 2e-5 as for the linear layers
            rel = ((got.double() - r[0]).norm() / r[0].norm()).item()
            assert rel < (u.half_step(dt) if dtype == "bf16" else 2e-5), (what, name, rel)
    assert torch.equal(b.op_gated_ffn_backward(dy, x, w_in, w_out, saved, act)[1], grads[1]), what


# rows: one token, a few (at both sides of what one matrix instruction takes), several tiles; sizes that are multiples of the tiles and
# slices, one off them, and of nothing
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 129, 257, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_ffn_rows(M, dtype):
    _ffn_case(M, 128, 320, "silu", dtype)
    _ffn_case(M, 96, 200, "gelu", dtype)


@pytest.mark.parametrize("D,F", [(1, 1), (1, 64), (64, 1), (2, 3), (7, 5), (8, 8), (31, 33), (63, 65), (64, 64), (65, 63), (72, 40), (100, 260),
                                 (127, 129), (129, 127), (192, 512), (250, 1000), (256, 128), (320, 897), (384, 1536), (1001, 333)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_ffn_widths(D, F, dtype):
    for M in (1, 5, 70):
        _ffn_case(M, D, F, "silu", dtype)


@pytest.mark.parametrize("M,D,F,act,dtype", [(512, 1152, 4608, "gelu", "bf16"), (1000, 1152, 2000, "silu", "bf16"), (2048, 384, 1536, "gelu", "bf16"),
                                             (700, 768, 2048, "silu", "fp32"), (24, 2048, 5120, "silu", "bf16"), (1, 2048, 5121, "gelu", "bf16"),
                                             (2, 4096, 10240, "silu", "bf16"), (1500, 1024, 1024, "silu", "bf16"), (5, 1152, 4608, "silu", "fp32")])
def test_ffn_sizes_in_use(M, D, F, act, dtype):
    _ffn_case(M, D, F, act, dtype)


# every tile of every product of the two passes, with K whole and in parts: (256 x 256, 128 x 256) down 4100, 9000; in parts 6000, 2060; dx
# 9000, 6000; in parts 3001, 1500; weights 200 (256), 9000 and 6000 in parts; the gated gradient on 256 x 256 2060; gate and up in parts 33;
# ragged rows in all of them
@pytest.mark.parametrize("M,D,F", [(4100, 2048, 1024), (9000, 512, 512), (6000, 320, 6400), (2060, 1152, 4608), (9000, 1536, 2048),
                                   (6000, 1152, 4608), (3001, 1152, 4608), (1500, 1152, 4608), (200, 1536, 2048), (9000, 256, 1024),
                                   (6000, 768, 2048), (2060, 320, 6400), (33, 2048, 1024)])
def test_ffn_tiles(M, D, F):
    _ffn_case(M, D, F, "silu", "bf16")


# widths that are multiples of 8 and not of a slice: ragged K of every product, the seam of [dg | du], K whole and in parts
@pytest.mark.parametrize("M,D,F", [(33, 72, 40), (100, 8, 8), (70, 136, 2000), (257, 1000, 72), (300, 1160, 2744), (1001, 200, 1000), (40, 1096, 4104),
                                   (2100, 1144, 4616), (6000, 328, 1544), (9000, 264, 1032)])
def test_ffn_ragged_slices(M, D, F):
    _ffn_case(M, D, F, "silu", "bf16")


def test_ffn_not_finite_weights():
    """What an infinite weight next to a ragged row's end reaches: the gate value it belongs to, not its neighbour's column."""
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(21)
    M, D, F = 50, 72, 136
    dt = torch.bfloat16
    x, w_in, w_out = _rnd(g, M, D, dtype=dt), _rnd(g, 2 * F, D, std=0.1, dtype=dt), _rnd(g, D, F, std=0.1, dtype=dt)
    clean = b.op_gated_ffn(x, w_in, w_out)
    w_out[6, 0] = float("inf")                             # read behind the end of row 5
    got = b.op_gated_ffn(x, w_in, w_out)
    keep = torch.arange(D, device="cuda") != 6
    assert torch.equal(got[:, keep], clean[:, keep]) and not torch.isfinite(got[:, 6]).any()
    # one infinite input: its row alone, though the row before is read into it
    w_out[6, 0] = 0.1
    x[7, 0] = float("nan")
    clean, got = b.op_gated_ffn(x.nan_to_num(0.0), w_in, w_out), b.op_gated_ffn(x, w_in, w_out)
    rows = torch.arange(M, device="cuda") != 7
    assert torch.equal(got[rows], clean[rows]) and torch.isnan(got[7]).all()


@pytest.mark.parametrize("M,D,F", [(40, 256, 4096), (600, 1152, 1152), (3000, 128, 512), (2500, 768, 1536), (130, 1024, 64)])
def test_ffn_tiles_fp32(M, D, F):
    """64 x 64 and 128 x 128 tiles, K whole and in parts."""
    _ffn_case(M, D, F, "gelu", "fp32")


@pytest.mark.parametrize("scale", [1e-22, 1e-12, 1e15])
def test_ffn_fp32_scales(scale):
    """Gradients far below 2^-64, where the three-part products are computed again in fp32, and far above one."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    g = _gen(16)
    for M, D, F in ((70, 128, 192), (333, 96, 100), (1000, 384, 512)):
        x, w_in, w_out = _rnd(g, M, D), _rnd(g, 2 * F, D, std=D ** -0.5), _rnd(g, D, F, std=F ** -0.5)
        dy = _rnd(g, M, D, std=scale)
        saved = torch.empty(b.gated_ffn_saved_bytes(M, D, F, "fp32"), dtype=torch.uint8, device="cuda")
        out = b.op_gated_ffn(x, w_in, w_out, saved=saved)
        got = (out, *b.op_gated_ffn_backward(dy, x, w_in, w_out, saved))
        for k, r, name in zip(got, u.ffn_reference(x, w_in, w_out, "silu", dy), ("out", "dx", "dw_in", "dw_out")):
            u.check(k, r, f"scale {scale} {name}")


def test_ffn_gradient_not_finite_rows_stay_alone():
    """dx has a row per token; what a token's infinite gradient reaches in the weights' gradients is not finite either."""
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(17)
    for dtype in ("bf16", "fp32"):
        dt = _t(dtype)
        M, D, F = 90, 128, 192
        x, w_in, w_out = _rnd(g, M, D, dtype=dt), _rnd(g, 2 * F, D, std=0.1, dtype=dt), _rnd(g, D, F, std=0.1, dtype=dt)
        dy = _rnd(g, M, D, dtype=dt)
        saved = torch.empty(b.gated_ffn_saved_bytes(M, D, F, dtype), dtype=torch.uint8, device="cuda")
        b.op_gated_ffn(x, w_in, w_out, saved=saved)
        clean = b.op_gated_ffn_backward(dy, x, w_in, w_out, saved)
        dy[41, 3] = float("inf")
        dx, dw_in, dw_out = b.op_gated_ffn_backward(dy, x, w_in, w_out, saved)
        keep = torch.arange(M, device="cuda") != 41
        assert torch.equal(dx[keep], clean[0][keep]) and not torch.isfinite(dx[41]).any()
        assert not torch.isfinite(dw_in).any() and not torch.isfinite(dw_out[3]).any()
        rest = torch.arange(D, device="cuda") != 3
        assert torch.equal(dw_out[rest], clean[2][rest])


@pytest.mark.parametrize("M", [1, 20, 33, 500])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_ffn_what_buffers_held(M, dtype):
    """Workspaces and kept state that start as NaN, and memory behind every output left as it was; even and padded widths."""
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(18, M)
    dt = _t(dtype)
    for D, F in ((128, 192), (72, 1100), (33, 65)):
        x, w_in, w_out = _rnd(g, M, D, dtype=dt), _rnd(g, 2 * F, D, std=0.1, dtype=dt), _rnd(g, D, F, std=0.1, dtype=dt)
        dy = _rnd(g, M, D, dtype=dt)
        results = []
        for fill in (0, 255):
            byte = lambda n: torch.full((n,), fill, dtype=torch.uint8, device="cuda")
            ws, saved = byte(b.gated_ffn_workspace_bytes(M, D, F, dtype, True)), byte(b.gated_ffn_saved_bytes(M, D, F, dtype))
            small = byte(b.gated_ffn_workspace_bytes(M, D, F, dtype))
            room = [torch.full((n + 64,), 7.0, dtype=dt, device="cuda") for n in (M * D, M * D, M * D, 2 * F * D, D * F)]
            outs = [r[:r.numel() - 64].view(s) for r, s in zip(room, ((M, D), (M, D), (M, D), (2 * F, D), (D, F)))]
            b.op_gated_ffn(x, w_in, w_out, out=outs[0], workspace=small)
            b.op_gated_ffn(x, w_in, w_out, out=outs[1], saved=saved, workspace=small)
            b.op_gated_ffn_backward(dy, x, w_in, w_out, saved, out=outs[2:], workspace=ws)
            for r in room:
                assert (r[-64:] == 7.0).all()
            results.append(outs)
        for a, e in zip(*results):
            assert torch.equal(a, e) and torch.isfinite(a).all()


def test_ffn_extreme_gates():
    """Gates far out on both sides: the activation is 0 or the gate, its slope 0 or 1, and nothing is NaN."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    for dtype in ("bf16", "fp32"):
        dt = _t(dtype)
        for act in ("silu", "gelu"):
            M, D, F = 40, 64, 128
            g = _gen(12)
            x = _rnd(g, M, D, std=40.0, dtype=dt)
            w_in, w_out, dy = _rnd(g, 2 * F, D, dtype=dt), _rnd(g, D, F, dtype=dt), _rnd(g, M, D, dtype=dt)
            saved = torch.empty(b.gated_ffn_saved_bytes(M, D, F, dtype), dtype=torch.uint8, device="cuda")
            out = b.op_gated_ffn(x, w_in, w_out, act, saved=saved)
            got = (out, *b.op_gated_ffn_backward(dy, x, w_in, w_out, saved, act))
            for k, r in zip(got, u.ffn_reference(x, w_in, w_out, act, dy)):
                u.check(k, r, f"extreme gates {act} {dtype}")


def test_ffn_not_finite_rows_stay_alone():
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(13)
    for M in (7, 200):
        x = _rnd(g, M, 128, dtype=torch.bfloat16)
        w_in, w_out = _rnd(g, 512, 128, std=0.1, dtype=torch.bfloat16), _rnd(g, 128, 256, std=0.1, dtype=torch.bfloat16)
        clean = b.op_gated_ffn(x, w_in, w_out)
        x[3, 5], x[M - 1, 0] = float("nan"), float("inf")
        got = b.op_gated_ffn(x, w_in, w_out)
        bad = torch.zeros(M, dtype=torch.bool, device="cuda")
        bad[3] = bad[M - 1] = True
        assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], clean[~bad])


def test_ffn_gradient_against_differences():
    import torch
    from paper_2511_20390_amd import binding as b
    g = _gen(14)
    M, D, F = 6, 16, 24
    x, w_in, w_out, dy = _rnd(g, M, D), _rnd(g, 2 * F, D, std=0.25), _rnd(g, D, F, std=0.2), _rnd(g, M, D)
    for act in ("silu", "gelu"):
        saved = torch.empty(b.gated_ffn_saved_bytes(M, D, F, "fp32"), dtype=torch.uint8, device="cuda")
        b.op_gated_ffn(x, w_in, w_out, act, saved=saved)
        grads = b.op_gated_ffn_backward(dy, x, w_in, w_out, saved, act)
        loss = lambda *a: (b.op_gated_ffn(*a, act).double() * dy.double()).sum().item()
        h = 2.0 ** -6                 # h^2 and the results' roundings (1e-6 of the loss over 2 h) both below 1e-2 of the largest gradient
        for k, t in enumerate((x, w_in, w_out)):
            for i in range(0, t.numel(), 29):
                args = [[x, w_in, w_out], [x, w_in, w_out]]
                for a, step in zip(args, (h, -h)):
                    a[k] = t.clone().flatten()
                    a[k][i] += step
                    a[k] = a[k].view_as(t)
                diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
                assert abs(diff - grads[k].flatten()[i].item()) < 1e-2 * max(1.0, grads[k].abs().max().item())


def test_ffn_far_rows():
    """Saved state and products past 2^32 bytes."""
    import torch
    from paper_2511_20390_amd import binding as b
    from tests import block_ops_util as u
    g = _gen(15)
    M, D, F = 140_001, 64, 4096
    dt = torch.bfloat16
    x = _rnd(g, M, D, dtype=dt)
    w_in, w_out = _rnd(g, 2 * F, D, std=0.12, dtype=dt), _rnd(g, D, F, std=0.015, dtype=dt)
    dy = torch.zeros(M, D, dtype=dt, device="cuda")
    dy[-9:] = _rnd(g, 9, D, dtype=dt)
    saved = torch.empty(b.gated_ffn_saved_bytes(M, D, F, "bf16"), dtype=torch.uint8, device="cuda")
    out = b.op_gated_ffn(x, w_in, w_out, saved=saved)
    got = b.op_gated_ffn_backward(dy, x, w_in, w_out, saved)
    ref = u.ffn_reference(x[-9:], w_in, w_out, "silu", dy[-9:])
    u.check(out[-9:], ref[0], "far out")
    u.check(got[0][-9:], ref[1], "far dx")
    u.check(got[1], ref[2], "far dw_in")
    u.check(got[2], ref[3], "far dw_out")
    assert not got[0][:-9].any()


# ---- together, streams, graphs -------------------------------------------------------------------------------------------
def test_no_rows():
    import torch
    from paper_2511_20390_amd import binding as b
    x = torch.empty(0, 64, device="cuda")
    assert b.op_layer_norm(x).shape == (0, 64)
    dx, dw, db = b.op_layer_norm_backward(x, x, out=(x, torch.ones(64, device="cuda"), torch.ones(64, device="cuda")))
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    assert b.op_rope_axes(x, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), 1, 64, [64]).shape == (0, 64)
    for dt in (torch.float32, torch.bfloat16):
        e, w_in, w_out = x.to(dt), torch.ones(96, 64, dtype=dt, device="cuda"), torch.ones(64, 48, dtype=dt, device="cuda")
        saved = torch.empty(512, dtype=torch.uint8, device="cuda")
        assert b.op_gated_ffn(e, w_in, w_out, saved=saved).shape == (0, 64)
        dx, dw_in, dw_out = b.op_gated_ffn_backward(e, e, w_in, w_out, saved, out=(e, w_in.clone(), w_out.clone()))
        assert dx.shape == (0, 64) and not dw_in.any() and not dw_out.any()


class _Block:
    """One pre-norm block on B states of 8 x 8 tokens: layer norm, QKV layer, rotary positions, attention, output layer, layer norm, gated
    feed-forward, and the gradient of its second half."""

    def __init__(self, mode, B=2, heads=4, dh=64, F=512, seed=0):
        import torch
        from paper_2511_20390_amd import binding as b
        g = _gen(20, seed)
        self.mode, self.B, self.N, self.heads, self.dh = mode, B, 64, heads, dh
        D = heads * dh
        self.dt = dt = _t(mode)
        self.x = _rnd(g, B * 64, D)
        self.w = dict(n1=_rnd(g, D, std=0.1) + 1, b1=_rnd(g, D, std=0.1), n2=_rnd(g, D, std=0.1) + 1, b2=_rnd(g, D, std=0.1),
                      qkv=_rnd(g, 3 * D, D, std=D ** -0.5, dtype=dt), qkv_b=_rnd(g, 3 * D, std=0.1), proj=_rnd(g, D, D, std=D ** -0.5, dtype=dt),
                      proj_b=_rnd(g, D, std=0.1), w_in=_rnd(g, 2 * F, D, std=D ** -0.5, dtype=dt), w_out=_rnd(g, D, F, std=F ** -0.5, dtype=dt))
        self.gate = torch.ones(1, D, device="cuda")
        self.pos = torch.stack(torch.meshgrid(torch.arange(8, device="cuda"), torch.arange(8, device="cuda"), indexing="ij"), -1).view(64, 2).int()
        self.dy = _rnd(g, B * 64, D, dtype=dt)
        self.saved = torch.empty(b.gated_ffn_saved_bytes(B * 64, D, F, mode), dtype=torch.uint8, device="cuda")
        self.ws = torch.empty(b.gated_ffn_workspace_bytes(B * 64, D, F, mode, True), dtype=torch.uint8, device="cuda")
        self.nws = torch.empty(b.layer_norm_backward_workspace_bytes(B * 64, D), dtype=torch.uint8, device="cuda")

    def run(self):
        from paper_2511_20390_amd import binding as b
        w, D = self.w, self.heads * self.dh
        resid = self.x.clone()
        qkv = b.op_linear(b.op_layer_norm(resid, w["n1"], w["b1"], self.mode), w["qkv"], w["qkv_b"], self.mode)
        b.op_rope_axes(qkv[:, :2 * D], self.pos, 2 * self.heads, self.dh, [32, 32], out=qkv[:, :2 * D])
        att = b.op_attention(qkv, self.B, self.N, self.heads, self.dh, self.mode)
        b.op_linear(att, w["proj"], w["proj_b"], self.mode, b.EPI_GATE_RESID, resid=resid, gate=self.gate, rows_per_sample=resid.shape[0])
        n = b.op_layer_norm(resid, w["n2"], w["b2"], self.mode)
        out = b.op_gated_ffn(n, w["w_in"], w["w_out"], "silu", saved=self.saved, workspace=self.ws)
        dn, dw_in, dw_out = b.op_gated_ffn_backward(self.dy, n, w["w_in"], w["w_out"], self.saved, "silu", workspace=self.ws)
        dr, dn2, db2 = b.op_layer_norm_backward(dn, resid, w["n2"], workspace=self.nws)
        return [resid, out, dw_in, dw_out, dr, dn2, db2]

    def reference(self):
        """The same with torch in 64 bits, gradients by its own differentiation."""
        import torch
        w = {k: v.double() for k, v in self.w.items()}
        D, H, dh = self.heads * self.dh, self.heads, self.dh
        norm = lambda v, a, c: torch.nn.functional.layer_norm(v, (D,), a, c, 1e-6)
        x = self.x.double()
        qkv = (norm(x, w["n1"], w["b1"]) @ w["qkv"].T + w["qkv_b"]).view(self.B, 64, 3, H, dh)
        inv = 10000.0 ** (-torch.arange(0, 32, 2, device="cuda").double() / 32)
        angle = (self.pos.double()[:, :, None] * inv).flatten(1)[:, None]                         # [64, 1, 32]: both sections' pairs
        turn = lambda v: torch.stack([v[..., 0::2] * angle.cos() - v[..., 1::2] * angle.sin(),
                                      v[..., 0::2] * angle.sin() + v[..., 1::2] * angle.cos()], -1).flatten(-2)
        q, k, v = turn(qkv[:, :, 0]), turn(qkv[:, :, 1]), qkv[:, :, 2]
        p = torch.softmax((q[:, :, None] * k[:, None]).sum(-1) / dh ** 0.5, dim=2)                # [B, q, k, H]
        att = (p[..., None] * v[:, None]).sum(2).reshape(-1, D)
        resid = (x + att @ w["proj"].T + w["proj_b"]).requires_grad_(True)
        for name in ("n2", "b2", "w_in", "w_out"):
            w[name].requires_grad_(True)
        n = norm(resid, w["n2"], w["b2"])
        gu = n @ w["w_in"].T
        F = gu.shape[1] // 2
        out = (torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]) @ w["w_out"].T
        out.backward(self.dy.double())
        return [t.detach() for t in (resid, out, w["w_in"].grad, w["w_out"].grad, resid.grad, w["n2"].grad[None], w["b2"].grad[None])]


@pytest.mark.parametrize("mode", ["fp32", "bf16"])
def test_block(mode):
    from tests import block_ops_util as u
    import torch
    block = _Block(mode)
    # bf16: up to ten tensors on the way to a gradient are rounded, each 2^-8 / sqrt(3) of itself at most and independent, carried on with
    # a gain of about one: sqrt(10 / 3) 2^-8, doubled.  fp32: ten products of 2e-5 at most, as for the linear layers
    tol = 2 * (10 / 3) ** 0.5 * 2.0 ** -8 if mode == "bf16" else 1e-4
    for got, ref, name in zip(block.run(), block.reference(), ("resid", "out", "dw_in", "dw_out", "dresid", "dn2", "db2")):
        rel = ((got.double() - ref).norm() / ref.norm()).item()
        assert rel < tol, (name, rel)


@pytest.mark.parametrize("mode", ["fp32", "bf16"])
def test_block_in_a_graph(mode):
    """Captured and replayed, with eager runs and other inputs in between; every replay equals the eager result on its inputs."""
    import torch
    block, other = _Block(mode), _Block(mode, seed=1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block.run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = block.run()
    for k in range(4):
        block.x.copy_(_rnd(_gen(30, k), *block.x.shape))
        block.dy.copy_(_rnd(_gen(31, k), *block.dy.shape))
        other.run()
        graph.replay()
        got = [t.clone() for t in held]
        torch.cuda.synchronize()
        for a, e in zip(got, block.run()):
            assert torch.equal(a, e), k


def test_two_streams_at_once():
    """Calls in flight on two streams, each with buffers of its own."""
    import torch
    blocks = [_Block("bf16", B=8, F=1024, seed=k) for k in range(2)]
    refs = [k.run() for k in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    got = []
    for _ in range(3):
        for block, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                got.append(block.run())
    torch.cuda.synchronize()
    for k, r in enumerate(got):
        for a, e in zip(r, refs[k % 2]):
            assert torch.equal(a, e)


def test_on_a_side_stream():
    """Calls go to the stream that is current when they are made."""
    import torch
    block = _Block("bf16")
    ref = block.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = block.run()
    s.synchronize()
    for a, e in zip(got, ref):
        assert torch.equal(a, e)
