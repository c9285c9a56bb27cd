"""The operators of rotary, gated blocks in 64 bits, each with a bound on how far fp32 arithmetic with the stated roundings can be from
it, element by element."""
import math

import torch

U = 2.0 ** -24                       # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_within(got, ref, bound, what):
    """|got - ref| <= bound + the rounding to got's type, everywhere; NaN and infinities in the same places."""
    got, ref, bound = got.double(), ref.double(), bound.double()
    assert got.shape == ref.shape, what
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN elsewhere"
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)]), f"{what}: infinities elsewhere"
    over = ((got - ref).abs() - bound)[fine]
    if over.numel():
        assert over.max() <= 0, f"{what}: {over.max().item():.3g} over the bound, {(over > 0).sum().item()} of {over.numel()} values"


def norm_reference(x, weight, bias, rows, plus_one, eps, dout=None):
    """(out, bound), and with dout also (dx, bound), (dw, bound), (db, bound), without the rounding to the results' types."""
    x = x.double()
    M, D = x.shape
    dev = x.device
    sample = torch.arange(M, device=dev) // rows
    n = max(1, -(-M // rows))
    w = torch.ones(M, D, dtype=torch.float64, device=dev) if weight is None else weight.double().reshape(n, D)[sample] + (1.0 if plus_one else 0.0)
    b = torch.zeros(M, D, dtype=torch.float64, device=dev) if bias is None else bias.double().reshape(n, D)[sample]
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    r = 1.0 / torch.sqrt((xc * xc).mean(1, keepdim=True) + eps)
    xh = xc * r
    # A lane adds up to 32 values, then 64 lanes and 16 wavefronts are added: under 56 roundings in a chain; they and the products'
    # make the mean off by 64 U mean|x|, x - mean by U |x| more, and r by 64 U of itself.
    e_xh = 64 * U * ((x.abs().mean(1, keepdim=True) + x.abs()) * r + xh.abs())
    out, e_out = xh * w + b, e_xh * w.abs() + 4 * U * ((xh * w).abs() + b.abs())
    if dout is None:
        return (out, e_out)
    dy = dout.double()
    g = dy * w
    m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = r * (g - m1 - xh * m2)
    e_dx = r * (64 * U * (2 * g.abs() + 2 * g.abs().mean(1, keepdim=True) + 2 * xh.abs() * (g * xh).abs().mean(1, keepdim=True)) +
                xh.abs() * (g.abs() * e_xh).mean(1, keepdim=True) + e_xh * m2.abs())
    zero = lambda: torch.zeros(n, D, dtype=torch.float64, device=dev)
    dw, db = zero().index_add_(0, sample, dy * xh), zero().index_add_(0, sample, dy)
    # a chain of additions: the rows of a wavefront, four wavefronts, the partial rows of a thread, sixteen threads
    chain = 160 * U
    e_dw = chain * zero().index_add_(0, sample, (dy * xh).abs()) + zero().index_add_(0, sample, dy.abs() * e_xh)
    e_db = chain * zero().index_add_(0, sample, dy.abs())
    return (out, e_out), (dx, e_dx), (dw, e_dw), (db, e_db)


def rope_reference(x, pos, heads, dh, dims, theta, pairs, inverse):
    """(out, bound) without the rounding to the result's type."""
    rows = x.shape[0]
    v = x.double().reshape(rows, heads, dh).clone()
    e = torch.zeros_like(v)
    at = 0
    where = torch.arange(rows, device=x.device) % pos.shape[0]
    for a, d in enumerate(dims):
        for i in range(d // 2):
            p, q = (at + 2 * i, at + 2 * i + 1) if pairs else (at + i, at + i + d // 2)
            angle = pos[where, a].double() * (theta ** (-2.0 * i / d)) * (-1.0 if inverse else 1.0)
            c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
            u, w = v[:, :, p].clone(), v[:, :, q].clone()
            v[:, :, p], v[:, :, q] = u * c - w * s, u * s + w * c
            # angle: half a step of a value up to pi, 2^-32 turns, and the reference's own 2^-53 of the angle; sine and cosine two steps;
            # two products and a sum
            e[:, :, p] = e[:, :, q] = (u.abs() + w.abs()) * (10 * U + 2.0 ** -51 * angle.abs()[:, None])
        at += d
    return v.reshape(rows, -1), e.reshape(rows, -1)


def _act(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    k, c = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(k * (g + c * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * c * g * g)


def ffn_reference(x, w_in, w_out, act, dout=None):
    """[(out, bound)], and with dout also of dx, dw_in, dw_out, without the rounding to the results' type."""
    half = half_step(x.dtype) if x.dtype != torch.float32 else U
    x, w_in, w_out = x.double(), w_in.double(), w_out.double()
    M, D = x.shape
    F = w_out.shape[1]
    # a sum of n products: n roundings of U at most, each of at most the sum of the absolute values
    total = lambda n: (n + 8) * U
    gu, e_gu = x @ w_in.T, total(D) * (x.abs() @ w_in.abs().T)
    g, u, e_g, e_u = gu[:, :F], gu[:, F:], e_gu[:, :F], e_gu[:, F:]
    a, da = _act(g, act)
    h = a * u
    # both activations have slopes below 1.13 and second derivatives below 1.2; the functions themselves: 16 U of a value and of |g|,
    # from the exponential's argument
    e_a, e_da = 1.2 * e_g + 16 * U * (a.abs() + g.abs() * U), 1.2 * e_g + 32 * U * (1 + da.abs())
    e_h = e_a * u.abs() + a.abs() * e_u + e_a * e_u + half * h.abs() + 2.0 ** -126
    res = [(h @ w_out.T, (1 + total(F)) * (e_h @ w_out.abs().T) + total(F) * (h.abs() @ w_out.abs().T))]
    if dout is None:
        return res
    dy = dout.double()
    dh, e_dh = dy @ w_out, total(D) * (dy.abs() @ w_out.abs())
    du, dg = dh * a, dh * u * da
    e_du = e_dh * a.abs() + dh.abs() * e_a + e_dh * e_a
    e_dg = (e_dh * u.abs() + dh.abs() * e_u + e_dh * e_u) * (da.abs() + e_da) + dh.abs() * u.abs() * e_da
    d = torch.cat([dg, du], 1)
    e_d = (1 + half) * torch.cat([e_dg, e_du], 1) + (half + 4 * U) * d.abs() + 2.0 ** -126
    res.append((d @ w_in, (1 + total(2 * F)) * (e_d @ w_in.abs()) + total(2 * F) * (d.abs() @ w_in.abs())))
    res.append((d.T @ x, (1 + total(M)) * (e_d.T @ x.abs()) + total(M) * (d.abs().T @ x.abs())))
    res.append((dy.T @ h, (1 + total(M)) * (dy.abs().T @ e_h) + total(M) * (dy.abs().T @ h.abs())))
    return res


def check(got, ref_bound, what):
    """got (rounded to its type) against (reference, bound)."""
    ref, bound = ref_bound
    assert_within(got, ref, bound + half_step(got.dtype) * (ref.abs() + bound) + 2.0 ** -126, what)
