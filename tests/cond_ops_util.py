"""Cross attention and the projection with adapters in 64 bits, each with a bound on how far fp32 arithmetic with the stated roundings can be from
it, element by element."""
import math

import torch

from tests.block_ops_util import U, half_step


def _operand(dtype):
    """Half a step of the rounding of an operand of a product: none in fp32."""
    return half_step(dtype) if dtype != torch.float32 else 0.0


def cross_reference(q, k, v, B, heads, kv, dh, scale, keys, dout=None):
    """keys: bool [B, Nk].  [(out, bound), (lse, bound)], and with dout also of dq, dk, dv, without the rounding to the results' type.  Rows
    are [rows, heads * dh] as the operator has them."""
    h, kind = _operand(q.dtype), q.dtype
    group, Nk = heads // kv, k.shape[0] // B
    Nq = q.shape[0] // B
    first = lambda t, n: t.double().reshape(B, -1, n, dh).transpose(1, 2)
    rows = lambda t: t.transpose(1, 2).reshape(B * t.shape[2], -1)
    share = lambda t: t.repeat_interleave(group, dim=1)
    there = keys[:, None, None, :]
    # what stands in keys that do not count has no influence
    clean = lambda t: torch.where(keys[:, None, :, None], first(t, kv), torch.zeros((), dtype=torch.float64, device=t.device))
    Q, K, V = first(q, heads), share(clean(k)), share(clean(v))
    s = scale * (Q @ K.transpose(2, 3))
    e_s = scale * (dh + 8) * U * (Q.abs() @ K.abs().transpose(2, 3))
    s = torch.where(there, s, torch.full_like(s, -math.inf))
    some = keys.any(1)[:, None, None, None]
    lse = torch.where(some, torch.logsumexp(s, dim=3, keepdim=True), torch.zeros_like(s[..., :1]))
    p = torch.where(there & some, torch.exp(s - lse), torch.zeros_like(s))
    size = torch.where(there, s.abs(), torch.zeros_like(s)).amax(3, keepdim=True)
    # a probability's relative error: its score's, and the exponent's argument, rounded where it is formed; a maximum that moves multiplies the
    # sums by a factor of the same kind: at most once for every tile of 32 keys and every part (64), and for four wavefronts
    moves = (Nk + 31) // 32 + 70
    e_p = 1.1 * (e_s + 4 * U * (2 + 2 * size) * (1 + 0.05 * moves) + 4 * U)
    e_p = torch.where(there, e_p, torch.zeros_like(e_p))
    chain = lambda n: (n + 80) * U
    out = p @ V
    pv = p @ V.abs()
    e_l = (p * e_p).sum(3, keepdim=True) + chain(Nk)
    # A probability (before the division by a sum of at least one) or a score's gradient below the smallest normal number of fp32 and bf16 may count as
    # zero, as it does where an instruction flushes subnormal results or operands: it is off by itself, less than 2^-126.
    least = torch.where(there, torch.full_like(p, 2.0 ** -126), torch.zeros_like(p))
    e_out = (p * (h + (1 + h) * e_p) + least) @ V.abs() + pv * (e_l + h) + chain(Nk) * pv
    e_lse = torch.where(some, 1.1 * e_l + 8 * U * (lse.abs() + size + 1), torch.zeros_like(lse))
    res = [(rows(out), rows(e_out)), (torch.where(some, lse, torch.full_like(lse, -math.inf))[..., 0], e_lse[..., 0])]
    if dout is None:
        return res
    G = first(dout, heads)
    e_p = e_p + 1.1 * (e_lse + half_step(torch.float32) * lse.abs() + 4 * U * (size + lse.abs()))
    e_p = torch.where(there, e_p, torch.zeros_like(e_p))
    dp, e_dp = G @ V.transpose(2, 3), (dh + 8) * U * (G.abs() @ V.abs().transpose(2, 3))
    delta = (G * out).sum(3, keepdim=True)
    e_delta = (G.abs() * (e_out * (1 + half_step(kind)) + (half_step(kind) + (dh + 8) * U) * out.abs())).sum(3, keepdim=True)
    ds = p * (dp - delta)
    e_ds = (p * e_p) * (dp - delta).abs() + p * (1 + e_p) * (e_dp + e_delta + 2 * U * (dp.abs() + delta.abs()))
    e_ds = (1 + h) * e_ds + h * ds.abs() + least * (1 + (dp - delta).abs())
    dq, e_dq = scale * (ds @ K), scale * ((e_ds + chain(Nk) * (ds.abs() + e_ds)) @ K.abs())
    n = chain(Nq * group)
    by_key = lambda t: t.reshape(B, kv, group, Nk, dh).sum(2)
    T = lambda t: t.transpose(2, 3)
    dk, e_dk = scale * (T(ds) @ Q), scale * (T(e_ds + n * (ds.abs() + e_ds)) @ Q.abs())
    e_pr = p * (h + (1 + h) * e_p) + least
    dv, e_dv = T(p) @ G, T(e_pr + n * (p + e_pr)) @ G.abs()
    return res + [(rows(dq), rows(e_dq)), (rows(by_key(dk)), rows(by_key(e_dk))), (rows(by_key(dv)), rows(by_key(e_dv)))]


def keys_that_count(B, Nk, key_len, key_mask, device):
    keys = torch.ones(B, Nk, dtype=torch.bool, device=device)
    if key_len is not None:
        keys &= torch.arange(Nk, device=device)[None, :] < key_len[:, None]
    if key_mask is not None:
        keys &= key_mask != 0
    return keys


def adapters_reference(x, w, bias, a, b, adapter, scale, rows, dout=None):
    """[(out, bound)], and with dout also of dx, dA, dB, without the rounding to the results' type."""
    h = half_step(x.dtype) if x.dtype != torch.float32 else U
    x, w, a, b = x.double(), w.double(), a.double(), b.double()
    M, K = x.shape
    n, r, N = a.shape[0], a.shape[1], w.shape[0]
    s = torch.ones(n, dtype=torch.float64, device=x.device) if scale is None else scale.double()
    which = adapter.long()[torch.arange(M, device=x.device) // rows]
    total = lambda k: (k + 16) * U
    out, e_out = x @ w.T, total(K + r) * (x.abs() @ w.abs().T)
    if bias is not None:
        out, e_out = out + bias.double(), e_out + total(K + r) * bias.double().abs()
    if dout is not None:
        g = dout.double()
        dx, e_dx = g @ w, total(N + r) * (g.abs() @ w.abs())
        da, db, e_da, e_db = torch.zeros_like(a), torch.zeros_like(b), torch.zeros_like(a), torch.zeros_like(b)
    for i in range(n):
        at = (which == i).nonzero()[:, 0]
        if at.numel() == 0:
            continue
        # a sum, a factor, and the rounding to the operand's type
        thin = lambda v, m, k: (s[i] * (v @ m), s[i].abs() * (total(k) + h) * (1 + h) * (v.abs() @ m.abs()) + 2.0 ** -126)
        t, e_t = thin(x[at], a[i].T, K)
        out[at] += t @ b[i].T
        e_out[at] += (e_t + total(K + r) * (t.abs() + e_t)) @ b[i].abs().T
        if dout is None:
            continue
        u, e_u = thin(g[at], b[i], N)
        dx[at] += u @ a[i]
        e_dx[at] += (e_u + total(N + r) * (u.abs() + e_u)) @ a[i].abs()
        m = at.numel()
        da[i], e_da[i] = u.T @ x[at], (e_u + total(m + 64) * (u.abs() + e_u)).T @ x[at].abs()
        db[i], e_db[i] = g[at].T @ t, g[at].abs().T @ (e_t + total(m + 64) * (t.abs() + e_t))
    return [(out, e_out)] if dout is None else [(out, e_out), (dx, e_dx), (da, e_da), (db, e_db)]
