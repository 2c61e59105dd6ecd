"""The operators of a transformer step from their definitions, in 64 bits row by row and
head by head; no code shared with the library.  Next to every result stands the bound that rounding
gives an implementation which holds its sums in fp32, rounds intermediate matrix operands to the
inputs' type and its results once (`u`: unit roundoff of that type).

    E = 2^-24 is fp32's unit roundoff; a sum of n terms formed in fp32 in any order is off by at
    most (n - 1) E times the sum of the terms' magnitudes.
"""
from __future__ import annotations

import math

import torch

E = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F = torch.float64


def qk_norm_rope(x, w, cos, sin, positions, eps, dy=None):
    """One of q, k: (y, bound) and, with dy, (dx, bound, dw, bound)."""
    u = U[x.dtype]
    x, w = x.to(F), w.to(F)
    T, H, D = x.shape
    half = D // 2
    c, s = cos.to(F)[positions.long()][:, None, :], sin.to(F)[positions.long()][:, None, :]
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * r
    t = n * w
    t1, t2 = t[..., :half], t[..., half:]
    y = torch.cat((t1 * c - t2 * s, t2 * c + t1 * s), -1)
    size = torch.cat((t1.abs() * c.abs() + t2.abs() * s.abs(), t2.abs() * c.abs() + t1.abs() * s.abs()), -1)
    # r: the mean's D roundings (halved by the root), root, then three products and a sum an element
    rel_r = (D / 2 + 4) * E
    out = [y, u * y.abs() + (rel_r + 6 * E) * size * 1.01]
    if dy is None:
        return out
    dy = dy.to(F)
    g1, g2 = dy[..., :half], dy[..., half:]
    du = torch.cat((g1 * c + g2 * s, g2 * c - g1 * s), -1)
    du_size = torch.cat((g1.abs() * c.abs() + g2.abs() * s.abs(), g2.abs() * c.abs() + g1.abs() * s.abs()), -1)
    dn = du * w
    dn_size = du_size * w.abs()
    back = (dn * n).mean(-1, keepdim=True)
    back_size = (dn_size * n.abs()).mean(-1, keepdim=True)
    dx = r * (dn - n * back)
    dx_size = r * (dn_size + n.abs() * back_size)
    dw, dw_size = (du * n).sum((0, 1)), (du_size * n.abs()).sum((0, 1))
    out += [dx, u * dx.abs() + (4 * rel_r + (D + 12) * E) * dx_size * 1.01]
    out += [dw, u * dw.abs() + (rel_r + (T * H + 8) * E) * dw_size * 1.01]
    return out


def attention(q, k, v, cu, scale, dout=None):
    """dict of out, lse and, with dout, dq, dk, dv: (value, bound)."""
    u = U[q.dtype]
    q, k, v = q.to(F), k.to(F), v.to(F)
    T, H, D = q.shape
    Hk = k.shape[1]
    out, ob = (torch.zeros(T, H, D, dtype=F, device=q.device) for _ in range(2))
    lse, lb = torch.full((H, T), -math.inf, dtype=F, device=q.device), torch.zeros(H, T, dtype=F, device=q.device)
    grads = {}
    if dout is not None:
        dout = dout.to(F)
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            grads[name] = [torch.zeros_like(like), torch.zeros_like(like)]
    for a, b in zip(cu[:-1], cu[1:]):
        n = b - a
        if n <= 0:
            continue
        for h in range(H):
            g = h // (H // Hk)
            Q, K, V = q[a:b, h], k[a:b, g], v[a:b, g]
            later = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1)
            s = scale * (Q @ K.t())
            # products of D terms, the scale folded into the exponential's base-2 argument
            s_err = ((D + 6) * E * scale * (Q.abs() @ K.abs().t())).masked_fill(later, 0).amax(1, keepdim=True) + \
                8 * E * s.abs().masked_fill(later, 0).amax(1, keepdim=True)
            s = s.masked_fill(later, -math.inf)
            L = torch.logsumexp(s, 1, keepdim=True)
            p = torch.exp(s - L)
            rel_p = 2 * s_err + (2 * n + 16) * E        # numerator and normaliser
            lse[h, a:b] = L[:, 0]
            lb[h, a:b] = (s_err + (n + 16) * E + 4 * E * L.abs())[:, 0]
            o = p @ V
            o_size = p @ V.abs()
            out[a:b, h] = o
            ob[a:b, h] = (u + rel_p + (n + 4) * E) * o_size * 1.01 + u * o.abs()
            if dout is None:
                continue
            do = dout[a:b, h]
            dv, dv_size = p.t() @ do, p.t() @ do.abs()
            dv_err = (u + (n + 4) * E) * dv_size + (p * (rel_p + 4 * E * L.abs())).t() @ do.abs()
            dp, dp_size = do @ V.t(), do.abs() @ V.abs().t()
            delta = (do * o).sum(1, keepdim=True)
            d_err = (D + 4) * E * (dp_size + (do.abs() * o_size).sum(1, keepdim=True)) + \
                (do.abs() * ob[a:b, h]).sum(1, keepdim=True)
            ds = p * (dp - delta)
            ds_err = u * ds.abs() + p * d_err + (rel_p + 4 * E * L.abs() + 4 * E) * ds.abs()
            grads["dq"][0][a:b, h] = scale * (ds @ K)
            grads["dq"][1][a:b, h] = scale * (ds_err @ K.abs() + (n + 4) * E * (ds.abs() @ K.abs())) * 1.01
            grads["dk"][0][a:b, g] += scale * (ds.t() @ Q)
            grads["dk"][1][a:b, g] += scale * (ds_err.t() @ Q.abs() + (n * (H // Hk) + 4) * E * (ds.abs().t() @ Q.abs())) * 1.01
            grads["dv"][0][a:b, g] += dv
            grads["dv"][1][a:b, g] += dv_err * 1.01 + (n * (H // Hk)) * E * dv_size
    for name in grads:
        grads[name][1] += u * grads[name][0].abs()
    return {"out": (out, ob), "lse": (lse, lb), **{n: tuple(t) for n, t in grads.items()}}


def cross_entropy(x, w, target, dloss=None):
    """dict of loss, lse and, with dloss, dx, dw: (value, bound).  Targets lie in the vocabulary or
    are negative."""
    u = U[x.dtype]
    x, w = x.to(F), w.to(F)
    rows, d = x.shape
    V = w.shape[0]
    logits = x @ w.t()
    l_err = ((d + 2) * E * (x.abs() @ w.abs().t())).amax(1)
    lse = torch.logsumexp(logits, 1)
    # a sum of V exponentials, at most 2^-22 off each relative to arguments of the row's size
    s_err = l_err + (V + 16) * E + 8 * E * logits.abs().amax(1) + 4 * E * lse.abs()
    counted = target >= 0
    at = torch.where(counted, target, 0)
    each = torch.arange(rows, device=x.device)
    right = logits[each, at]
    zero = torch.zeros(rows, dtype=F, device=x.device)
    result = {"loss": (torch.where(counted, lse - right, zero),
                       torch.where(counted, s_err + l_err + 2 * E * (lse - right).abs(), zero)),
              "lse": (lse, s_err)}
    if dloss is None:
        return result
    p = torch.exp(logits - lse[:, None])
    one = torch.zeros_like(p)
    one[each, at] = 1.0
    g = torch.where(counted, dloss.to(F), zero)[:, None]
    dl = g * (p - one)
    dl_err = u * dl.abs() + g.abs() * (p * (s_err + l_err)[:, None] + 2 * E * (p + one))
    dx, dw = dl @ w, dl.t() @ x
    result["dx"] = (dx, (dl_err @ w.abs() + (V + 8) * E * (dl.abs() @ w.abs())) * 1.01 + u * dx.abs())
    result["dw"] = (dw, (dl_err.t() @ x.abs() + (rows + 8) * E * (dl.abs().t() @ x.abs())) * 1.01 + u * dw.abs())
    return result
