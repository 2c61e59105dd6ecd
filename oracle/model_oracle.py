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


# additions one after the other in a sum over a row: 16 values a lane, 6 steps inside a wavefront, 16 wavefronts
ROW = 38


def layer_norm(s, w, b, eps, dy=None, ds=None):
    """The norm of the stored rows s: dict of y, mean, r and, with dy, dx, dw, db: (value, bound)."""
    u = U[s.dtype]
    s, w = s.to(F), w.to(F)
    rows, d = s.shape
    depth = min(d, ROW) + 2
    m = s.mean(1, keepdim=True)
    # the mean is formed in 64 bits, up to 42 roundings one after the other, and used to 48 bits; it is rounded once to fp32
    # where it is stored, for the backward pass
    m_err = 2.0 ** -47 * s.abs().mean(1, keepdim=True)
    stored = m_err + E * m.abs()
    c = s - m
    var = c.square().mean(1, keepdim=True)
    r = (var + eps) ** -0.5
    # squares around a mean that is off by m_err are larger by its square; the root halves, and rounds itself
    rel_r = ((depth + 8) * E * var + m_err.square() + 2 * E * m_err * c.abs().mean(1, keepdim=True)) * r.square() / 2 + 4 * E
    n = c * r
    n_err = (m_err + 2 * E * c.abs()) * r + n.abs() * (rel_r + 2 * E)
    y = n * w + (0 if b is None else b.to(F))
    size = (n * w).abs() + (0 if b is None else b.to(F).abs())
    out = {"y": (y, (w.abs() * n_err + 3 * E * size) * 1.01 + u * y.abs()), "mean": (m[:, 0], stored[:, 0] * 1.01),
           "r": (r[:, 0], (rel_r * r)[:, 0])}
    if dy is None:
        return out
    n_err = (stored + E * (c.abs() + stored)) * r + n.abs() * (rel_r + 2 * E)
    dy = dy.to(F)
    dn = dy * w
    even, even_err = dn.mean(1, keepdim=True), (depth + 2) * E * dn.abs().mean(1, keepdim=True)
    along = (dn * n).mean(1, keepdim=True)
    along_err = (depth + 3) * E * (dn * n).abs().mean(1, keepdim=True) + (dn.abs() * n_err).mean(1, keepdim=True)
    inner = dn - even - n * along
    size = dn.abs() + even.abs() + (n * along).abs()
    dx = r * inner
    err = r * (even_err + n_err * along.abs() + n.abs() * along_err + 4 * E * size) + dx.abs() * rel_r
    if ds is not None:
        dx = dx + ds.to(F)
        err = err + 2 * E * ds.to(F).abs()
    out["dx"] = (dx, err * 1.01 + u * dx.abs())
    # rows one after the other: those of a group of lanes, of a workgroup's groups, of 64 slices of up to 512 workgroups
    deep = min(rows, rows // 512 + 16 + 8 + 64) + 4
    dw, db = (dy * n).sum(0), dy.sum(0)
    out["dw"] = (dw, (deep * E * (dy * n).abs().sum(0) + (dy.abs() * n_err).sum(0)) * 1.01 + u * dw.abs())
    out["db"] = (db, deep * E * dy.abs().sum(0) * 1.01 + u * db.abs())
    return out


def frequencies(part, base, scaling="none", factor=1.0, original=0.0, low=1.0, high=32.0):
    """Angles of one position, pair by pair."""
    out = []
    for i in range(part // 2):
        f = base ** (-2 * i / part)
        if scaling == "linear":
            f = f / factor
        if scaling == "base":
            f = (base * factor ** (part / (part - 2))) ** (-2 * i / part)
        if scaling == "parts":
            turns = original * f / (2 * math.pi)
            keep = 1.0 if turns >= high else 0.0 if turns <= low else (turns - low) / (high - low)
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return torch.tensor(out, dtype=F)


def rotary(x, cos, sin, positions, interleaved, back=False):
    """One of q, k: (y, bound); back: turned the other way, as its gradient is."""
    u = U[x.dtype]
    x = x.to(F)
    half = cos.shape[1]
    c, s = cos.to(F)[positions.long()][:, None, :], sin.to(F)[positions.long()][:, None, :]
    s = -s if back else s
    y, size = x.clone(), torch.zeros_like(x)
    at = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, b * c + a * s
    size[..., at[0]], size[..., at[1]] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    moved = size.abs() > 0
    return y, torch.where(moved, u * y.abs() + 2 * E * size, 0.0) * 1.01


def distillation(x, w, index, logits, tau, dloss=None, pieces=1):
    """dict of loss, lse, picked and, with dloss, dx, dw: (value, bound).  Words lie in the vocabulary or are negative.
    pieces: 2 where the gradients of logits are kept with what their first rounding leaves, rounded in turn."""
    u = U[x.dtype]
    x, w = x.to(F), w.to(F)
    rows, d = x.shape
    V, K = w.shape[0], index.shape[1]
    l = x @ w.t()
    l_err = ((d + 2) * E * (x.abs() @ w.abs().t())).amax(1, keepdim=True)
    lse = torch.logsumexp(l / tau, 1, keepdim=True)
    s_err = l_err / tau + (V + 16) * E + 10 * E * l.abs().amax(1, keepdim=True) / tau + 4 * E * lse.abs()
    used = (index >= 0) & (logits != -math.inf)
    counted = used.any(1, keepdim=True)
    at = torch.where(used, index, 0)
    picked = torch.where(used, l.gather(1, at), 0.0)
    t = torch.where(used, logits.to(F) / tau, -math.inf)
    t_top = torch.where(counted, t.amax(1, keepdim=True), 0.0)
    log_q = torch.where(used, t - torch.where(counted, torch.logsumexp(t, 1, keepdim=True), 0.0), 0.0)
    q = torch.where(used, log_q.exp(), 0.0)
    far = torch.where(used, t_top - t, 0.0)
    # distances in the exponent, exponentials and their sum
    q_err = 6 * E * far + 6 * E * (q * far).sum(1, keepdim=True) + (16 + 8) * E
    log_p = torch.where(used, picked / tau - lse, 0.0)
    term = torch.where(used, log_q - log_p, 0.0)
    term_err = q_err + l_err / tau + s_err + 6 * E * (log_q.abs() + log_p.abs())
    result = {"loss": ((q * term).sum(1), (q * (term_err + q_err * term.abs() + 16 * E * term.abs())).sum(1) * 1.01),
              "lse": (lse[:, 0], s_err[:, 0]), "picked": (picked, torch.where(used, l_err, 0.0))}
    if dloss is None:
        return result
    p = torch.exp(l / tau - lse)
    share, share_err = torch.zeros_like(p), torch.zeros_like(p)
    share.scatter_add_(1, at, q)
    share_err.scatter_add_(1, at, q * q_err)
    g = torch.where(counted[:, 0], dloss.to(F), 0.0)[:, None] / tau
    dl = g * (p - share)
    dl_err = u ** pieces * dl.abs() + g.abs() * (p * (s_err + l_err / tau) + share_err + 4 * E * (p + share))
    dx, dw = dl @ w, dl.t() @ x
    # (two pieces are two terms of a sum each)
    result["dx"] = (dx, (dl_err @ w.abs() + (pieces * V + 8) * E * (dl.abs() @ w.abs())) * 1.01 + u * dx.abs())
    result["dw"] = (dw, (dl_err.t() @ x.abs() + (pieces * rows + 8) * E * (dl.abs().t() @ x.abs())) * 1.01 + u * dw.abs())
    return result
