"""Plain 64-bit forms of the router, its losses and gradients and the experts' 4-bit products (tests only)."""
import math

import torch


def scores(x, score):
    """x float64 [..., E] -> scores, normaliser and availability."""
    ok = x > -math.inf
    if score == "sigmoid":
        p = torch.sigmoid(x)
        return p, p.sum(-1), ok
    live = ok.any(-1, keepdim=True)      # from differences to the largest: the lowest value of a type is a logit as any other
    p = torch.softmax(torch.where(live, x, torch.zeros_like(x)), -1)
    return torch.where(live, p, torch.zeros_like(p)), torch.logsumexp(x, -1), ok


def select(x, k, score, bias=None):
    """ids [..., k] (-1 where none is left) by the stable descending order of the logits, or of score + bias."""
    p, _, ok = scores(x, score)
    key = x if bias is None else torch.where(ok, p + bias, torch.full_like(x, -math.inf))
    value, at = torch.sort(key, dim=-1, descending=True, stable=True)
    return torch.where(value[..., :k] > -math.inf, at[..., :k], torch.full_like(at[..., :k], -1))


def gates(x, ids, score, renorm, scale):
    p, _, _ = scores(x, score)
    have = ids >= 0
    g = torch.where(have, p.gather(-1, ids.clamp_min(0)), torch.zeros((), dtype=x.dtype))
    if renorm:
        if score == "softmax":  # the softmax over the selected alone: also where their scores are too small to be held
            y = torch.where(have, x.gather(-1, ids.clamp_min(0)), torch.full((), -math.inf, dtype=x.dtype))
            g = torch.where(have, torch.softmax(torch.where(have[..., :1], y, torch.zeros_like(y)), -1), 0.0)
        else:
            total = g.sum(-1, keepdim=True)
            g = g / torch.where(total > 0, total, torch.ones_like(total))
    return scale * g


def losses(x, ids, off, score):
    """D, tokens [F][L], balance, z of x [L][N][E] (differentiable; the selection is constant)."""
    L, N, E = x.shape
    k, F = ids.shape[2], len(off) - 1
    p, norm, ok = scores(x, score)
    live = ok.any(-1)
    share = p if score == "softmax" else p / torch.where(norm > 0, norm, torch.ones_like(norm)).unsqueeze(-1)
    D = torch.zeros((F, L, E), dtype=torch.int64)
    tokens = torch.zeros((F, L), dtype=torch.int64)
    balance, z = [], []
    for f in range(F):
        for l in range(L):
            a, b = int(off[f]), int(off[f + 1])
            keep = live[l, a:b]
            T = int(keep.sum())
            sel = ids[l, a:b]
            count = torch.bincount(sel[sel >= 0].flatten(), minlength=E)
            D[f, l] = count
            tokens[f, l] = T
            if T == 0:
                balance.append(torch.zeros((), dtype=x.dtype))
                z.append(torch.zeros((), dtype=x.dtype))
                continue
            balance.append((count * share[l, a:b][keep].sum(0)).sum() * E / (k * T * T))
            z.append((norm[l, a:b][keep] ** 2).sum() / T)
    return D, tokens, torch.stack(balance).reshape(F, L), torch.stack(z).reshape(F, L)


def total(x, ids, off, score, renorm, scale, gg=None, gb=None, gz=None):
    """The number whose gradient tacg_route_backward returns."""
    out = torch.zeros((), dtype=x.dtype)
    if gg is not None:
        out = out + (torch.where(ids >= 0, gg, torch.zeros_like(gg)) * gates(x, ids, score, renorm, scale)).sum()
    if gb is not None or gz is not None:
        _, _, b, z = losses(x, ids, off, score)
        if gb is not None:
            out = out + (gb * b).sum()
        if gz is not None:
            out = out + (gz * z).sum()
    return out


def gradient(x, ids, off, score, renorm, scale, gg=None, gb=None, gz=None):
    """The gradient by its formula, and the sum of its terms' magnitudes (what rounding errors go by)."""
    L, N, E = x.shape
    k = ids.shape[2]
    p, norm, ok = scores(x, score)
    live = ok.any(-1)
    D, tokens, _, _ = losses(x, ids, off, score)
    c = torch.zeros_like(x)
    zc = torch.zeros((L, N), dtype=x.dtype)
    for f in range(len(off) - 1):
        a, b = int(off[f]), int(off[f + 1])
        for l in range(L):
            T = max(int(tokens[f, l]), 1)
            if gb is not None:
                c[l, a:b] = gb[f, l] * E / (k * T * T) * D[f, l]
            if gz is not None:
                zc[l, a:b] = gz[f, l] * 2 / T
    have = ids >= 0
    at = ids.clamp_min(0)
    ps = torch.where(have, p.gather(2, at), torch.zeros((), dtype=x.dtype))
    u = torch.zeros_like(ps) if gg is None else torch.where(have, gg, torch.zeros_like(gg))
    if renorm:
        w = gates(x, ids, score, True, 1.0)
        mean = (w * u).sum(2, keepdim=True)
        if score == "softmax":
            straight, su_abs = scale * w * (u - mean), scale * w * (u.abs() + (w * u.abs()).sum(2, keepdim=True))
            u, u_abs = torch.zeros_like(u), torch.zeros_like(u)
        else:
            inner = ps.sum(2, keepdim=True)
            inner = torch.where(inner > 0, inner, torch.ones_like(inner))
            straight, su_abs = torch.zeros_like(u), torch.zeros_like(u)
            u, u_abs = have.to(x.dtype) * scale / inner * (u - mean), have.to(x.dtype) * scale / inner * (u.abs() + mean.abs())
    else:
        straight, su_abs = torch.zeros_like(u), torch.zeros_like(u)
        u, u_abs = scale * u, scale * u.abs()
    spread = lambda v: torch.zeros_like(x).scatter_add(2, at, torch.where(have, v, torch.zeros_like(v)))  # noqa: E731
    U, U_abs, S, S_abs = spread(u), spread(u_abs), spread(straight), spread(su_abs)
    if score == "softmax":
        nz = torch.where(live, zc * torch.where(live, norm, 0.0), torch.zeros_like(zc)).unsqueeze(-1)
        d = c + U
        g = p * (d - (p * d).sum(-1, keepdim=True) + nz) + S
        mag = p * (c.abs() + U_abs + (p * (c.abs() + U_abs)).sum(-1, keepdim=True) + nz.abs()) + S_abs
    else:
        n = torch.where(norm > 0, norm, torch.ones_like(norm)).unsqueeze(-1)
        n = torch.where(norm.unsqueeze(-1) > 0, n, torch.full_like(n, math.inf))
        g = p * (1 - p) * ((c - (p * c).sum(-1, keepdim=True) / n) / n + U)
        mag = p * ((c.abs() + (p * c.abs()).sum(-1, keepdim=True) / n) / n + U_abs)
    return g, mag


def dequantise(q, scales, zeros, K, group):
    """Weights [H][N][K] in float64, column by column."""
    c = torch.arange(K, device=q.device)
    byte = q[:, :, c // 2]
    level = torch.where(c % 2 == 1, byte >> 4, byte & 15).double()
    zero = 8.0 if zeros is None else zeros[:, :, c // group].double()
    return (level - zero) * scales[:, :, c // group].double()


def products(x, ids, q, scales, zeros, group, mode, slot=None, gate=None):
    """The products and a bound of what their 32-bit sums may be off, both float64."""
    T, k = ids.shape
    K, (H, N) = x.shape[-1], q.shape[:2]
    w = dequantise(q, scales, zeros, K, group)
    wide = scales.double().repeat_interleave(group, 2)[:, :, :K]
    y = torch.zeros((T, k, N), dtype=torch.float64, device=x.device)
    off = torch.zeros_like(y)
    for t in range(T):
        for j in range(k):
            e = int(ids[t, j])
            h = -1 if e < 0 else e if slot is None else int(slot[e])
            if not 0 <= h < H:
                continue
            v = (x[t, j] if x.dim() == 3 else x[t]).double()
            y[t, j] = w[h] @ v
            # a level may be held with an offset of up to 128 + 8: sixteen roundings of a sum of such terms
            off[t, j] = 16 * 2.0 ** -24 * 151 * (wide[h].abs() @ v.abs())
    if mode == "glu":
        a, b = y[..., :N // 2], y[..., N // 2:]
        da, db = off[..., :N // 2], off[..., N // 2:]
        s = a * torch.sigmoid(a)
        return s * b, 1.1 * da * b.abs() + s.abs() * db + 1.1 * da * db + 2.0 ** -20 * (s * b).abs()
    if mode == "sum":
        g = gate.double().unsqueeze(-1)
        return (g * y).sum(1), (g.abs() * off).sum(1) + 16 * 2.0 ** -24 * (g * y).abs().sum(1)
    return y, off
