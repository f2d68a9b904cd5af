"""Plain 64-bit statements (CPU, float64) of the RMS norm, rows in 8 bits, activations, dense
products and routing by scores, with the magnitudes their rounding errors are measured against
(rows_ref.py has the other operators' and the conventions).
"""
import math

import numpy as np
import torch

TOP, LEAST = 448.0, 2.0 ** -100      # the largest e4m3 number; the least a scale is made for
F8 = torch.float8_e4m3fn
A, B = 2 * math.sqrt(2 / math.pi), 0.044715


def packed(x):
    """(q, scale) of fp32 or bf16 rows, bit for bit: two fp32 roundings and one to e4m3."""
    x = x.float()
    top = x.abs().amax(1, keepdim=True)
    fine = top < math.inf            # (false for NaN)
    top = torch.where(fine, top, torch.ones(())).clamp(min=LEAST)
    q = torch.where(fine, x * (torch.tensor(TOP) / top), torch.zeros(())).to(F8)
    scale = torch.where(fine, top / torch.tensor(TOP), torch.full((), math.nan))
    return q, scale.reshape(-1)


def stands_for(q, scale):
    return q.double() * scale.double()[:, None]


def act(z, kind):
    if kind == "relu":
        return torch.where(z < 0, torch.zeros((), dtype=z.dtype), z)
    if kind == "gelu":
        return z * torch.sigmoid(A * (z + B * z ** 3))
    if kind == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, kind):
    if kind == "relu":
        return torch.where(z <= 0, torch.zeros((), dtype=z.dtype), torch.ones((), dtype=z.dtype))
    if kind == "gelu":
        s = torch.sigmoid(A * (z + B * z ** 3))
        return s + z * s * torch.sigmoid(-A * (z + B * z ** 3)) * A * (1 + 3 * B * z ** 2)
    if kind == "silu":
        s = torch.sigmoid(z)
        return s + z * s * torch.sigmoid(-z)
    return torch.ones_like(z)


def rms(h, gamma, eps):
    """y, rstd"""
    rstd = 1.0 / torch.sqrt((h * h).sum(1) / h.shape[1] + eps)
    y = h * rstd[:, None]
    return y if gamma is None else y * gamma, rstd


def rms_grad(dy, h, rstd, gamma, dh):
    """(dx, dgamma) and their magnitudes, for the rstd given"""
    C, z = h.shape[1], h * rstd[:, None]
    g = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (g - z * (g * z).sum(1, keepdim=True) / C)
    mag = rstd[:, None] * (g.abs() + z.abs() * (g * z).abs().sum(1, keepdim=True) / C)
    if dh is not None:
        dx, mag = dx + dh, mag + dh.abs()
    return (dx, (dy * z).sum(0)), (mag, (dy * z).abs().sum(0))


def linear(x, w, bias):
    """z, its magnitude"""
    z, mag = x @ w, x.abs() @ w.abs()
    return (z, mag) if bias is None else (z + bias, mag + bias.abs())


def scores(logits, kind):
    """float64 [n, E]; 0 for a row that is all closed"""
    x = logits.double()
    if kind == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    top = x.max(1, keepdim=True).values
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(1, keepdim=True)
    return torch.where(total == 0, torch.zeros_like(e), e / total)


def _above(p, i, q, j):
    """Whether score p of place i goes before q of place j: NaN is the largest, ties by place."""
    pn, qn = math.isnan(p), math.isnan(q)
    if pn or qn:
        return pn and (not qn or i < j)
    return p > q or (p == q and i < j)


def choose(logits, bias, kind, groups, top_groups, k):
    """experts [n, k] (-1 for none), one comparison at a time"""
    x, s = logits.double(), scores(logits, kind)
    v = s if bias is None else s + bias.double()
    v = torch.where(x == -math.inf, torch.full_like(v, -math.inf), v).numpy()
    n, E = v.shape
    per, out = E // groups, np.full((n, k), -1, np.int64)

    def best(values, places, count):
        left, got = list(places), []
        while left and len(got) < count:
            m = left[0]
            for p in left[1:]:
                if _above(values[p], p, values[m], m):
                    m = p
            left.remove(m)
            if values[m] == -math.inf:
                break
            got.append(m)
        return got
    for r in range(n):
        open_ = range(E)
        if groups > 1:
            worth = []
            for g in range(groups):
                two = best(v[r], range(g * per, (g + 1) * per), 2)
                worth.append(sum(v[r][e] for e in two) if two else -math.inf)
            stay = best(worth, range(groups), top_groups)
            open_ = [e for g in sorted(stay) for e in range(g * per, (g + 1) * per)]
        got = best(v[r], open_, k)
        out[r, :len(got)] = got
    return torch.from_numpy(out)


def weights(logits, experts, kind, normalize, scale):
    s, some = scores(logits, kind), experts >= 0
    w = torch.where(some, s.gather(1, experts.clamp(min=0)), torch.zeros((), dtype=torch.float64))
    if normalize:
        total = w.sum(1, keepdim=True)
        w = torch.where(total == 0, torch.zeros_like(w), w / total)
    return w * scale


def weights_grad(logits, experts, kind, normalize, scale, dw):
    """dlogits and its magnitude, through the scores"""
    s, some = scores(logits, kind), experts >= 0
    e = experts.clamp(min=0)
    zero = torch.zeros((), dtype=torch.float64)
    c = torch.where(some, s.gather(1, e), zero)
    d = torch.where(some, dw * scale, zero)
    mag = d.abs()
    if normalize:
        total = c.sum(1, keepdim=True)
        one = torch.where(total == 0, torch.ones_like(total), total)
        dead = total == 0
        mean, mm = (d * c / one).sum(1, keepdim=True), (mag * c / one).sum(1, keepdim=True)
        d = torch.where(dead, zero, (d - mean) / one)
        mag = torch.where(dead, zero, (mag + mm) / one)
        d, mag = torch.where(some, d, zero), torch.where(some, mag, zero)
    ds = torch.zeros_like(s).scatter_add_(1, e, d)
    dm = torch.zeros_like(s).scatter_add_(1, e, mag)
    if kind == "sigmoid":
        back = s * (1.0 / (1.0 + torch.exp(logits.double())))
        return ds * back, dm * back
    return (s * (ds - (ds * s).sum(1, keepdim=True)), s * (dm + (dm * s).sum(1, keepdim=True)))
