"""Plain 64-bit statements of the operators on feature rows (CPU, float64), with
the magnitudes their rounding errors are measured against.

Every function returns what the operator returns; a `*_mag` value is the sum of
the absolute values of the terms of the result, so that an fp32 evaluation of n
terms in any order is within about n * 2^-24 of it.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24                       # fp32 rounding unit
BF16 = 2.0 ** -8                     # one bf16 rounding, relative (twice its unit)


def layer_norm(x, gamma, beta, eps):
    """y, mean, rstd, y_mag"""
    C = x.shape[1]
    mean = x.sum(1) / C
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / C + eps)
    g = torch.ones(C, dtype=torch.float64) if gamma is None else gamma
    b = torch.zeros(C, dtype=torch.float64) if beta is None else beta
    y = d * rstd[:, None] * g + b
    # the mean's own rounding is of the size of the row's largest elements
    size = x.abs() + x.abs().mean(1, keepdim=True)
    return y, mean, rstd, size * rstd[:, None] * g.abs() * 2 + b.abs()


def layer_norm_grad(dy, x, mean, rstd, gamma):
    """dx, dgamma, dbeta and their magnitudes, for the statistics given"""
    C = x.shape[1]
    g = torch.ones(C, dtype=torch.float64) if gamma is None else gamma
    z = (x - mean[:, None]) * rstd[:, None]
    zm = (x.abs() + mean.abs()[:, None]) * rstd[:, None]
    h = dy * g
    dx = rstd[:, None] * (h - h.sum(1, keepdim=True) / C - z * (h * z).sum(1, keepdim=True) / C)
    mag = rstd[:, None] * (h.abs() + h.abs().mean(1, keepdim=True) +
                           zm * (h.abs() * zm).mean(1, keepdim=True))
    return (dx, (dy * z).sum(0), dy.sum(0)), (mag, (dy.abs() * zm).sum(0), dy.abs().sum(0))


def philox(counter, key, rounds):
    """Philox4x32 (Salmon, Moraes, Dror and Shaw, 2011): counter uint32 [.., 4], key (2 words)."""
    c = [counter[..., j].astype(np.uint64) for j in range(4)]
    k = [int(key[0]), int(key[1])]
    m = np.uint64(0xFFFFFFFF)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & m,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(c, -1).astype(np.uint32)


def kept(first, count, p, seed, offset):
    """Whether elements first .. first + count stay."""
    i = np.arange(first // 4, -(-(first + count) // 4), dtype=np.uint64)
    c = np.empty((len(i), 4), np.uint32)
    c[:, 0], c[:, 1] = i & np.uint64(0xFFFFFFFF), i >> np.uint64(32)
    c[:, 2], c[:, 3] = offset % 2 ** 32, offset // 2 ** 32 % 2 ** 32
    u = philox(c, (seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32), 7).reshape(-1)
    at = first - first // 4 * 4
    return u[at:at + count].astype(np.uint64) >= np.uint64(round(p * 2 ** 32))


def route(logits, k, normalize):
    """experts, weights, offsets, rows, pos: one row and one slot at a time."""
    n, E = logits.shape
    experts, weights = np.full((n, k), -1, np.int64), np.zeros((n, k))
    for r in range(n):
        row = [float(v) for v in logits[r]]
        left = [e for e in range(E) if row[e] != -math.inf]
        nan = any(math.isnan(v) for v in row)
        for s in range(min(k, len(left))):
            best = max(left, key=lambda e: (math.isnan(row[e]), 0.0 if math.isnan(row[e]) else
                                            row[e], -e))
            experts[r, s] = best
            left.remove(best)
        got = [e for e in experts[r] if e >= 0]
        if not got:
            continue
        if nan or math.isinf(row[got[0]]):
            # exp and / of what the softmax has to work with
            t = np.array([row[e] for e in (got if normalize else range(E))])
            with np.errstate(all="ignore"):
                top = row[got[0]]
                w = np.exp(np.array([row[e] for e in got]) - top) / np.exp(t - top).sum()
        else:
            top = max(row)
            z = sum(math.exp(row[e] - top) for e in (got if normalize else range(E)))
            w = [math.exp(row[e] - top) / z for e in got]
        weights[r, :len(got)] = w
    pairs = sorted((int(e), i) for i, e in enumerate(experts.reshape(-1)) if e >= 0)
    rows, pos = np.full(n * k, -1, np.int64), np.full(n * k, -1, np.int64)
    for at, (e, i) in enumerate(pairs):
        rows[at], pos[i] = i // k, at
    offsets = np.array([sum(e < b for e, _ in pairs) for b in range(E)] + [len(pairs)])
    return experts, weights, offsets, rows, pos.reshape(n, k)


def route_grad(dweights, logits, experts, weights, normalize):
    n, E = logits.shape
    d = np.zeros((n, E))
    for r in range(n):
        got = [(int(e), s) for s, e in enumerate(experts[r]) if e >= 0]
        dot = sum(weights[r, s] * dweights[r, s] for _, s in got)
        if not normalize and np.isfinite(logits[r]).any():
            x = np.exp(logits[r] - logits[r].max())
            d[r] = -x / x.sum() * dot
        for e, s in got:
            d[r, e] += weights[r, s] * (dweights[r, s] - (dot if normalize else 0.0))
    return d


def groups(offsets, m):
    return [(e, int(a), int(b)) for e, (a, b) in enumerate(zip(offsets[:-1], offsets[1:]))]


def take(x, rows, m):
    """x's rows per position; an index out of range is a row of zeros."""
    if rows is None:
        return x
    ok = (rows >= 0) & (rows < len(x))
    return torch.where(ok[:, None], x[torch.where(ok, rows, 0)], 0.0)


def grouped(x, w, offsets, rows, bias, relu):
    """y, y_mag"""
    m = len(x) if rows is None else len(rows)
    x = take(x, rows, m)
    y = torch.zeros((m, w.shape[2]), dtype=torch.float64)
    mag = torch.zeros_like(y)
    for e, a, b in groups(offsets, m):
        y[a:b] = x[a:b] @ w[e] + (0.0 if bias is None else bias[e])
        mag[a:b] = x[a:b].abs() @ w[e].abs() + (0.0 if bias is None else bias[e].abs())
    return (torch.where(y < 0, 0.0, y) if relu else y), mag


def grouped_grad(x, dy, w, offsets, rows, mask):
    """(dx, dw, db), their magnitudes"""
    m = len(dy)
    x = take(x, rows, m)
    E, ci, co = w.shape
    out = [torch.zeros((m, ci), dtype=torch.float64), torch.zeros_like(w),
           torch.zeros((E, co), dtype=torch.float64)]
    mag = [torch.zeros_like(t) for t in out]
    for e, a, b in groups(offsets, m):
        for t, f in ((out, lambda v: v), (mag, torch.abs)):
            t[0][a:b] = f(dy[a:b]) @ f(w[e]).T
            t[1][e] = f(x[a:b]).T @ f(dy[a:b])
            t[2][e] = f(dy[a:b]).sum(0)
    if mask is not None:
        out[0] = torch.where(mask <= 0, 0.0, out[0])
    return out, mag


def combine(y, pos, weights, residual):
    """out, out_mag"""
    n, k = pos.shape
    out = torch.zeros((n, y.shape[1]), dtype=torch.float64) if residual is None else residual
    mag = out.abs()
    for s in range(k):
        ok = ((pos[:, s] >= 0) & (pos[:, s] < len(y)))[:, None]
        v = torch.where(ok, y[torch.where(ok[:, 0], pos[:, s], 0)], 0.0)
        w = 1.0 if weights is None else torch.where(ok, weights[:, s:s + 1], 0.0)
        out = out + w * v
        mag = mag + (w * v).abs()
    return out, mag


def combine_grad(dout, y, pos, weights):
    """dy, dweights, dweights_mag"""
    n, k = pos.shape
    dy = torch.zeros_like(y)
    dw = torch.zeros((n, k), dtype=torch.float64)
    mag = torch.zeros_like(dw)
    for r in range(n):
        for s in range(k):
            p = int(pos[r, s])
            if 0 <= p < len(y):
                dy[p] = dout[r] * (1.0 if weights is None else weights[r, s])
                dw[r, s] = (dout[r] * y[p]).sum()
                mag[r, s] = (dout[r] * y[p]).abs().sum()
    return dy, dw, mag
