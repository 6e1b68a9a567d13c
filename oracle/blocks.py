"""What surrounds the products of experts, in float64 (numpy), from its definitions: routing, the join of the experts' results,
activations in 8 bits, the root-mean-square norm, and their gradients.  Test infrastructure; shares no code with the GPU path."""
from __future__ import annotations

import numpy as np


def scores(logits, sigmoid):
    """Softmax (zeros where a row has no finite logit) or sigmoid of float64 logits."""
    with np.errstate(over="ignore", invalid="ignore"):
        if sigmoid:
            e = np.exp(-np.abs(logits))
            return np.where(logits >= 0, 1.0 / (1.0 + e), e / (1.0 + e))
        high = logits.max(1, keepdims=True)
        e = np.exp(logits - np.where(np.isneginf(high), 0.0, high))
        total = e.sum(1, keepdims=True)
        return e / np.where(total == 0, 1.0, total)


def route(logits, bias, fan, groups=1, top_groups=1, group_best=1, sigmoid=False, renormalise=True, scale=1.0):
    """(choice [n, fan], gate [n, fan])."""
    n, E = logits.shape
    s = scores(logits, sigmoid)
    choice, gate = np.full((n, fan), -1, dtype=np.int64), np.zeros((n, fan))
    for t in range(n):
        shut = np.isneginf(logits[t]) | (False if bias is None else np.isneginf(bias))
        if np.isnan(logits[t]).any() or (not sigmoid and np.isposinf(logits[t]).any()) or (bias is not None and np.isnan(bias[~np.isneginf(logits[t])]).any()):
            gate[t] = np.nan
            continue
        by_score = bias is not None or (groups > 1 and group_best > 1)
        rank = s[t] + (0.0 if bias is None else bias) if by_score else logits[t]
        open_ = [e for e in range(E) if not shut[e]]
        if groups > 1:
            size, of = E // groups, []
            for g in range(groups):
                inside = sorted((rank[e] for e in open_ if e // size == g), reverse=True)
                if inside:
                    of.append((-sum(inside[:group_best]), g))
            kept = {g for _, g in sorted(of)[:top_groups]}
            open_ = [e for e in open_ if e // size in kept]
        # without a bias experts go by their logits, whatever the groups go by
        key = (lambda e: (-rank[e], e)) if bias is not None else (lambda e: (-logits[t, e], e))
        for j, e in enumerate(sorted(open_, key=key)[:fan]):
            choice[t, j] = e
        there = choice[t] >= 0
        gate[t, there] = scale * weights(logits[t], choice[t][there], sigmoid) if renormalise else scale * s[t, choice[t][there]]
    return choice, gate


def weights(l, chosen, sigmoid):
    """Chosen scores over their sum, from their logarithms, so that tiny ones do not vanish."""
    x = l[chosen].astype(np.float64)
    with np.errstate(over="ignore"):
        log = -np.logaddexp(0.0, -x) if sigmoid else x
    if not len(x):
        return x
    e = np.exp(log - log.max())
    return e / e.sum()


def route_grad(logits, choice, dgate, sigmoid=False, renormalise=True, scale=1.0):
    """(dlogits, sum of the magnitudes that each is the sum of)."""
    n, E = logits.shape
    s = scores(logits, sigmoid)
    out, mag = np.zeros((n, E)), np.zeros((n, E))
    for t in range(n):
        j = np.nonzero((choice[t] >= 0) & (choice[t] < E))[0]
        if not len(j):
            continue
        c, up = choice[t][j], scale * dgate[t][j]
        if renormalise:
            w = weights(logits[t], c, sigmoid)
            slope = 1.0 - s[t, c] if sigmoid else np.ones(len(j))
            if sigmoid:
                slope = scores(-logits[t][None].astype(np.float64), True)[0, c]
            np.add.at(out[t], c, w * (up - (up * w).sum()) * slope)
            np.add.at(mag[t], c, w * (np.abs(up) + (np.abs(up) * w).sum()) * slope)
        elif sigmoid:
            slope = s[t, c] * scores(-logits[t][None].astype(np.float64), True)[0, c]
            np.add.at(out[t], c, up * slope)
            np.add.at(mag[t], c, np.abs(up) * slope)
        else:
            u, ua = np.zeros(E), np.zeros(E)
            np.add.at(u, c, up)
            np.add.at(ua, c, np.abs(up))
            out[t] = s[t] * (u - (up * s[t, c]).sum())
            mag[t] = s[t] * (ua + (np.abs(up) * s[t, c]).sum())
    return out, mag


def combine(y, gate, fan, residual):
    """(out, magnitude); y [n, dim], gate [n] or None, residual [n / fan, dim] or None."""
    n, dim = y.shape
    g = np.ones(n) if gate is None else gate.astype(np.float64)
    terms = (g[:, None] * y).reshape(n // fan, fan, dim)
    out, mag = terms.sum(1), np.abs(terms).sum(1)
    return (out, mag) if residual is None else (out + residual, mag + np.abs(residual))


def combine_grad(y, gate, fan, dout):
    """(dy, dgate, magnitude of dgate)."""
    n = y.shape[0]
    up = np.repeat(dout, fan, 0)
    g = np.ones(n) if gate is None else gate.astype(np.float64)
    return g[:, None] * up, (up * y).sum(1), np.abs(up * y).sum(1)


def e4m3_values():
    """What the 256 bytes stand for: sign, four exponent bits (bias 7), three of the fraction; 0x7F and 0xFF are NaN."""
    v = np.zeros(256)
    for b in range(256):
        field, low = (b >> 3) & 15, b & 7
        m = low * 2.0 ** -9 if field == 0 else (8 + low) * 2.0 ** (field - 10)
        v[b] = np.nan if b & 0x7F == 0x7F else (-m if b & 0x80 else m)
    return v


def to_e4m3(u):
    """The bytes nearest to values of magnitude up to 448, ties to the even byte; NaN to NaN."""
    table = e4m3_values()[:127]
    a = np.abs(u)
    above = np.searchsorted(table, np.where(np.isnan(a), 0.0, a)).clip(0, 126)
    below = (above - 1).clip(0)
    da, db = table[above] - a, a - table[below]
    byte = np.where((db < da) | ((db == da) & (below % 2 == 0)), below, above)
    byte = np.where(np.isnan(u), 0x7F, byte)
    return (byte | np.where(np.signbit(u), 0x80, 0)).astype(np.uint8)


def keep(x):
    """(q bytes, scale bytes) of rows of float64 values."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    q, e = np.zeros((rows, cols), dtype=np.uint8), np.zeros((rows, blocks), dtype=np.int64)
    for b in range(blocks):
        v = x[:, 32 * b:32 * b + 32]
        fine = np.isfinite(v)
        high = np.where(fine, np.abs(v), 0.0).max(1)
        exponent = np.full(rows, -117)
        for k in range(-116, 120):
            exponent = np.where(high > 448.0 * 2.0 ** (k - 1), k, exponent)
        u = np.where(fine, v, 0.0) / 2.0 ** exponent[:, None]
        u = np.where(fine, np.clip(u, -448.0, 448.0), np.copysign(np.nan, v))
        q[:, 32 * b:32 * b + 32] = to_e4m3(u)
        e[:, b] = exponent
    return q, (e + 127).astype(np.uint8)


def restore(q, scales):
    power = 2.0 ** (scales.astype(np.float64) - 127.0)
    return e4m3_values()[q] * np.repeat(power, 32, 1)[:, :q.shape[1]]


def rms_norm(h, gamma, eps):
    """(y, r) of float64 rows."""
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return gamma * h * r, r


def rms_norm_grad(dy, h, gamma, eps, dstream):
    """(dh, its magnitude, dgamma, its magnitude, mean of squares)."""
    _, r = rms_norm(h, gamma, eps)
    u, g = h * r, gamma * dy
    along = (g * u).mean(1, keepdims=True)
    dh, mag = r * (g - u * along), r * (np.abs(g) + np.abs(u) * np.abs(g * u).mean(1, keepdims=True))
    if dstream is not None:
        dh, mag = dh + dstream, mag + np.abs(dstream)
    p = dy * u
    return dh, mag, p.sum(0), np.abs(p).sum(0), (p * p).mean(0) if len(p) else (p * p).sum(0)
