"""Token and expert layers in float64 (numpy), from their definitions: segments, embedding, dropout, products grouped by expert,
their gradients and Kronecker factors.  Test infrastructure; shares no code with the GPU path."""
from __future__ import annotations

import numpy as np


def segments(ids, num):
    """order (stable, ids outside [0, num) last), offsets [num + 1]."""
    ids = np.asarray(ids, dtype=np.int64)
    key = np.where((ids >= 0) & (ids < num), ids, num)
    order = np.argsort(key, kind="stable").astype(np.int32)
    counts = np.bincount(key, minlength=num + 1)[:num]
    return order, np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def embedding(ids, table, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for i, t in enumerate(ids):
        if 0 <= t < table.shape[0]:
            out[i] = scale * table[t].astype(np.float64)
    return out


def embedding_grad(ids, grad_out, scale, vocab):
    """(dW, counts, sum of magnitudes): the last is what the rounding of the sums is measured against."""
    dW, mag = np.zeros((vocab, grad_out.shape[1])), np.zeros((vocab, grad_out.shape[1]))
    counts = np.zeros(vocab, dtype=np.int64)
    ok = (np.asarray(ids) >= 0) & (np.asarray(ids) < vocab)
    g = grad_out[ok].astype(np.float64)
    np.add.at(dW, np.asarray(ids)[ok], g)
    np.add.at(mag, np.asarray(ids)[ok], np.abs(g))
    np.add.at(counts, np.asarray(ids)[ok], 1)
    return scale * dW, counts, abs(scale) * mag


def philox4x32(counter, key):
    """Philox4x32-10 (Salmon et al., SC 2011), one block: four words of counter, two of key, plain integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_keep(first, n, p, seed, offset):
    """Which of the elements first .. first + n - 1 are kept."""
    keep = np.zeros(n, dtype=bool)
    low = 0xFFFFFFFF
    words, at = None, None
    for i in range(n):
        e = first + i
        if at != e // 8:
            at = e // 8
            words = philox4x32([at & low, at >> 32, offset & low, offset >> 32], [seed & low, seed >> 32])
        keep[i] = ((words[(e % 8) // 2] >> (16 * (e % 2))) & 0xFFFF) >= round(p * 65536)
    return keep


def dropout(x, residual, p, seed, offset):
    """x, residual (or None): [rows, cols]."""
    keep = dropout_keep(0, x.size, p, seed, offset).reshape(x.shape)
    t = round(p * 65536)
    y = np.zeros(x.shape)
    if t < 65536:
        y[keep] = x[keep].astype(np.float64) * (65536.0 / (65536.0 - t))
    return y if residual is None else y + residual.astype(np.float64)


def expert_forward(choice, x, W, c_in, bias, fan):
    """(y, magnitude); choice [n], W [E, c_out, >= c_in + bias]."""
    n, E, co = len(choice), W.shape[0], W.shape[1]
    y, mag = np.zeros((n, co)), np.zeros((n, co))
    for e in range(E):
        c = np.nonzero(np.asarray(choice) == e)[0]
        xe, We = x[c // fan].astype(np.float64), W[e, :, :c_in].astype(np.float64)
        y[c], mag[c] = xe @ We.T, np.abs(xe) @ np.abs(We).T
        if bias:
            b = W[e, :, c_in].astype(np.float64)
            y[c] += b
            mag[c] += np.abs(b)
    return y, mag


def expert_grad_input(choice, dy, W, c_in):
    n = len(choice)
    dx, mag = np.zeros((n, c_in)), np.zeros((n, c_in))
    for e in range(W.shape[0]):
        c = np.nonzero(np.asarray(choice) == e)[0]
        d, We = dy[c].astype(np.float64), W[e, :, :c_in].astype(np.float64)
        dx[c], mag[c] = d @ We, np.abs(d) @ np.abs(We)
    return dx, mag


def _with_bias(x, bias):
    return np.concatenate([x, np.ones((x.shape[0], 1))], 1) if bias else x


def expert_grad_weight(choice, x, dy, experts, bias, fan):
    out = np.zeros((experts, dy.shape[1], x.shape[1] + bias))
    mag = np.zeros_like(out)
    for e in range(experts):
        c = np.nonzero(np.asarray(choice) == e)[0]
        xe, d = _with_bias(x[c // fan].astype(np.float64), bias), dy[c].astype(np.float64)
        out[e], mag[e] = d.T @ xe, np.abs(d).T @ np.abs(xe)
    return out, mag


def expert_factors(choice, rows, experts, bias, fan):
    """(mean of outer products of every expert's rows, magnitude, rows of every expert)."""
    d = rows.shape[1] + bias
    out, mag, count = np.zeros((experts, d, d)), np.zeros((experts, d, d)), np.zeros(experts, dtype=np.int64)
    for e in range(experts):
        c = np.nonzero(np.asarray(choice) == e)[0]
        count[e] = len(c)
        if len(c):
            r = _with_bias(rows[c // fan].astype(np.float64), bias)
            out[e], mag[e] = r.T @ r / len(c), np.abs(r).T @ np.abs(r) / len(c)
    return out, mag, count
