"""The token models' operators in fp64, one mini-batch at a time, from their formulas.

* embedding: Y[t] = scale E[token[t]], zeros outside the table; its gradient is the sum of
  each token's rows;
* recurrence: a = sigmoid(g + bias), h_t = a h_{t-1} + (1 - a) x_t, and its gradients from
  the chain rule, last token first;
* 8-bit activations: whole numbers of at most 127 on the smallest power-of-two step that
  holds the 32 tokens of a channel; the weight gradient of a layer is A^T dY of their values.

Beside each result stands a bound on what a computation in 32 bits may be off by, carried
through the same recursion (u = 2^-24, half a step of fp32): a gate of z = g + bias is off
by (6 |z| + 10) u of its value (z's own rounding, the scaled argument of the exponential,
its last place, and 1 + e, the reciprocal and a product on top), each product and sum by u.

Pins (tests/test_oracle_tokens.py): torch autograd in float64 and central differences.
"""

from __future__ import annotations

import numpy as np

U = 2.0 ** -24
BLOCK = 32


def embed(E, tokens, scale):
    tokens = np.asarray(tokens)
    inside = (tokens >= 0) & (tokens < len(E))
    Y = np.zeros((len(tokens), E.shape[1]))
    Y[inside] = scale * np.asarray(E, np.float64)[tokens[inside]]
    return Y


def embed_grad(dY, tokens, vocab, scale):
    """(gradient [vocab, dim], bound)."""
    tokens = np.asarray(tokens)
    G, S, k = np.zeros((vocab, dY.shape[1])), np.zeros((vocab, dY.shape[1])), np.zeros(vocab)
    for t in np.flatnonzero((tokens >= 0) & (tokens < vocab)):
        G[tokens[t]] += np.asarray(dY[t], np.float64)
        S[tokens[t]] += np.abs(np.asarray(dY[t], np.float64))
        k[tokens[t]] += 1
    return scale * G, (k[:, None] + 1) * U * abs(scale) * S


def gates(g, bias):
    z = np.asarray(g, np.float64) + np.asarray(bias, np.float64)
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z)), (6 * np.minimum(np.abs(z), 1e3) + 10) * U


def scan(x, g, bias, h0, length):
    """One sequence [T, C]: (h, states before every token, last state) and their bounds."""
    a, rest, off = gates(g, bias)
    T, C = a.shape
    h, before, eh, eb = np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C))
    s, e = np.array(h0, np.float64), np.zeros(C)
    for t in range(T):
        before[t], eb[t] = s, e
        if t < length:
            keep, put = a[t] * s, rest[t] * np.asarray(x[t], np.float64)
            e = a[t] * e + (off[t] + 2 * U) * (np.abs(keep) + np.abs(put)) + 1e-37
            s = keep + put
            h[t], eh[t] = s, e
    return (h, before, s), (eh, eb, e)


def scan_grad(x, g, bias, h0, length, dh, dh_last):
    """(dx, dg, dh0, dbias) of one sequence and their bounds."""
    a, rest, off = gates(g, bias)
    (_, before, _), (_, eb, _) = scan(x, g, bias, h0, length)
    T, C = a.shape
    dx, dg, ex, eg = np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C))
    mu, e = np.array(dh_last, np.float64), np.zeros(C)
    for t in range(min(T, length) - 1, -1, -1):
        d = np.asarray(dh[t], np.float64)
        lam, el = d + mu, e + U * (np.abs(d) + np.abs(mu))
        gap = before[t] - np.asarray(x[t], np.float64)
        egap = eb[t] + U * (np.abs(before[t]) + np.abs(np.asarray(x[t], np.float64)))
        dx[t] = lam * rest[t]
        ex[t] = rest[t] * el + (off[t] + U) * np.abs(dx[t])
        dg[t] = dx[t] * a[t] * gap
        eg[t] = (ex[t] * np.abs(gap) + np.abs(dx[t]) * egap) * a[t] + (off[t] + 3 * U) * np.abs(dg[t])
        mu, e = a[t] * lam, a[t] * el + (off[t] + 2 * U) * a[t] * (np.abs(d) + np.abs(mu)) + 1e-37
    db, edb = dg.sum(0), eg.sum(0) + T * U * np.abs(dg).sum(0)
    return (dx, dg, mu, db), (ex, eg, e, edb)


def act8(A):
    """(whole numbers [T, dim], step of every entry) of activations [T, dim]; NaN steps where a
    block holds an infinity or a NaN."""
    A = np.asarray(A, np.float64)
    q, step = np.zeros(A.shape), np.zeros(A.shape)
    for t in range(0, len(A), BLOCK):
        for c in range(A.shape[1]):
            v = A[t:t + BLOCK, c]
            if not np.isfinite(v).all():
                step[t:t + BLOCK, c] = np.nan
                continue
            k = -126
            while k < 121 and np.abs(np.rint(v / 2.0 ** k)).max() > 127:
                k += 1
            q[t:t + BLOCK, c] = np.clip(np.rint(v / 2.0 ** k), -127, 127)
            step[t:t + BLOCK, c] = 2.0 ** k
    return q, step


def act_grad(values, dY):
    """A^T dY of the 8-bit values [T, dim] and dY [T, out], and the bound of T sums in fp32, each
    off by a whole step at most (the matrix cores may truncate)."""
    v, d = np.asarray(values, np.float64), np.asarray(dY, np.float64)
    return v.T @ d, (len(v) + 1) * 2 * U * (np.abs(v).T @ np.abs(d)) + 1e-36
