"""CPU oracle for serving many sequences from a paged cache: appending, attention of the newest tokens, linear layers.

TEST INFRASTRUCTURE ONLY.  Plain fp64 numpy; only tests may import it.  It shares no code with the HIP path and imports nothing
from the product package.

The batch of a call: ``lens[s]`` tokens of sequence s with the call's own, ``cu`` the first row of each sequence (None: row i is
sequence i's only one), ``table[s]`` its pages.  A row's place is its token's index in its sequence, counted from 0; the place has a
slot (page, token in the page) unless it is negative, lies behind the table's row, or its page is outside the pool.

Rotary embedding of a row at position p: pair i of the first ``rope_dim`` features turns by p * theta^(-2 i / rope_dim); pairs are
neighbours ("pairs") or half of rope_dim apart ("halves"); "grid" divides D / 2 neighbouring pairs into frame, row and column, with
D // 6 pairs for each of the last two.
"""
from __future__ import annotations

import math

import numpy as np


def rows_of(lens, cu, n_tokens):
    """(sequence, place) of every row of a call; None for rows of no sequence."""
    out = [None] * n_tokens
    for s, n in enumerate(lens):
        first, end = (s, s + 1) if cu is None else (int(cu[s]), int(cu[s + 1]))
        for r in range(max(first, 0), min(end, n_tokens)):
            out[r] = (s, int(n) - (end - r))
    return out


def slot(table, n_pages, page_tokens, s, place):
    """(page, token in the page) of a place, or None."""
    if place < 0 or place >= len(table[s]) * page_tokens:
        return None
    page = int(table[s][place // page_tokens])
    return (page, place % page_tokens) if 0 <= page < n_pages else None


def angles(rope, rope_dim, theta, position):
    """Angle of each pair; position: a number, or (frame, row, column)."""
    if rope == "none":
        return np.zeros(0)
    if rope == "grid":
        n_x = rope_dim // 6
        parts = [(rope_dim // 2 - 2 * n_x, position[0]), (n_x, position[1]), (n_x, position[2])]
        return np.array([p * float(theta) ** (-i / n) for n, p in parts for i in range(n)])
    return np.array([position * float(theta) ** (-2.0 * i / rope_dim) for i in range(rope_dim // 2)])


def turn(x, rope, rope_dim, theta, position):
    """x [heads, D] turned by the embedding at ``position``."""
    a = angles(rope, rope_dim, theta, position)
    out = np.array(x, dtype=np.float64)
    for i, t in enumerate(a):
        f, g = (i, i + rope_dim // 2) if rope == "halves" else (2 * i, 2 * i + 1)
        out[:, f] = x[:, f] * math.cos(t) - x[:, g] * math.sin(t)
        out[:, g] = x[:, g] * math.cos(t) + x[:, f] * math.sin(t)
    return out


def appended(lens, cu, table, n_pages, page_tokens, q, k, v, rope, rope_dim, theta, positions=None):
    """What one append stores and returns: {(page, token in it): (turned key, value)} and {row: turned, scaled query}."""
    stored, queries = {}, {}
    for r, at in enumerate(rows_of(lens, cu, len(k))):
        if at is None:
            continue
        position = at[1] if positions is None else positions[r]
        if q is not None:
            queries[r] = turn(q[r], rope, rope_dim, theta, position) * (math.log2(math.e) / math.sqrt(q.shape[-1]))
        to = slot(table, n_pages, page_tokens, *at)
        if to is not None:
            stored[to] = (turn(k[r], rope, rope_dim, theta, position), v[r])
    return stored, queries


def sees(i, j, sink, window):
    return j <= i and (window == 0 or j < sink or j > i - window)


def attended(lens, cu, table, page_tokens, q, keys, values, sink, window, max_new=1):
    """Per row: (output [q_heads, D], sum of |weight * value| / sum of weights, largest sum of |q_d k_d|), zeros where a row sees no key.
    keys, values: the pool [n_pages, page_tokens, kv_heads, D]; q carries log2(e) / sqrt(D).  Rows of no sequence and rows behind
    the max_new-th of a sequence are left out."""
    out = {}
    n_pages, _, kv_heads, d = keys.shape
    group = q.shape[1] // kv_heads
    for r, at in enumerate(rows_of([max(int(n), 0) for n in lens], cu, len(q))):
        if at is None:
            continue
        s, i = at
        if cu is not None and r - int(cu[s]) >= max_new:
            continue
        slots = [slot(table, n_pages, page_tokens, s, j) for j in range(min(i + 1, len(table[s]) * page_tokens)) if sees(i, j, sink, window)]
        slots = [x for x in slots if x is not None]
        o, mag, big = np.zeros((q.shape[1], d)), np.zeros((q.shape[1], d)), np.zeros(q.shape[1])
        if slots:
            pages, tokens = (np.array(x) for x in zip(*slots))
            for h in range(q.shape[1]):
                k, v = keys[pages, tokens, h // group], values[pages, tokens, h // group]
                z = k @ q[r, h]
                w = np.exp2(z - z.max())
                o[h], mag[h], big[h] = w @ v / w.sum(), w @ np.abs(v) / w.sum(), (np.abs(k) @ np.abs(q[r, h])).max()
        out[r] = (o, mag, big)
    return out


def activation(y, name):
    if name == "gelu_tanh":
        return 0.5 * y * (1 + np.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    if name == "gelu":
        return np.array([0.5 * t * math.erfc(-t / math.sqrt(2)) for t in y.ravel()]).reshape(y.shape)
    if name == "silu":
        return y / (1 + np.exp(-y))
    return y


def linear(x, w, bias=None, act="none", residual=None):
    """(act(x w^T + bias) + residual, sum of |x w| + |bias|)"""
    y, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    y = activation(y, act)
    return (y if residual is None else y + residual), mag
