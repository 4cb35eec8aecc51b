"""CPU oracle for the layer norm and for the attention to an encoder's states, with their gradients.

TEST INFRASTRUCTURE ONLY.  Plain fp64 numpy; only tests may import it.  It shares no code with the HIP path and imports nothing from the
product package.  Beside each result stands what a kernel that computes in fp32 and rounds where the library says it does may be off by.

U: a rounding to fp32.  B: one to bfloat16.  Sums of n terms by at most 64 additions one after the other and trees are off by at most (n + 2) U of
the terms' absolute sum; rows of up to 16384 features are summed by 32 additions and trees of depth 9 and 8: 64 U.
"""
from __future__ import annotations

import math

import numpy as np

U, B = 2.0 ** -24, 2.0 ** -8
TINY = 2.0 ** -126        # a weight, or a weight's product, below the smallest normal number may count as 0: so much is lost of each term of the sums it goes into


def group_of(rows, group_rows):
    return np.arange(rows) // group_rows if group_rows else np.zeros(rows, dtype=np.int64)


def norm(x, w, b, eps, group_rows, y_step):
    """((y, how far it may be off), (mean, 1 / sqrt(var + eps))): x [m, n], w and b [groups, n] or None."""
    m, n = x.shape
    g = group_of(m, group_rows)
    mean = x.mean(1, keepdims=True)
    r = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    h = (x - mean) * r
    wr = np.ones((1, n)) if w is None else w[g]
    br = np.zeros((1, n)) if b is None else b[g]
    y = h * wr + br
    off = np.abs(wr) * h_off(x, h, r) + 4 * U * (np.abs(h * wr) + np.abs(br)) + y_step * np.abs(y) + 1e-38
    return (y, off), (mean[:, 0], r[:, 0])


def h_off(x, h, r):
    """How far (x - mean) r may be off: the mean by 66 U of the mean absolute value, the variance by the square of that and 70 U of itself, r by half of it."""
    lost = 66 * U * np.abs(x).mean(1, keepdims=True) * r
    return np.abs(h) * (64 * U + lost ** 2) + lost


def norm_backward(dy, x, w, eps, group_rows, residual, dx_step):
    """((dx, off), (dweight, off), (dbias, off))"""
    m, n = x.shape
    g = group_of(m, group_rows)
    mean = x.mean(1, keepdims=True)
    r = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    h = (x - mean) * r
    eh = h_off(x, h, r)
    t = dy if w is None else dy * w[g]
    a, b = t.mean(1, keepdims=True), (t * h).mean(1, keepdims=True)
    res = 0.0 if residual is None else residual
    dx = r * (t - a - h * b) + res
    ea = 70 * U * np.abs(t).mean(1, keepdims=True)
    eb = 70 * U * np.abs(t * h).mean(1, keepdims=True) + (np.abs(t) * eh).mean(1, keepdims=True)
    off = r * (4 * U * np.abs(t) + ea + np.abs(h) * eb + np.abs(b) * eh + 70 * U * (np.abs(t) + np.abs(a) + np.abs(h * b))) + 4 * U * (np.abs(dx) + np.abs(res))
    off = off + dx_step * np.abs(dx) + 1e-38
    groups = int(g[-1]) + 1 if m else 1
    out = [np.zeros((groups, n)) for _ in range(4)]
    for i in range(m):
        out[0][g[i]] += dy[i] * h[i]
        out[1][g[i]] += np.abs(dy[i]) * eh[i] + (m + 20) * U * np.abs(dy[i] * h[i])
        out[2][g[i]] += dy[i]
        out[3][g[i]] += (m + 20) * U * np.abs(dy[i])
    return (dx, off), (out[0], out[1] + 1e-38), (out[2], out[3] + 1e-38)


def spans(cu, lens, n_seqs, total, most):
    """(first row, rows that are seen, rows) of each sequence."""
    out = []
    for s in range(n_seqs):
        begin, end = (s * (total // n_seqs), (s + 1) * (total // n_seqs)) if cu is None else (int(cu[s]), int(cu[s + 1]))
        begin = min(max(begin, 0), total)
        end = min(max(end, begin), total)
        n = end - begin if lens is None else min(max(int(lens[s]), 0), end - begin)
        out.append((begin, min(n, most), end - begin))
    return out


def attention(q, k, v, scale):
    """((out, off), (lse, off)) of one sequence and head: q [m, D], k, v [n, D]."""
    m, d = q.shape
    if len(k) == 0:
        return (np.zeros((m, d)), np.zeros((m, d))), (np.full(m, -math.inf), np.zeros(m))
    z = scale * (q @ k.T)
    top = z.max(1, keepdims=True)
    p = np.exp(z - top)
    total = p.sum(1, keepdims=True)
    p /= total
    out, lse = p @ v, (top + np.log(total))[:, 0]
    arg = score_off(q, k, scale, z)
    off = p @ np.abs(v) * (B + 2 * arg.max(1, keepdims=True) + (len(k) + 70) * U) + B * np.abs(out) + TINY * (1 + np.abs(v).sum(0))
    return (out, off), (lse, arg.max(1) + (len(k) + 70) * U + 8 * U * np.abs(lse))


def score_off(q, k, scale, z):
    """A score in nats: D products added up in fp32, a product with the scale, an exponential of a difference, and the exponential's own 2^-21."""
    return (q.shape[1] + 2) * U * scale * (np.abs(q) @ np.abs(k).T) + 8 * U * np.abs(z) + 2.0 ** -21


def attention_backward(dout, q, k, v, scale):
    """((dq, off), (dk, off), (dv, off)) of one sequence and head.  The weights and dS are rounded to bfloat16 for their products; delta is off by up to 2^-10 of
    the row's sum of P |dP - delta|, and by what the sums in fp32 lose."""
    m, d = q.shape
    n = len(k)
    if n == 0 or m == 0:
        return tuple((np.zeros(t.shape), np.zeros(t.shape)) for t in (q, k, v))
    z = scale * (q @ k.T)
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    lse = np.abs(z.max(1, keepdims=True)) + math.log(n)
    arg = score_off(q, k, scale, z)
    ep = 2 * (arg + arg.max(1, keepdims=True)) + 20 * U * lse + (n + 70) * U                    # of a weight, before it is rounded
    dp = dout @ v.T
    delta = (p * dp).sum(1, keepdims=True)
    ds = p * (dp - delta) if n > 1 else np.zeros_like(p)
    edp = (d + 2) * U * (np.abs(dout) @ np.abs(v).T)
    edelta = 1.1 * 2.0 ** -10 * np.abs(ds).sum(1, keepdims=True) + (p * (np.abs(dp) * (ep + (n + 4) * U) + edp)).sum(1, keepdims=True)
    eds = p * ((B + ep) * np.abs(dp - delta) + edp + edelta) + TINY * (1 + np.abs(dp - delta)) if n > 1 else np.zeros_like(p)
    dq, dk, dv = scale * (ds @ k), scale * (ds.T @ q), p.T @ dout
    sums = (max(m, n) + 40) * U
    return ((dq, scale * (eds + sums * np.abs(ds)) @ np.abs(k) + 1.01 * B * np.abs(dq) + TINY), (dk, scale * (eds + sums * np.abs(ds)).T @ np.abs(q) + 1.01 * B * np.abs(dk) + TINY),
            (dv, (p * (B + ep + sums) + TINY).T @ np.abs(dout) + 1.01 * B * np.abs(dv) + TINY))


def attended(q, k, v, scale, n_seqs, cu_q, cu_k, k_lens, max_q, max_k, dout=None):
    """Whole tensors {name: (value, off)}; NaN where nothing is written.  q [n_q, q_heads, D], k and v [n_k, kv_heads, D]."""
    hq, hkv = q.shape[1], k.shape[1]
    made = {"out": q.shape, "lse": (hq, len(q))}
    if dout is not None:
        made |= {"dq": q.shape, "dk": k.shape, "dv": k.shape}
    got = {name: (np.full(shape, math.nan), np.zeros(shape)) for name, shape in made.items()}
    for (a, m, _), (b, n, rows) in zip(spans(cu_q, None, n_seqs, len(q), max_q), spans(cu_k, k_lens, n_seqs, len(k), max_k)):
        at, to = slice(a, a + m), slice(b, b + n)
        if dout is not None:
            for name in ("dk", "dv"):
                got[name][0][b:b + rows] = 0.0
        for h in range(hq):
            g = h // (hq // hkv)
            one = attention(q[at, h], k[to, g], v[to, g], scale)
            for i in range(2):
                got["out"][i][at, h] = one[0][i]
                got["lse"][i][h, at] = one[1][i]
            if dout is not None:
                dq, dk, dv = attention_backward(dout[at, h], q[at, h], k[to, g], v[to, g], scale)
                for i in range(2):
                    got["dq"][i][at, h] = dq[i]
                    got["dk"][i][to, g] += dk[i]
                    got["dv"][i][to, g] += dv[i]
    return got
