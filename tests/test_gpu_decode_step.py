"""A small decoder's layers as they are served: the product that makes q, k and v, the append, the attention over the pages, the output projection added to the
stream, the two products of the feed-forward block.  Prompts of different lengths first, then one token a sequence, the steps captured once and replayed.

Every stage's output is held against the fp64 oracle on that stage's own inputs (the numbers the kernels in front of it left), with the tolerances derived in
test_gpu_paged.py and test_gpu_linear.py, so that nothing accumulates; the replays are held against eager calls bit for bit.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged_serving as O
from paper_2509_22622_amd import binding as B

from test_gpu_paged import f64, normal

pytestmark = pytest.mark.gpu

LAYERS, HIDDEN, HQ, HKV, D, PAGE, WIDE = 2, 192, 6, 2, 64, 16, 520
QKV = (HQ + 2 * HKV) * D


class Decoder:
    """Weights, caches and buffers of `rows` rows, as a serving program keeps them."""

    def __init__(self, n_pages, kv_format):
        self.cache = B.PagedCache(LAYERS, HQ, HKV, D, PAGE, n_pages, rope="halves", rope_theta=500000.0, kv_format=kv_format)
        self.w, self.b, self.packed = [], [], []
        for layer in range(LAYERS):
            shapes = {"qkv": (QKV, HIDDEN), "out": (HIDDEN, HQ * D), "up": (WIDE, HIDDEN), "down": (HIDDEN, WIDE)}
            self.w.append({n: normal(s, 10 * layer + i, s[1] ** -0.5) for i, (n, s) in enumerate(shapes.items())})
            self.b.append({n: normal((s[0],), 100 + 10 * layer + i, 0.3) for i, (n, s) in enumerate(shapes.items())})
            self.packed.append({n: B.Linear(w) for n, w in self.w[-1].items()})

    def buffers(self, rows, seqs, max_new, max_len):
        new = lambda n: torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
        return {"x": new(HIDDEN), "qkv": new(QKV), "q": torch.empty(rows, HQ, D, dtype=torch.bfloat16, device="cuda"), "attn": new(HQ * D).zero_(), "mid": new(HIDDEN),
                "wide": new(WIDE), "ws": self.cache.attn_workspace(seqs, max_new=max_new, max_len=max_len), "max_new": max_new, "max_len": max_len}

    def layer(self, layer, buf, lens, table, cu, seen=None):
        """One layer on buf["x"], in place.  `seen`: a function that is shown each stage."""
        p, b, c = self.packed[layer], self.b[layer], self.cache
        q, k, v = (t.unflatten(1, (-1, D)) for t in buf["qkv"].split([HQ * D, HKV * D, HKV * D], 1))
        attn = buf["attn"].unflatten(1, (HQ, D))
        show = seen or (lambda *a: None)
        p["qkv"].forward(buf["x"], buf["qkv"], bias=b["qkv"])
        show("linear", "qkv", buf["x"], buf["qkv"], "none", None)
        c.append(layer, lens, table, k, v, q=q, q_out=buf["q"], cu_tokens=cu)
        show("append", q, k, v, buf["q"])
        c.attn(layer, lens, table, buf["q"], attn, buf["ws"], cu_tokens=cu, max_new=buf["max_new"], max_len=buf["max_len"])
        show("attend", buf["q"], attn)
        was = buf["x"].clone() if seen else None
        p["out"].forward(buf["attn"], buf["mid"], bias=b["out"], residual=buf["x"])
        show("linear", "out", buf["attn"], buf["mid"], "none", was)
        p["up"].forward(buf["mid"], buf["wide"], bias=b["up"], activation="gelu_tanh")
        show("linear", "up", buf["mid"], buf["wide"], "gelu_tanh", None)
        was = buf["mid"].clone() if seen else None
        p["down"].forward(buf["wide"], buf["mid"], bias=b["down"], residual=buf["mid"])      # onto the stream itself
        show("linear", "down", buf["wide"], buf["mid"], "none", was)
        buf["x"].copy_(buf["mid"])


def checker(dec, layer, lens, table, cu, max_new):
    rows_of = lambda n: O.rows_of(lens, cu, n)

    def linear(name, x, y, act, residual):
        w, b = f64(dec.w[layer][name]), f64(dec.b[layer][name])
        want, mag = O.linear(f64(x), w, b, act, None if residual is None else f64(residual))
        plain = want if residual is None else want - f64(residual)
        tol = 1.13 * (w.shape[1] + 1) * 2.0 ** -24 * mag + 2.0 ** -17 * np.abs(plain) + 2.0 ** -8 * np.abs(want) + 1e-30
        assert (np.abs(f64(y) - want) <= tol).all(), name

    def pool(values):
        x = dec.cache.values(layer) if values else dec.cache.keys(layer)
        bits = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
        return f64(bits.reshape(dec.cache.n_pages, PAGE, HKV, D).contiguous().view(x.dtype))

    def append(q, k, v, q_out):
        stored, queries = O.appended(lens, cu, table, dec.cache.n_pages, PAGE, f64(q), f64(k), f64(v), "halves", D, 500000.0)
        keys, values = pool(False), pool(True)
        half, top = (2.0 ** -8, math.inf) if dec.cache.kv_format == "bf16" else (2.0 ** -4, 448.0)      # 8 bits: clamped first
        for at, kv in stored.items():
            want_k, want_v = (np.clip(t, -top, top) for t in kv)
            assert (np.abs(keys[at] - want_k) <= np.maximum(np.abs(want_k) * half, 2.0 ** -10 if half > 0.01 else 0) + 4e-6).all()
            assert (np.abs(values[at] - want_v) <= (0 if half < 0.01 else np.maximum(np.abs(want_v) * half, 2.0 ** -10))).all()
        got = f64(q_out)
        for r, want in queries.items():
            assert (np.abs(got[r] - want) <= np.abs(want) * 2.0 ** -8 + 4e-6).all()

    def attend(q, out):
        want, got = O.attended(lens, cu, table, PAGE, f64(q), pool(False), pool(True), 0, 0, max_new), f64(out)
        assert len(want) == sum(at is not None for at in rows_of(len(got)))
        for r, (o, mag, big) in want.items():
            tol = mag * (2.0 ** -8 + 2 * math.log(2) * D * 2.0 ** -24 * big[:, None] + 2.0 ** -20) + np.abs(o) * 2.0 ** -8 + 1e-30
            assert (np.abs(got[r] - o) <= tol).all(), r

    return lambda what, *a: {"linear": linear, "append": append, "attend": attend}[what](*a)


@pytest.mark.parametrize("kv_format", ["bf16", "fp8_e4m3"])
def test_prompts_then_tokens(kv_format):
    prompts, steps, cols = [5, 64, 33, 1], 24, 8
    rng = np.random.default_rng(3)
    n_pages = len(prompts) * cols
    table = rng.permutation(n_pages).astype(np.int32).reshape(len(prompts), cols)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    eager, graphed = Decoder(n_pages, kv_format), Decoder(n_pages, kv_format)
    tab, lens = dev(table), np.array(prompts)
    cu = np.concatenate([[0], np.cumsum(prompts)])
    for dec in (eager, graphed):                                  # the prompts, all at once
        buf = dec.buffers(int(cu[-1]), len(prompts), max(prompts), max(prompts))
        buf["x"].copy_(normal((int(cu[-1]), HIDDEN), 77))
        for layer in range(LAYERS):
            dec.layer(layer, buf, dev(lens), tab, dev(cu), checker(dec, layer, lens, table, cu, max(prompts)) if dec is eager else None)
    first = buf["x"][torch.tensor(cu[1:] - 1, device="cuda")]     # what follows each prompt

    bufs = [dec.buffers(len(prompts), len(prompts), 1, cols * PAGE) for dec in (eager, graphed)]
    n = dev(lens)

    def step(dec, buf, seen=lambda layer: None):
        for layer in range(LAYERS):
            dec.layer(layer, buf, n, tab, None, seen(layer))

    # the step is captured without having run: lengths of 0 make the warm-up one that stores nothing
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        n.zero_()
        bufs[1]["x"].copy_(first)
        step(graphed, bufs[1])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed, bufs[1])
    for buf in bufs:
        buf["x"].copy_(first)
    n.copy_(dev(lens))
    for i in range(steps):
        n += 1
        lens = lens + 1
        if i == 10:                                               # a sequence ends: its place in the batch idles
            n[2], lens[2] = -1000, -1000
        graph.replay()
        step(eager, bufs[0], lambda layer: checker(eager, layer, lens, table, None, 1) if i % 6 == 0 else None)
        torch.cuda.synchronize()
        for name in ("q", "attn", "x"):
            assert torch.equal(bufs[0][name], bufs[1][name]), (i, name)
    for layer in range(LAYERS):
        for values in (False, True):
            a, b = ((d.cache.values(layer) if values else d.cache.keys(layer)) for d in (eager, graphed))
            assert torch.equal(a.view(torch.uint8) if kv_format != "bf16" else a, b.view(torch.uint8) if kv_format != "bf16" else b)
