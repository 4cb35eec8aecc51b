"""ll_linear on the GPU against the fp64 oracle (oracle/paged_serving.py).

Tolerance: K fp32 products and additions and the bias are off by at most (K + 1) 2^-24 of sum |x w| + |bias|; no activation here is steeper
than 1.13, and its own arithmetic (an exponential of an fp32 argument t: |t| + 8 units of 2^-24, |t| <= 90 where it matters) moves it by at
most 2^-17 of |y|; one addition of the residual, one rounding to bfloat16, 2^-8 of the result.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged_serving as O
from paper_2509_22622_amd import binding as B

pytestmark = pytest.mark.gpu


def normal(shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16).cuda()


def apart(t, extra, fill=math.nan):
    """The same rows, `extra` numbers further apart; between them `fill`."""
    wide = torch.full((t.shape[0], t.shape[1] + extra), fill, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]], wide


def check(m, n, k, bias=True, act="none", residual=True, x_extra=0, y_extra=0, r_extra=0, w_extra=0, seed=0):
    x, w = normal((m, k), seed + 1), normal((n, k), seed + 2, k ** -0.5)
    b = normal((n,), seed + 3) if bias else None
    r = normal((m, n), seed + 4) if residual else None
    want, mag = O.linear(*(None if t is None else t.double().cpu().numpy() for t in (x, w, b)), act, None if r is None else r.double().cpu().numpy())
    layer = B.Linear(apart(w, w_extra)[0])
    y, whole = apart(torch.empty(m, n, dtype=torch.bfloat16, device="cuda"), y_extra, 7.0)
    layer.forward(apart(x, x_extra)[0], y, bias=b, activation=act, residual=None if r is None else apart(r, r_extra)[0])
    torch.cuda.synchronize()
    got = y.double().cpu().numpy()
    tol = 1.13 * (k + 1) * 2.0 ** -24 * mag + 2.0 ** -17 * np.abs(want - (0 if r is None else r.double().cpu().numpy())) + 2.0 ** -8 * np.abs(want) + 1e-30
    err = np.abs(got - want)
    assert np.isfinite(got).all() and (err <= tol).all(), (err / tol).max()
    assert (whole[:, n:] == 7.0).all()
    return layer, x, b, r, y


ROWS = [1, 2, 15, 16, 17, 31, 33, 48, 63, 64, 65, 100, 127, 129, 200, 257, 300]


@pytest.mark.parametrize("m", ROWS)
def test_rows(m):
    check(m, 192, 320, seed=m)


@pytest.mark.parametrize("n", [1, 2, 3, 7, 15, 16, 17, 33, 66, 127, 130, 513])
@pytest.mark.parametrize("m", [5, 40, 130])
def test_features_out(m, n):
    check(m, n, 128, seed=n)


@pytest.mark.parametrize("k", [8, 16, 24, 56, 64, 72, 120, 136, 200, 456, 1000])
@pytest.mark.parametrize("m", [3, 20, 50, 90, 400])
def test_features_in(m, k):
    """A row's end inside a step: what lies behind it (NaN here) is not part of the product."""
    check(m, 80, k, x_extra=8, seed=k)


@pytest.mark.parametrize("act", ["none", "gelu_tanh", "gelu", "silu"])
@pytest.mark.parametrize("m", [1, 24, 60, 140])
def test_activations(m, act):
    check(m, 100, 256, act=act, seed=m)
    check(m, 100, 256, act=act, residual=False, bias=False, seed=m + 1)


@pytest.mark.parametrize("m", [4, 70, 300])
def test_strides(m):
    check(m, 68, 96, x_extra=40, y_extra=12, r_extra=4, w_extra=8)
    check(m, 68, 96, x_extra=8, y_extra=3, r_extra=0)
    check(m, 68, 96, y_extra=4, r_extra=1)
    check(m, 67, 96, y_extra=5, r_extra=1)


@pytest.mark.parametrize("m, n, k", [(4680, 384, 256), (700, 1536, 1536), (2400, 200, 72), (1, 4200, 512), (16, 4100, 1000), (64, 8192, 256), (600, 256, 64), (257, 4111, 136)])
def test_larger(m, n, k):
    check(m, n, k, act="gelu_tanh", seed=9)


@pytest.mark.parametrize("m, n, k", [(3, 33, 840), (3, 33, 72), (1029, 33, 72), (17, 4107, 72), (33, 3001, 456), (4111, 33, 72), (4111, 33, 456), (50, 4107, 456),
                                     (4111, 161, 72), (131, 6149, 200), (131, 8203, 200), (2570, 1537, 72), (1029, 8203, 72)])
def test_each_block_of_outputs(m, n, k):
    """Sizes that select each shape of block (csrc/linear.h), none of them a multiple of it."""
    check(m, n, k, act="silu", x_extra=8, r_extra=3, y_extra=1, seed=5)


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("m, n, k", [(131, 4104, 200), (131, 6152, 456), (131, 8200, 456), (519, 8200, 200), (645, 8200, 200), (1029, 6152, 456), (1601, 8200, 72)])
def test_each_tile_of_aligned_rows(m, n, k, act):
    """Sizes that select each tile of 64 rows and more (csrc/linear.h); rows of y and of the residual are 16-byte aligned, the last tile's columns are some of
    them past the end."""
    check(m, n, k, act=act, seed=6)
    check(m, n, k, act=act, bias=False, residual=False, y_extra=8, seed=7)


@pytest.mark.parametrize("m", [2, 30, 61, 333])
def test_residual_in_place_and_repeats(m):
    layer, x, b, r, y = check(m, 136, 264, seed=m)
    again = torch.empty_like(y)
    layer.forward(x, again, bias=b, residual=r)
    layer.forward(x, r, bias=b, residual=r)
    assert torch.equal(again, y) and torch.equal(r, y)


@pytest.mark.parametrize("m", [3, 40, 150])
def test_numbers_that_are_none(m):
    """NaN and infinities stay in their row (of x) or column (of w), whatever the activation."""
    for act in ("none", "gelu_tanh", "gelu", "silu"):
        x, w = normal((m, 72), 1), normal((50, 72), 2)
        x[1, 70], x[2, 3], w[7, 71] = math.nan, math.inf, math.nan
        y = torch.empty(m, 50, dtype=torch.bfloat16, device="cuda")
        B.Linear(w).forward(x, y, activation=act)
        bad = ~torch.isfinite(y)
        want = torch.zeros_like(bad)
        want[1], want[:, 7] = True, True
        clean = torch.zeros_like(bad)
        clean[2] = True                                          # infinite, or zero where an activation takes minus infinity there
        assert torch.equal(bad[~clean], want[~clean])
        assert torch.isnan(y[1]).all() and torch.isnan(y[:, 7]).all()
        if act == "none":
            assert torch.isinf(y[2, [c for c in range(50) if c != 7]]).all()


def test_far_values_of_the_activations():
    """Very large and very small products: the activations end in x, in 0, and never in NaN."""
    x = torch.tensor([[v] + [0.0] * 7 for v in (-3e38, -1e20, -300.0, -88.0, -20.0, -6.0, -1e-30, 0.0, 1e-30, 6.0, 88.0, 1e20, 3e38)], dtype=torch.bfloat16).cuda()
    w = torch.zeros(4, 8, dtype=torch.bfloat16, device="cuda")
    w[:, 0] = 1.0
    for act in ("gelu_tanh", "gelu", "silu"):
        y = torch.empty(len(x), 4, dtype=torch.bfloat16, device="cuda")
        B.Linear(w).forward(x, y, activation=act)
        v = x[:, 0].double()
        if act == "silu":
            want = v * torch.sigmoid(v)
        elif act == "gelu":
            want = 0.5 * v * torch.special.erfc(-v * math.sqrt(0.5))
        else:
            want = v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
        # fp32 arguments of the exponential: relative error |t| 2^-23 of a result that is itself tiny there
        assert torch.isfinite(y).all()
        assert ((y[:, 0].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -12) + 1e-37).all(), (act, y[:, 0], want)


def test_graph():
    for m in (8, 200):
        layer, x, b, r, y = check(m, 144, 200, act="silu", seed=m)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer.forward(x, y, bias=b, residual=r)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.forward(x, y, bias=b, residual=r)
        for i in range(5):
            x.copy_(normal(x.shape, 50 + i))
            graph.replay()
            want = torch.empty_like(y)
            layer.forward(x, want, bias=b, residual=r)
            torch.cuda.synchronize()
            assert torch.equal(y, want)
