"""ll_layer_norm and ll_layer_norm_backward on the GPU against the fp64 oracle (oracle/norm_and_encoder.py, which derives the tolerances)."""
import math

import numpy as np
import pytest
import torch

from oracle import norm_and_encoder as O
from paper_2509_22622_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def normal(shape, seed, dtype=BF16, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std + mean).to(dtype).cuda()


def apart(t, extra, shift=0, fill=math.nan):
    """The same rows, `extra` numbers further apart and `shift` numbers into their row; between them `fill`."""
    if extra == 0 and shift == 0:
        return t, t
    wide = torch.full((t.shape[0], shift + t.shape[1] + extra), fill, dtype=t.dtype, device=t.device)
    wide[:, shift:shift + t.shape[1]] = t
    return wide[:, shift:shift + t.shape[1]], wide


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def near(got, want, what):
    err = np.abs(f64(got) - want[0])
    assert np.isfinite(f64(got)).all() and (err <= want[1]).all(), (what, (err / want[1]).max())


def check(m, n, xt=BF16, yt=BF16, wt=BF16, weight=True, bias=True, group=0, residual=False, extra=0, shift=0, eps=1e-5, mean=0.3, std=1.5, seed=0, back=True):
    groups = -(-m // group) if group else 1
    x, dy = normal((m, n), seed + 1, xt, std, mean), normal((m, n), seed + 2, yt)
    w = normal((groups, n), seed + 3, wt, 0.3, 1.0) if weight else None
    b = normal((groups, n), seed + 4, wt, 0.3) if bias else None
    res = normal((m, n), seed + 5, xt) if residual else None
    norm = B.LayerNorm(n, eps)
    (want, stats_want) = O.norm(f64(x), f64(w), f64(b), eps, group, STEP[yt])
    y, y_all = apart(torch.zeros(m, n, dtype=yt, device="cuda"), extra, shift, 7.0)
    xs = apart(x, extra, shift)[0]
    stats = torch.empty(m, 2, device="cuda")
    norm.forward(xs, y, weight=w, bias=b, group_rows=group, stats=stats)
    torch.cuda.synchronize()
    near(y, want, "y")
    outside = torch.ones_like(y_all, dtype=torch.bool)
    outside[:, shift:shift + n] = False
    assert (y_all[outside] == 7.0).all()
    absolute = np.abs(f64(x)).mean(1)
    assert (np.abs(f64(stats[:, 0]) - stats_want[0]) <= 66 * O.U * absolute + 1e-38).all()
    assert (np.abs(f64(stats[:, 1]) - stats_want[1]) <= stats_want[1] * (64 * O.U + (66 * O.U * absolute * stats_want[1]) ** 2)).all()
    if not back:
        return
    want_dx, want_dw, want_db = O.norm_backward(f64(dy), f64(x), f64(w), eps, group, f64(res), STEP[xt])
    dx, dx_all = apart(torch.zeros(m, n, dtype=xt, device="cuda"), extra, shift, 7.0)
    dw, db = torch.full((groups, n), 9.0, device="cuda"), torch.full((groups, n), 9.0, device="cuda")
    ws = norm.backward_workspace(m, group)
    norm.backward(apart(dy, extra, shift)[0], xs, stats, dx, weight=w, dweight=dw, dbias=db, group_rows=group, residual=None if res is None else apart(res, extra, shift)[0], workspace=ws)
    torch.cuda.synchronize()
    near(dx, want_dx, "dx")
    near(dw, want_dw, "dweight")
    near(db, want_db, "dbias")
    assert dx_all is dx or (dx_all[outside] == 7.0).all()


# every shape of rows (csrc/layer_norm.h), at its ends
WIDTHS = [1, 2, 7, 8, 9, 64, 127, 128, 129, 250, 256, 264, 511, 512, 520, 1000, 1024, 1032, 1536, 1537, 2000, 2048, 2056, 4096, 4097, 6144, 6152, 8191, 8192, 8200, 12288,
          12296, 16000, 16383, 16384]


@pytest.mark.parametrize("n", WIDTHS)
def test_widths(n):
    check(5, n, residual=True, seed=n)
    check(19, n, F32, F32, F32, seed=n)


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 15, 16, 17, 63, 65, 333, 1025, 2049, 4500])
@pytest.mark.parametrize("n", [72, 700])
def test_rows(m, n):
    check(m, n, F32, BF16, residual=True, seed=m)


@pytest.mark.parametrize("xt, yt", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("wt", [BF16, F32])
@pytest.mark.parametrize("n", [40, 333, 1536, 2500, 9000])
def test_types(n, wt, xt, yt):
    check(37, n, xt, yt, wt, residual=True, seed=1)
    check(6, n, xt, yt, wt, weight=False, bias=False, seed=2)
    check(6, n, xt, yt, wt, bias=False, seed=3)
    check(6, n, xt, yt, wt, weight=False, seed=4)


@pytest.mark.parametrize("m, group", [(1, 1), (7, 1), (40, 3), (100, 50), (101, 50), (99, 50), (50, 100), (1500, 7), (4000, 1999), (6000, 1560), (2100, 2)])
@pytest.mark.parametrize("n", [96, 1040])
def test_groups(m, group, n):
    check(m, n, group=group, residual=True, seed=m)


@pytest.mark.parametrize("extra, shift", [(8, 0), (8, 8), (5, 0), (3, 1), (16, 3), (0, 1)])
@pytest.mark.parametrize("n", [64, 61, 1536, 2321, 8200])
def test_strides(n, extra, shift):
    check(21, n, residual=True, extra=extra, shift=shift)
    check(6, n, F32, BF16, F32, residual=True, extra=extra, shift=shift)


def test_levels():
    """Rows whose mean is far from 0, whose variance is nothing, and the smallest and largest eps."""
    check(20, 1536, F32, F32, F32, mean=1000.0, std=1.0)
    check(20, 100, F32, F32, F32, mean=-3e4, std=1e-2)
    check(20, 100, F32, F32, F32, std=1e-12, mean=0.0, eps=1e-12)
    check(20, 2500, F32, F32, F32, std=1e15, mean=0.0)
    check(20, 2500, std=0.0, mean=3.0, residual=True)
    check(20, 96, std=0.0, mean=0.0, eps=1e-30)
    check(20, 96, eps=100.0)


@pytest.mark.parametrize("n", [48, 1000, 3000])
def test_in_place(n):
    """y over x; dx over dy, over x and over the residual: the same numbers."""
    m = 70
    norm, x, dy, res = B.LayerNorm(n), normal((m, n), 1), normal((m, n), 2), normal((m, n), 3)
    w = normal((n,), 4)
    y, stats = torch.empty_like(x), torch.empty(m, 2, device="cuda")
    norm.forward(x, y, weight=w, stats=stats)
    over = x.clone()
    norm.forward(over, over, weight=w)
    assert torch.equal(over, y)
    ws = norm.backward_workspace(m)
    dx, dw, db = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    norm.backward(dy, x, stats, dx, weight=w, dweight=dw, dbias=db, residual=res, workspace=ws)
    for i in range(3):
        a = [dy.clone(), x.clone(), res.clone()]
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        norm.backward(a[0], a[1], stats, a[i], weight=w, dweight=dw2, dbias=db2, residual=a[2], workspace=ws)
        assert torch.equal(a[i], dx) and torch.equal(dw2, dw) and torch.equal(db2, db), i


def test_parts_and_repeats():
    """Gradients one by one are those of one call, without a workspace where none is needed; a call repeated gives the same bits."""
    m, n = 3000, 1000
    norm, x, dy, w = B.LayerNorm(n), normal((m, n), 1), normal((m, n), 2), normal((n,), 4)
    stats, y = torch.empty(m, 2, device="cuda"), torch.empty_like(x)
    norm.forward(x, y, weight=w, stats=stats)
    ws = norm.backward_workspace(m)
    dx, dw, db = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    norm.backward(dy, x, stats, dx, weight=w, dweight=dw, dbias=db, workspace=ws)
    one = [torch.empty_like(t) for t in (dx, dw, db)]
    norm.backward(dy, x, stats, one[0], weight=w)
    assert torch.equal(one[0], dx)
    norm.backward(dy, x, stats, one[0], weight=w, dweight=one[1], workspace=ws)
    norm.backward(dy, x, stats, one[0], weight=w, dbias=one[2], workspace=ws)
    assert torch.equal(one[1], dw) and torch.equal(one[2], db)
    for _ in range(3):
        again = [torch.empty_like(t) for t in (dx, dw, db)]
        norm.backward(dy, x, stats, again[0], weight=w, dweight=again[1], dbias=again[2], workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))


def test_no_rows():
    norm = B.LayerNorm(64)
    none, dw, db = torch.empty(0, 64, dtype=BF16, device="cuda"), torch.full((64,), 5.0, device="cuda"), torch.full((64,), 5.0, device="cuda")
    stats = torch.empty(0, 2, device="cuda")
    norm.forward(none, none.clone(), weight=torch.ones(64, device="cuda"), stats=stats)
    norm.backward(none, none.clone(), stats, none.clone(), dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()
    norm.backward(none, none.clone(), stats, none.clone(), dweight=torch.empty(0, 64, device="cuda"), group_rows=3)


def test_numbers_that_are_none():
    """NaN and infinities stay in their row, and reach the weight's gradient only in columns that hold them there."""
    for m, n in ((40, 100), (40, 1536), (9, 5000)):
        x, dy = normal((m, n), 1), normal((m, n), 2)
        x[3, n - 1], x[5, 0] = math.nan, math.inf
        norm, y, stats = B.LayerNorm(n), torch.empty_like(x), torch.empty(m, 2, device="cuda")
        norm.forward(x, y, stats=stats)
        bad = ~torch.isfinite(y)
        assert bad[3].all() and bad[5].all() and not bad[[r for r in range(m) if r not in (3, 5)]].any()
        dy[7, 2] = math.inf
        dx = torch.empty_like(x)
        norm.backward(dy, x, stats, dx)
        assert torch.isfinite(dx[[r for r in range(m) if r not in (3, 5, 7)]]).all()


def test_differences():
    """The gradients against differences of the forward pass in 32 bits: (f(t + e) - f(t - e)) / 2 e of f = sum(y dy), off by e^2 and by the sum's rounding."""
    m, n, e = 3, 24, 2.0 ** -6
    norm = B.LayerNorm(n)
    x, dy, w, b = normal((m, n), 1, F32), normal((m, n), 2, F32), normal((n,), 3, F32), normal((n,), 4, F32)

    def f(x, w, b):
        y = torch.empty_like(x)
        norm.forward(x, y, weight=w, bias=b)
        return (y.double() * dy.double()).sum().item()

    y, stats, dx, dw, db = torch.empty_like(x), torch.empty(m, 2, device="cuda"), torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    norm.forward(x, y, weight=w, bias=b, stats=stats)
    norm.backward(dy, x, stats, dx, weight=w, dweight=dw, dbias=db, workspace=norm.backward_workspace(m))
    for t, g in ((x, dx), (w, dw), (b, db)):
        flat, grad = t.view(-1), g.view(-1)
        for i in range(0, flat.numel(), 5):
            old = flat[i].item()
            flat[i] = old + e
            up = f(x, w, b)
            flat[i] = old - e
            down = f(x, w, b)
            flat[i] = old
            assert abs((up - down) / (2 * e) - grad[i].item()) <= 20 * e * e + 2.0 ** -24 * 200 / e, (i, (up - down) / (2 * e), grad[i].item())


def test_graph_and_streams():
    m, n = 300, 1536
    norm, x, dy, w, b = B.LayerNorm(n), normal((m, n), 1), normal((m, n), 2), normal((3, n), 3), normal((3, n), 4)

    def step(ws, out):
        norm.forward(x, out[0], weight=w, bias=b, group_rows=100, stats=out[1])
        norm.backward(dy, x, out[1], out[2], weight=w, dweight=out[3], dbias=out[4], group_rows=100, residual=dy, workspace=ws)

    make = lambda: [torch.empty_like(x), torch.empty(m, 2, device="cuda"), torch.empty_like(x), torch.empty(3, n, device="cuda"), torch.empty(3, n, device="cuda")]
    ws, out = norm.backward_workspace(m, 100), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(ws, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ws, out)
    for i in range(5):
        x.copy_(normal((m, n), 50 + i))
        graph.replay()
        want = make()
        step(norm.backward_workspace(m, 100), want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, want)), i


@pytest.mark.parametrize("n", [100, 700, 5000])
def test_far_rows(n):
    """Rows 2^21 numbers apart, all of a call's tensors side by side in one array of 2.3e9 numbers: the same bits as without gaps."""
    m, far = 1100, 1 << 21
    base = torch.empty(m * far, dtype=BF16, device="cuda")
    norm, w, b = B.LayerNorm(n), normal((n,), 3), normal((n,), 4)
    x, dy, res, results = normal((m, n), 1), normal((m, n), 2), normal((m, n), 5), []
    for make in (lambda i: torch.empty(m, n, dtype=BF16, device="cuda"), lambda i: base.as_strided((m, n), (far, 1), i * n)):
        xs, dys, rs, y, dx = make(0).copy_(x), make(1).copy_(dy), make(2).copy_(res), make(3), make(4)
        stats, dw, db = torch.empty(m, 2, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        norm.forward(xs, y, weight=w, bias=b, stats=stats)
        norm.backward(dys, xs, stats, dx, weight=w, dweight=dw, dbias=db, residual=rs, workspace=norm.backward_workspace(m))
        torch.cuda.synchronize()
        results.append((y, stats, dx, dw, db))
    assert all(torch.equal(a, c) for a, c in zip(*results))


def test_many_rows_and_groups():
    """More groups than workgroups, each of one row, and rows of a few numbers; sums by torch in 64 bits."""
    for m, n, group in ((1 << 21, 3, 1), (3_000_000, 5, 0), (1_100_000, 16, 2)):
        groups = -(-m // group) if group else 1
        x, dy, w = normal((m, n), 1), normal((m, n), 2), normal((groups, n), 3)
        norm, y, dx, stats = B.LayerNorm(n, 1e-3), torch.empty_like(x), torch.empty_like(x), torch.empty(m, 2, device="cuda")
        dw, db = torch.empty(groups, n, device="cuda"), torch.empty(groups, n, device="cuda")
        norm.forward(x, y, weight=w, group_rows=group, stats=stats)
        norm.backward(dy, x, stats, dx, weight=w, dweight=dw, dbias=db, group_rows=group, workspace=norm.backward_workspace(m, group))
        torch.cuda.synchronize()
        rows = torch.arange(m, device="cuda") // (group or m)
        xd, mean = x.double(), x.double().mean(1, keepdim=True)
        h = (xd - mean) / (((xd - mean) ** 2).mean(1, keepdim=True) + 1e-3).sqrt()
        want = h * w.double()[rows]
        # The mean of up to 16 numbers is a sum in at most 12 steps and a quotient, off by 13 x 2^-24 |x|; times rstd <= 1 / sqrt(1e-3), once in x - mean and |h| <= 4 times in
        # rstd: 1.3e-4 |x|.  y is rounded to bfloat16 besides.
        off = 1.3e-4 * xd.abs().amax(1, keepdim=True) + 70 * 2.0 ** -24 * h.abs()
        assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * off * w.double()[rows].abs() + 1e-38).all(), (m, n)
        for got, terms, slack in ((dw, dy.double() * h, dy.double().abs() * off), (db, dy.double(), torch.zeros_like(h))):
            add = lambda t: torch.zeros(groups, n, dtype=torch.float64, device="cuda").index_add_(0, rows, t) if group else t.sum(0, keepdim=True)
            total = add(terms)
            # a sum's depth: a row a round and team, 16 teams and up to 1024 chunks in strands of 128, less than sqrt(rows) + 30
            much = add(terms.abs() * ((group or m) ** 0.5 + 30) * 2.0 ** -24 + slack)
            assert ((got.double() - total).abs() <= much + 1e-38).all(), (m, n)
