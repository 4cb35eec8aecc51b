"""ll_layer_norm and ll_layer_norm_backward at the limits of 32 bits: rows of finite numbers whose sum, whose squares or whose differences from the mean pass 3.4e38."""
import numpy as np
import pytest
import torch

from oracle import norm_and_encoder as O
from paper_2509_22622_amd import binding as B
from test_gpu_layer_norm import BF16, F32, STEP, f64, near, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("xt, yt", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("n, extra", [(100, 0), (200, 0), (1536, 0), (1536, 3), (8192, 0), (9000, 0)])
def test_large_rows(n, extra, xt, yt):
    """Rows whose sum of squared differences is above 3.4e38 come out as the bias, with dx the residual and nothing for dweight; those a little below it as ever."""
    i = torch.arange(n)
    sign = torch.where(i % 2 == 0, 1.0, -1.0)
    most = (2.0 ** 128 / n) ** 0.5                           # in every place: the squares add up to 2^128
    large = [sign * (1.1 * most), sign * 1e36, torch.full((n,), 1e36) + sign * 1e35, torch.where(i == 5, 3.2e38, 3.3e38), torch.where(i % 2 == 0, 3e38, 2e38), sign * 3.3e38,
             torch.where(i < n // 2, 3.3e38, -3.3e38), torch.where(i == n // 3, -3.3e38, 3.3e38), torch.where(i == n - 1, 3.3e38, 0.0)]
    fine = [sign * (0.9 * most), sign * 1e15 + 3e15]
    g = torch.Generator().manual_seed(n)
    rows = [r for pair in zip(large, [torch.randn(n, generator=g) for _ in large]) for r in pair] + fine * 3
    x = torch.zeros(len(rows), n + extra, dtype=xt, device="cuda")[:, :n]
    x.copy_(torch.stack(rows).to(xt))
    m, out = len(rows), np.array([i < 2 * len(large) and i % 2 == 0 for i in range(len(rows))])
    dy, w, b, res = normal((m, n), 2, yt), normal((n,), 3, F32, 0.3, 1.0), normal((n,), 4, F32, 0.3), normal((m, n), 5, xt)
    norm, y, stats = B.LayerNorm(n), torch.empty(m, n, dtype=yt, device="cuda"), torch.empty(m, 2, device="cuda")
    norm.forward(x, y, weight=w, bias=b, stats=stats)
    dx, dw, db = torch.empty(m, n, dtype=xt, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    norm.backward(dy, x, stats, dx, weight=w, dweight=dw, dbias=db, residual=res, workspace=norm.backward_workspace(m))
    torch.cuda.synchronize()
    wide = f64(x)
    assert (np.abs(f64(stats[:, 0]) - wide.mean(1)) <= 66 * O.U * np.abs(wide).mean(1) + 1e-38).all(), stats[:, 0]
    assert (f64(stats[:, 1])[out] == 0).all(), stats[:, 1]
    assert (y[out] == b.to(yt)).all()
    assert torch.equal(dx[out], res[out])
    kept = ~out
    pick = lambda t: f64(t)[kept]
    (want, _) = O.norm(pick(x), f64(w)[None], f64(b)[None], 1e-5, 0, STEP[yt])
    near(y[kept], want, "y")
    want_dx, want_dw, _ = O.norm_backward(pick(dy), pick(x), f64(w)[None], 1e-5, 0, pick(res), STEP[xt])
    near(dx[kept], want_dx, "dx")
    near(dw[None], (want_dw[0], want_dw[1] + (m + 20) * O.U * np.abs(want_dw[0])), "dweight")
    assert (np.abs(f64(db) - f64(dy).sum(0)) <= (m + 20) * O.U * np.abs(f64(dy)).sum(0)).all()


def test_infinities_still_show():
    """An infinity or NaN among a row's numbers leaves no number in that row, nor one that looks like a row out of range."""
    x = torch.ones(5, 1536, dtype=BF16, device="cuda")
    x[0, 7], x[1, 7], x[2, 3], x[2, 900], x[3, 1535] = torch.inf, -torch.inf, torch.inf, -torch.inf, torch.nan
    norm, y, stats = B.LayerNorm(1536), torch.empty_like(x), torch.empty(5, 2, device="cuda")
    norm.forward(x, y, stats=stats)
    assert torch.isnan(y[:4]).all() and torch.isnan(stats[:4, 1]).all() and (y[4] == 0).all()
