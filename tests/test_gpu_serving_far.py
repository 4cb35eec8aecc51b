"""The serving operators where offsets pass 32 bits: rows as far apart as the calls allow, page tables that are part of a wider one, sequences of millions of
tokens.  Tolerances as derived in test_gpu_paged.py and test_gpu_linear.py."""
import math

import pytest
import torch

from paper_2509_22622_amd import binding as B

from test_gpu_linear import check
from test_gpu_paged import Batch, check_append, check_attn, fill, natural, normal, poison_unused

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n, k", [(33, 72), (200, 136), (4107, 72)])
def test_linear_rows_far_apart(n, k):
    """Rows of x, y and the residual 2^21 numbers apart, the most that is allowed: the last of 1100 lie 4.6 GB behind the first."""
    far = 1 << 21
    check(1100, n, k, act="silu", x_extra=far - k, y_extra=far - n, r_extra=far - n, seed=3)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fmt, d", [("bf16", 128), ("fp8_e4m3", 64)])
def test_paged_rows_far_apart(fmt, d):
    """Rows of q, k, v and of the outputs 2^26 numbers apart, and a page table whose rows are part of longer ones."""
    b = Batch([60, 17, 200], [30, 3, 7], 32, 4, extra_rows=2)
    cache = B.PagedCache(1, 6, 2, d, 32, b.n_pages, rope="halves", kv_format=fmt)
    cache.k_exp = cache.v_exp = 0
    wide = torch.zeros(b.rows, 1 << 26, dtype=torch.bfloat16, device="cuda")
    parts = [wide[:, at:at + h * d].unflatten(1, (h, d)) for at, h in ((8, 6), (1 << 12, 2), (1 << 13, 2), (1 << 14, 6), (1 << 15, 6))]
    q, k, v, q_out, out = parts
    for i, t in enumerate((q, k, v)):
        t.copy_(normal(t.shape, i + 1))
    table, device = torch.full((3, b.table.shape[1] + 9), 2 ** 31 - 1, dtype=torch.int32, device="cuda"), b.device()
    table[:, 4:4 + b.table.shape[1]] = device["page_table"]
    device["page_table"] = table[:, 4:4 + b.table.shape[1]]
    assert q.stride(0) == 1 << 26 and not device["page_table"].is_contiguous()
    b.device = lambda: device
    check_append(cache, b, q, k, v, q_out, rope="halves", rope_dim=d, theta=10000.0)
    fill(cache, 6)
    poison_unused(cache, b)
    q.mul_(math.log2(math.e) / math.sqrt(d))
    check_attn(cache, b, q, out, max_new=30, max_len=200)
    del wide, parts, q, k, v, q_out, out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fmt, d, length", [("bf16", 128, 1 << 24), ("fp8_e4m3", 64, (1 << 25) + 16 * 1024)])
def test_attn_millions_of_tokens(fmt, d, length):
    """16 pages of 1024 tokens, again and again: every key counts as often as any other, and the result is that of the pages once.
    An fp32 sum takes in 32 (64) keys a step: at head_dim 128 2^24 / 32 steps over 256 workgroups of four waves, 512 a wave; at 64 the same.  A step's product
    rounds 32 (64) times at most, so that sums are off by at most 2^15 * 2^-24 of the sum of |weight * value| if all fall one way; at random, as here, by the
    root of that many: 2^-16, and the weights' sum as much; 2^-13 is asked for."""
    page, n_pages, hq = 1024, 16, 4
    cache = B.PagedCache(1, hq, 1, d, page, n_pages, kv_format=fmt)
    fill(cache, 3)
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda").repeat(-(-length // (page * n_pages)))[None].contiguous()
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    q = normal((1, hq, d), 4, 2 * math.log2(math.e) / math.sqrt(d))
    out, ws = torch.empty_like(q), cache.attn_workspace(1, max_len=length)
    assert ws.numel() > 0
    cache.attn(0, lens, table, q, out, ws, max_len=length)
    keys, values = (natural(cache, i).double().reshape(-1, d) if fmt == "bf16" else natural(cache, i).float().double().reshape(-1, d) for i in (False, True))
    score = q[0].double() @ keys.t()
    big = (q[0].double().abs() @ keys.abs().t()).amax(-1, keepdim=True)
    weight = torch.softmax(score * math.log(2), -1)
    want, mag = weight @ values, weight @ values.abs()
    tol = mag * (2.0 ** -8 + 2 * math.log(2) * d * 2.0 ** -24 * big + 2.0 ** -13) + want.abs() * 2.0 ** -8
    assert ((out[0].double() - want).abs() <= tol).all(), ((out[0].double() - want).abs() / tol).max()


def test_attn_window_far_out():
    """A window at the end of 2^24 tokens and a sink at their beginning: only those tokens, whatever lies between (pages that are none)."""
    page, length, sink, window = 16, 1 << 24, 40, 100
    cols = length // page
    cache = B.PagedCache(1, 4, 2, 128, page, 12)
    fill(cache, 8)
    table = torch.full((1, cols), -1, dtype=torch.int32, device="cuda")
    table[0, :3], table[0, -7:] = torch.arange(3, device="cuda").int(), torch.arange(4, 11, device="cuda").int()
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    q = normal((1, 4, 128), 4, math.log2(math.e) / math.sqrt(128))
    out = torch.empty_like(q)
    kw = {"max_len": length, "sink_tokens": sink, "window_tokens": window}
    cache.attn(0, lens, table, q, out, cache.attn_workspace(1, **kw), **kw)
    keys, values = (natural(cache, i).double() for i in (False, True))
    near = [t.flatten(0, 1) for t in (keys, values)]
    at = torch.tensor(list(range(sink)) + list(range(11 * page - window, 11 * page)), device="cuda")
    for h in range(4):
        k, v = near[0][at, h // 2], near[1][at, h // 2]
        w = torch.softmax(k @ q[0, h].double() * math.log(2), -1)
        big, mag, want = (k.abs() @ q[0, h].double().abs()).max(), w @ v.abs(), w @ v
        tol = mag * (2.0 ** -8 + 2 * math.log(2) * 128 * 2.0 ** -24 * big + 2.0 ** -20) + want.abs() * 2.0 ** -8
        assert ((out[0, h].double() - want).abs() <= tol).all()
