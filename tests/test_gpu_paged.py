"""The paged cache on the GPU: ll_paged_append and ll_paged_attn against the fp64 oracle (oracle/paged_serving.py).

Tolerances.  A rounding to bfloat16 is off by at most 2^-8 of the value, one to E4M3 by 2^-4 of it (2^-10 below the normal numbers).
Appended keys and queries: one rounding of a value computed in fp32 from an angle good to 2^-23 of a circle's radian (6e-7 of the pair's
length, with 2e-6 to spare); values: none in bfloat16.
Attention, from the stored bits: the weights' rounding moves the output by at most 2^-8 of sum |w v| / sum w, the output's by 2^-8 of itself;
the scores are fp32 sums of D products, off by at most D 2^-24 times sum |q_d k_d|, which moves each weight by ln 2 times that, once up
and once in the sum; 2^-20 covers the exponentials and the fp32 sums over the keys.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged_serving as O
from oracle.fp8_cache import e4m3_table
from paper_2509_22622_amd import binding as B

pytestmark = pytest.mark.gpu
CODES = e4m3_table()


def f64(t):
    if t.dtype == torch.float8_e4m3fn:
        return CODES[t.contiguous().view(torch.uint8).cpu().numpy()]
    return t.to(torch.float64).cpu().numpy()


class Batch:
    """A batch of sequences over a pool: lengths, rows, a page table whose pages lie in a random order."""

    def __init__(self, lens, news, page, seed, spare=3, cu=None, extra_rows=0, extra_cols=1):
        rng = np.random.default_rng(seed)
        self.lens, self.page = list(lens), page
        need = [-(-max(n, 0) // page) for n in lens]
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        cols = max(need) + extra_cols
        self.table = np.full((len(lens), cols), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.unused = order[at:]
        self.cu = None if news is None else np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        if cu is not None:
            self.cu = np.array(cu, dtype=np.int32)
        self.rows = (len(lens) if self.cu is None else int(self.cu[-1])) + extra_rows

    def device(self):
        put = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
        return {"seq_lens": put(self.lens), "page_table": put(self.table), "cu_tokens": put(self.cu)}


def normal(shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16).cuda()


def natural(cache, values):
    x = (cache.values(0) if values else cache.keys(0))
    codes = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
    return codes.reshape(cache.n_pages, cache.page_tokens, cache.kv_heads, cache.head_dim).contiguous().view(x.dtype)


def fill(cache, seed):
    """Random numbers everywhere in layer 0."""
    shape = (cache.n_pages, cache.page_tokens, cache.kv_heads, cache.head_dim)
    for i, view in enumerate((cache.keys(0), cache.values(0))):
        x = normal(shape, seed + i)
        if view.dtype == torch.float8_e4m3fn:
            view.view(torch.uint8).copy_(x.to(torch.float8_e4m3fn).view(torch.uint8).view(view.shape))
        else:
            view.copy_(x.view(view.shape))


# ---- append ------------------------------------------------------------------------------------------------------

def check_append(cache, b, q, k, v, q_out, positions=None, **rope):
    """One append into a pool of known numbers: what it stores, and that it leaves everything else alone."""
    fill(cache, 77)
    before = [natural(cache, i) for i in (False, True)]
    q_out.fill_(7.0)
    cache.append(0, k=k, v=v, q=q, q_out=q_out, positions=None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda"), **b.device())
    torch.cuda.synchronize()
    stored, queries = O.appended(b.lens, b.cu, b.table, b.n_pages, b.page, f64(q), f64(k), f64(v), positions=positions, **rope)
    after = [natural(cache, i) for i in (False, True)]
    touched = torch.zeros(b.n_pages, b.page, dtype=torch.bool)
    for (page, t), _ in stored.items():
        touched[page, t] = True
    for x, y in zip(before, after):
        bits = torch.uint8 if x.dtype == torch.float8_e4m3fn else torch.int16
        keep = ~touched.cuda()
        assert torch.equal(x.view(bits)[keep], y.view(bits)[keep]), "a slot that is none of the call's has changed"
    keys, values = (f64(x) for x in after)
    slots = list(stored)
    if slots:
        at = tuple(np.array(x) for x in zip(*slots))
        want_k, want_v = (np.stack([stored[s][i] for s in slots]) for i in (0, 1))
        if cache.kv_format == "bf16":
            assert np.array_equal(values[at], want_v)
            err = np.abs(keys[at] - want_k)
            assert (err <= np.abs(want_k) * 2.0 ** -8 + 2e-6).all(), err.max()
        else:
            for got, want, slack in ((keys[at], want_k * 2.0 ** -cache.k_exp, 2e-6 * 2.0 ** -cache.k_exp), (values[at], want_v * 2.0 ** -cache.v_exp, 0.0)):
                want = np.clip(want, -448.0, 448.0)
                err = np.abs(got - want)
                assert (err <= np.maximum(np.abs(want) * 2.0 ** -4, 2.0 ** -10) + slack).all(), err.max()
    got = f64(q_out)
    for r in range(len(got)):
        if r in queries:
            err = np.abs(got[r] - queries[r])
            assert (err <= np.abs(queries[r]) * 2.0 ** -8 + 2e-6).all(), (r, err.max())
        else:
            assert (got[r] == 7.0).all(), f"row {r} is none of the call's"


APPENDS = [
    # fmt, D, q heads, kv heads, page, rope, rope_dim, lens, news (None: one each)
    ("bf16", 64, 4, 4, 16, "pairs", 64, [1, 17, 40], None),
    ("bf16", 128, 8, 2, 32, "halves", 128, [1, 5, 16, 33, 0, 100, 31, 32], None),
    ("bf16", 128, 3, 1, 48, "halves", 64, [70, 3, 50], [70, 2, 9]),
    ("bf16", 64, 5, 5, 16, "halves", 32, [130, 7, 64], [65, 0, 64]),
    ("bf16", 128, 2, 2, 64, "none", 0, [40, 90], [1, 90]),
    ("bf16", 128, 12, 12, 16, "grid", 128, [100, 37], [33, 37]),
    ("bf16", 64, 6, 3, 32, "grid", 64, [61], [61]),
    ("fp8_e4m3", 128, 8, 2, 16, "halves", 128, [1, 2, 3, 4, 5, 6, 7, 64, 65], None),
    ("fp8_e4m3", 64, 4, 4, 32, "pairs", 16, [200, 3, 35], [129, 3, 33]),
    ("fp8_e4m3", 128, 5, 5, 48, "grid", 128, [97], [97]),
    ("fp8_e4m3", 64, 7, 7, 16, "none", 0, [18, 1], [18, 1]),
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append(case):
    fmt, d, hq, hkv, page, rope, rope_dim, lens, news = APPENDS[case]
    b = Batch(lens, news, page, case, extra_rows=0 if news is None else 5)
    exps = {"k_exp": -2, "v_exp": 1} if fmt != "bf16" else {}
    cache = B.PagedCache(1, hq, hkv, d, page, b.n_pages, rope=rope, rope_dim=rope_dim, kv_format=fmt, **exps)
    cache.k_exp, cache.v_exp = exps.get("k_exp", 0), exps.get("v_exp", 0)
    qkv = normal((b.rows, (hq + 2 * hkv) * d), 100 + case, 3.0)         # q, k, v side by side: rows further apart than they are long
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], 1))
    positions = np.stack([np.arange(b.rows) % 7 + 40, np.arange(b.rows) % 30, np.arange(b.rows) % 52], 1) if rope == "grid" else None
    check_append(cache, b, q, k, v, torch.empty(b.rows, hq, d, dtype=torch.bfloat16, device="cuda"), positions, rope=rope, rope_dim=rope_dim, theta=10000.0)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_append_pages_and_lengths_that_are_none(fmt):
    """Pages outside the pool, places behind the table and before the sequence, offsets that skip rows: those tokens are left out."""
    b = Batch([60, 30, 2, 500, -5, 20], None, 16, 5, cu=[3, 43, 43, 48, 50, 51, 60], extra_rows=4, extra_cols=0)
    b.table[0, 2] = b.n_pages
    b.table[0, 1] = -1
    b.table[5, 0] = np.iinfo(np.int32).max
    b.table[5, 1] = np.iinfo(np.int32).min
    cache = B.PagedCache(1, 4, 2, 64, 16, b.n_pages, rope="halves", rope_dim=64, kv_format=fmt)
    cache.k_exp = cache.v_exp = 0
    q, k, v = normal((b.rows, 4, 64), 1), normal((b.rows, 2, 64), 2), normal((b.rows, 2, 64), 3)
    check_append(cache, b, q, k, v, torch.empty_like(q), rope="halves", rope_dim=64, theta=10000.0)


def test_append_positions_far_out():
    """Positions given by the caller, up to the last 32-bit one: the angles are taken in double."""
    b = Batch([64], [64], 16, 2)
    cache = B.PagedCache(1, 2, 2, 128, 16, b.n_pages, rope="halves", rope_theta=1e6)
    cache.k_exp = cache.v_exp = 0
    positions = np.concatenate([np.arange(40) * 524287, [2 ** 31 - 1, 2 ** 24 + 1, -1, -2 ** 31], np.arange(20) + 10 ** 6])
    q, k, v = (normal((64, 2, 128), s) for s in (1, 2, 3))
    check_append(cache, b, q, k, v, torch.empty_like(q), positions, rope="halves", rope_dim=128, theta=1e6)


def test_append_in_place_keys_only_and_odd_numbers():
    """q_out over q gives the same bits; without queries the cache is the same; infinities and NaN are stored as such (8 bits: clamped, and NaN)."""
    for fmt in ("bf16", "fp8_e4m3"):
        b = Batch([70, 3, 19], [37, 3, 2], 32, 3)
        caches = [B.PagedCache(1, 4, 2, 128, 32, b.n_pages, rope="pairs", kv_format=fmt) for _ in range(3)]
        q, k, v = normal((b.rows, 4, 128), 1), normal((b.rows, 2, 128), 2), normal((b.rows, 2, 128), 3)
        k[4, 1, 6], v[5, 0, 3], v[6, 1, 9], v[7, 1, 8] = math.nan, math.inf, -math.inf, math.nan
        out = torch.empty_like(q)
        caches[0].append(0, k=k, v=v, q=q, q_out=out, **b.device())
        same = q.clone()
        caches[1].append(0, k=k, v=v, q=same, q_out=same, **b.device())
        caches[2].append(0, k=k, v=v, **b.device())
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), same.view(torch.int16))
        assert torch.equal(caches[0].buffer, caches[1].buffer) and torch.equal(caches[0].buffer, caches[2].buffer)
        rows, keys, values = O.rows_of(b.lens, b.cu, b.rows), f64(natural(caches[0], False)), f64(natural(caches[0], True))
        at = [O.slot(b.table, b.n_pages, 32, *r) for r in rows]
        assert np.isnan(keys[at[4]][1, 6:8]).all() and np.isnan(keys[at[4]]).sum() == 2
        top = math.inf if fmt == "bf16" else 448.0
        assert values[at[5]][0, 3] == top and values[at[6]][1, 9] == -top and np.isnan(values[at[7]][1, 8])


# ---- attention ---------------------------------------------------------------------------------------------------

def check_attn(cache, b, q, out, sink=0, window=0, max_new=1, max_len=None):
    keys, values = (f64(natural(cache, i)) for i in (False, True))
    keys, values = np.nan_to_num(keys * 2.0 ** cache.k_exp), np.nan_to_num(values * 2.0 ** cache.v_exp)
    kw = {"max_new": max_new, "max_len": max_len, "sink_tokens": sink, "window_tokens": window}
    out.fill_(7.0)
    ws = cache.attn_workspace(len(b.lens), **kw)
    ws.fill_(0xFF)                                               # NaN: what no workgroup of this call has written must not be read
    cache.attn(0, q=q, out=out, workspace=ws, **kw, **b.device())
    torch.cuda.synchronize()
    want = O.attended(b.lens, b.cu, b.table, b.page, f64(q), keys, values, sink, window, max_new)
    got, d = f64(out), q.shape[-1]
    for r in range(len(got)):
        if r not in want:
            assert (got[r] == 7.0).all(), f"row {r} is none of the call's"
            continue
        o, mag, big = want[r]
        tol = mag * (2.0 ** -8 + 2 * math.log(2) * d * 2.0 ** -24 * big[:, None] + 2.0 ** -20) + np.abs(o) * 2.0 ** -8 + 1e-30
        err = np.abs(got[r] - o)
        assert np.isfinite(got[r]).all() and (err <= tol).all(), (r, (err / tol).max())


def poison_unused(cache, b):
    """NaN wherever no sequence has a token: behind the lengths and in pages of no sequence."""
    keep = torch.zeros(b.n_pages, b.page, dtype=torch.bool)
    for s, n in enumerate(b.lens):
        for j in range(max(n, 0)):
            at = O.slot(b.table, b.n_pages, b.page, s, j)
            if at is not None:
                keep[at] = True
    for view, values in ((cache.keys(0), False), (cache.values(0), True)):
        x = natural(cache, values)
        codes = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
        codes[~keep.cuda()] = 0x7F if x.dtype == torch.float8_e4m3fn else math.nan
        (view.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else view).copy_(codes.view(view.shape))


EDGES = [1, 0, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 127, 128, 129, 255, 257]
ATTENDS = [
    # fmt, D, q heads, kv heads, page, lens, news, sink, window, max_new, max_len
    ("bf16", 128, 4, 4, 16, EDGES, None, 0, 0, 1, 257),
    ("bf16", 64, 8, 2, 32, EDGES, None, 0, 0, 1, 257),
    ("fp8_e4m3", 128, 6, 2, 48, EDGES, None, 0, 0, 1, 257),
    ("fp8_e4m3", 64, 4, 1, 16, EDGES, None, 0, 0, 1, 257),
    ("bf16", 128, 32, 1, 64, [300, 77], None, 0, 0, 1, 300),            # more query heads a kv head than a tile has rows
    ("bf16", 128, 17, 1, 16, [100], None, 0, 0, 1, 100),
    ("bf16", 128, 8, 8, 16, [4000, 30, 0, 1555], None, 0, 0, 1, 4000),  # split over workgroups, one row a tile
    ("bf16", 64, 10, 2, 16, [5000, 30, 2049], None, 0, 0, 1, 5000),
    ("fp8_e4m3", 128, 8, 2, 128, [6000, 1025, 64], None, 0, 0, 1, 6000),
    ("fp8_e4m3", 64, 24, 3, 32, [4097, 5], None, 0, 0, 1, 4097),
    ("bf16", 128, 8, 2, 16, [4000, 900], None, 0, 0, 1, 64),            # much longer than max_len says
    ("bf16", 128, 8, 2, 16, [40, 9], None, 0, 0, 1, 100000),            # much shorter
    ("bf16", 128, 4, 2, 16, EDGES + [500], None, 20, 50, 1, 500),       # sink and window
    ("bf16", 64, 4, 2, 48, EDGES + [900], None, 0, 33, 1, 900),
    ("fp8_e4m3", 128, 4, 2, 16, EDGES + [700], None, 40, 1, 1, 700),
    ("bf16", 128, 4, 4, 32, [6000, 3000, 200], None, 100, 2500, 1, 6000),
    ("bf16", 128, 8, 2, 16, [100, 33, 0, 3, 64], [4, 1, 0, 3, 2], 0, 0, 4, 100),
    ("bf16", 64, 10, 2, 32, [2100, 70, 9], [7, 8, 9], 0, 0, 8, 2100),   # more new tokens than max_new: the last one is left alone
    ("fp8_e4m3", 128, 12, 12, 16, [130, 40], [20, 40], 0, 0, 64, 130),
    ("fp8_e4m3", 64, 5, 1, 16, [300, 64, 7], [5, 3, 7], 10, 37, 7, 300),
    ("bf16", 128, 4, 2, 16, [500, 65], [5, 5], 17, 16, 5, 500),
    ("bf16", 128, 3, 3, 16, [3, 2], [6, 2], 0, 0, 6, 16),               # more new tokens than the sequence has
    ("bf16", 64, 4, 2, 16, [300, 130, 0, 170], [300, 130, 0, 1], 0, 0, 300, 300),       # whole prompts, and one that goes on
    ("fp8_e4m3", 128, 2, 2, 48, [210, 99], [200, 99], 7, 40, 200, 210),
]


@pytest.mark.parametrize("case", range(len(ATTENDS)))
def test_attn(case):
    fmt, d, hq, hkv, page, lens, news, sink, window, max_new, max_len = ATTENDS[case]
    b = Batch(lens, news, page, 50 + case, extra_rows=0 if news is None else 3)
    exps = {"k_exp": 1, "v_exp": -1} if fmt != "bf16" else {}
    cache = B.PagedCache(1, hq, hkv, d, page, b.n_pages, kv_format=fmt, **exps)
    cache.k_exp, cache.v_exp = exps.get("k_exp", 0), exps.get("v_exp", 0)
    fill(cache, 200 + case)
    poison_unused(cache, b)
    q = normal((b.rows, 2 * hq * d), 300 + case, 2 * math.log2(math.e) / math.sqrt(d))[:, :hq * d].unflatten(1, (hq, d))
    out = torch.empty(b.rows, 3 * hq * d, dtype=torch.bfloat16, device="cuda")[:, hq * d:2 * hq * d].unflatten(1, (hq, d))
    check_attn(cache, b, q, out, sink, window, max_new, max_len)


def test_attn_pages_that_are_none():
    """Pages outside the pool inside a sequence: their tokens are left out; a row that has none left gives zeros."""
    for fmt in ("bf16", "fp8_e4m3"):
        b = Batch([100, 40, 20, 3000, 700], None, 16, 8)
        b.table[0, 1], b.table[0, 4], b.table[1, :], b.table[2, 0] = -1, b.n_pages, -7, 2 ** 31 - 1
        b.table[3, 3:90] = -1
        b.lens[4] = 10 ** 9                                      # as many as the table can name
        cache = B.PagedCache(1, 6, 2, 128, 16, b.n_pages, kv_format=fmt)
        cache.k_exp = cache.v_exp = 0
        fill(cache, 9)
        q = normal((5, 6, 128), 10, 0.2)
        out = torch.empty_like(q)
        b_lens, b.lens = b.lens, [min(n, b.table.shape[1] * 16) for n in b.lens]
        check_attn(cache, b, q, out, max_len=1000)
        want = out.clone()
        b.lens = b_lens
        cache.attn(0, q=q, out=out, workspace=cache.attn_workspace(5, max_len=1000), max_len=1000, **b.device())
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        assert (out[1] == 0).all()


@pytest.mark.parametrize("sink, window", [(0, 0), (5, 37), (0, 3)])
def test_attn_lengths_beyond_the_table(sink, window):
    """A sequence longer than its row of the page table names: its queries keep their places, and the tokens behind the row are none."""
    b = Batch([64, 64, 64], [1, 4, 2], 16, 8, extra_cols=0)
    b.lens = [70, 99, 5000]
    cache = B.PagedCache(1, 4, 2, 64, 16, b.n_pages)
    cache.k_exp = cache.v_exp = 0
    fill(cache, 9)
    q = normal((b.rows, 4, 64), 10, 0.2)
    check_attn(cache, b, q, torch.empty_like(q), sink, window, 4, 100)


def test_refusals():
    """What the binding refuses, and what the calls refuse before they enqueue anything."""
    b = Batch([4000, 33], None, 16, 8)
    cache, L = B.PagedCache(1, 4, 2, 64, 16, b.n_pages, rope="grid"), B.lib()
    d = b.device()
    q, k, v = normal((2, 4, 64), 1), normal((2, 2, 64), 2), normal((2, 2, 64), 3)
    out, pos, ws = torch.empty_like(q), torch.zeros(2, 3, dtype=torch.int32, device="cuda"), cache.attn_workspace(2, max_len=4000)
    before = cache.buffer.clone()
    for bad in (lambda: cache.append(0, k=k, v=v, q=q, positions=pos, **d), lambda: cache.append(0, k=k, v=v[:1], positions=pos, **d),
                lambda: cache.append(0, k=k.float(), v=v, positions=pos, **d), lambda: cache.append(0, k=k.cpu(), v=v, positions=pos, **d),
                lambda: cache.append(0, k=k, v=v, positions=pos[:, 0], **d), lambda: cache.append(0, k=k, v=v, positions=pos, **{**d, "seq_lens": d["seq_lens"].long()}),
                lambda: cache.append(0, k=k, v=v, positions=pos, **{**d, "page_table": d["page_table"][:1]}),
                lambda: cache.append(0, k=k, v=v, positions=pos, **{**d, "page_table": d["page_table"][:, ::2]}),
                lambda: cache.append(0, k=k, v=v, positions=pos, **{**d, "cu_tokens": d["seq_lens"]}),
                lambda: cache.attn(0, q=q, out=out[:1], workspace=ws, **d), lambda: cache.attn(0, q=q[:, :2], out=out, workspace=ws, **d),
                lambda: cache.attn(0, q=q, out=out.transpose(0, 1), workspace=ws, **d), lambda: cache.attn(0, q=q, out=out, workspace=ws.float(), **d)):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: cache.append(0, k=k, v=v, **d), 1), (lambda: cache.append(1, k=k, v=v, positions=pos, **d), 1),
                        (lambda: cache.append(0, k=k, v=v, q=q, q_out=k.view(1, 4, 64).expand(2, 4, 64), positions=pos, **d), 1),
                        (lambda: cache.append(0, k=k[:1], v=v[:1], positions=pos[:1], **d), 1), (lambda: cache.attn(0, q=q, out=q, workspace=ws, max_len=4000, **d), 1),
                        (lambda: cache.attn(0, q=q, out=out, max_len=4000, **d), 1), (lambda: cache.attn(0, q=q, out=out, workspace=ws[:-16], max_len=4000, **d), 3),
                        (lambda: cache.attn(0, q=q, out=out, workspace=ws[1:], max_len=4000, **d), 1), (lambda: cache.attn(0, q=q, out=out, workspace=ws, max_new=2, max_len=4000, **d), 1),
                        (lambda: cache.attn(0, q=q, out=out, workspace=ws, max_len=4000, sink_tokens=4, **d), 1),
                        (lambda: cache.attn(0, q=q, out=out, workspace=ws, max_len=0, **d), 1)):
        with pytest.raises(B.LongLiveError) as e:
            bad()
        assert e.value.status == status
    at = lambda t: t.data_ptr()
    call = lambda k_at=at(k), k_stride=128, out_at=None, q_at=None: L.ll_paged_append(cache._h, 0, 2, 2, None, at(d["seq_lens"]), at(d["page_table"]), 251, 251, at(pos), q_at, 256,
                                                                                     k_at, k_stride, at(v), 128, out_at, 256, None)
    assert call(k_at=None) == 1 and call(k_at=at(k) + 2) == 1 and call(k_stride=120) == 1 and call(k_stride=132) == 1 and call(q_at=at(q)) == 1
    assert call(q_at=at(q), out_at=at(k)) == 1
    torch.cuda.synchronize()
    assert torch.equal(cache.buffer, before)
    nothing = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(0, k=nothing, v=nothing, positions=pos[:0], **{**d, "cu_tokens": torch.zeros(3, dtype=torch.int32, device="cuda")})     # no row at all
    cache.attn(0, q=q[:0], out=out[:0], workspace=ws, max_len=4000, **{**d, "cu_tokens": torch.zeros(3, dtype=torch.int32, device="cuda")})
    cache.close()
    with pytest.raises(B.LongLiveError):
        cache.attn(0, q=q, out=out, workspace=ws, max_len=4000, **d)


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_attn_numbers_a_query_does_not_see(fmt):
    """NaN and infinities in keys and values that a row does not see leave it as it is; in those it sees they reach it, and no other row."""
    b = Batch([200], [5], 16, 4)
    cache = B.PagedCache(1, 4, 2, 128, 16, b.n_pages, kv_format=fmt)
    q = normal((5, 4, 128), 3, 0.3)

    def run(change):
        fill(cache, 6)
        for view, values in ((cache.keys(0), False), (cache.values(0), True)):
            x = natural(cache, values)
            for j, what in change.get("v" if values else "k", {}).items():
                x.view(torch.uint8 if fmt != "bf16" else torch.bfloat16)[O.slot(b.table, b.n_pages, 16, 0, j)] = what
            (view.view(torch.uint8) if fmt != "bf16" else view).copy_((x.view(torch.uint8) if fmt != "bf16" else x).view(view.shape))
        out = torch.empty_like(q)
        cache.attn(0, q=q, out=out, workspace=cache.attn_workspace(1, 5, 200, 32, 40), max_new=5, max_len=200, sink_tokens=32, window_tokens=40, **b.device())
        return out.cpu().float()

    nan = math.nan if fmt == "bf16" else 0x7F
    big = math.inf if fmt == "bf16" else 0x7E                     # 8 bits have no infinity: the largest number
    clean = run({})
    assert torch.isfinite(clean).all()
    hidden = run({"v": {j: nan for j in range(32, 156)} | {199: big}, "k": {j: big for j in range(33, 156)} | {199: nan, 40: nan}})
    assert torch.equal(hidden[:4], clean[:4]) and torch.isnan(hidden[4]).all()     # places 195 .. 198 do not see 199
    seen = run({"v": {156: nan}})                                 # seen by the first query only (window 156 .. 195)
    assert torch.equal(seen[1:], clean[1:]) and torch.isnan(seen[0]).all()
    sink = run({"k": {31: nan}})
    assert torch.isnan(sink).all()


@pytest.mark.parametrize("fmt, D, group, new", [("bf16", 128, 2, 8), ("bf16", 64, 3, 5), ("fp8_e4m3", 64, 5, 4), ("fp8_e4m3", 128, 1, 16)])
def test_attn_drafts_whose_last_values_are_none(fmt, D, group, new):
    """The newest tokens' values are NaN from one token on, keys and places behind the length too: the rows in front have the same bits, also where their
    step's other rows do not, and thousands of keys lie before it."""
    lens = [3001, 70, new + 1]
    b = Batch(lens, [new] * 3, 32, 5)
    cache = B.PagedCache(1, 2 * group, 2, D, 32, b.n_pages, kv_format=fmt)
    q = normal((3 * new, 2 * group, D), 4, 0.3)
    ws = cache.attn_workspace(3, new, 3001)

    def run(from_token):
        fill(cache, 8)
        x = natural(cache, True)
        codes = x.view(torch.uint8) if fmt != "bf16" else x
        for s, n in enumerate(lens):
            for j in range(n - new + from_token, n):
                codes[O.slot(b.table, b.n_pages, b.page, s, j)] = 0x7F if fmt != "bf16" else math.nan
        view = cache.values(0)
        (view.view(torch.uint8) if fmt != "bf16" else view).copy_(codes.view(view.shape))
        poison_unused(cache, b)
        out = torch.empty_like(q)
        cache.attn(0, q=q, out=out, workspace=ws, max_new=new, max_len=3001, **b.device())
        return out.view(3, new, -1).cpu()

    clean = run(new)
    assert torch.isfinite(clean.float()).all()
    for first in (1, new - 1):
        got = run(first)
        assert torch.equal(got[:, :first], clean[:, :first]) and torch.isnan(got[:, first:].float()).all()


def test_attn_one_key_and_scores_far_apart():
    """A lone key's weight is 1 whatever its score; scores of hundreds, rising and falling through the sequence, neither overflow nor vanish."""
    b = Batch([1, 700, 700], None, 16, 4)
    cache = B.PagedCache(1, 2, 1, 64, 16, b.n_pages)
    cache.k_exp = cache.v_exp = 0
    fill(cache, 8)
    keys = natural(cache, False)
    for s, ramp in ((1, 1), (2, -1)):
        for j in range(700):
            keys[O.slot(b.table, b.n_pages, 16, s, j)] *= (j if ramp > 0 else 700 - j) / 70.0
    cache.keys(0).copy_(keys.view(cache.keys(0).shape))
    q = normal((3, 2, 64), 1, 4.0)
    out = torch.empty_like(q)
    check_attn(cache, b, q, out, max_len=700)
    assert torch.equal(out[0], natural(cache, True)[b.table[0, 0], 0].expand(2, 64))


def test_attn_layers_and_repeats():
    """Layers do not touch each other, and the same call gives the same bits whatever lies in the workspace."""
    b = Batch([3000, 17], None, 16, 4)
    cache = B.PagedCache(3, 8, 2, 128, 16, b.n_pages, rope="halves")
    q, k, v = normal((2, 8, 128), 1), normal((2, 2, 128), 2), normal((2, 2, 128), 3)
    for layer in (0, 2):
        cache.keys(layer).copy_(normal(cache.keys(layer).shape, 10 + layer))
        cache.values(layer).copy_(normal(cache.values(layer).shape, 20 + layer))
    before = cache.keys(0).clone(), cache.values(2).clone()
    qr, outs = torch.empty_like(q), []
    cache.append(1, k=k, v=v, q=q, q_out=qr, **b.device())
    for i in range(3):
        ws, out = cache.attn_workspace(2, max_len=3000), torch.empty_like(q)
        assert ws.numel() > 0
        ws.fill_(85 * i)
        cache.attn(2, q=qr, out=out, workspace=ws, max_len=3000, **b.device())
        outs.append(out)
    assert torch.equal(cache.keys(0), before[0]) and torch.equal(cache.values(2), before[1])
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    assert cache.keys(1).count_nonzero() > 0
    other = torch.empty_like(q)
    cache.attn(1, q=qr, out=other, workspace=ws, max_len=3000, **b.device())
    assert not torch.equal(other, outs[0])


def test_pool_beyond_32_bits():
    """A pool of more than 4 GiB: its last pages are written and read like its first."""
    page, n_pages = 1024, 2200                                   # 2 MiB a page and head pair: 4.3 GiB
    cache = B.PagedCache(1, 4, 4, 128, page, n_pages, rope="none")
    lens = [page + 3, 40]
    for pages in ([0, 1], [n_pages - 1, n_pages - 2]):
        table = torch.tensor([[pages[0], 5], [pages[1], 6]], dtype=torch.int32, device="cuda")
        table[0, 1] = pages[0] // 2 + 7
        q, k, v = (normal((page + 43, 4, 128), s + pages[0]) for s in (1, 2, 3))
        cu = torch.tensor([0, page + 3, page + 43], dtype=torch.int32, device="cuda")
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        cache.append(0, n, table, k, v, cu_tokens=cu)
        last = torch.tensor([page + 2, page + 42], device="cuda")
        out = torch.empty(2, 4, 128, dtype=torch.bfloat16, device="cuda")
        qs = (q[last] * (math.log2(math.e) / math.sqrt(128))).contiguous()
        cache.attn(0, n, table, qs, out, cache.attn_workspace(2, max_len=page + 3), max_len=page + 3)
        for s, (a, z) in enumerate(((0, page + 3), (page + 3, page + 43))):
            score = (k[a:z].double().transpose(0, 1) @ qs[s].double()[..., None])[..., 0] * math.log(2)
            want = (torch.softmax(score, -1)[:, None] @ v[a:z].double().transpose(0, 1))[:, 0]
            assert (out[s].double() - want).norm() <= 5e-3 * want.norm()


def test_another_stream_and_graph():
    """Work goes to the current stream.  A captured step (append and attention) follows lengths, pages and inputs from replay to replay,
    with eager calls on the same handle in between."""
    page, steps = 16, 40
    b = Batch([5, 20, 1], None, page, 4)
    n_pages = 3 * 8
    table = np.arange(n_pages, dtype=np.int32).reshape(3, 8)[:, ::-1].copy()
    for fmt in ("bf16", "fp8_e4m3"):
        eager, graphed = (B.PagedCache(1, 4, 2, 64, page, n_pages, rope="halves", kv_format=fmt) for _ in range(2))
        for c in (eager, graphed):
            fill(c, 4)
        lens = torch.tensor(b.lens, dtype=torch.int32, device="cuda")
        tab = torch.tensor(table, device="cuda")
        q, k, v = normal((3, 4, 64), 1), normal((3, 2, 64), 2), normal((3, 2, 64), 3)
        qr, out = torch.empty_like(q), torch.empty_like(q)
        ws = graphed.attn_workspace(3, max_len=8 * page)

        def step(cache, qr, out, ws):
            cache.append(0, lens, tab, k, v, q=q, q_out=qr)
            cache.attn(0, lens, tab, qr, out, ws, max_len=8 * page)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(graphed, qr, out, ws)                            # warm-up, on a stream of its own
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(graphed, qr, out, ws)
        qe, oe = torch.empty_like(q), torch.empty_like(q)
        step(eager, qe, oe, ws)                                   # what the warm-up stored
        for i in range(steps):
            lens += 1
            q.copy_(normal(q.shape, 1000 + i))
            k.copy_(normal(k.shape, 2000 + i))
            v.copy_(normal(v.shape, 3000 + i))
            graph.replay()
            step(eager, qe, oe, eager.attn_workspace(3, max_len=8 * page))
            torch.cuda.synchronize()
            assert torch.equal(out, oe) and torch.equal(qr, qe), i
        for values in (False, True):
            assert torch.equal(natural(graphed, values).view(torch.uint8), natural(eager, values).view(torch.uint8))


def test_calls_at_once():
    """Two streams attend over one cache at the same time, each with a workspace of its own, beside appends to other pages; so do products with one packed
    weight.  Every result is the one the call has by itself."""
    b = Batch([6000, 20, 4100], None, 16, 8)
    cache = B.PagedCache(2, 8, 2, 128, 16, b.n_pages, rope="halves")
    fill(cache, 3)
    d, kw = b.device(), {"max_len": 6000}
    layer = B.Linear(normal((512, 1024), 5, 1 / 32))
    inputs = [(normal((3, 8, 128), 10 + i, 0.3), normal((300, 1024), 20 + i)) for i in range(2)]
    alone = []
    for q, x in inputs:
        out, y = torch.empty_like(q), torch.empty(300, 512, dtype=torch.bfloat16, device="cuda")
        cache.attn(0, q=q, out=out, workspace=cache.attn_workspace(3, **kw), **kw, **d)
        layer.forward(x, y, activation="silu")
        alone.append((out, y))
    k, v = normal((3, 2, 128), 1), normal((3, 2, 128), 2)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [(torch.empty_like(o), torch.empty_like(y), cache.attn_workspace(3, **kw)) for o, y in alone]
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, (q, x), (out, y, ws) in zip(streams, inputs, got):
            with torch.cuda.stream(stream):
                cache.attn(0, q=q, out=out, workspace=ws, **kw, **d)
                layer.forward(x, y, activation="silu")
        with torch.cuda.stream(streams[2]):
            cache.append(1, k=k, v=v, **d)
    torch.cuda.synchronize()
    for (out, y), (o, z, _) in zip(alone, got):
        assert torch.equal(out, o) and torch.equal(y, z)
