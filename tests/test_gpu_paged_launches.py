"""The paged cache on the GPU in the launches that full batches, prompts and chunks make: whole tiles of the append with several units a workgroup,
and every branch of the attention's split (csrc/paged.h).  Held against the fp64 oracle with the tolerances derived in test_gpu_paged.py;
test_paged_launches.py checks, without a GPU, that these sizes select what is said here.
"""
import math

import numpy as np
import pytest
import torch

from paper_2509_22622_amd import binding as B

from test_gpu_paged import Batch, check_append, check_attn, fill, normal, poison_unused

pytestmark = pytest.mark.gpu

# format, D, q heads, kv heads, page, rope, rope_dim, lens, news, units a workgroup at least (a unit: a kv head's K and V, or two query heads).
# A tile is 32 rows at D 128 and 64 at D 64.  All have workgroups with two kv heads, with the last kv head and the first queries, and a last query head by itself.
APPENDS = [
    ("bf16", 128, 33, 33, 32, "halves", 128, [700, 90, 41, 20], [660, 90, 41, 9], 2),
    ("bf16", 128, 35, 5, 64, "pairs", 64, [2400, 131], [2369, 131], 2),
    ("bf16", 64, 33, 33, 16, "halves", 64, [1200, 65, 190], [1145, 65, 190], 2),
    ("fp8_e4m3", 128, 99, 99, 48, "grid", 128, [801], [801], 4),
    ("fp8_e4m3", 64, 99, 33, 32, "pairs", 16, [700, 3, 900], [643, 3, 754], 2),
    ("bf16", 128, 15, 3, 128, "none", 0, [9000, 7500], [8985, 7477], 2),         # more than 512 tiles
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append_whole_tiles(case):
    fmt, d, hq, hkv, page, rope, rope_dim, lens, news, _ = APPENDS[case]
    b = Batch(lens, news, page, 30 + case, extra_rows=3)
    exps = {"k_exp": -2, "v_exp": 1} if fmt != "bf16" else {}
    cache = B.PagedCache(1, hq, hkv, d, page, b.n_pages, rope=rope, rope_dim=rope_dim, kv_format=fmt, **exps)
    cache.k_exp, cache.v_exp = exps.get("k_exp", 0), exps.get("v_exp", 0)
    qkv = normal((b.rows, (hq + 2 * hkv) * d), 400 + case, 3.0)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], 1))
    at = np.arange(b.rows)
    positions = np.stack([at // 1560 + 3, at % 1560 // 52, at % 52], 1) if rope == "grid" else None
    out = torch.empty(b.rows, hq, d, dtype=torch.bfloat16, device="cuda")
    check_append(cache, b, q, k, v, out, positions, rope=rope, rope_dim=rope_dim, theta=10000.0)
    # in place, and without queries: the same bits
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    pool, rows = cache.buffer.clone(), int(b.cu[-1])
    same = q.clone(memory_format=torch.contiguous_format)
    for queries in (same, None):
        fill(cache, 77)
        cache.append(0, k=k, v=v, q=queries, q_out=queries, positions=pos, **b.device())
        assert torch.equal(cache.buffer, pool)
    assert torch.equal(same[:rows], out[:rows]) and torch.equal(same[rows:], q[rows:])


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
def test_append_many_sequences(fmt):
    """300 sequences with offsets, which are searched in memory; every fifth brings nothing, some have no tokens at all."""
    rng = np.random.default_rng(11)
    news = [0 if s % 5 == 2 else int(rng.integers(1, 5)) for s in range(300)]
    lens = [0 if s % 25 == 2 else n + int(rng.integers(0, 40)) for s, n in enumerate(news)]
    b = Batch(lens, news, 16, 12, extra_rows=4)
    cache = B.PagedCache(1, 6, 2, 64, 16, b.n_pages, rope="halves", kv_format=fmt)
    cache.k_exp = cache.v_exp = 0
    q, k, v = normal((b.rows, 6, 64), 1), normal((b.rows, 2, 64), 2), normal((b.rows, 2, 64), 3)
    check_append(cache, b, q, k, v, torch.empty_like(q), rope="halves", rope_dim=64, theta=10000.0)
    check_attn(cache, b, q, torch.empty_like(q), max_new=4, max_len=max(lens))


def _few_long(n, long, seed):
    """Lengths of n sequences: the long ones first, the others idle or short."""
    rng = np.random.default_rng(seed)
    return list(long) + [0 if i % 3 == 1 else int(rng.integers(1, 90)) for i in range(n - len(long))]


# format, D, q heads, kv heads, page, lens, news (None: one each), sink, window, max_new, max_len, row tiles a sequence and kv head, splits
ATTENDS = [
    ("bf16", 128, 32, 8, 16, _few_long(11, [6400, 5123], 1), None, 0, 0, 1, 6400, 1, 5),                  # 88 tiles of 200 steps
    ("fp8_e4m3", 64, 8, 8, 48, _few_long(31, [12800, 777], 2), None, 0, 0, 1, 12800, 1, 5),               # 248 of 200
    ("bf16", 128, 32, 8, 64, _few_long(33, [2560, 2100, 33], 3), None, 0, 0, 1, 2560, 1, 5),              # 264 of 80
    ("fp8_e4m3", 64, 40, 8, 32, _few_long(50, [6144, 4000], 4), None, 0, 0, 1, 6144, 1, 5),               # 400 of 96
    ("fp8_e4m3", 128, 16, 8, 128, _few_long(64, [3072, 1030], 5), None, 0, 0, 1, 3072, 1, 5),             # 512 of 96
    ("bf16", 128, 8, 8, 16, _few_long(65, [8192, 8000, 1500], 6), None, 0, 0, 1, 8192, 1, 3),             # 520 of 256
    ("fp8_e4m3", 64, 12, 12, 16, _few_long(170, [16384, 600], 7), None, 0, 0, 1, 16384, 1, 3),            # 2040 of 256
    ("bf16", 128, 32, 8, 16, _few_long(11, [9000, 6401], 8), None, 0, 0, 1, 6400, 1, 5),                  # longer than max_len says
    ("bf16", 128, 12, 12, 16, _few_long(24, [7000, 3001, 2700], 9), None, 200, 2600, 1, 7000, 1, 5),      # 288 tiles, sink and window
    ("bf16", 128, 32, 8, 16, _few_long(6, [6400, 900], 10), [8, 8, 3, 0, 8, 1], 0, 0, 8, 6400, 2, 5),     # two row tiles
    ("fp8_e4m3", 64, 15, 3, 32, _few_long(11, [13000, 700], 11), [8, 5, 8, 0, 8, 1, 2, 0, 7, 8, 8], 0, 0, 8, 13000, 3, 5),   # three; the last set of 8 runs is not full
    ("bf16", 64, 20, 4, 16, _few_long(48, [17000, 400], 12), [8, 8] + [1, 0, 4] * 15 + [2], 30, 16400, 8, 17000, 3, 3),      # 576 tiles, sink and window
    ("bf16", 128, 32, 8, 64, [4000], None, 0, 0, 1, 120000, 1, 32),                                       # two of 32 partial results, in the wide join
    ("fp8_e4m3", 128, 16, 4, 16, [4096, 70], None, 0, 0, 1, 131072, 1, 32),
]


@pytest.mark.parametrize("case", range(len(ATTENDS)))
def test_attn_splits(case):
    fmt, d, hq, hkv, page, lens, news, sink, window, max_new, max_len, tiles, splits = ATTENDS[case]
    b = Batch(lens, news, page, 150 + case, extra_rows=0 if news is None else 2)
    exps = {"k_exp": 1, "v_exp": -1} if fmt != "bf16" else {}
    cache = B.PagedCache(1, hq, hkv, d, page, b.n_pages, kv_format=fmt, **exps)
    cache.k_exp, cache.v_exp = exps.get("k_exp", 0), exps.get("v_exp", 0)
    assert cache.attn_workspace_bytes(len(lens), max_new, max_len, sink, window) == len(lens) * hkv * tiles * splits * 16 * (d + 2) * 4
    fill(cache, 500 + case)
    poison_unused(cache, b)
    q = normal((b.rows, hq, d), 600 + case, 2 * math.log2(math.e) / math.sqrt(d))
    check_attn(cache, b, q, torch.empty_like(q), sink, window, max_new, max_len)
