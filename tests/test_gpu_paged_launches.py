"""The paged cache on the GPU in the launches that full batches, prompts and chunks make: whole tiles of the append with several units a
workgroup, offsets of many sequences (csrc/paged.h).  Held against the fp64 oracle with the tolerances derived in test_gpu_paged.py;
test_paged_launches.py checks, without a GPU, that these sizes select what is said here.
"""
import numpy as np
import pytest
import torch

from paper_2509_22622_amd import binding as B

from test_gpu_paged import Batch, check_append, check_attn, fill, normal

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
