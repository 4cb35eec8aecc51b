"""Row offsets that reach beyond the call's rows, on either side: what a sequence brings is the difference of its offsets all the same, so that its rows
keep their places; rows that the call does not have are left out.  Held against the fp64 oracle with the tolerances derived in test_gpu_paged.py."""
import math

import pytest
import torch

from paper_2509_22622_amd import binding as B

from test_gpu_paged import Batch, check_append, check_attn, fill, normal

pytestmark = pytest.mark.gpu

# lens, offsets, rows of the call
OFFSETS = [([40, 60], [0, 6, 30], 10), ([30, 50], [-4, 5, 12], 12), ([64], [-9, 64], 20), ([20, 2000, 9], [0, 3, 40, 44], 17), ([2 ** 31 - 1, 45], [0, 2 ** 31 - 1, 2 ** 31 - 1], 25),
           ([0, 7], [-2 ** 30, 5, 9], 12)]


def batch(case, page):
    lens, cu, rows = OFFSETS[case]
    b = Batch([min(n, 3000) for n in lens], None, page, 70 + case, cu=cu)
    b.lens, b.rows = list(lens), rows
    return b


@pytest.mark.parametrize("fmt", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("case", range(len(OFFSETS)))
def test_offsets_beyond_the_rows(case, fmt):
    b = batch(case, 16)
    cache = B.PagedCache(1, 6, 2, 64, 16, b.n_pages, rope="halves", kv_format=fmt)
    cache.k_exp = cache.v_exp = 0
    fill(cache, 5)
    q, k, v = normal((b.rows, 6, 64), 1), normal((b.rows, 2, 64), 2), normal((b.rows, 2, 64), 3)
    check_append(cache, b, q, k, v, torch.empty_like(q), rope="halves", rope_dim=64, theta=10000.0)
    fill(cache, 6)
    q = normal((b.rows, 6, 64), 4, math.log2(math.e) / 8)
    for sink, window in ((0, 0), (5, 30)):
        check_attn(cache, b, q, torch.empty_like(q), sink, window, 64, 3000)
