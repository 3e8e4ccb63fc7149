"""An infinity in q makes all of a row's scores infinities or NaN: the row is NaN, also where every score is -infinity, which is not
a row that sees nothing."""
import math

import pytest
import torch

from paper_2512_24449_amd import binding
from tests.test_gpu_fp4_cache import DEV, ints, page_table, rows, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.1, -0.1, 0.0])
@pytest.mark.parametrize("D, H, G, lens, new", [(128, 2, 1, [1], 1), (64, 1, 4, [1, 40], 1), (128, 1, 1, [1200], 1), (64, 1, 16, [20000], 1),
                                                (128, 16, 4, [300] * 4, 300), (64, 4, 4, [17000], 130)])
def test_rows_of_infinite_scores(D, H, G, lens, new, scale, dtype):
    gen = torch.Generator().manual_seed(D + H)
    total, n = sum(lens), new * len(lens)
    k, v = torch.rand(total, H, D, generator=gen) + 0.5, torch.randn(total, H, D, generator=gen)   # no K is 0 or negative
    table, n_pages = page_table(lens)
    cache = binding.FP4KVCache(n_pages, H, H * G, D)
    cache.kv_fp4_append(k.to(dtype).to(DEV), v.to(dtype).to(DEV),
                        binding.FP4Batch(ints(lens), max(lens), table, new_rows=ints(lens), first_row=ints(starts(lens))))
    batch = binding.FP4Batch(ints(lens), new, table)
    q = rows(n, H * G, D, dtype, 1)
    lse, good_lse = (torch.empty(n, H * G, device=DEV) for _ in range(2))
    good = cache.kv_fp4_attention(q.to(DEV), batch, scale, lse=good_lse)
    assert bool(torch.isfinite(good).all()) and bool(torch.isfinite(good_lse).all())
    at = torch.zeros(n, H * G, dtype=torch.bool)
    for i, (row, value) in enumerate(((0, -math.inf), (n // 2, math.inf), (n - 1, -math.inf))):
        head = (3 * i) % (H * G)
        q[row, head, (37 * i + 5) % D] = value
        at[row, head] = True
    got = cache.kv_fp4_attention(q.to(DEV), batch, scale, lse=lse)
    at = at.to(DEV)
    assert bool(torch.isnan(got[at]).all()) and bool(torch.isnan(lse[at]).all())
    assert torch.equal(got[~at], good[~at]) and torch.equal(lse[~at], good_lse[~at])


def test_such_a_row_that_sees_nothing():
    H, D = 2, 64
    cache = binding.FP4KVCache(2, H, H, D)
    x = rows(3, H, D, torch.float16, 2).to(DEV)
    x[0, 0, 3] = math.inf
    batch = binding.FP4Batch(ints([2]), 3, ints([[1]]))         # the first of three rows is at position -1
    cache.kv_fp4_append(rows(3, H, D, torch.float16, 3).to(DEV), rows(3, H, D, torch.float16, 4).to(DEV), batch)
    lse = torch.empty(3, H, device=DEV)
    out = cache.kv_fp4_attention(x, batch, 0.1, lse=lse)
    assert not out[0].any() and bool((lse[0] == -math.inf).all()) and bool(torch.isfinite(out).all())
