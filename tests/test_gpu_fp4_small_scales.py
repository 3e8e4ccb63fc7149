"""Scales of 0 and far below 1 with queries as large as bf16 holds: with 0 every visible token weighs the same, whatever the
scores; with others it is their product that counts."""
import math

import pytest
import torch

from paper_2512_24449_amd import binding
from tests import fp4_reference as ref
from tests.test_gpu_fp4_attention import check, filled
from tests.test_gpu_fp4_cache import DEV, ints

pytestmark = pytest.mark.gpu
# one token; some; split contexts; many rows in blocks of 128 columns
SHAPES = [(128, 2, 2, [1, 90], 1), (64, 1, 4, [700], 3), (128, 1, 1, [5000], 1), (128, 16, 4, [300] * 4, 300), (64, 4, 4, [17000], 130)]


def queries(n, heads, D, size, seed):
    return (torch.randn(n, heads, D, generator=torch.Generator().manual_seed(seed)) * size).bfloat16()


@pytest.mark.parametrize("zero", [0.0, -0.0])
@pytest.mark.parametrize("size", [1.0, 1e30, 5e37])
@pytest.mark.parametrize("D, H, G, lens, new", SHAPES)
def test_scale_zero(D, H, G, lens, new, size, zero):
    cache, k, v, table = filled(lens, H, H * G, D, torch.bfloat16)
    n = new * len(lens)
    q = queries(n, H * G, D, size, 3)
    lse = torch.empty(n, H * G, device=DEV)
    out = torch.empty(n, H * G, D, device=DEV)
    cache.kv_fp4_attention(q.to(DEV), binding.FP4Batch(ints(lens), new, table), zero, out=out, lse=lse)
    check(cache, k, v, lens, [new] * len(lens), torch.zeros_like(q), out, lse, 0.0)


@pytest.mark.parametrize("sm_scale, size", [(1e-31, 1e30), (-3e-36, 1e35), (1e-37, 1e36), (2e-39, 5e37)])
@pytest.mark.parametrize("D, H, G, lens, new", SHAPES)
def test_small_scales(D, H, G, lens, new, sm_scale, size):
    """(2e-39 is below fp32's normal range; held there to 2^-21: in the scores, which are of order 1, less than their sums' roundings)"""
    cache, k, v, table = filled(lens, H, H * G, D, torch.bfloat16, size=0.1)
    n = new * len(lens)
    q = queries(n, H * G, D, size / math.sqrt(D), 4)
    lse = torch.empty(n, H * G, device=DEV)
    out = torch.empty(n, H * G, D, device=DEV)
    cache.kv_fp4_attention(q.to(DEV), binding.FP4Batch(ints(lens), new, table), sm_scale, out=out, lse=lse)
    held = torch.tensor(sm_scale, dtype=torch.float32).double().item()
    check(cache, k, v, lens, [new] * len(lens), q, out, lse, held)


def test_scale_zero_keeps_nan_and_infinity():
    cache, k, v, table = filled([200], 2, 4, 128, torch.float16)
    q = torch.randn(3, 4, 128, generator=torch.Generator().manual_seed(5)).half()
    batch = binding.FP4Batch(ints([200]), 3, table)
    good = cache.kv_fp4_attention(q.to(DEV), batch, 0.0)
    q[1, 2, 17], q[2, 0, 0], q[2, 3, 1] = float("nan"), float("inf"), float("-inf")
    got = cache.kv_fp4_attention(q.to(DEV), batch, 0.0)
    bad = torch.zeros(3, 4, dtype=torch.bool, device=DEV)
    bad[1, 2] = bad[2, 0] = bad[2, 3] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], good[~bad])
