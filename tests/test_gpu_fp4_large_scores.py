"""Scores far beyond what the exponential's argument can hold to a fraction: the difference from the row's largest score is what
counts, however large that score is.

The scores of these tests are exact in fp32 whatever the order of the sum: one channel gives 1.5 * 2^30 (q 32768, K 49152, the largest
value the cache holds), one channel of another group adds 128 times one of 0, 1, 2, 3, 4, 6, and 128 is the spacing of fp32 there.  What may be off
is then the weights' rounding to fp16, half a step 2^-11 of their size, the exponential's argument, a few roundings of a difference of at most
40 (2^-24 each: 2^-16 together), the sums over the tokens in fp32 (counted as in fp4_reference), and the output's own rounding."""
import math

import pytest
import torch

from paper_2512_24449_amd import binding
from tests import fp4_reference as ref
from tests.test_gpu_fp4_cache import DEV, ints, page_table, starts

pytestmark = pytest.mark.gpu


def cache_of(k, v, lens, H, Hq, D, seed):
    table, n_pages = page_table(lens, seed=seed)
    cache = binding.FP4KVCache(n_pages, H, Hq, D)
    cache.kv_fp4_append(k.to(DEV), v.to(DEV), binding.FP4Batch(ints(lens), max(lens), table, new_rows=ints(lens),
                                                               first_row=ints(starts(lens))))
    return cache, ref.quantise(k)[0], ref.quantise(v)[0], table


# one token; a few; split and joined by the last workgroup, by a kernel; many rows in blocks of 128 columns, whole and split contexts
SHAPES = [(128, 2, 1, [1], 1), (64, 1, 4, [40], 2), (128, 1, 1, [1200], 1), (128, 1, 4, [20000], 1), (64, 1, 16, [20000], 1),
          (128, 16, 4, [300] * 4, 300), (64, 4, 4, [17000], 130)]


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("sm_scale", [2.0 ** -9, 1.0, 2.0 ** 90])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D, H, G, lens, new", SHAPES)
def test_exact_large_scores(D, H, G, lens, new, dtype, sm_scale, sign):
    """Weights of 2^-9 as usual; with 1 and more the tokens of the largest score share all the weight."""
    gen = torch.Generator().manual_seed(D + H + sum(lens))
    total = sum(lens)
    step = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0])[torch.randint(0, 6, (total, H), generator=gen)]
    k = torch.zeros(total, H, D)
    k[:, :, 5], k[:, :, 40] = 49152.0, step                     # (groups of 32: each value is held as it is)
    v = torch.randn(total, H, D, generator=gen).to(dtype)
    cache, _, held, table = cache_of(k.to(dtype), v, lens, H, H * G, D, seed=total)
    n = new * len(lens)
    q = torch.zeros(n, H * G, D)
    q[:, :, 5], q[:, :, 40] = sign * 32768.0, sign * 128.0
    batch = binding.FP4Batch(ints(lens), new, table)
    lse = torch.empty(n, H * G, device=DEV)
    out = torch.empty(n, H * G, D, device=DEV)
    cache.kv_fp4_attention(q.to(dtype).to(DEV), batch, sign * sm_scale, out=out, lse=lse)
    out, lse = out.cpu().double(), lse.cpu().double()
    at = 0
    for b, length in enumerate(lens):
        above = (step[at:at + length].double() - 6.0) * 128.0 * sm_scale               # scores, 1.5 * 2^30 + 768 less
        hv = held[at:at + length]
        rows = [0, new // 2, new - 1] if new > 2 else range(new)
        for i in rows:
            p = length - new + i
            s = above[:p + 1]
            w = torch.exp(s - s.amax(0))
            total_w = w.sum(0)
            want = torch.einsum("th,thd->hd", w, hv[:p + 1]) / total_w[:, None]
            around = torch.einsum("th,thd->hd", w, hv[:p + 1].abs()) / total_w[:, None]
            bound = around * (2.0 ** -11 + 2.0 ** -15 + (p / 4 + 128) * 2.0 ** -24) + 2.0 ** -37 * hv[:p + 1].abs().sum(0)
            got = out[b * new + i].view(H, G, D)
            assert bool(((got - want[:, None]).abs() <= bound[:, None] + want.abs()[:, None] * 2.0 ** -24).all()), (b, i)
            want_lse = torch.log(total_w) + s.amax(0) + (1.5 * 2.0 ** 30 + 768) * sm_scale
            assert bool(((lse[b * new + i].view(H, G) - want_lse[:, None]).abs() <= 2.0 ** -21 * (1 + want_lse.abs())[:, None]).all())
        at += length


@pytest.mark.parametrize("D, H, G, lens, new", SHAPES)
def test_largest_values(D, H, G, lens, new):
    """Every row is a mean of visible values, its logarithm finite, with all of q and K as large as fp16 and the cache hold."""
    gen = torch.Generator().manual_seed(D + H)
    total, n = sum(lens), new * len(lens)
    k = (49152.0 - 16000.0 * torch.rand(total, H, D, generator=gen)).half()
    v = torch.randn(total, H, D, generator=gen).half()
    q = (60000.0 - 20000.0 * torch.rand(n, H * G, D, generator=gen)).half()
    cache, _, held, table = cache_of(k, v, lens, H, H * G, D, seed=1)
    lse = torch.empty(n, H * G, device=DEV)
    for flip in (1, -1):
        out = cache.kv_fp4_attention((flip * q).to(DEV), binding.FP4Batch(ints(lens), new, table), 1 / math.sqrt(D), lse=lse)
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
        out, at = out.cpu().double().view(len(lens), new, H, G, D), 0
        for b, length in enumerate(lens):
            lo, hi = held[at:at + length].amin(0), held[at:at + length].amax(0)
            # a rounding of the weights each way, and the output's
            assert bool((out[b] >= (lo - 2.0 ** -9 * lo.abs() - 1e-7)[None, :, None]).all())
            assert bool((out[b] <= (hi + 2.0 ** -9 * hi.abs() + 1e-7)[None, :, None]).all())
            at += length
        if lens == [1]:
            assert torch.equal(out[0, 0], held[0][:, None].expand(H, G, D))
