"""Splits longer than the page numbers that a wave holds at a time -- 256 steps of 32 tokens in the kernel for few rows, 64 pages in
the one for many --, split contexts of many rows through a window, pages that sequences share, and page tables much wider than
the sequences.  The sequences of a batch are prefixes of one, over the same pages: many of them use up the workgroups, so that
none is split, and the cache stays small.  Steps and pages of the longest split, by the launcher's rule, stand beside the cases."""
import math

import pytest
import torch

from paper_2512_24449_amd import binding
from tests import fp4_reference as ref
from tests.test_gpu_fp4_attention import run
from tests.test_gpu_fp4_cache import DEV, ints, page_table, rows, starts

pytestmark = pytest.mark.gpu


def stored(length, H, Hq, D, dtype, wide=None):
    """A cache with one sequence, its values as it holds them, and its row of the page table (to `wide` pages)."""
    table, n_pages = page_table([length], seed=length)
    cache = binding.FP4KVCache(n_pages, H, Hq, D)
    cache.pages.fill_(255)
    gen = torch.Generator(device=DEV).manual_seed(length)
    k, v = (torch.randn(length, H, D, generator=gen, device=DEV) for _ in range(2))
    k[:, :, 3:D:D // 4] *= 4.0
    whole = binding.FP4Batch(ints([length]), length, table)
    cache.kv_fp4_append(k.to(dtype), v.to(dtype), whole)
    k, v = (t.cpu() for t in cache.kv_fp4_read(whole, length, torch.float32))
    if wide:
        table = torch.cat([table, torch.full((1, wide - table.shape[1]), -1, dtype=torch.int32, device=DEV)], 1)
    return cache, k, v, table


def agree(out, lse, q, k, v, length, n, scale, window=0, sinks=0):
    want, want_lse, bound, lse_bound = ref.attention(q.cpu(), k[:length], v[:length], n, scale, window, sinks)
    step = torch.finfo(out.dtype).eps / 2
    off = (out.cpu().double() - want).abs() - bound - (want.abs() + bound) * step
    assert bool((off <= 1e-7).all()), float(off.max())          # 1e-7: fp16 below its normal range
    assert bool(((lse.cpu().double() - want_lse).abs() <= lse_bound).all())


@pytest.mark.parametrize("longest, D, G, dtype, window, sinks", [
    (9003, 128, 1, torch.float16, 0, 0),         # 282 steps: 256 and 26
    (17500, 64, 2, torch.bfloat16, 0, 0),        # 547: 256, 256, 35
    (17500, 64, 1, torch.float16, 8400, 70),     # 266, three of them first tokens
])
def test_few_rows(longest, D, G, dtype, window, sinks):
    H, batch, scale = 12, 64, 1 / math.sqrt(D)
    cache, k, v, table = stored(longest, H, H * G, D, dtype)
    lens = [longest - b % 3 for b in range(batch)]
    q = rows(1, H * G, D, dtype, 1).to(DEV)
    lse = torch.empty(batch, H * G, device=DEV)
    out = torch.empty(batch, H * G, D, dtype=dtype, device=DEV)
    shared = binding.FP4Batch(ints(lens), 1, table.repeat(batch, 1))
    cache.kv_fp4_attention(q.repeat(batch, 1, 1), shared, scale, window, sinks, out=out, lse=lse)
    for b in range(3):
        agree(out[b:b + 1], lse[b:b + 1], q, k, v, lens[b], 1, scale, window, sinks)
        assert torch.equal(out[b::3], out[b:b + 1].expand_as(out[b::3])) and torch.equal(lse[b::3], lse[b:b + 1].expand_as(lse[b::3]))


@pytest.mark.parametrize("D, dtype, window, sinks", [(64, torch.float16, 0, 0),          # 140 pages: 64, 64, 12
                                                     (128, torch.bfloat16, 0, 0),
                                                     (64, torch.bfloat16, 4300, 70)])    # 71, two of them first tokens
def test_many_rows(D, dtype, window, sinks):
    H, G, new, batch, scale = 4, 4, 32, 100, 1 / math.sqrt(D)
    lens = [4200 + 48 * b for b in range(batch)]
    cache, k, v, table = stored(lens[-1], H, H * G, D, dtype)
    q = rows(batch * new, H * G, D, dtype, 2).to(DEV)
    lse = torch.empty(batch * new, H * G, device=DEV)
    out = torch.empty(batch * new, H * G, D, dtype=dtype, device=DEV)
    cache.kv_fp4_attention(q, binding.FP4Batch(ints(lens), new, table.repeat(batch, 1)), scale, window, sinks, out=out, lse=lse)
    for b in (0, 1, 21, 47, 81, 98, 99):
        part = slice(b * new, (b + 1) * new)
        agree(out[part], lse[part], q[part], k, v, lens[b], new, scale, window, sinks)


@pytest.mark.parametrize("D, H, G, lens, new, window, sinks", [
    (64, 4, 4, [20000], [130], 16500, 70),              # 22 pages in one of 12 splits
    (64, 4, 4, [20000, 18000], [130, 70], 16500, 70),   # 53
    (128, 2, 4, [18100], [600], 16400, 3)])
def test_many_rows_split_through_a_window(D, H, G, lens, new, window, sinks):
    run(lens, new, H, G, D, torch.float16, window, sinks, seed=H)


@pytest.mark.parametrize("H, G, lens, new", [(1, 1, [1000], 1), (2, 4, [1, 300, 65], 3), (8, 2, [129] * 3, 1), (4, 4, [200, 130], 130)])
def test_tables_wider_than_the_sequences(H, G, lens, new):
    """Room for 131072 tokens: the longest sequence is what counts."""
    D, scale = 128, 0.1
    longest = max(lens)
    cache, k, v, table = stored(longest, H, H * G, D, torch.float16, wide=2048)
    q = rows(len(lens) * new, H * G, D, torch.float16, 3).to(DEV)
    take = [min(new, n) for n in lens]
    for window, sinks in ((0, 0), (50, 4)):
        lse = torch.empty(len(lens) * new, H * G, device=DEV)
        out = torch.empty(len(lens) * new, H * G, D, dtype=torch.float16, device=DEV)
        batch = binding.FP4Batch(ints(lens), new, table.repeat(len(lens), 1), new_rows=ints(take), first_row=ints(starts(take)))
        cache.kv_fp4_attention(q, batch, scale, window, sinks, out=out, lse=lse)
        for length, n, at in zip(lens, take, starts(take)):
            agree(out[at:at + n], lse[at:at + n], q[at:at + n], k, v, length, n, scale, window, sinks)


def test_append_behind_shared_pages():
    """Two sequences that share a prefix of full pages go on in pages of their own."""
    H, D, prefix, more = 2, 128, 128, 37
    cache = binding.FP4KVCache(4, H, H, D)
    table = ints([[3, 1, 0], [3, 1, 2]])
    k, v = (rows(prefix + 2 * more, H, D, torch.float16, s) for s in (4, 5))
    cache.kv_fp4_append(k[:prefix].to(DEV), v[:prefix].to(DEV), binding.FP4Batch(ints([prefix]), prefix, table[:1].contiguous()))
    before = cache.pages.view(4, -1)[[3, 1]].clone()
    cache.kv_fp4_append(k[prefix:].to(DEV), v[prefix:].to(DEV), binding.FP4Batch(ints([prefix + more] * 2), more, table))
    assert torch.equal(cache.pages.view(4, -1)[[3, 1]], before)
    got = cache.kv_fp4_read(binding.FP4Batch(ints([prefix + more] * 2), prefix + more, table), 2 * (prefix + more), torch.float32)
    for g, x in zip(got, (k, v)):
        want = ref.quantise(x)[0]
        for b in range(2):
            part = g[b * (prefix + more):(b + 1) * (prefix + more)].cpu().double()
            assert torch.equal(part[:prefix], want[:prefix])
            assert torch.equal(part[prefix:], want[prefix + b * more:prefix + (b + 1) * more])
