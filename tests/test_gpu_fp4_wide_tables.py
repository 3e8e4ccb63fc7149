"""Page tables of many pages, around a cache's budget: selections in more parts than a wave has lanes, weights of so many heads and pages that
workgroups take several groups of pages."""
import pytest
import torch

from paper_2512_24449_amd import binding
from tests import budget_reference as ref
from tests import fp4_reference
from tests.test_gpu_fp4_budget import close, ints, query

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def sorted_choice(mass, length, keep, sinks, recent):
    """The same by a stable sort, for long sequences (mass [H, tokens], no NaN)."""
    if length <= keep:
        return torch.arange(length, device=DEV).expand(mass.shape[0], -1)
    most = torch.sort(-mass[:, sinks:length - recent], dim=1, stable=True).indices[:, :keep - sinks - recent] + sinks
    fixed = torch.cat([torch.arange(sinks, device=DEV), torch.arange(length - recent, length, device=DEV)])
    return torch.cat([most, fixed.expand(mass.shape[0], -1)], 1).sort(1).values


def test_the_sorted_choice_is_the_rules():
    m = torch.randint(0, 5, (2, 700), generator=torch.Generator().manual_seed(1)).float()
    for keep, sinks, recent in ((1, 0, 0), (300, 4, 20), (699, 0, 1), (700, 3, 3)):
        got = sorted_choice(m.to(DEV), 700, keep, sinks, recent)
        assert got.tolist() == [ref.kept(x.tolist(), 700, keep, sinks, recent) for x in m]


# parts of 8192 tokens: 65, 74, 129, 245 and 256 of them
@pytest.mark.parametrize("tokens", [64 * 8192 + 1, 600_000, 128 * 8192 + 77, 2_000_003, 256 * 8192])
def test_select_in_more_parts_than_lanes(tokens):
    pages = -(-tokens // 64)
    cache = binding.FP4KVCache(1, 2, 2, 128)
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    spread = torch.exp(3 * torch.randn(1, 2, tokens, generator=gen, device=DEV))
    spread[torch.rand(1, 2, tokens, generator=gen, device=DEV) < 0.2] = 0.0
    one_digit = 1.0 + torch.rand(1, 2, tokens, generator=gen, device=DEV) / 8          # more keys with the digit than LDS holds
    tied = (one_digit * 64).round() / 64
    for mass in (spread, one_digit, tied, torch.zeros_like(spread)):
        for length in (tokens, tokens - 70_001, 9000):
            batch = binding.FP4Batch(ints([length]), 0, table_pages=pages)
            for keep, sinks, recent in ((4096, 4, 512), (tokens // 2, 0, 0), (tokens // 3, 100_000, 70_000), (20, 20, 0)):
                kept, count = cache.kv_fp4_select(mass, batch, keep, sinks, recent)
                want = sorted_choice(mass[0], length, keep, sinks, recent)
                assert int(count) == want.shape[1]
                assert torch.equal(kept[0, :, :want.shape[1]].long(), want) and bool((kept[0, :, want.shape[1]:] == -1).all())


# a block of columns, some (64 pages to a wave), many
@pytest.mark.parametrize("new, pages", [(1, 90_000), (40, 900_000), (130, 90_000)])
def test_weights_of_thousands_of_heads_in_a_wide_table(new, pages):
    """More groups of pages than a launch has workgroups for with this many heads."""
    heads, lens = 5000, [130]
    cache = binding.FP4KVCache(3, heads, heads, 64)
    k = torch.randn(130, heads, 64, generator=torch.Generator().manual_seed(2)).half()
    table = torch.full((1, pages), -1, dtype=torch.int32)
    table[0, :3] = torch.tensor([2, 0, 1])
    narrow = binding.FP4Batch(ints(lens), 130, table[:, :3].contiguous().to(DEV))
    cache.kv_fp4_append(k.to(DEV), k.to(DEV), narrow)
    q = query(new, heads, 64, torch.float16, 3).to(DEV)
    lse = torch.empty(new, heads, device=DEV)
    narrow = binding.FP4Batch(ints(lens), new, table[:, :3].contiguous().to(DEV))
    cache.kv_fp4_attention(q, narrow, 0.1, lse=lse)
    past = torch.rand(1, heads, 200, device=DEV)
    want = cache.kv_fp4_weights(q, lse, narrow, 0.1, past=past, out=torch.full_like(past, -3.0))
    wide = binding.FP4Batch(ints(lens), new, table.to(DEV))
    got = cache.kv_fp4_weights(q, lse, wide, 0.1, past=past, out=torch.full_like(past, -3.0))
    assert torch.equal(got, want) and bool((got[..., 130:] == -3.0).all())
    some = [0, 1, 2499, 4999]
    exact, bound = ref.weights(q[:, some], fp4_reference.quantise(k[:, some])[0], lse[:, some], new, 0.1)
    exact[:, :130 - new] += past[0, some, :130 - new].cpu().double()
    close(got[0, some, :130], exact, bound + ref.STEP * exact)
    if new > 1:
        return
    # a sequence that fills the table, all of its pages missing but the last, for which mass has no place
    far = torch.full((1, pages), -1, dtype=torch.int32)
    far[0, pages - 1] = 2
    end = 64 * pages
    batch = binding.FP4Batch(ints([end]), 1, far.to(DEV))
    one = q[:1].contiguous()
    cache.kv_fp4_attention(one, batch, 0.1, lse=lse[:1])
    out = cache.kv_fp4_weights(one, lse[:1], batch, 0.1, past=past, out=torch.full_like(past, -3.0))
    assert torch.equal(out, past)
