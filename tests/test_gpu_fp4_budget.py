"""Attention weights of cached tokens, which of them are kept, and their rows moved together, against plain 64-bit arithmetic
(budget_reference, fp4_reference)."""
import math

import pytest
import torch

from paper_2512_24449_amd import binding
from tests import budget_reference as ref
from tests import fp4_reference
from tests.test_gpu_fp4_cache import DEV, ints, page_table, rows, starts

pytestmark = pytest.mark.gpu
NAN = float("nan")


class Filled:
    """A cache with sequences of lens tokens in pages anywhere, and what it holds."""

    def __init__(self, lens, kv_heads, group, dim, dtype, seed, more_pages=0, extra=0):
        self.lens, self.H, self.G, self.D, self.dtype = lens, kv_heads, group, dim, dtype
        self.table, self.n_pages = page_table(lens, extra, seed)
        self.cache = binding.FP4KVCache(self.n_pages + more_pages, kv_heads, kv_heads * group, dim)
        self.cache.pages.fill_(255)                              # bytes that no append wrote are NaNs and infinities
        k, v = rows(sum(lens), kv_heads, dim, dtype, seed + 1), rows(sum(lens), kv_heads, dim, dtype, seed + 2)
        self.cache.kv_fp4_append(k.to(DEV), v.to(DEV), self.batch(lens))
        self.k, self.v = (list(fp4_reference.quantise(x)[0].split(lens)) for x in (k, v))

    def batch(self, new, first=None, table=None, lens=None, max_new=None):
        return binding.FP4Batch(ints(lens or self.lens), max(new) if max_new is None else max_new, self.table if table is None else table,
                                new_rows=ints(new), first_row=ints(starts(new) if first is None else first))


def query(n, heads, dim, dtype, seed):
    return torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(seed)).to(dtype)


def close(got, want, bound):
    off = (got.cpu().double() - want).abs()
    assert bool((off <= bound).all()), (float((off - bound).max()), int((off > bound).sum()))


def check_weights(held, new, window=0, sinks=0, sm_scale=None, past=True, seed=50, room=None):
    sm_scale = held.D ** -0.5 if sm_scale is None else sm_scale
    q = query(sum(new), held.H * held.G, held.D, held.dtype, seed).to(DEV)
    batch = held.batch(new)
    lse = torch.empty(q.shape[:2], device=DEV)
    held.cache.kv_fp4_attention(q, batch, sm_scale, window, sinks, lse=lse)
    room = room or max(1, max(held.lens)) + 5
    old = torch.rand(len(held.lens), held.H, room, generator=torch.Generator().manual_seed(seed + 1)) + 0.01
    for b, (length, n) in enumerate(zip(held.lens, new)):        # what may not be read, or written
        old[b, :, max(length - n, 0):] = NAN
    out = torch.full(old.shape, -3.0, device=DEV)
    got = held.cache.kv_fp4_weights(q, lse, batch, sm_scale, window, sinks, past=old.to(DEV) if past else None, out=out)
    assert got is out
    at = 0
    for b, (length, n) in enumerate(zip(held.lens, new)):
        upto = min(length, room)
        m = min(n, length)                                       # (rows before the first token see nothing)
        if m:
            want, bound = ref.weights(q[at + n - m:at + n], held.k[b], lse[at + n - m:at + n], m, sm_scale, window, sinks)
        else:
            want = bound = torch.zeros(held.H, length, dtype=torch.float64)
        before = torch.where(torch.isnan(old[b]), 0.0, old[b]).double() if past else torch.zeros(held.H, room, dtype=torch.float64)
        want, bound = want[:, :upto] + before[:, :upto], bound[:, :upto]
        close(got[b, :, :upto], want, bound + ref.STEP * want)
        assert bool((got[b, :, upto:] == -3.0).all())
        at += n
    if past:                                                     # into past itself: the same bits
        same = old.to(DEV)
        held.cache.kv_fp4_weights(q, lse, batch, sm_scale, window, sinks, past=same, out=same)
        for b, length in enumerate(held.lens):
            upto = min(length, room)
            assert torch.equal(same[b, :, :upto], got[b, :, :upto])
    again = held.cache.kv_fp4_weights(q, lse, batch, sm_scale, window, sinks, past=old.to(DEV) if past else None, out=torch.full_like(out, -3.0))
    assert torch.equal(again, got)
    return got


CASES = [  # lens, new, H, G, D
    ([1], [1], 1, 1, 128), ([1000], [1], 1, 1, 128), ([63, 64, 65], [1, 1, 1], 2, 4, 64), ([300, 0, 7], [1, 1, 1], 3, 5, 128),
    ([513], [1], 2, 16, 128), ([130, 257], [5, 3], 2, 3, 64), ([200], [32], 2, 4, 128), ([640, 77], [100, 77], 2, 2, 128),
    ([200, 129], [200, 129], 1, 4, 64), ([700], [333], 1, 7, 128), ([90, 40], [0, 40], 2, 1, 128), ([5], [9], 1, 2, 64),
    ([1500], [17], 1, 1, 128), ([2100], [64], 1, 12, 64)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens, new, H, G, D", CASES)
def test_weights(lens, new, H, G, D, dtype):
    held = Filled(lens, H, G, D, dtype, 20)
    check_weights(held, new)
    check_weights(held, new, past=False, seed=51)


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 3), (40, 0), (64, 64), (100, 4), (129, 70), (5000, 2), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_weights_through_windows(window, sinks):
    for lens, new, H, G, D in (([900, 70], [1, 1], 2, 2, 128), ([400, 333], [150, 64], 1, 3, 64), ([700], [700], 1, 1, 128)):
        check_weights(Filled(lens, H, G, D, torch.float16, 21), new, window, sinks)


@pytest.mark.parametrize("sm_scale", [0.0, -0.2, 1e-30, 3.0, 40.0])
def test_weights_of_any_scale(sm_scale):
    for dtype in (torch.float16, torch.bfloat16):
        held = Filled([300, 65], 2, 3, 128, dtype, 22)
        check_weights(held, [1, 2], sm_scale=sm_scale)
        check_weights(held, [40, 65], sm_scale=sm_scale)


def test_weights_of_a_narrow_tensor_and_of_a_wide_table():
    held = Filled([300, 200], 2, 1, 128, torch.float16, 23, extra=40)
    check_weights(held, [1, 30], room=100)
    check_weights(held, [1, 30], room=1)
    q = query(2, 2, 128, torch.float16, 1).to(DEV)
    batch = held.batch([1, 1])
    lse = torch.empty(2, 2, device=DEV)
    held.cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
    made = held.cache.kv_fp4_weights(q, lse, batch, 0.1)
    assert made.shape == (2, 2, 64 * batch.table_pages)
    assert bool((made[0, :, 300:] == 0).all()) and bool((made[1, :, 200:] == 0).all())
    # A row's weights are 1 in all, but for the error of lse that the call was given (the sum of exp(s - lse) is exp(true lse - lse),
    # and lse may be off by lse_bound) and for their own.
    for b in range(2):
        _, _, _, lse_bound = fp4_reference.attention(q[b:b + 1].cpu(), held.k[b], held.v[b], 1, 0.1)
        want, bound = ref.weights(q[b:b + 1], held.k[b], lse[b:b + 1], 1, 0.1)
        close(made[b].double().sum(-1), torch.ones(2, dtype=torch.float64), torch.expm1(lse_bound[0]) + bound.sum(-1))


def test_weights_of_missing_pages_and_rows_outside():
    held = Filled([300, 200], 2, 2, 64, torch.float16, 24)
    table = held.table.clone()
    table[0, 1], table[0, 3], table[1, 0] = -1, held.n_pages, 2 ** 31 - 1
    new = [70, 3]
    q = query(100, 4, 64, torch.float16, 61).to(DEV)
    batch = held.batch(new, first=[45, -1], table=table)         # rows 100 .. of the first and -1 of the second are not there
    lse = torch.full((100, 4), NAN, device=DEV)
    held.cache.kv_fp4_attention(q, batch, 0.2, lse=lse)
    past = torch.rand(2, 2, 300, device=DEV)
    got = held.cache.kv_fp4_weights(q, lse, batch, 0.2, past=past)
    for b, (length, n, first) in enumerate(((300, 70, 45), (200, 3, -1))):
        present = torch.ones(length, dtype=torch.bool)
        for page in ((1, 3) if b == 0 else (0,)):
            present[64 * page:64 * page + 64] = False
        row = torch.arange(first, first + n)
        there = (row >= 0) & (row < 100)
        at = row.clamp(0, 99)
        want, bound = ref.weights(q[at.to(DEV)], held.k[b], torch.where(there[:, None], lse.cpu()[at], 0.0), n, 0.2, present=present, rows=there)
        want[:, :length - n] += past[b, :, :length - n].cpu().double()
        close(got[b, :, :length], want, bound + ref.STEP * want)


def test_weights_of_rows_that_are_not_finite():
    held = Filled([130], 2, 2, 128, torch.float16, 25)
    q = query(3, 4, 128, torch.float16, 62)
    q[1, 2, 7], q[2, 1, 0] = NAN, float("inf")
    q = q.to(DEV)
    batch = held.batch([3])
    lse = torch.empty(3, 4, device=DEV)
    held.cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
    assert torch.isnan(lse[1, 2]) and torch.isnan(lse[2, 1])
    got = held.cache.kv_fp4_weights(q, lse, batch, 0.1)[0].cpu()
    # kv-head 1 has the NaN row (tokens 0 .. 128), kv-head 0 the infinite one (all)
    assert torch.isnan(got[1, :129]).all() and torch.isfinite(got[1, 129]) and torch.isnan(got[0, :130]).all()
    lse[1, 2] = lse[2, 1] = -math.inf                            # a row said to see nothing gives nothing
    q[1, 2], q[2, 1] = 0, 0
    got = held.cache.kv_fp4_weights(q, lse, batch, 0.1)[0]
    want, bound = ref.weights(q, held.k[0], lse, 3, 0.1)
    close(got[:, :130], want, bound + ref.STEP * want)


def test_weights_of_no_rows():
    held = Filled([100, 30], 2, 2, 64, torch.bfloat16, 26)
    past = torch.rand(2, 2, 100, device=DEV)
    none = held.cache.kv_fp4_weights(query(0, 4, 64, torch.bfloat16, 1).to(DEV), torch.empty(0, 4, device=DEV), held.batch([0, 0], max_new=0), 0.1,
                                     past=past)
    assert torch.equal(none[0], past[0]) and torch.equal(none[1, :, :30], past[1, :, :30]) and bool((none[1, :, 30:] == 0).all())


def test_queries_in_parts_of_wider_rows():
    held = Filled([300], 2, 2, 128, torch.float16, 27)
    wide = torch.randn(20, 8 * 128, device=DEV).half()
    q = wide[:, 256:768].unflatten(1, (4, 128))
    batch = held.batch([20])
    lse = torch.empty(20, 4, device=DEV)
    held.cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
    assert torch.equal(held.cache.kv_fp4_weights(q, lse, batch, 0.1), held.cache.kv_fp4_weights(q.contiguous(), lse, batch, 0.1))


def test_weights_of_several_pages_to_a_wave():
    """Wide tables: what a wave takes follows the table's width; pages that rows see and do not see in turn."""
    for lens, new, G in (([3000, 700], [1, 1], 2), ([3000, 700], [20, 9], 3)):
        held = Filled(lens, 2, G, 64, torch.float16, 28, extra=4000)
        check_weights(held, new)
        check_weights(held, new, window=300, sinks=70, seed=52)
        check_weights(held, new, window=1, past=False, seed=53)


def check_long(tokens, new, dim=64):
    """One head, values that repeat: what the cache holds by kv_fp4_read, scores in 64 bits on the GPU."""
    gen = torch.Generator(device=DEV).manual_seed(54)
    k = torch.randn(tokens, 1, dim, generator=gen, device=DEV).half()
    n_pages = -(-tokens // 64)
    cache = binding.FP4KVCache(n_pages, 1, 1, dim)
    batch = binding.FP4Batch(ints([tokens]), tokens, table_pages=n_pages)
    cache.kv_fp4_append(k, k, batch)
    values = cache.kv_fp4_read(batch, tokens, torch.float16)[0][:, 0]
    q = torch.randn(new, 1, dim, generator=gen, device=DEV).half()
    rows_of = binding.FP4Batch(ints([tokens]), new, table_pages=n_pages)
    lse = torch.empty(new, 1, device=DEV)
    cache.kv_fp4_attention(q, rows_of, 0.1, lse=lse)
    got = cache.kv_fp4_weights(q, lse, rows_of, 0.1)
    want, bound = torch.zeros(tokens, dtype=torch.float64, device=DEV), torch.zeros(tokens, dtype=torch.float64, device=DEV)
    t = torch.arange(tokens, device=DEV)
    for i in range(new):                                         # (the bound of budget_reference.weights)
        s = values.double() @ q[i, 0].double() * 0.1
        size = values.double().abs() @ q[i, 0].double().abs() * 0.1
        p = torch.where(t <= tokens - new + i, torch.exp(s - lse[i, 0].double()), 0.0)
        want += p
        bound += p * torch.expm1((dim + 8) * ref.STEP * size + 3 * ref.STEP * (s.abs() + lse[i, 0].double().abs()) + 2 * ref.STEP)
    bound += (new + 2) * ref.STEP * want + new * 2.0 ** -126
    assert bool(((got[0, 0, :tokens].double() - want).abs() <= bound).all())
    return cache, got, rows_of


def test_more_pages_than_a_launch_has_workgroups_for():
    check_long(1_100_000, 200)
    cache, mass, batch = check_long(6_400_001, 1)
    kept, count = cache.kv_fp4_select(mass, batch, 100_000, 4, 1000)
    middle = mass[0, 0, 4:6_400_001 - 1000].double()
    most = torch.sort(-middle, stable=True).indices[:100_000 - 1004] + 4
    want = torch.cat([most, torch.arange(4, device=DEV), torch.arange(6_400_001 - 1000, 6_400_001, device=DEV)]).sort().values
    assert torch.equal(kept[0, 0].long(), want) and int(count) == 100_000


# ---- which tokens are kept ----

def heavy(shape, seed, zeros=0.2):
    gen = torch.Generator().manual_seed(seed)
    m = torch.exp(3 * torch.randn(shape, generator=gen))
    m[torch.rand(shape, generator=gen) < zeros] = 0.0
    return m


def check_select(mass, lens, keep, sinks, recent, budgets=None, table_pages=None):
    B, H, T = mass.shape
    cache = binding.FP4KVCache(1, H, H, 64)
    pages = table_pages or max(1, -(-max(lens) // 64))
    batch = binding.FP4Batch(ints(lens), 0, table_pages=pages)
    kept, count = cache.kv_fp4_select(mass.to(DEV), batch, keep, sinks, recent, budgets=None if budgets is None else ints(budgets))
    kept, count = kept.cpu(), count.cpu()
    for b in range(B):
        length = min(lens[b], 64 * pages)
        for h in range(H):
            want = ref.kept(mass[b, h].tolist(), length, keep, sinks, recent, None if budgets is None else budgets[b])
            assert kept[b, h].tolist() == want + [-1] * (keep - len(want)), (b, h)
            assert int(count[b]) == len(want)


@pytest.mark.parametrize("lens, keep, sinks, recent", [
    ([1], 1, 0, 0), ([2], 1, 0, 0), ([2], 1, 1, 0), ([2], 1, 5, 5), ([2], 1, 0, 1), ([70, 0, 64], 64, 4, 16), ([1000, 999, 12], 200, 4, 32),
    ([1000], 999, 0, 0), ([1000], 1000, 0, 0), ([1000], 2000, 3, 3), ([5000, 4097], 37, 0, 0), ([5000], 2500, 2500, 7), ([5000], 2500, 100, 5000),
    ([20000, 8193], 4096, 4, 512), ([1025], 1024, 0, 1023), ([66000], 30000, 4, 100)])
def test_select(lens, keep, sinks, recent):
    check_select(heavy((len(lens), 2, max(lens)), len(lens) + keep), lens, keep, sinks, recent)


def test_select_among_equal_weights_takes_the_first():
    check_select(torch.ones(1, 2, 3000), [3000], 700, 3, 10)
    check_select(torch.zeros(1, 1, 1300), [1300], 100, 0, 0)
    m = torch.randint(0, 3, (2, 3, 5000), generator=torch.Generator().manual_seed(1)).float()
    check_select(m, [5000, 4001], 2222, 4, 100)
    m[m == 0] = -0.0
    m[:, :, ::7] = 0.0                                           # both zeros are the same weight
    check_select(m, [5000, 4001], 4500, 0, 0)
    # weights that differ in the last bit only, and by sign
    bits = 0x3F800000 + torch.randint(0, 9, (1, 2, 4000), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    check_select(bits.view(torch.float32), [4000], 1000, 0, 0)
    m = torch.randn(1, 2, 4000, generator=torch.Generator().manual_seed(3))
    check_select(m, [4000], 3000, 0, 0)


def test_select_among_infinities_and_nans():
    m = torch.randn(2, 2, 2000, generator=torch.Generator().manual_seed(4))
    m[..., 5::17], m[..., 3::19], m[..., 1::23] = NAN, float("inf"), -float("inf")
    m[1, 0, 5] = -torch.tensor(NAN)
    for keep in (50, 200, 1900, 1990):
        check_select(m, [2000, 1500], keep, 2, 9)
    m.fill_(NAN)
    check_select(m, [2000, 100], 99, 0, 0)


def test_select_with_budgets_narrow_tensors_and_narrow_tables():
    lens = [900, 800, 700, 600, 50, 0]
    m = heavy((6, 2, 900), 6)
    check_select(m, lens, 300, 4, 20, budgets=[300, 299, 0, -5, 400, 10])
    check_select(m, lens, 300, 4, 20, budgets=[1, 2 ** 31 - 1, -2 ** 31, 24, 25, 1])
    check_select(m[..., :100].contiguous(), lens, 300, 4, 20)    # tokens without a place have weight 0
    check_select(m[..., :1].contiguous(), lens, 20, 0, 0)
    check_select(m, lens, 150, 4, 20, table_pages=10)
    check_select(m, [-5, 800, 700, 2 ** 31 - 1, 50, 3], 150, 4, 20, table_pages=10)


@pytest.mark.parametrize("pages", [600, 1025])
def test_select_in_long_tables(pages):
    """Tables of more than 32768 tokens: sequences of all lengths in them, few and many tokens with the decisive weight's first digits."""
    lens = [64 * pages, 40000, 8192, 8193, 3, 0]
    m = heavy((6, 1, 64 * pages), 7)
    check_select(m, lens, 5000, 4, 100, table_pages=pages)
    check_select(m, lens, 37000, 0, 0, table_pages=pages, budgets=[37000, 36999, 5000, 8193, 0, 9])
    check_select(m, lens, 3000, 3000, 9, table_pages=pages)
    check_select(m, lens, 40000, 10000, 20000, table_pages=pages)
    check_select(m[..., :30000].contiguous(), lens, 20000, 4, 100, table_pages=pages)
    m = (1.0 + torch.rand(6, 1, 64 * pages, generator=torch.Generator().manual_seed(8)) / 8)      # one first digit for all
    check_select(m, lens, 20000, 4, 100, table_pages=pages)
    check_select((m * 64).round() / 64, lens, 20001, 0, 100, table_pages=pages)
    check_select(torch.zeros(6, 1, 64 * pages), lens, 33333, 1, 1, table_pages=pages)


def test_select_of_many_heads_in_long_tables():
    """More than the workspace takes in parts: a workgroup to a head all the same."""
    lens, heads = [40000, 100], 300
    m = heavy((2, heads, 40000), 9)
    cache = binding.FP4KVCache(1, heads, heads, 64)
    batch = binding.FP4Batch(ints(lens), 0, table_pages=700)
    kept, count = cache.kv_fp4_select(m.to(DEV), batch, 1000, 4, 100)
    assert count.tolist() == [1000, 100]
    for b, h in ((0, 0), (0, 299), (1, 7), (0, 123)):
        want = ref.kept(m[b, h].tolist(), lens[b], 1000, 4, 100)
        assert kept[b, h].tolist() == want + [-1] * (1000 - len(want))


# ---- rows moved together ----

@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens, H, D, keep", [([1], 1, 128, 1), ([300], 2, 128, 77), ([64, 200, 0, 9], 3, 64, 64), ([700, 130], 2, 128, 200),
                                              ([500, 20], 1, 64, 65)])
def test_compact(lens, H, D, keep, dtype):
    B, kept_pages = len(lens), -(-keep // 64)
    held = Filled(lens, H, 1, D, dtype, 30, more_pages=B * kept_pages)
    n = [min(length, keep - (3 if b % 2 else 0)) for b, length in enumerate(lens)]
    gen = torch.Generator().manual_seed(31)
    kept = torch.full((B, H, keep), -1, dtype=torch.int32)
    for b in range(B):
        for h in range(H):
            kept[b, h, :n[b]] = torch.randperm(lens[b], generator=gen)[:n[b]].sort().values.int()
            kept[b, h, n[b]:] = 5                                # (behind n_kept: not looked at)
    mass = torch.rand(B, H, max(lens) + 3, generator=gen)
    to_table = held.n_pages + torch.arange(B * kept_pages, dtype=torch.int32).view(B, kept_pages).flip(0)
    count = ints(n)
    to = binding.FP4Batch(count, keep, to_table.contiguous().to(DEV), new_rows=count)
    mass_out = torch.full((B, H, keep + 7), -3.0, device=DEV)
    before = held.cache.pages.clone()
    got = held.cache.kv_fp4_compact(kept.to(DEV), count, held.batch([0] * B, max_new=0), to, mass=mass.to(DEV), mass_out=mass_out)
    assert got is mass_out
    page = H * 64 * (D + D // 16)
    assert torch.equal(held.cache.pages[:held.n_pages * page], before[:held.n_pages * page])   # what they came from stays
    out = [torch.full((B * keep, H, D), 9.0, device=DEV) for _ in range(2)]
    held.cache.kv_fp4_read(to, B * keep, torch.float32, k=out[0], v=out[1])
    for b in range(B):
        for h in range(H):
            index = kept[b, h, :n[b]].long()
            for x, y in zip((held.k, held.v), out):
                assert torch.equal(y[b * keep:b * keep + n[b], h].cpu().double(), x[b][index, h])
            assert torch.equal(mass_out[b, h, :n[b]].cpu(), mass[b, h, index])
        assert bool((mass_out[b, :, n[b]:] == -3.0).all())
    made = held.cache.kv_fp4_compact(kept.to(DEV), count, held.batch([0] * B, max_new=0), to, mass=mass.to(DEV))
    assert made.shape == (B, H, keep) and all(torch.equal(made[b, :, :n[b]], mass_out[b, :, :n[b]]) for b in range(B))
    assert held.cache.kv_fp4_compact(kept.to(DEV), count, held.batch([0] * B, max_new=0), to) is None


@pytest.mark.parametrize("B, H, D, keep", [(4, 8, 64, 2603), (8, 8, 128, 4101), (3, 30, 64, 1441)])
def test_compact_of_many_tokens(B, H, D, keep):
    """Several eights to a wave, ends inside them, tokens that are not there among them: against what reading back and gathering give."""
    gen = torch.Generator(device=DEV).manual_seed(33)
    lens = [keep + 1500 - 37 * b for b in range(B)]
    most, kept_pages = max(lens), -(-keep // 64)
    pages = -(-most // 64)
    cache = binding.FP4KVCache(B * (pages + kept_pages), H, H, D)
    order = torch.randperm(B * (pages + kept_pages), generator=gen, device=DEV).int()
    table, to_table = order[:B * pages].view(B, pages).contiguous(), order[B * pages:].view(B, kept_pages).contiguous()
    n = ints(lens)
    whole = binding.FP4Batch(n, most, table, new_rows=n)
    k, v = (torch.randn(B * most, H, D, generator=gen, device=DEV).half() for _ in range(2))
    cache.kv_fp4_append(k, v, whole)
    held = [x.view(B, most, H, D) for x in cache.kv_fp4_read(whole, B * most)]
    kept = torch.randint(0, most + 20, (B, H, keep), generator=gen, device=DEV, dtype=torch.int32)   # (some behind the end)
    count = ints([keep - 5 * b for b in range(B)])
    to = binding.FP4Batch(count, keep, to_table, new_rows=count)
    mass = torch.rand(B, H, most, generator=gen, device=DEV)
    moved = cache.kv_fp4_compact(kept, count, whole, to, mass=mass)
    out = [x.view(B, keep, H, D) for x in cache.kv_fp4_read(to, B * keep)]
    for b in range(B):
        m = keep - 5 * b
        there = kept[b, :, :m] < lens[b]
        index = kept[b, :, :m].clamp(max=lens[b] - 1).long()
        assert torch.equal(moved[b, :, :m], torch.where(there, mass[b].gather(1, index), 0.0)) and bool((moved[b, :, m:] == 0).all())
        for x, y in zip(held, out):
            want = x[b].gather(0, index.T[..., None].expand(-1, -1, D))
            assert torch.equal(y[b, :m], torch.where(there.T[..., None], want, torch.zeros_like(want)))


def test_compact_of_odd_positions():
    """Out of order, the same twice, not there, of a missing page; to a missing page; fewer and more than there is room for."""
    held = Filled([300, 100], 2, 1, 128, torch.float16, 32, more_pages=6)
    table = held.table.clone()
    table[0, 1] = -1
    source = binding.FP4Batch(ints([300, 100]), 0, table)
    kept = torch.tensor([[[299, 0, 0, 64, 300, -1, 127, 128, 2 ** 31 - 1, -2 ** 31, 63, 63] + [10] * 128] * 2,
                         [[99, 100, 98] + [7] * 137] * 2], dtype=torch.int32, device=DEV)
    first = held.n_pages
    to_table = torch.tensor([[first, -1, first + 1], [first + 2, first + 3, 2 ** 30]], dtype=torch.int32, device=DEV)
    count = ints([140, 500])                                     # (more than keep: keep)
    to = binding.FP4Batch(count, 140, to_table, new_rows=ints([140, 140]))
    mass = torch.arange(2 * 2 * 200, dtype=torch.float32, device=DEV).view(2, 2, 200)
    mass_out = torch.full((2, 2, 100), -3.0, device=DEV)
    held.cache.pages[first * 2 * 64 * 136:] = 255
    held.cache.kv_fp4_compact(kept, count, source, to, mass=mass, mass_out=mass_out)
    k, v = (x.cpu().double().view(2, 140, 2, 128) for x in held.cache.kv_fp4_read(binding.FP4Batch(ints([140, 140]), 140, to_table), 280, torch.float32))
    for b, length in enumerate((300, 100)):
        for i in range(140):
            t = int(kept[b, 0, i])
            there = 0 <= t < length and not (b == 0 and 64 <= t < 128) and not (b == 0 and 64 <= i < 128) and not (b == 1 and i >= 128)
            for x, y in ((held.k, k), (held.v, v)):
                assert torch.equal(y[b, i], x[b][t] if there else torch.zeros(2, 128, dtype=torch.float64)), (b, i, t)
            if i < 100:
                want = mass[b, :, t].cpu() if 0 <= t < min(length, 200) else torch.zeros(2)
                assert torch.equal(mass_out[b, :, i].cpu(), want)


def test_pages_beyond_4_gib():
    heads, n_pages = 64, 9000
    cache = binding.FP4KVCache(n_pages, heads, heads, 128)       # 5 GB
    k, v = rows(130, heads, 128, torch.float16, 40).to(DEV), rows(130, heads, 128, torch.float16, 41).to(DEV)
    batch = binding.FP4Batch(ints([130]), 130, ints([[8999, 3, 8998]]))
    cache.kv_fp4_append(k, v, batch)
    q = query(130, heads, 128, torch.float16, 42).to(DEV)
    lse = torch.empty(130, heads, device=DEV)
    cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
    got = cache.kv_fp4_weights(q, lse, batch, 0.1)
    want, bound = ref.weights(q, fp4_reference.quantise(k.cpu())[0], lse, 130, 0.1)
    close(got[0, :, :130], want, bound + ref.STEP * want)
    kept, count = cache.kv_fp4_select(got, batch, 70)
    to = binding.FP4Batch(count, 70, ints([[8997, 5000]]), new_rows=count)
    cache.kv_fp4_compact(kept, count, batch, to)
    out, index = cache.kv_fp4_read(to, 70, torch.float32), kept[0].long().T[..., None].expand(-1, -1, 128).cpu()
    for x, y in zip((k, v), out):
        assert torch.equal(y.cpu().double(), fp4_reference.quantise(x.cpu())[0].gather(0, index))


def test_weights_beyond_2_to_the_31():
    tokens = 420_000_000                                         # 10 GB
    held = Filled([100, 70, 90], 2, 1, 64, torch.float16, 43, more_pages=6)
    q = query(3, 2, 64, torch.float16, 44).to(DEV)
    batch = held.batch([1, 1, 1])
    lse = torch.empty(3, 2, device=DEV)
    held.cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
    small = held.cache.kv_fp4_weights(q, lse, batch, 0.1)
    out = torch.empty(3, 2, tokens, device=DEV)
    held.cache.kv_fp4_weights(q, lse, batch, 0.1, out=out)
    for b, n in enumerate(held.lens):
        assert torch.equal(out[b, :, :n], small[b, :, :n])
    kept = held.cache.kv_fp4_select(out, batch, 40)
    want = held.cache.kv_fp4_select(small, batch, 40)
    assert torch.equal(kept[0], want[0]) and torch.equal(kept[1], want[1])
    to = binding.FP4Batch(want[1], 40, held.n_pages + ints([[0], [1], [2]]))
    moved = held.cache.kv_fp4_compact(*want, batch, to, mass=out)
    assert torch.equal(moved, torch.gather(small, 2, want[0].long()))


# ---- together ----

def step_inputs(B, H, G, D, step, dtype):
    gen = torch.Generator().manual_seed(700 + step)
    return [torch.randn(B, h, D, generator=gen).to(dtype) for h in (H * G, H, H)]


@pytest.mark.parametrize("captured", [False, True])
def test_a_decoding_batch_within_a_budget(captured):
    """Turn, append, attend, weigh; when the cache is full, select and move: against the same in 64 bits, every step's output."""
    B, H, G, D, dtype, keep, full = 2, 2, 2, 128, torch.float16, 40, 70
    scale, sinks, recent = D ** -0.5, 2, 8
    cache = binding.FP4KVCache(2 * 2 * B, H, H * G, D)
    rotary = binding.Rotary(D, 64, scaling="bands", factor=4.0, original=32)
    tables = [ints([[0, 1], [2, 3]]), ints([[4, 5], [6, 7]])]
    table, spare = tables[0].clone(), tables[1].clone()
    lens, pos = ints([0, 0]), torch.tensor([1000, 5], dtype=torch.int32, device=DEV)
    q, k, v = (torch.zeros(B, h, D, dtype=dtype, device=DEV) for h in (H * G, H, H))
    lse, mass, moved = torch.empty(B, H * G, device=DEV), torch.zeros(B, H, 128, device=DEV), torch.zeros(B, H, 128, device=DEV)
    n_kept = ints([0, 0])
    batch = binding.FP4Batch(lens, 1, table)
    cut = binding.FP4Batch(n_kept, 1, spare)
    q_turned, k_turned, out = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)

    def step():
        lens.add_(1)
        rotary.kv_rotary(q, pos, k=k, out=q_turned, k_out=k_turned)
        cache.kv_fp4_append(k_turned, v, batch)
        cache.kv_fp4_attention(q_turned, batch, scale, out=out, lse=lse)
        cache.kv_fp4_weights(q_turned, lse, batch, scale, past=mass, out=mass)
        pos.add_(1)

    def drop():
        kept, _ = cache.kv_fp4_select(mass, batch, keep, sinks, recent, n_kept=n_kept)
        cache.kv_fp4_compact(kept, n_kept, batch, cut, mass=mass, mass_out=moved)
        mass.copy_(moved)
        lens.copy_(n_kept)
        old = table.clone()
        table.copy_(spare)
        spare.copy_(old)
        return kept

    graph = None
    if captured:
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        lens.zero_()
        pos.sub_(1)
        torch.cuda.synchronize()
    held = [[torch.zeros(0, H, D, dtype=torch.float64) for _ in range(2)] for _ in range(B)]
    sums = [torch.zeros(H, 0, dtype=torch.float64) for _ in range(B)]
    bounds = [torch.zeros(H, 0, dtype=torch.float64) for _ in range(B)]
    for i in range(2 * full):
        for to, x in zip((q, k, v), step_inputs(B, H, G, D, i, dtype)):
            to.copy_(x)
        where = pos.cpu()
        graph.replay() if graph else step()
        torch.cuda.synchronize()
        for x, y in ((q, q_turned), (k, k_turned)):
            want, bound = ref.turned(x, where, rotary.frequencies, rotary.magnitude, False)
            close(y, want, ref.rounded(want, bound, dtype))
        for b in range(B):
            for j, x in enumerate((k_turned, v)):
                held[b][j] = torch.cat([held[b][j], fp4_reference.quantise(x[b:b + 1].cpu())[0]])
            length = held[b][0].shape[0]
            assert length == int(lens[b])
            want, _, bound, _ = fp4_reference.attention(q_turned[b:b + 1].cpu(), *held[b], 1, scale)
            close(out[b:b + 1], want, ref.rounded(want, bound, dtype))
            more, off = ref.weights(q_turned[b:b + 1], held[b][0], lse[b:b + 1], 1, scale)
            new = torch.zeros(H, 1, dtype=torch.float64)
            sums[b], bounds[b] = torch.cat([sums[b], new], 1) + more, torch.cat([bounds[b], new], 1) + off
            bounds[b] += ref.STEP * sums[b]
            close(mass[b, :, :length], sums[b], bounds[b])
        if int(lens.max()) == full:
            before = mass.cpu()
            kept = drop().cpu()
            for b in range(B):
                for h in range(H):
                    assert kept[b, h].tolist() == ref.kept(before[b, h].tolist(), full, keep, sinks, recent)
                index = kept[b].long()
                held[b] = [x.gather(0, index.T[..., None].expand(-1, -1, D)) for x in held[b]]
                sums[b], bounds[b] = sums[b].gather(1, index), bounds[b].gather(1, index)


def test_calls_on_another_stream_and_replays():
    held = Filled([500, 300], 2, 4, 128, torch.float16, 45, more_pages=6)
    q = query(6, 8, 128, torch.float16, 46).to(DEV)
    batch = held.batch([4, 2])
    lse = torch.empty(6, 8, device=DEV)
    held.cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
    to_table = held.n_pages + ints([[0, 1], [2, 3]])

    def all_of_it(stream=None):
        mass = held.cache.kv_fp4_weights(q, lse, batch, 0.1, stream=stream)
        kept, count = held.cache.kv_fp4_select(mass, batch, 100, 4, 10, stream=stream)
        to = binding.FP4Batch(count, 100, to_table, new_rows=count)
        moved = held.cache.kv_fp4_compact(kept, count, batch, to, mass=mass, stream=stream)
        return [mass, kept, count, moved, *held.cache.kv_fp4_read(to, 200, torch.float16, stream=stream)]
    want = all_of_it()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = all_of_it(stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of_it()
    for turn in range(3):
        q.mul_(-0.5)
        held.cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
        for t in got:
            t.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        want = all_of_it()
        torch.cuda.synchronize()
        n = want[2].tolist()
        assert torch.equal(got[2], want[2]) and all(torch.equal(got[i], want[i]) for i in (1,))
        for b in range(2):
            assert torch.equal(got[0][b, :, :held.lens[b]], want[0][b, :, :held.lens[b]])
            assert torch.equal(got[3][b, :, :n[b]], want[3][b, :, :n[b]])
            for i in (4, 5):
                assert torch.equal(got[i][100 * b:100 * b + n[b]], want[i][100 * b:100 * b + n[b]])
