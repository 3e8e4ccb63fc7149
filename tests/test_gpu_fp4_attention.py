"""Attention over the 4-bit paged cache against 64-bit arithmetic on the values the cache holds, within the bound that
fp4_reference.attention derives, and half a step of the output's type."""
import math

import pytest
import torch

from paper_2512_24449_amd import binding
from tests import fp4_reference as ref
from tests.test_gpu_fp4_cache import DEV, ints, page_table, rows, starts

pytestmark = pytest.mark.gpu


def filled(lens, H, Hq, D, dtype, seed=0, size=1.0, table=None):
    """A cache that holds `lens` tokens of random K (four large channels a head) and V, their values, and the page table."""
    made, n_pages = page_table(lens, extra=1, seed=seed)
    table = made if table is None else table(made)
    cache = binding.FP4KVCache(n_pages, H, Hq, D)
    cache.pages.fill_(255)                                      # where nothing is written: NaN and infinity as scales
    gen = torch.Generator().manual_seed(seed)
    total = sum(lens)
    k, v = torch.randn(total, H, D, generator=gen) * size, torch.randn(total, H, D, generator=gen)
    k[:, :, 3:D:D // 4] *= 10.0
    k, v = k.to(dtype), v.to(dtype)
    if total:
        cache.kv_fp4_append(k.to(DEV), v.to(DEV), binding.FP4Batch(ints(lens), max(lens), table, new_rows=ints(lens),
                                                                   first_row=ints(starts(lens))))
    return cache, ref.quantise(k)[0], ref.quantise(v)[0], table


def check(cache, k, v, lens, new, q, out, lse, scale, window=0, sinks=0, present=None):
    at = row = 0
    for b, (length, n) in enumerate(zip(lens, new)):
        m = min(n, length)
        got, got_lse = out[row:row + n].cpu().double(), lse[row:row + n].cpu().double()
        assert not got[:n - m].any() and bool((got_lse[:n - m] == -math.inf).all())   # positions below 0
        at, row = at + length, row + n
        if m == 0:
            continue
        got, got_lse = got[n - m:], got_lse[n - m:]
        want, want_lse, bound, lse_bound = ref.attention(q[row - m:row].cpu(), k[at - length:at], v[at - length:at], m, scale,
                                                         window, sinks, None if present is None else present[b])
        step = torch.finfo(out.dtype).eps / 2
        off = (got - want).abs() - bound - (want.abs() + bound) * step
        assert bool((off <= 1e-7).all()), (b, length, n, float(off.max()), float((got - want).abs().max()))   # 1e-7: fp16 below its normal range
        empty = want_lse == -math.inf
        assert torch.equal(empty, got_lse == -math.inf) and not got[empty].any()
        assert bool(((got_lse - want_lse).abs()[~empty] <= lse_bound[~empty]).all())


def run(lens, new, H, G, D, dtype, window=0, sinks=0, seed=0, out_dtype=None, size=1.0, scale=None):
    cache, k, v, table = filled(lens, H, H * G, D, dtype, seed, size)
    q = rows(sum(new), H * G, D, dtype, seed + 1)
    scale = 1 / math.sqrt(D) if scale is None else scale
    batch = binding.FP4Batch(ints(lens), max(max(new), 1), table, new_rows=ints(new), first_row=ints(starts(new)))
    lse = torch.full((sum(new), H * G), 7.0, dtype=torch.float32, device=DEV)
    out = torch.full((sum(new), H * G, D), 7.0, dtype=out_dtype or dtype, device=DEV)
    got = cache.kv_fp4_attention(q.to(DEV), batch, scale, window, sinks, out=out, lse=lse)
    assert got is out
    check(cache, k, v, lens, new, q, out, lse, scale, window, sinks)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D, H, G, lens", [(128, 1, 1, [1]), (128, 2, 1, [2, 31, 32, 33]), (128, 1, 4, [64, 65, 127]),
                                           (64, 3, 2, [128, 1, 700]), (128, 2, 16, [1000]), (64, 1, 17, [999]),
                                           (128, 1, 3, [5000]), (128, 5, 8, [63, 0, 300])])
def test_single_tokens(D, H, G, lens, dtype):
    run(lens, [1] * len(lens), H, G, D, dtype, seed=len(lens) + G)


@pytest.mark.parametrize("D, H, G, lens, new", [(128, 2, 4, [300, 17], [5, 3]), (64, 1, 1, [129], [2]), (128, 1, 1, [77], [77]),
                                                (128, 2, 2, [64, 200], [64, 0]), (64, 2, 3, [513, 40], [130, 40]),
                                                (128, 1, 4, [1100], [300]), (128, 1, 8, [90], [90]), (64, 1, 40, [50], [9]),
                                                (128, 3, 1, [20, 3, 0], [33, 5, 2])])   # more new rows than tokens
def test_several_rows(D, H, G, lens, new):
    run(lens, new, H, G, D, torch.float16, seed=G)
    run(lens, new, H, G, D, torch.bfloat16, seed=G + 1, out_dtype=torch.float32)


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 4), (7, 1), (32, 0), (33, 31), (64, 64), (100, 33), (500, 4), (5000, 3),
                                           (2 ** 31 - 1, 2 ** 31 - 1), (40, 2 ** 31 - 1)])
@pytest.mark.parametrize("new", [[1, 1, 1], [4, 1, 9], [150, 33, 1]])
def test_windows(window, sinks, new):
    run([700, 33, 129], new, 2, 3, 128, torch.float16, window, sinks, seed=window % 97)


def test_window_heads_of_64():
    run([300, 1500], [200, 77], 2, 2, 64, torch.bfloat16, 90, 5, seed=3)


@pytest.mark.parametrize("out_dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_output_types(out_dtype):
    for D in (64, 128):
        run([200, 2000], [3, 1], 2, 2, D, torch.float16, out_dtype=out_dtype)


@pytest.mark.parametrize("scale, size", [(0.0, 1.0), (-0.1, 1.0), (1.0, 1.0), (0.05, 300.0), (0.1, 1e-4), (3.0, 4.0)])
def test_scales(scale, size):
    """Uniform weights, negative scales, one token that takes all the weight."""
    run([450, 90], [2, 30], 1, 2, 128, torch.float16, scale=scale, size=size)


def test_tokens_that_no_row_sees_are_not_read():
    """A window: pages below it may be missing, what a page of it holds below it may be any bits."""
    H, G, D, length, window, sinks = 2, 2, 128, 1000, 200, 3
    cache, k, v, table = filled([length], H, H * G, D, torch.float16)
    q = rows(4, H * G, D, torch.float16, 1)
    batch = binding.FP4Batch(ints([length]), 4, table)
    begin = length - 4 - window + 1
    first = begin // 64 * 64
    block = cache.pages.view(cache.n_pages, H, -1)
    page = block[int(table[0, begin // 64])]
    v_scales = 64 * 64 + 256 + 64 * 64                          # of a head's block
    page[:, v_scales:].view(H, 4, 64)[:, :, :begin - first] = 255
    page[:, 4096:4352].view(H, 64, 4)[:, :begin - first] = 255
    sink = block[int(table[0, 0])]
    sink[:, v_scales:].view(H, 4, 64)[:, :, sinks:] = 255
    sink[:, 4096:4352].view(H, 64, 4)[:, sinks:] = 255
    table[0, 1:first // 64] = -1
    lse = torch.empty(4, H * G, device=DEV)
    out = cache.kv_fp4_attention(q.to(DEV), batch, 0.1, window, sinks, lse=lse)
    check(cache, k, v, [length], [4], q, out, lse, 0.1, window, sinks)


def test_missing_pages_and_rows_of_no_sequence():
    H, G, D, lens = 1, 4, 64, [300, 130, 64]
    gone = [(0, 2), (2, 0)]

    def without(table):
        for b, i in gone:
            table[b, i] = 10 ** 6 if b else -1
        return table
    cache, k, v, table = filled(lens, H, H * G, D, torch.float16, table=without)
    present = [torch.ones(n, dtype=torch.bool) for n in lens]
    for b, i in gone:
        present[b][64 * i:64 * i + 64] = False
    new = [5, 2, 6]                                             # the third's rows see nothing
    q = rows(13, H * G, D, torch.float16, 2).to(DEV)
    batch = binding.FP4Batch(ints(lens), 6, table, new_rows=ints(new), first_row=ints([0, 5, 7]))
    lse = torch.empty(13, H * G, device=DEV)
    out = cache.kv_fp4_attention(q, batch, 0.125, lse=lse)
    check(cache, k, v, lens, new, q, out, lse, 0.125, present=present)
    assert not out[7:].any() and bool((lse[7:] == -math.inf).all())
    # the same rows behind others, and the last of them outside the tensors
    wide = torch.full((20, H * G, D), 5.0, dtype=torch.float16, device=DEV)
    more = torch.zeros(20, H * G, D, dtype=torch.float16, device=DEV)
    more[9:20] = q[:11]
    batch = binding.FP4Batch(ints(lens), 6, table, new_rows=ints(new), first_row=ints([9, 14, 16]))
    cache.kv_fp4_attention(more, batch, 0.125, out=wide)
    assert bool((wide[:9] == 5.0).all()) and torch.equal(wide[9:20], out[:11])


def test_not_a_number_stays_with_its_row_and_head():
    cache, k, v, table = filled([300, 300], 2, 4, 128, torch.float16)
    q = rows(6, 4, 128, torch.float16, 3)
    batch = binding.FP4Batch(ints([300, 300]), 3, table)
    good = cache.kv_fp4_attention(q.to(DEV), batch, 0.1)
    q[1, 2, 17], q[5, 0, 0] = float("nan"), float("inf")
    got = cache.kv_fp4_attention(q.to(DEV), batch, 0.1)
    bad = torch.zeros(6, 4, dtype=torch.bool)
    bad[1, 2] = bad[5, 0] = True
    assert torch.isnan(got[1, 2]).all() and not torch.isfinite(got[5, 0]).all()
    assert torch.equal(got[~bad.to(DEV)], good[~bad.to(DEV)])


def test_strided_queries():
    cache, k, v, table = filled([90, 41], 2, 4, 128, torch.bfloat16)
    qkv = rows(60, 4 + 2 + 2, 128, torch.bfloat16, 4).to(DEV)
    q = qkv[:, :4]
    batch = binding.FP4Batch(ints([90, 41]), 30, table)
    want = cache.kv_fp4_attention(q.contiguous(), batch, 0.1)
    assert torch.equal(cache.kv_fp4_attention(q, batch, 0.1), want)
    assert torch.equal(cache.kv_fp4_attention(q.unflatten(0, (2, 30)), batch, 0.1).flatten(0, 1), want)
    assert not torch.equal(want, torch.zeros_like(want))


def test_reproducible():
    """Bit for bit, again and again."""
    cache, k, v, table = filled([3000, 800, 40], 2, 8, 128, torch.float16)
    q = rows(9, 8, 128, torch.float16, 5).to(DEV)
    batch = binding.FP4Batch(ints([3000, 800, 40]), 3, table)
    a = cache.kv_fp4_attention(q, batch, 0.1)
    assert all(torch.equal(a, cache.kv_fp4_attention(q, batch, 0.1)) for _ in range(5))


def test_decoding_captured():
    """A step -- append, attention -- captured once and replayed as the sequences grow, other work of the program between."""
    H, G, D, lens0, steps = 2, 4, 128, [61, 200], 70
    lens = [n + steps for n in lens0]
    k, v = rows(sum(lens), H, D, torch.float16, 6), rows(sum(lens), H, D, torch.float16, 7)
    qs = rows(2 * steps, H * G, D, torch.float16, 8)
    table, n_pages = page_table(lens)
    cache = binding.FP4KVCache(n_pages, H, H * G, D)
    first = starts(lens)
    which = torch.cat([torch.arange(f, f + n) for f, n in zip(first, lens0)])
    cache.kv_fp4_append(k[which].to(DEV), v[which].to(DEV), binding.FP4Batch(ints(lens0), max(lens0), table, new_rows=ints(lens0),
                                                                             first_row=ints(starts(lens0))))
    held = ints(lens0)
    batch = binding.FP4Batch(held, 1, table)
    nk, nv, nq = (torch.zeros(2, h, D, dtype=torch.float16, device=DEV) for h in (H, H, H * G))
    out, lse = torch.empty(2, H * G, D, dtype=torch.float16, device=DEV), torch.empty(2, H * G, device=DEV)
    eager = torch.empty_like(out)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                                          # two graphs that share the cache's workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.add_(1)
            cache.kv_fp4_append(nk, nv, batch)
            cache.kv_fp4_attention(nq, batch, 0.09, out=out, lse=lse)
        graphs.append(graph)
    for step in range(steps):
        rows_now = [f + n + step for f, n in zip(first, lens0)]
        nk.copy_(k[rows_now]), nv.copy_(v[rows_now]), nq.copy_(qs[2 * step:2 * step + 2])
        graphs[step % 2].replay()
        if step % 10 == 0 or step == steps - 1:
            cache.kv_fp4_attention(nq, batch, 0.09, out=eager)
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
            now = [n + step + 1 for n in lens0]
            keep = torch.cat([torch.arange(f, f + n) for f, n in zip(first, now)])
            check(cache, ref.quantise(k[keep])[0], ref.quantise(v[keep])[0], now, [1, 1], nq, out, lse, 0.09)


def test_joining_over_parts():
    """Two results over parts of a sequence joined with their lse are the result over the whole."""
    H, G, D, n = 2, 2, 128, 500
    cache, k, v, table = filled([n], H, H * G, D, torch.float16)
    q = rows(1, H * G, D, torch.float16, 9).to(DEV)
    full, full_lse = torch.empty(1, H * G, D, device=DEV), torch.empty(1, H * G, device=DEV)
    cache.kv_fp4_attention(q, binding.FP4Batch(ints([n]), 1, table), 0.1, out=full, lse=full_lse)
    parts = []
    for pages, length in ((table[:, :4].contiguous(), 256), (table[:, 4:].contiguous(), n - 256)):
        o, s = torch.empty_like(full), torch.empty_like(full_lse)
        cache.kv_fp4_attention(q, binding.FP4Batch(ints([length]), 1, pages), 0.1, out=o, lse=s)
        parts.append((o, s))
    joined = torch.logaddexp(parts[0][1], parts[1][1])
    out = sum(o * torch.exp(s - joined)[..., None] for o, s in parts)
    # each side's weights are rounded to fp16 by itself: half a step of the values around, twice
    around = ref.attention(q.cpu(), k, v.abs(), 1, 0.1)[0]
    assert bool(((out - full).abs().cpu().double() <= 3 * 2.0 ** -11 * around + 1e-5).all())
    assert bool(((joined - full_lse).abs() < 1e-4).all())


def test_pages_behind_4_gib():
    H, D = 64, 128
    page = H * 64 * (D + D // 16)
    n_pages = (1 << 32) // page + 3
    cache = binding.FP4KVCache(n_pages, H, H, D)
    k, v, q = (rows(70, H, D, torch.float16, s).to(DEV) for s in (10, 11, 12))
    batch = binding.FP4Batch(ints([70]), 70, ints([[n_pages - 1, n_pages - 2]]))
    cache.kv_fp4_append(k, v, batch)
    lse = torch.empty(70, H, device=DEV)
    out = cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
    check(cache, ref.quantise(k.cpu())[0], ref.quantise(v.cpu())[0], [70], [70], q, out, lse, 0.1)


@pytest.mark.parametrize("H, G, lens", [(2, 1, [9000] + [5] * 20), (1, 4, [40, 6000, 41]), (2, 2, [100] * 70 + [3000] + [1] * 5),
                                        (1, 16, [7000, 0, 900]), (1, 1, [130] * 129)])
def test_very_different_lengths(H, G, lens):
    """A long sequence among short ones is split over more workgroups; more sequences than one wave shares out."""
    run(lens, [1] * len(lens), H, G, 64, torch.float16, seed=len(lens))
    run(lens, [min(n, 2) for n in lens], H, G, 64, torch.bfloat16, 50, 3, seed=len(lens))


@pytest.mark.parametrize("G", [1, 2, 3, 5, 8, 16])
def test_joined_by_the_last_workgroup_and_by_a_kernel(G):
    """Splits of one sequence: few rows (joined where they are made) and many."""
    for lens in ([1200], [20000]):
        run(lens, [1], 1, G, 128 if G < 4 else 64, torch.float16, seed=G)


@pytest.mark.parametrize("D, H, G, lens, new, window, sinks", [
    (128, 12, 4, [600] * 8, [150, 300, 160, 1, 20, 600, 31, 0], 0, 0), (64, 16, 3, [500, 300, 900] * 5, [200, 170, 130] * 5, 0, 0),
    (64, 24, 1, [1200] * 4, [1000, 100, 513, 1200], 300, 70), (128, 8, 16, [400] * 4, [400, 64, 399, 10], 33, 5),
    (64, 4, 4, [17000, 16500], [70, 130], 0, 0), (128, 3, 8, [20000], [100], 0, 0), (128, 16, 5, [333] * 8, [333] * 8, 1, 0)])
def test_many_rows(D, H, G, lens, new, window, sinks):
    """The kernel for many rows: blocks of 128 columns, full and ragged, split contexts, windows that end inside a page."""
    run(lens, new, H, G, D, torch.float16, window, sinks, seed=H)
    run(lens[:4], new[:4], H, G, D, torch.bfloat16, window, sinks, seed=H + 1, out_dtype=torch.float32)


def test_padded_batch():
    """Rows at b * max_new, fewer than max_new of some sequences: the others are left as they were."""
    lens, new, most = [70, 200, 9], [3, 5, 0], 6
    cache, k, v, table = filled(lens, 2, 4, 64, torch.float16)
    q = rows(18, 4, 64, torch.float16, 4)
    batch = binding.FP4Batch(ints(lens), most, table, new_rows=ints(new))
    out, lse = torch.full((18, 4, 64), 7.0, dtype=torch.float16, device=DEV), torch.full((18, 4), 7.0, device=DEV)
    cache.kv_fp4_attention(q.to(DEV).view(3, 6, 4, 64), batch, 0.1, out=out.view(3, 6, 4, 64), lse=lse.view(3, 6, 4))
    which = torch.tensor([0, 1, 2, 6, 7, 8, 9, 10])
    check(cache, k, v, lens, new, q[which], out[which.to(DEV)], lse[which.to(DEV)], 0.1)
    left = [i for i in range(18) if i not in which.tolist()]
    assert bool((out[left] == 7.0).all()) and bool((lse[left] == 7.0).all())


@pytest.mark.parametrize("batch", [1025, 32768, 33000])
def test_thousands_of_sequences(batch):
    """As many sequences in one call give what they give a thousand at a time."""
    lens = torch.randint(0, 65, (batch,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(DEV)
    cache = binding.FP4KVCache(batch, 1, 2, 64)
    gen = torch.Generator(device=DEV).manual_seed(2)
    k, v = (torch.randn(64 * batch, 1, 64, generator=gen, device=DEV).half() for _ in range(2))
    q = torch.randn(batch, 2, 64, generator=gen, device=DEV).half()
    table = torch.randperm(batch, generator=torch.Generator().manual_seed(3), dtype=torch.int32).view(-1, 1).to(DEV)
    first = 64 * torch.arange(batch, dtype=torch.int32, device=DEV)
    cache.kv_fp4_append(k, v, binding.FP4Batch(lens, 64, table, new_rows=lens, first_row=first))
    out = cache.kv_fp4_attention(q, binding.FP4Batch(lens, 1, table), 0.125)
    for at in range(0, batch, 1000):
        part = cache.kv_fp4_attention(q[at:at + 1000], binding.FP4Batch(lens[at:at + 1000], 1, table[at:at + 1000]), 0.125)
        assert torch.equal(part, out[at:at + 1000])
    assert not out[lens == 0].any() and bool(torch.isfinite(out).all()) and bool(out[lens > 0].any(2).all())
