"""Writing rows into the 4-bit paged cache and reading them back, against the plain arithmetic of fp4_reference: equal, always."""
import random

import pytest
import torch

from paper_2512_24449_amd import binding
from tests import fp4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def starts(x):
    return [sum(x[:i]) for i in range(len(x))]


def page_table(lens, extra=0, seed=0):
    """Pages anywhere, one table row to a sequence; (table [batch, most pages], pages of the cache)."""
    pages = [-(-n // 64) for n in lens]
    order = list(range(sum(pages) + 2))
    random.Random(seed).shuffle(order)
    table = torch.full((len(lens), max(1, max(pages)) + extra), -1, dtype=torch.int32)
    for b, n in enumerate(pages):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    return table.to(DEV), sum(pages) + 2


def rows(n, heads, dim, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(n, heads, dim, generator=gen) * torch.exp(2.0 * torch.randn(n, heads, 1, generator=gen))
    return x.to(dtype)


def equal(got, want):
    return torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim, heads, lens", [(128, 1, [1]), (128, 3, [64]), (128, 2, [65, 1, 31]), (64, 5, [130, 7]),
                                              (64, 1, [63, 64, 129]), (128, 8, [200, 0, 33])])
def test_whole_sequences(dim, heads, lens, dtype):
    table, n_pages = page_table(lens)
    cache = binding.FP4KVCache(n_pages, heads, heads, dim)
    k, v = rows(sum(lens), heads, dim, dtype, 1), rows(sum(lens), heads, dim, dtype, 2)
    batch = binding.FP4Batch(ints(lens), max(lens), table, new_rows=ints(lens), first_row=ints(starts(lens)))
    cache.kv_fp4_append(k.to(DEV), v.to(DEV), batch)
    for out in (torch.float16, torch.bfloat16, torch.float32):
        got = cache.kv_fp4_read(batch, sum(lens), out)
        assert got[0].dtype == out and equal(got[0], ref.quantise(k)[0]) and equal(got[1], ref.quantise(v)[0])


def test_layout_of_a_page():
    for dim, heads in ((128, 2), (64, 3)):
        cache = binding.FP4KVCache(3, heads, heads, dim)
        k, v = rows(64, heads, dim, torch.float16, 3), rows(64, heads, dim, torch.float16, 4)
        cache.kv_fp4_append(k.to(DEV), v.to(DEV), binding.FP4Batch(ints([64]), 64, ints([[2]])))
        page = cache.pages.cpu().reshape(3, -1)[2]
        for h in range(heads):
            K, V = ref.read_page(page, h, dim, heads)
            assert torch.equal(K, ref.quantise(k[:, h])[0]) and torch.equal(V, ref.quantise(v[:, h])[0])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_every_value_and_every_scale(dtype):
    """All 16-bit patterns, NaNs and infinities among them, each beside larger and smaller neighbours of its group."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    parts = []
    for shift in (0, 1, 3):
        x = bits.clone()
        x[shift::32] = torch.tensor(3.0 * 2.0 ** (5 * shift - 9), dtype=dtype)
        parts.append(x)
    x = torch.cat(parts).reshape(-1, 1, 128)
    order = torch.randperm(x.numel(), generator=torch.Generator().manual_seed(5))
    x = torch.cat([x, x.flatten()[order].reshape(x.shape)])
    n = x.shape[0]
    cache = binding.FP4KVCache(-(-n // 64), 1, 1)
    batch = binding.FP4Batch(ints([n]), n, table_pages=-(-n // 64))
    cache.kv_fp4_append(x.to(DEV), x.flip(0).to(DEV), batch)
    got = cache.kv_fp4_read(batch, n, torch.float32)
    want = ref.quantise(x)[0]
    assert torch.isfinite(got[0]).all() and equal(got[0], want) and equal(got[1], want.flip(0))
    # and all the edges between two codes, at the least, an ordinary and the greatest scale
    for e in (-23, -22, -14, 0, 12, 13):
        edge = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.0], dtype=torch.float64)
        y = torch.cat([edge * 2.0 ** e, -edge * 2.0 ** e, torch.zeros(14, dtype=torch.float64)]).to(dtype)
        y = torch.cat([y, torch.nextafter(y.float(), torch.tensor(9e9)).to(dtype), y * 0.5, y * 0]).reshape(1, 1, 128)
        one = binding.FP4Batch(ints([1]), 1, table_pages=1)
        cache.kv_fp4_append(y.to(DEV), y.to(DEV), one)
        got = cache.kv_fp4_read(one, 1, torch.float32)
        assert equal(got[0], ref.quantise(y)[0]) and equal(got[1], ref.quantise(y)[0])


def test_groups_with_nan_and_infinity_keep_their_other_values():
    x = rows(4, 1, 128, torch.float16, 6)
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 41], x[3, 0, 127] = float("nan"), float("inf"), float("-inf"), float("nan")
    cache = binding.FP4KVCache(1, 1, 1)
    batch = binding.FP4Batch(ints([4]), 4, table_pages=1)
    cache.kv_fp4_append(x.to(DEV), x.to(DEV), batch)
    k, v = (t.cpu() for t in cache.kv_fp4_read(batch, 4, torch.float32))
    assert torch.equal(k, v) and equal(k, ref.quantise(x)[0])
    assert k[0, 0, 5] == 0 and k[1, 0, 40] == 49152 and k[2, 0, 41] == -49152 and k[3, 0, 127] == 0


@pytest.mark.parametrize("dim", [128, 64])
def test_token_by_token_and_in_pieces(dim):
    """However the tokens arrive, the cache reads the same; those already there keep their values."""
    lens, heads = [150, 97, 64], 2
    k, v = rows(sum(lens), heads, dim, torch.float16, 7), rows(sum(lens), heads, dim, torch.float16, 8)
    first = starts(lens)
    table, n_pages = page_table(lens)
    want = [ref.quantise(t)[0] for t in (k, v)]
    for pieces in ([1] * 150, [3, 5, 64, 1, 7, 8, 33, 29], [149, 1], [8, 142]):
        cache = binding.FP4KVCache(n_pages, heads, heads, dim)
        cache.pages.fill_(255)
        at = [0] * 3
        for step in pieces:
            new = [min(step, n - a) for a, n in zip(at, lens)]
            which = torch.cat([torch.arange(f + a, f + a + n) for f, a, n in zip(first, at, new)])
            at = [a + n for a, n in zip(at, new)]
            batch = binding.FP4Batch(ints(at), step, table, new_rows=ints(new), first_row=ints(starts(new)))
            cache.kv_fp4_append(k[which].to(DEV), v[which].to(DEV), batch)
        assert at == lens
        whole = binding.FP4Batch(ints(lens), max(lens), table, new_rows=ints(lens), first_row=ints(first))
        got = cache.kv_fp4_read(whole, sum(lens), torch.float32)
        assert equal(got[0], want[0]) and equal(got[1], want[1]), pieces[:3]


def test_strided_inputs_and_four_axes():
    """K and V as parts of one projection's output, and of a [batch, n, heads, D] tensor."""
    B, n, Hq, H, D = 3, 37, 4, 2, 128
    qkv = rows(B * n, Hq + 2 * H, D, torch.bfloat16, 9).to(DEV)
    k, v = qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    cache = binding.FP4KVCache(B, H, Hq, D)
    batch = binding.FP4Batch(ints([n] * B), n, table_pages=1)
    for view in (lambda t: t, lambda t: t.unflatten(0, (B, n))):
        cache.pages.zero_()
        cache.kv_fp4_append(view(k), view(v), batch)
        got = cache.kv_fp4_read(batch, B * n, torch.bfloat16)
        assert equal(got[0], ref.quantise(k.cpu())[0]) and equal(got[1], ref.quantise(v.cpu())[0])


def test_rows_of_no_sequence_and_missing_pages():
    H, D, lens, new = 2, 64, [100, 70, 5], [40, 10, 9]          # (the third has more new rows than tokens)
    first = [3, 50, 70]
    table, n_pages = page_table(lens)
    table[0, 0] = -1                                            # positions 60 .. 63 of the first are missing
    table[1, 1] = n_pages                                       # and positions 64 .. 69 of the second
    cache = binding.FP4KVCache(n_pages, H, H, D)
    cache.pages.fill_(3)
    k, v = rows(75, H, D, torch.float16, 10), rows(75, H, D, torch.float16, 11)   # rows 75 .. 78 do not exist
    batch = binding.FP4Batch(ints(lens), 40, table, new_rows=ints(new), first_row=ints(first))
    cache.kv_fp4_append(k.to(DEV), v.to(DEV), batch)
    got = [torch.full((75, H, D), 7.0, dtype=torch.float32, device=DEV) for _ in range(2)]
    cache.kv_fp4_read(batch, 75, torch.float32, *got)
    for g, x in zip(got, (k, v)):
        want = torch.full((75, H, D), 7.0, dtype=torch.float64)
        want[3:7] = 0
        want[7:43] = ref.quantise(x[7:43])[0]
        want[50:54] = ref.quantise(x[50:54])[0]                 # positions 60 .. 63
        want[54:60] = 0
        want[70:74] = 0                                         # positions -4 .. -1
        want[74:75] = ref.quantise(x[74:75])[0]                 # position 0
        assert equal(g, want)
    # pages of no sequence keep their bytes
    used = {int(p) for p in table.flatten().tolist() if 0 <= p < n_pages}
    pages = cache.pages.cpu().reshape(n_pages, -1)
    assert all(bool((pages[p] == 3).all()) for p in range(n_pages) if p not in used)


def test_lengths_behind_the_table_and_below_zero():
    cache = binding.FP4KVCache(2, 1, 1, 128)
    x = rows(200, 1, 128, torch.float16, 12)
    batch = binding.FP4Batch(ints([190, -5]), 100, ints([[0], [1]]), first_row=ints([0, 100]))   # room for 64 tokens each
    cache.pages.fill_(9)
    cache.kv_fp4_append(x.to(DEV), x.to(DEV), batch)            # positions 90 .. 189: none held
    assert bool((cache.pages == 9).all())
    k, v = cache.kv_fp4_read(batch, 200, k=torch.ones(200, 1, 128, dtype=torch.float16, device=DEV))
    assert not k.any()
    far = binding.FP4Batch(ints([2 ** 31 - 1]), 2 ** 20, ints([[0]]))
    cache.kv_fp4_append(x.to(DEV), x.to(DEV), far)
    cache.kv_fp4_read(far, 200)
    assert bool((cache.pages == 9).all())


def test_on_another_stream_and_captured():
    """A captured append and read follow what the batch's tensors hold at each replay."""
    H, D = 2, 128
    cache = binding.FP4KVCache(4, H, H, D)
    lens = ints([1, 1])
    batch = binding.FP4Batch(lens, 1, ints([[0, 1], [2, 3]]))
    k, v = (torch.zeros(2, H, D, dtype=torch.float16, device=DEV) for _ in range(2))
    ks, vs = rows(200, H, D, torch.float16, 13), rows(200, H, D, torch.float16, 14)
    out = [torch.empty(2, H, D, dtype=torch.float16, device=DEV) for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        cache.kv_fp4_append(k, v, batch)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.kv_fp4_append(k, v, batch)
        cache.kv_fp4_read(batch, 2, k=out[0], v=out[1])
    for step in range(100):
        k.copy_(ks[2 * step:2 * step + 2])
        v.copy_(vs[2 * step:2 * step + 2])
        lens.fill_(step + 1)
        graph.replay()
        if step % 33 == 0:
            assert equal(out[0], ref.quantise(ks[2 * step:2 * step + 2])[0])
            assert equal(out[1], ref.quantise(vs[2 * step:2 * step + 2])[0])
    whole = cache.kv_fp4_read(binding.FP4Batch(ints([100, 100]), 100, ints([[0, 1], [2, 3]])), 200, torch.float32,
                              stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert equal(whole[0], ref.quantise(torch.cat([ks[0::2], ks[1::2]]))[0])
    assert equal(whole[1], ref.quantise(torch.cat([vs[0::2], vs[1::2]]))[0])


def test_far_pages():
    """Pages behind the 4 GiB and 2^31 marks of the buffer."""
    H, D = 64, 128
    page = H * 64 * (D + D // 16)
    n_pages = (1 << 32) // page + 3
    cache = binding.FP4KVCache(n_pages, H, H, D)
    x = rows(3, H, D, torch.float16, 15)
    table = ints([[n_pages - 1], [(1 << 31) // page + 1], [0]])
    batch = binding.FP4Batch(ints([1, 1, 1]), 1, table)
    cache.kv_fp4_append(x.to(DEV), x.to(DEV), batch)
    got = cache.kv_fp4_read(batch, 3)
    assert equal(got[0], ref.quantise(x)[0]) and equal(got[1], ref.quantise(x)[0])


def test_native_calls_and_python_calls_agree():
    """The binding's two ways of making a call give the same, for the layouts that one of them leaves to the other too."""
    H, D, B, n = 2, 128, 2, 9
    qkv = rows(B * n, 4 + 2 * H, D, torch.float16, 16).to(DEV)
    k, v, q = qkv[:, 4:6], qkv[:, 6:], qkv[:, :4]
    batch = binding.FP4Batch(ints([n, n]), n, table_pages=1)
    got = []
    for python in (False, True):
        cache = binding.FP4KVCache(B, H, 4, D)
        if python:
            cache._calls = binding._PythonCalls()
        cache.kv_fp4_append(k, v, batch)
        kr, vr = cache.kv_fp4_read(batch, B * n, torch.bfloat16)
        cache.kv_fp4_append(k.unflatten(0, (B, n)), v.unflatten(0, (B, n)), batch)
        out = cache.kv_fp4_attention(q, batch, 0.1, window=4, sinks=1)
        assert torch.equal(cache.kv_fp4_attention(q.unflatten(0, (B, n)), batch, 0.1, 4, 1).flatten(0, 1), out)
        assert torch.equal(cache.kv_fp4_attention(q, batch, 0.1, 4, 1, stream=torch.cuda.current_stream().cuda_stream), out)
        got.append((kr, vr, out))
        with pytest.raises(binding.PackKVError):
            cache.kv_fp4_attention(q, batch, float("nan"))
        with pytest.raises(binding.PackKVError):
            cache.kv_fp4_attention(q, batch, 0.1, window=-1)
        with pytest.raises(binding.PackKVError):
            cache.kv_fp4_append(k[:, :1].expand(-1, 2, -1), v, batch)
        cache.close()
        with pytest.raises(binding.PackKVError):
            cache.kv_fp4_read(batch, B * n)
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][2].dtype == torch.float16
