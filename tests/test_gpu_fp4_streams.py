"""Calls on another stream than the current one while that stream is behind: what the program drops is not reused under them, and
their outputs are not in memory that the current stream still writes."""
import pytest
import torch

from paper_2512_24449_amd import binding
from tests.test_gpu_fp4_cache import DEV, ints, page_table, rows, starts

pytestmark = pytest.mark.gpu
LENS, H, G, D = [130, 70], 2, 2, 128


def busy(stream):
    """Some milliseconds of work."""
    with torch.cuda.stream(stream):
        a = torch.ones(4096, 4096, device=DEV)
        for _ in range(12):
            a = (a @ a) * (1.0 / 4096)


def waste():
    """Fills what the allocator hands out again in the sizes of the calls' tensors."""
    total = sum(LENS)
    kept = [torch.full((2,), -1, dtype=torch.int32, device=DEV) for _ in range(40)]
    kept += [torch.full((2, 3), -1, dtype=torch.int32, device=DEV) for _ in range(40)]
    kept += [torch.full((total, h, D), float("nan"), dtype=torch.float16, device=DEV) for h in (H, H * G) for _ in range(8)]
    return kept


@pytest.mark.parametrize("raw", [False, True])
def test_tensors_dropped_after_the_call(raw):
    total = sum(LENS)
    table, n_pages = page_table(LENS)
    k, v, q = rows(total, H, D, torch.float16, 1), rows(total, H, D, torch.float16, 2), rows(total, H * G, D, torch.float16, 3)

    def batch():
        return binding.FP4Batch(ints(LENS), max(LENS), table.clone(), new_rows=ints(LENS), first_row=ints(starts(LENS)))
    plain = binding.FP4KVCache(n_pages, H, H * G, D)
    plain.kv_fp4_append(k.to(DEV), v.to(DEV), batch())
    want = [*plain.kv_fp4_read(batch(), total), plain.kv_fp4_attention(q.to(DEV), batch(), 0.1)]

    cache = binding.FP4KVCache(n_pages, H, H * G, D)
    side = torch.cuda.Stream()
    stream = side.cuda_stream if raw else side
    torch.cuda.synchronize()
    busy(side)
    done = torch.cuda.Event()
    side.wait_stream(torch.cuda.current_stream())
    cache.kv_fp4_append(k.to(DEV), v.to(DEV), batch(), stream=stream)
    first = waste()
    side.wait_stream(torch.cuda.current_stream())
    got = [*cache.kv_fp4_read(batch(), total, stream=stream), cache.kv_fp4_attention(q.to(DEV), batch(), 0.1, stream=stream)]
    done.record(side)
    second = waste()
    del cache                                                   # the pages too
    third = [torch.full((n_pages * H * 64 * (D + D // 16),), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
    done.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert len(first) + len(second) + len(third)


def test_outputs_beside_work_of_the_current_stream():
    """The current stream is behind and still writes what it has dropped; the call's stream is not behind it."""
    total = sum(LENS)
    table, n_pages = page_table(LENS)
    k, v, q = (rows(total, h, D, torch.float16, 4 + h).to(DEV) for h in (H, H, H * G))
    batch = binding.FP4Batch(ints(LENS), max(LENS), table, new_rows=ints(LENS), first_row=ints(starts(LENS)))
    cache = binding.FP4KVCache(n_pages, H, H * G, D)
    cache.kv_fp4_append(k, v, batch)
    want = [*cache.kv_fp4_read(batch, total), cache.kv_fp4_attention(q, batch, 0.1)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    old = [torch.empty_like(t) for t in want for _ in range(4)]
    busy(torch.cuda.current_stream())
    for t in old:
        t.fill_(7.0)
    del old, t
    got = [*cache.kv_fp4_read(batch, total, stream=side), cache.kv_fp4_attention(q, batch, 0.1, stream=side)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
