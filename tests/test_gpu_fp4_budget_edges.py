"""Calls around a cache's budget at the edges of what they write and take."""
import pytest
import torch

from paper_2512_24449_amd import binding
from tests.test_gpu_fp4_budget import Filled, ints, query

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_tensors_next_to_each_other_in_one_buffer():
    """What a call writes may begin where what it reads ends."""
    held = Filled([500, 300], 2, 4, 128, torch.float16, 70, more_pages=4)
    q = query(6, 8, 128, torch.float16, 71)
    shapes = dict(past=(2, 2, 500), mass=(2, 2, 500), n_kept=(2,), budgets=(2,), kept=(2, 2, 100), lse=(6, 8), mass_out=(2, 2, 77), lens=(2,))
    place, at = {}, 0
    for name, shape in shapes.items():
        n = torch.Size(shape).numel()
        place[name] = (at, at + n, shape)
        at += n

    def together():
        flat = torch.zeros(at, dtype=torch.int32, device=DEV)
        t = {name: flat[a:b].view(shape) for name, (a, b, shape) in place.items()}
        return {name: x if name in ("n_kept", "budgets", "kept", "lens") else x.view(torch.float32) for name, x in t.items()}

    def apart():
        return {name: x.clone() for name, x in together().items()}

    results = []
    for t in (together(), apart()):
        t["past"].copy_(torch.rand(2, 2, 500, generator=torch.Generator().manual_seed(72)))
        t["lens"].copy_(ints(held.lens)), t["budgets"].copy_(ints([90, 100]))
        batch = binding.FP4Batch(t["lens"], 4, held.table, new_rows=ints([4, 2]), first_row=ints([0, 4]))
        held.cache.kv_fp4_attention(q.to(DEV), batch, 0.1, lse=t["lse"])
        held.cache.kv_fp4_weights(q.to(DEV), t["lse"], batch, 0.1, past=t["past"], out=t["mass"])
        held.cache.kv_fp4_select(t["mass"], batch, 100, 4, 10, budgets=t["budgets"], kept=t["kept"], n_kept=t["n_kept"])
        to = binding.FP4Batch(t["n_kept"], 100, held.n_pages + ints([[0, 1], [2, 3]]), new_rows=t["n_kept"])
        held.cache.kv_fp4_compact(t["kept"], t["n_kept"], batch, to, mass=t["mass"], mass_out=t["mass_out"])
        results.append(t)
    assert results[0]["n_kept"].tolist() == [90, 100]
    assert all(torch.equal(results[0][name], results[1][name]) for name in shapes)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [[1, 9, 64], [7, 8, 15], [63, 65, 0], [121, 3, 127]])
def test_compaction_clears_the_rest_of_the_last_eight(n, D):
    """Tokens behind the last one, up to a whole eight, are zeros in pages that held anything; those of the next eight stay."""
    lens, H, keep = [150, 140, 130], 2, 128
    held = Filled(lens, H, 1, D, torch.float16, 73, more_pages=6)
    page = H * 64 * (D + D // 16)
    held.cache.pages[held.n_pages * page:] = 255
    to_table = held.n_pages + ints([[3, 0], [5, 1], [2, 4]])
    kept = torch.arange(keep, dtype=torch.int32, device=DEV).flip(0).expand(3, H, keep).contiguous()
    count = ints(n)
    held.cache.kv_fp4_compact(kept, count, held.batch([0] * 3, max_new=0), binding.FP4Batch(count, keep, to_table))
    whole = binding.FP4Batch(ints([keep] * 3), keep, to_table)
    for x, y in zip((held.k, held.v), held.cache.kv_fp4_read(whole, 3 * keep, torch.float32)):
        y = y.cpu().double().view(3, keep, H, D)
        for b, m in enumerate(n):
            end = -(-m // 8) * 8
            assert torch.equal(y[b, :m], x[b][kept[b, 0, :m].long().cpu()])
            assert bool((y[b, m:end] == 0).all())
            assert not torch.isfinite(y[b, end:]).any()          # (scales of 255 as they were)


@pytest.mark.parametrize("new, G", [(3, 2), (20, 3), (50, 4)])   # one block of columns, some, many
@pytest.mark.parametrize("dtype, value", [(torch.float16, float("inf")), (torch.float16, -float("inf")), (torch.bfloat16, float("nan")),
                                          (torch.bfloat16, 3e38), (torch.bfloat16, -3e38)])
def test_a_row_whose_logarithm_is_minus_infinity_gives_nothing(new, G, dtype, value):
    """Whatever its query is: infinite, NaN, or finite with scores that are not."""
    held = Filled([200], 2, G, 128, dtype, 74)
    q = query(new, 2 * G, 128, dtype, 75).to(DEV)
    batch = held.batch([new])
    lse = torch.empty(new, 2 * G, device=DEV)
    held.cache.kv_fp4_attention(q, batch, 0.1, lse=lse)
    lse[1, 1] = lse[new - 1, 2 * G - 1] = -float("inf")
    plain = held.cache.kv_fp4_weights(q, lse, batch, 0.1)
    assert torch.isfinite(plain).all()
    q[1, 1], q[new - 1, 2 * G - 1, ::3] = value, value
    assert torch.equal(held.cache.kv_fp4_weights(q, lse, batch, 0.1), plain)
