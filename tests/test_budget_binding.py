"""The native part of the binding, calls around a cache's budget: it leaves what it does not expect, and gives what the Python code gives."""
import ctypes as C

import pytest
import torch

from paper_2512_24449_amd import binding


class _Sub(torch.Tensor):
    pass


def test_leaves_what_it_does_not_expect():
    """With addresses that must never be followed: every one of these is left to the Python code."""
    binding.lib()
    never = binding._native.FP4Calls(2, 4, 128, "cpu")
    never.set_handle(0xDEAD0)
    b = binding.FP4Batch(torch.ones(2, dtype=torch.int32), 3, table_pages=1)
    at, on = b._address, -1
    f, i = torch.zeros, lambda *s: torch.zeros(*s, dtype=torch.int32)
    q, lse, mass, kept, count = f(6, 4, 128).half(), f(6, 4), f(2, 2, 64), i(2, 2, 10), i(2)
    no = NotImplemented
    for change in ({0: q.float()}, {0: q[:, :2]}, {0: q.as_subclass(_Sub)}, {1: lse.double()}, {1: lse[:5]}, {1: lse.T.contiguous()}, {2: None},
                   {3: 0}, {4: 1}, {4: None}, {5: -1}, {5: 1.0}, {6: 2 ** 31}, {7: mass[:, :, :3].contiguous()}, {7: mass.half()}, {8: None},
                   {8: mass[..., ::2]}, {8: f(3, 2, 64)}, {9: 0}):
        args = [q, lse, at, on, 0.1, 0, 0, None, mass, None]
        for k, v in change.items():
            args[k] = v
        assert never.weights(*args) is no
    for change in ({0: mass.double()}, {0: f(2, 3, 64)}, {0: mass.as_subclass(_Sub)}, {3: 0}, {3: 2 ** 31}, {3: 1.0}, {4: -1}, {5: None}, {6: i(3)},
                   {6: f(2)}, {7: 0}):
        args = [mass, at, on, 10, 0, 0, None, None]
        for k, v in change.items():
            args[k] = v
        assert never.select(*args) is no
    for change in ({0: kept.long()}, {0: i(2, 3, 10)}, {1: i(3)}, {1: f(2)}, {4: None}, {5: 7}, {6: mass}, {7: mass}, {6: mass.half(), 7: mass},
                   {6: mass, 7: f(1, 2, 64)}, {8: 0}):
        args = [kept, count, at, on, at, on, None, None, None]
        for k, v in change.items():
            args[k] = v
        assert never.compact(*args) is no
    table = binding.kv_rotary_t(128, 128, 0, 1.0, 0xDEAD0)
    turn = binding._native.RotaryCalls(C.addressof(table), 128, "cpu").turn
    p = i(6)
    for change in ({0: q.int()}, {0: q[0]}, {0: q[..., :64]}, {0: q.transpose(0, 1)}, {0: q.as_subclass(_Sub)}, {1: p.long()}, {1: p[:5]}, {1: p[None]},
                   {2: q.float()}, {2: q[:5]}, {3: q[:, :2]}, {3: q.float()}, {4: q}, {5: 1}, {5: None}, {6: 0}):
        args = [q, p, None, None, None, False, None]
        for k, v in change.items():
            args[k] = v
        assert turn(*args) is no
    with torch.overrides.BaseTorchFunctionMode():
        assert turn(q, p, None, None, None, False, None) is no and never.select(mass, at, on, 10, 0, 0, None, None) is no
    never.set_handle(0)
    assert never.weights(q, lse, at, on, 0.1, 0, 0, None, mass, None) is no


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_same_results_and_errors_as_the_python_code(dtype):
    dev, H, G, D, lens = "cuda:0", 2, 3, 128, [150, 70]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    gen = torch.Generator().manual_seed(1)
    k, v, q = (torch.randn(220, h, D, generator=gen).to(dtype).to(dev) for h in (H, H, H * G))
    got, side = [], torch.cuda.Stream()
    for native in (True, False):
        cache, rotary = binding.FP4KVCache(8, H, H * G, D), binding.Rotary(D, 64)
        if not native:
            cache._calls = rotary._calls = binding._PythonCalls()
        whole = binding.FP4Batch(ints(lens), 150, ints([[0, 1, 2], [3, 4, 5]]), new_rows=ints(lens), first_row=ints([0, 150]))
        pos = ints([*range(150), *range(70)])
        results = []

        def run():
            a, b = rotary.kv_rotary(q, pos, k=k)
            results.extend([a, b, rotary.kv_rotary(q, pos, inverse=True)])
            out = [torch.empty_like(q), torch.empty_like(k)]
            assert rotary.kv_rotary(q, pos, k=k, out=out[0], k_out=out[1])[1] is out[1]
            results.extend(out)
            cache.kv_fp4_append(b, v, whole)
            lse = torch.empty(220, H * G, device=dev)
            cache.kv_fp4_attention(a, whole, 0.1, lse=lse)
            mass = torch.zeros(2, H, 192, device=dev)
            assert cache.kv_fp4_weights(a, lse, whole, 0.1, window=100, sinks=4, out=mass) is mass
            results.append(cache.kv_fp4_weights(a, lse, whole, 0.1, past=mass, out=torch.zeros_like(mass)))
            count = ints([0, 0])
            kept, n = cache.kv_fp4_select(mass, whole, 60, 4, 10, n_kept=count)
            assert n is count
            results.extend([mass, kept, n, cache.kv_fp4_select(mass, whole, 33, recent=5)[0]])
            cut = binding.FP4Batch(n, 60, ints([[6], [7]]), new_rows=n)
            moved = torch.zeros(2, H, 64, device=dev)
            assert cache.kv_fp4_compact(kept, n, whole, cut, mass=mass, mass_out=moved) is moved
            assert cache.kv_fp4_compact(kept, n, whole, cut) is None
            to = [torch.zeros(120, H, D, dtype=dtype, device=dev) for _ in range(2)]
            assert cache.kv_fp4_read(cut, 120, dtype, k=to[0], v=to[1])[0] is to[0]
            results.extend([moved, *to])
        run()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            run()
        side.synchronize()
        errors = []
        f = torch.zeros
        for call in (lambda: rotary.kv_rotary(q, pos[:3]), lambda: rotary.kv_rotary(q[:, ::2], pos), lambda: rotary.kv_rotary(q.expand(2, 220, 6, D), pos),
                     lambda: rotary.kv_rotary(q[:1].expand(220, 6, D), pos), lambda: cache.kv_fp4_weights(q, f(3), whole, 0.1, out=f(2, H, 9, device=dev)),
                     lambda: cache.kv_fp4_weights(q, results[0], whole, 0.1), lambda: cache.kv_fp4_weights(q, f(220, 6, device=dev), whole, float("nan"), out=f(2, H, 9, device=dev)),
                     lambda: cache.kv_fp4_select(f(2, H, 0, device=dev), whole, 5), lambda: cache.kv_fp4_select(f(2, H, 9, device=dev), whole, 0),
                     lambda: cache.kv_fp4_compact(f(2, H, 0, dtype=torch.int32, device=dev), ints([0, 0]), whole, whole)):
            with pytest.raises(binding.PackKVError) as e:
                call()
            errors.append((e.value.code, str(e.value).split("\n")[0]))
        got.append((results, errors))
    assert len(got[0][0]) == len(got[1][0]) and all(torch.equal(a, b) for a, b in zip(got[0][0], got[1][0]))
    assert got[0][1] == got[1][1]
