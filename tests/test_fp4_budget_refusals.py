"""What the operators around a cache's budget refuse, and what their calls on another stream keep: no GPU is touched."""
import ctypes as C
import math
import types

import pytest
import torch

from paper_2512_24449_amd import binding
from tests import budget_reference as ref
from tests.test_fp4_refusals import ARG, BAD_BATCHES, SOME, UNSUPPORTED, batch, cache, python_cache, refused  # noqa: F401 (fixtures)
from tests.test_fp4_streams import Stream, calls, half, made_batch  # noqa: F401


def weights(c, b=None, q=SOME, qs=512, type=0, rows=6, scale=1.0, window=0, sinks=0, lse=SOME, past=None, mass=SOME, tokens=256):
    return binding.lib().kv_fp4_weights(c, batch() if b is None else b, q, qs, type, rows, scale, window, sinks, lse, past, mass, tokens, None)


def select(c, b=None, mass=SOME, tokens=256, keep=10, budgets=None, sinks=0, recent=0, kept=SOME, n_kept=SOME):
    return binding.lib().kv_fp4_select(c, batch() if b is None else b, mass, tokens, keep, budgets, sinks, recent, kept, n_kept, None)


def compact(c, b=None, to=None, kept=SOME, keep=10, n_kept=SOME, mass=None, tokens=0, mass_out=None, out_tokens=0):
    return binding.lib().kv_fp4_compact(c, batch() if b is None else b, batch() if to is None else to, kept, keep, n_kept, mass, tokens,
                                        mass_out, out_tokens, None)


@pytest.mark.parametrize("change, want", BAD_BATCHES)
def test_batches(cache, change, want):  # noqa: F811
    assert weights(cache, batch(**change)) == want and select(cache, batch(**change)) == want
    assert compact(cache, batch(**change)) == want and compact(cache, to=batch(**change)) == want


def test_no_cache_or_batch(cache):  # noqa: F811
    L = binding.lib()
    for c, b in ((None, batch()), (cache, None)):
        assert L.kv_fp4_weights(c, b, SOME, 512, 0, 6, 1.0, 0, 0, SOME, None, SOME, 256, None) == ARG
        assert L.kv_fp4_select(c, b, SOME, 256, 10, None, 0, 0, SOME, SOME, None) == ARG
        assert L.kv_fp4_compact(c, b, batch(), SOME, 10, SOME, None, 0, None, 0, None) == ARG
    assert L.kv_fp4_compact(cache, batch(), None, SOME, 10, SOME, None, 0, None, 0, None) == ARG


def test_arguments(cache):  # noqa: F811
    for bad in (dict(q=None), dict(q=SOME + 8), dict(qs=504), dict(qs=513), dict(type=2), dict(type=-1), dict(rows=-1), dict(scale=math.nan),
                dict(scale=math.inf), dict(scale=2.4e38), dict(window=-1), dict(sinks=-1), dict(lse=None), dict(lse=SOME + 2),
                dict(past=SOME + 1), dict(mass=None), dict(mass=SOME + 2), dict(tokens=0)):
        assert weights(cache, **bad) == ARG, bad
    assert weights(cache, batch(max_new=2 ** 31 - 1)) == UNSUPPORTED
    for bad in (dict(mass=None), dict(mass=SOME + 2), dict(tokens=0), dict(keep=0), dict(keep=-1), dict(budgets=SOME + 2), dict(sinks=-1),
                dict(recent=-1), dict(kept=None), dict(kept=SOME + 1), dict(n_kept=None), dict(n_kept=SOME + 2)):
        assert select(cache, **bad) == ARG, bad
    for bad in (dict(kept=None), dict(kept=SOME + 2), dict(keep=0), dict(n_kept=None), dict(n_kept=SOME + 1), dict(to=batch(batch=3)),
                dict(mass=SOME), dict(mass_out=SOME), dict(mass=SOME, tokens=1, mass_out=SOME), dict(mass=SOME, mass_out=SOME, out_tokens=1),
                dict(mass=SOME + 2, tokens=1, mass_out=SOME, out_tokens=1), dict(mass=SOME, tokens=1, mass_out=SOME + 2, out_tokens=1)):
        assert compact(cache, **bad) == ARG, bad


def rotary(head_dim=64, dims=64, magnitude=1.0, turns=SOME, positions=SOME, rows=3, type=0, q=SOME, qs=256, heads=4, out=SOME, outs=256,
           k=None, ks=0, k_heads=0, k_out=None, k_outs=0, table=True):
    held = binding.kv_rotary_t(head_dim, dims, 0, magnitude, turns)
    return binding.lib().kv_rotary(C.byref(held) if table else None, positions, rows, type, 0, q, qs, heads, out, outs, k, ks, k_heads, k_out, k_outs, None)


def test_rotary_arguments():
    k = dict(k=SOME, ks=128, k_heads=2, k_out=SOME, k_outs=128)
    for bad in (dict(head_dim=0), dict(head_dim=65), dict(dims=63), dict(dims=0), dict(dims=66), dict(magnitude=math.inf), dict(magnitude=math.nan),
                dict(turns=None), dict(turns=SOME + 4), dict(positions=None), dict(positions=SOME + 2), dict(rows=-1), dict(type=3), dict(type=-1),
                dict(q=None), dict(q=SOME + 1), dict(type=2, q=SOME + 2), dict(out=None), dict(out=SOME + 1), dict(qs=255), dict(outs=255),
                dict(heads=-1), dict(heads=0), dict(k, k=None), dict(k, ks=127), dict(k, k_outs=100), dict(k, k_out=None), dict(k, k_heads=-1),
                dict(table=False)):
        assert rotary(**bad) == ARG, bad
    assert rotary(head_dim=514, dims=2, qs=4000, outs=4000) == UNSUPPORTED
    assert rotary(heads=65536, qs=2 ** 30, outs=2 ** 30) == UNSUPPORTED
    assert rotary(rows=2 ** 41) == UNSUPPORTED and rotary(rows=2 ** 35) == UNSUPPORTED
    assert rotary(rows=0) == 0 and rotary(rows=0, q=None, out=None, positions=None) == 0


def test_binding_refuses(python_cache):  # noqa: F811
    c = python_cache
    b = binding.FP4Batch(torch.ones(2, dtype=torch.int32), 3, table_pages=1)
    f = lambda *s: torch.zeros(*s)
    q, lse, mass = half(6, 4, 128), f(6, 4), f(2, 2, 64)
    for bad in (dict(q=q.float()), dict(q=half(6, 2, 128)), dict(lse=lse.half()), dict(lse=f(5, 4)), dict(lse=f(4, 6).T), dict(past=f(2, 64)),
                dict(past=f(2, 2, 60), out=mass), dict(past=f(1, 2, 64)), dict(out=mass.half()), dict(out=f(2, 64, 2).transpose(1, 2)),
                dict(window=-1), dict(sinks=2 ** 31)):
        with refused():
            c.kv_fp4_weights(**dict(dict(q=q, lse=lse, batch=b, sm_scale=1.0), **bad))
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)
    for bad in (dict(mass=f(2, 64)), dict(mass=mass.half()), dict(mass=f(2, 3, 64)), dict(keep=0), dict(keep=2 ** 31), dict(sinks=-1), dict(recent=-1),
                dict(budgets=ints(3)), dict(budgets=f(2)), dict(kept=ints(2, 2, 9)), dict(kept=f(2, 2, 10)), dict(n_kept=ints(2, 1))):
        with refused():
            c.kv_fp4_select(**dict(dict(mass=mass, batch=b, keep=10), **bad))
    other = binding.FP4Batch(ints(3), 3, table_pages=1)
    for bad in (dict(kept=ints(2, 3, 10)), dict(kept=f(2, 2, 10)), dict(n_kept=ints(3)), dict(n_kept=f(2)), dict(to=other), dict(mass_out=mass),
                dict(mass=f(2, 3, 64)), dict(mass=f(2, 64)), dict(mass=mass, mass_out=f(2, 2, 64).half()), dict(mass=mass, mass_out=f(2, 64))):
        with refused():
            c.kv_fp4_compact(**dict(dict(kept=ints(2, 2, 10), n_kept=ints(2), batch=b, to=b), **bad))
    c.handle = None
    for call in (lambda: c.kv_fp4_weights(q, lse, b, 1.0), lambda: c.kv_fp4_select(mass, b, 10),
                 lambda: c.kv_fp4_compact(ints(2, 2, 10), ints(2), b, b)):
        with refused():
            call()


def test_rotary_tables_and_refusals():
    for bad in (dict(head_dim=63), dict(head_dim=64, dims=0), dict(head_dim=64, dims=66), dict(head_dim=64, dims=3), dict(head_dim=64, base=1.0),
                dict(head_dim=64, factor=0.0), dict(head_dim=64, scaling="odd"), dict(head_dim=64, dims=2, scaling="base"),
                dict(head_dim=64, scaling="bands", low=4.0, high=4.0), dict(head_dim=64, scaling="ramp", slow=3.0, fast=2.0),
                dict(head_dim=64, frequencies=[1.0]), dict(head_dim=64, dims=2, frequencies=[math.inf]), dict(head_dim=64, magnitude=math.nan)):
        with refused():
            binding.Rotary(device="cpu", **bad)
    r = binding.Rotary(64, 8, base=16.0, frequencies=[2 * math.pi * 0.75, -2 * math.pi * 0.25, 0.0, 2 * math.pi * 3.5], device="cpu")
    assert [t % 2 ** 64 / 2.0 ** 64 for t in r._turns.tolist()] == [0.75, 0.75, 0.0, 0.5]
    ramp = binding.Rotary(64, scaling="ramp", factor=8.0, original=4096, device="cpu")
    plain, slow = binding.Rotary(64, device="cpu").frequencies, binding.Rotary(64, scaling="linear", factor=8.0, device="cpu").frequencies
    assert ramp.magnitude == 0.1 * math.log(8.0) + 1.0 and ramp.frequencies[0] == plain[0] and abs(ramp.frequencies[-1] / slow[-1] - 1) < 1e-12
    bands = binding.Rotary(64, scaling="bands", factor=8.0, original=4096, device="cpu").frequencies
    assert all(s * (1 - 1e-12) <= b <= p * (1 + 1e-12) for s, b, p in zip(slow, bands, plain)) and bands[0] == plain[0]
    assert abs(bands[-1] / slow[-1] - 1) < 1e-12
    base = binding.Rotary(64, scaling="base", factor=8.0, device="cpu").frequencies
    assert base[0] == 1.0 and abs(base[-1] / slow[-1] - 1) < 1e-9
    q, p = half(6, 4, 64), torch.zeros(6, dtype=torch.int32)
    for bad in (dict(positions=p.long()), dict(positions=p[:5]), dict(positions=p[None]), dict(positions=torch.zeros(12, dtype=torch.int32)[::2]),
                dict(q=q.int()), dict(q=q[0]), dict(q=half(6, 4, 32)), dict(k=half(6, 4, 32)), dict(k=half(5, 2, 64)), dict(k=q.float()),
                dict(k_out=q), dict(out=half(6, 3, 64)), dict(out=q.float()), dict(q=half(6, 64, 4).transpose(1, 2)), dict(q=half(6, 8, 64)[:, ::2])):
        with refused():
            binding.Rotary(64, device="cpu").kv_rotary(**dict(dict(q=q, positions=p), **bad))


@pytest.mark.parametrize("stream", [Stream(22), 22])
def test_what_a_call_on_another_stream_uses_is_kept(calls, monkeypatch, stream):  # noqa: F811
    c = calls.cache
    zeros = torch.zeros

    def made(*args, **kw):
        t = zeros(*args, **kw)
        calls.made.append((t.data_ptr(), calls.at[-1].cuda_stream))
        return t

    def launch(*args):
        calls.launched.append(args[-1])
        return 0
    b, held = made_batch()
    to, to_held = made_batch()
    q, lse, mass, budgets = half(6, 4, 128), torch.zeros(6, 4), torch.zeros(2, 2, 64), torch.zeros(2, dtype=torch.int32)
    kept, n_kept = torch.zeros(2, 2, 10, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    monkeypatch.setattr(torch, "zeros", made)
    monkeypatch.setattr(binding, "_lib", types.SimpleNamespace(kv_fp4_weights=launch, kv_fp4_select=launch, kv_fp4_compact=launch, kv_rotary=launch))
    always = {t.data_ptr() for t in (c.pages, c.workspace, *held)}
    for call, used in ((lambda: [c.kv_fp4_weights(q, lse, b, 1.0, past=mass, stream=stream)], (q, lse, mass)),
                       (lambda: c.kv_fp4_select(mass, b, 10, budgets=budgets, stream=stream), (mass, budgets)),
                       (lambda: [c.kv_fp4_compact(kept, n_kept, b, to, mass=mass, stream=stream)], (kept, n_kept, mass, *to_held))):
        calls.kept.clear(), calls.made.clear()
        out = call()
        assert calls.kept[22] >= always | {t.data_ptr() for t in used}
        assert calls.made == [(t.data_ptr(), 22) for t in out] and calls.kept[11] == {t.data_ptr() for t in out}
    r = binding.Rotary(128, device="cpu")
    p = torch.ones(6, dtype=torch.int32)
    calls.kept.clear(), calls.made.clear()
    out = r.kv_rotary(q, p, k=q, stream=stream)
    assert calls.kept[22] >= {t.data_ptr() for t in (q, p, r._turns)} and calls.kept[11] == {t.data_ptr() for t in out}
    assert calls.made == [(t.data_ptr(), 22) for t in out] and calls.launched == [22] * 4


def test_reference_keeps_what_the_rules_say():
    """The plain rules by hand."""
    m = [5.0, 1.0, 4.0, 4.0, 2.0, 9.0, 0.0, 3.0]
    assert ref.kept(m, 8, 3, 0, 0) == [0, 2, 5] and ref.kept(m, 8, 4, 0, 0) == [0, 2, 3, 5] and ref.kept(m, 8, 3, 2, 0) == [0, 1, 5]
    assert ref.kept(m, 8, 3, 0, 2) == [5, 6, 7] and ref.kept(m, 8, 3, 2, 2) == [0, 1, 7] and ref.kept(m, 8, 2, 5, 5) == [0, 1]
    assert ref.kept(m, 8, 8, 0, 0) == list(range(8)) and ref.kept(m, 8, 5, 0, 0, budget=0) == []
    assert ref.kept([1.0, math.nan, 2.0, math.inf], 4, 2, 0, 0) == [1, 3]
