"""What the 4-bit paged cache refuses, and that its host-only parts behave: no GPU is touched."""
import ctypes as C

import pytest
import torch

from paper_2512_24449_amd import binding
from tests import fp4_reference as ref

ARG, UNSUPPORTED = binding.KV_ERR_ARG, binding.KV_ERR_UNSUPPORTED
SOME = 1 << 20          # an aligned address that is never followed


def sizes(*cfg):
    out = binding.kv_fp4_sizes_t()
    return binding.lib().kv_fp4_query_sizes(C.byref(binding.kv_fp4_config_t(*cfg)), C.byref(out)), out


def test_sizes_and_configurations():
    rc, s = sizes(8, 32, 128, 10)
    assert rc == 0 and s.pages == 10 * 8 * 64 * (64 + 4 + 64 + 4) and s.workspace > 0
    rc, s = sizes(3, 3, 64, 7)
    assert rc == 0 and s.pages == 7 * 3 * 64 * 68
    for cfg, want in (((0, 1, 128, 1), ARG), ((1, 0, 128, 1), ARG), ((4, 6, 128, 1), ARG), ((1, 1, 128, 0), ARG),
                      ((1, 1, 128, 2 ** 31), ARG), ((1, 1, 96, 1), UNSUPPORTED), ((1, 1, 256, 1), UNSUPPORTED),
                      ((1, 65536, 128, 1), UNSUPPORTED), ((1024, 1024, 128, 2 ** 31 - 1), UNSUPPORTED)):
        assert sizes(*cfg)[0] == want, cfg
    assert binding.lib().kv_fp4_query_sizes(None, None) == ARG
    assert binding.lib().kv_fp4_query_sizes(C.byref(binding.kv_fp4_config_t(1, 1, 128, 1)), None) == ARG


class Handle(C.Structure):
    """What kv_fp4_cache_t holds (csrc/fp4.h): creating one takes a GPU, being refused with one does not."""
    _fields_ = [("cfg", binding.kv_fp4_config_t), ("pages", C.c_void_p), ("workspace", C.c_void_p)]


@pytest.fixture
def cache():
    held = Handle(binding.kv_fp4_config_t(2, 4, 128, 5), SOME, SOME)
    yield C.cast(C.pointer(held), C.c_void_p)


def test_creation():
    L, handle = binding.lib(), C.c_void_p()
    cfg = binding.kv_fp4_config_t(2, 4, 128, 5)
    _, s = sizes(2, 4, 128, 5)
    create = L.kv_fp4_cache_create
    assert create(C.byref(cfg), None, SOME, C.byref(s), C.byref(handle)) == ARG
    assert create(C.byref(cfg), SOME, None, C.byref(s), C.byref(handle)) == ARG
    assert create(C.byref(cfg), SOME + 64, SOME, C.byref(s), C.byref(handle)) == ARG
    assert create(C.byref(cfg), SOME, SOME, None, C.byref(handle)) == ARG
    assert create(C.byref(cfg), SOME, SOME, C.byref(s), None) == ARG
    assert create(None, SOME, SOME, C.byref(s), C.byref(handle)) == ARG
    for field in ("pages", "workspace"):
        small = binding.kv_fp4_sizes_t(s.pages, s.workspace)
        setattr(small, field, getattr(s, field) - 1)
        assert create(C.byref(cfg), SOME, SOME, C.byref(small), C.byref(handle)) == ARG
    assert L.kv_fp4_cache_destroy(None) == ARG


def batch(**change):
    fields = dict(batch=2, max_new=3, table_pages=4, lens=SOME, new_rows=None, first_row=None, page_table=None)
    fields.update(change)
    return C.byref(binding.kv_fp4_batch_t(**fields))


BAD_BATCHES = [(dict(batch=0), ARG), (dict(max_new=-1), ARG), (dict(table_pages=0), ARG), (dict(lens=None), ARG),
               (dict(lens=SOME + 2), ARG), (dict(new_rows=SOME + 1), ARG), (dict(first_row=SOME + 2), ARG),
               (dict(page_table=SOME + 3), ARG), (dict(table_pages=2 ** 24 + 1), UNSUPPORTED), (dict(batch=65536), UNSUPPORTED)]


@pytest.mark.parametrize("change, want", BAD_BATCHES)
def test_batches(cache, change, want):
    L = binding.lib()
    assert L.kv_fp4_append(cache, batch(**change), SOME, 256, SOME, 256, 0, 6, None) == want
    assert L.kv_fp4_read(cache, batch(**change), SOME, SOME, 0, 6, None) == want
    assert L.kv_fp4_attention(cache, batch(**change), SOME, 512, 0, 6, 1.0, 0, 0, SOME, 0, None, None) == want


def test_no_cache_or_batch(cache):
    L = binding.lib()
    for c, b in ((None, batch()), (cache, None)):
        assert L.kv_fp4_append(c, b, SOME, 256, SOME, 256, 0, 6, None) == ARG
        assert L.kv_fp4_read(c, b, SOME, SOME, 0, 6, None) == ARG
        assert L.kv_fp4_attention(c, b, SOME, 512, 0, 6, 1.0, 0, 0, SOME, 0, None, None) == ARG


def test_append_arguments(cache):
    def call(k=SOME, ks=256, v=SOME, vs=256, type=0, rows=6):
        return binding.lib().kv_fp4_append(cache, batch(), k, ks, v, vs, type, rows, None)
    for bad in (dict(k=None), dict(v=None), dict(k=SOME + 8), dict(v=SOME + 2), dict(ks=255), dict(vs=248), dict(ks=260),
                dict(vs=257), dict(type=2), dict(type=-1), dict(rows=-1)):
        assert call(**bad) == ARG, bad
    assert call(rows=0) == 0 and call(k=None, v=None, rows=0) == 0


def test_read_arguments(cache):
    def call(k=SOME, v=SOME, type=0, rows=6):
        return binding.lib().kv_fp4_read(cache, batch(), k, v, type, rows, None)
    for bad in (dict(k=None, v=None), dict(k=SOME + 8), dict(v=SOME + 4), dict(type=3), dict(type=-1), dict(rows=-1)):
        assert call(**bad) == ARG, bad
    assert call(rows=0) == 0


def test_attention_arguments(cache):
    def call(q=SOME, qs=512, type=0, rows=6, scale=1.0, window=0, sinks=0, out=SOME, out_type=0, lse=None):
        return binding.lib().kv_fp4_attention(cache, batch(), q, qs, type, rows, scale, window, sinks, out, out_type, lse, None)
    for bad in (dict(q=None), dict(q=SOME + 8), dict(qs=504), dict(qs=513), dict(type=2), dict(rows=-1), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(window=-1), dict(sinks=-1), dict(out=None), dict(out=SOME + 8), dict(out_type=3),
                dict(out_type=-1), dict(lse=SOME + 2)):
        assert call(**bad) == ARG, bad
    assert call(rows=0) == 0
    many = binding.kv_fp4_batch_t(1, 2 ** 31 - 1, 4, SOME, None, None, None)
    assert binding.lib().kv_fp4_attention(cache, C.byref(many), SOME, 512, 0, 6, 1.0, 0, 0, SOME, 0, None, None) == UNSUPPORTED


def test_no_new_rows_is_no_work(cache):
    L = binding.lib()
    none = dict(max_new=0)
    assert L.kv_fp4_append(cache, batch(**none), SOME, 256, SOME, 256, 0, 6, None) == 0
    assert L.kv_fp4_read(cache, batch(**none), SOME, SOME, 0, 6, None) == 0
    assert L.kv_fp4_attention(cache, batch(**none), SOME, 512, 0, 6, 1.0, 0, 0, SOME, 0, None, None) == 0


def refused():
    return pytest.raises(binding.PackKVError)


def test_binding_batches():
    lens = torch.ones(2, dtype=torch.int32)
    table = torch.zeros(2, 3, dtype=torch.int32)
    ok = binding.FP4Batch(lens, 1, table)
    assert ok.table_pages == 3 and binding.FP4Batch(lens, 1, table_pages=7).table_pages == 7
    for bad in (lambda: binding.FP4Batch(lens.long(), 1, table), lambda: binding.FP4Batch(lens[None], 1, table),
                lambda: binding.FP4Batch(lens[:0], 1, table[:0]), lambda: binding.FP4Batch(lens, 1),
                lambda: binding.FP4Batch(lens, -1, table), lambda: binding.FP4Batch(lens, 2 ** 31, table),
                lambda: binding.FP4Batch(lens, 1, table.long()), lambda: binding.FP4Batch(lens, 1, table[:1]),
                lambda: binding.FP4Batch(lens, 1, table[:, ::2]), lambda: binding.FP4Batch(lens, 1, table, table_pages=2),
                lambda: binding.FP4Batch(lens, 1, table, new_rows=lens[:1]), lambda: binding.FP4Batch(lens, 1, table, first_row=lens.float()),
                lambda: binding.FP4Batch(lens, 1, torch.zeros(2, 0, dtype=torch.int32)), lambda: binding.FP4Batch(lens, 1, table_pages=0)):
        with refused():
            bad()


@pytest.fixture
def python_cache(cache):
    """The binding's object around the handle, its tensors on the CPU: what it refuses never reaches the library."""
    c = binding.FP4KVCache.__new__(binding.FP4KVCache)
    c._calls = binding._PythonCalls()
    c.handle, c.device, c.n_pages, c.n_kv_heads, c.n_q_heads, c.head_dim = cache, torch.device("cpu"), 5, 2, 4, 128
    yield c
    c.handle = None


def test_binding_calls(python_cache):
    c = python_cache
    b = binding.FP4Batch(torch.ones(2, dtype=torch.int32), 3, table_pages=1)
    half = lambda *s: torch.zeros(*s, dtype=torch.float16)
    kv, q = half(6, 2, 128), half(6, 4, 128)
    for k, v in ((kv.float(), kv.float()), (kv, kv.bfloat16()), (kv, half(5, 2, 128)), (half(6, 3, 128), half(6, 3, 128)),
                 (half(6, 2, 64), half(6, 2, 64)), (half(6, 128, 2).transpose(1, 2), kv), (half(6, 4, 128)[:, ::2], kv),
                 (half(6, 2, 256)[..., ::2], kv), (half(2, 5, 2, 128)[:, :3], half(2, 5, 2, 128)[:, :3]), (half(768), half(768))):
        with refused():
            c.kv_fp4_append(k, v, b)
    for bad in (dict(q=q.float()), dict(q=half(6, 2, 128)), dict(q=q.transpose(0, 1)), dict(window=-1), dict(sinks=-1),
                dict(window=2 ** 31), dict(out=half(6, 4, 64)), dict(out=half(5, 4, 128)), dict(out=q.int()),
                dict(out=half(6, 128, 4).transpose(1, 2)), dict(lse=torch.zeros(6, 4, dtype=torch.float16)),
                dict(lse=torch.zeros(6, 3)), dict(lse=torch.zeros(4, 6).T)):
        args = dict(q=q, batch=b, sm_scale=1.0)
        args.update(bad)
        with refused():
            c.kv_fp4_attention(**args)
    for bad in (dict(dtype=torch.int32), dict(k=half(5, 2, 128)), dict(v=kv.float()), dict(k=half(6, 128, 2).transpose(1, 2))):
        with refused():
            c.kv_fp4_read(b, 6, **bad)
    c.handle = None
    with refused():
        c.kv_fp4_append(kv, kv, b)


def test_reference_rounds_to_the_nearest():
    """The plain arithmetic itself: no value is further than half a gap, ties are even, the scale is the least that fits."""
    x = torch.randn(50, 64, dtype=torch.float64, generator=torch.Generator().manual_seed(0))
    values, codes, e = ref.quantise(x)
    top = x.unflatten(-1, (2, 32)).abs().amax(-1)
    assert bool((top <= 7 * 2.0 ** e.double()).all()) and bool((top > 7 * 2.0 ** (e.double() - 1)).all())
    assert bool(((values - x).abs().unflatten(-1, (2, 32)) <= (2.0 ** e.double())[..., None]).all())
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9] + [0.0] * 24, dtype=torch.float64)
    assert ref.quantise(ties)[0][:8].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
