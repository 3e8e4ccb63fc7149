"""Which tensors a call on a stream of the program's choosing keeps from being reused, and whose memory its outputs get: stand-ins
for the streams and the library, no GPU."""
import contextlib
import types

import pytest
import torch

from paper_2512_24449_amd import binding
from tests.test_fp4_refusals import cache, python_cache  # noqa: F401 (fixtures)


class Stream:
    def __init__(self, pointer):
        self.cuda_stream = pointer


CURRENT = Stream(11)


@pytest.fixture
def calls(monkeypatch, python_cache):  # noqa: F811
    c = python_cache
    c.pages, c.workspace = torch.zeros(1, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8)
    seen = types.SimpleNamespace(cache=c, kept={}, made=[], at=[CURRENT], launched=[])

    def record(tensor, stream):
        seen.kept.setdefault(stream.cuda_stream, set()).add(tensor.data_ptr())

    @contextlib.contextmanager
    def stream(s):
        seen.at.append(s)
        yield
        seen.at.pop()
    empty = torch.empty

    def made(*args, **kw):
        t = empty(*args, **kw)
        seen.made.append((t.data_ptr(), seen.at[-1].cuda_stream))
        return t

    def launch(handle, batch, *args):
        seen.launched.append(args[-1])
        return 0
    monkeypatch.setattr(torch.Tensor, "record_stream", record)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: CURRENT)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda pointer, device=None: Stream(pointer))
    monkeypatch.setattr(torch, "empty", made)
    monkeypatch.setattr(binding, "_current_device", lambda: None)
    monkeypatch.setattr(binding, "_lib", types.SimpleNamespace(kv_fp4_append=launch, kv_fp4_read=launch, kv_fp4_attention=launch))
    return seen


def made_batch():
    ints = lambda *s: torch.ones(*s, dtype=torch.int32)
    tensors = ints(2), ints(2, 3), ints(2), ints(2)
    return binding.FP4Batch(tensors[0], 3, tensors[1], new_rows=tensors[2], first_row=tensors[3]), tensors


def half(*shape):
    return torch.zeros(*shape, dtype=torch.float16)


@pytest.mark.parametrize("stream", [Stream(22), 22])
def test_what_a_call_on_another_stream_uses_is_kept(calls, stream):
    c = calls.cache
    for given in (False, True):
        batch, held = made_batch()
        k, v, q = half(6, 2, 128), half(6, 2, 128), half(6, 4, 128)
        lse = torch.zeros(6, 4)
        calls.kept.clear()
        c.kv_fp4_append(k, v, batch, stream=stream)
        assert calls.kept[22] == {t.data_ptr() for t in (k, v, c.pages, c.workspace, *held)}
        calls.kept.clear(), calls.made.clear()
        out = c.kv_fp4_read(batch, 6, k=k if given else None, v=v if given else None, stream=stream)
        assert calls.kept[22] >= {t.data_ptr() for t in (c.pages, c.workspace, *held)} | ({t.data_ptr() for t in out} if given else set())
        assert calls.made == ([] if given else [(t.data_ptr(), 22) for t in out])
        assert given or calls.kept[11] == {t.data_ptr() for t in out}     # (used there next)
        calls.kept.clear(), calls.made.clear()
        to = half(6, 4, 128) if given else None
        out = c.kv_fp4_attention(q, batch, 1.0, out=to, lse=lse, stream=stream)
        want = {t.data_ptr() for t in (q, lse, c.pages, c.workspace, *held)}
        assert calls.kept[22] >= (want | {out.data_ptr()} if given else want)
        assert calls.made == ([] if given else [(out.data_ptr(), 22)])
        assert given or calls.kept[11] == {out.data_ptr()}
    assert calls.launched == [22] * 6 and calls.at == [CURRENT]


def test_calls_on_the_current_stream_keep_nothing(calls, monkeypatch):
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream=None: 11)
    c, (batch, _) = calls.cache, made_batch()
    c.kv_fp4_append(half(6, 2, 128), half(6, 2, 128), batch)
    made = [*c.kv_fp4_read(batch, 6), c.kv_fp4_attention(half(6, 4, 128), batch, 1.0)]
    assert not calls.kept and calls.made == [(t.data_ptr(), 11) for t in made]
