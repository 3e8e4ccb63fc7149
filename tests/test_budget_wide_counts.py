"""Tensors with more values along an axis than the library's 32-bit counts hold do not become small ones: no GPU is touched.  (The
tensors' memory is never written.)"""
import types

import pytest
import torch

from paper_2512_24449_amd import binding
from tests.test_fp4_refusals import cache, python_cache, refused  # noqa: F401 (fixtures)
from tests.test_fp4_streams import calls  # noqa: F401


@pytest.mark.parametrize("more", [0, 5, 2 ** 31 + 7])
def test_kept_tokens(python_cache, monkeypatch, more):  # noqa: F811
    seen = []
    monkeypatch.setattr(binding, "_lib", types.SimpleNamespace(kv_fp4_compact=lambda *args: seen.append(args) or 0))
    c = python_cache
    c.n_kv_heads = 1
    b = binding.FP4Batch(torch.ones(1, dtype=torch.int32), 3, table_pages=1)
    kept = torch.empty(1, 1, 2 ** 31 + more, dtype=torch.int32)
    with refused():
        c.kv_fp4_compact(kept, torch.ones(1, dtype=torch.int32), b, b)
    assert not seen


def test_heads(calls, monkeypatch):  # noqa: F811
    seen = []
    monkeypatch.setattr(binding, "_lib", types.SimpleNamespace(kv_rotary=lambda *args: seen.append(args) or 0))
    r = binding.Rotary(2, device="cpu")
    for heads in (4, 65536, 2 ** 32 + 4):
        q = torch.empty(1, heads, 2, dtype=torch.float16)
        r.kv_rotary(q, torch.ones(1, dtype=torch.int32), out=q, stream=22)
    assert [args[7] for args in seen] == [4, 65536, 65536]       # (more than 65535: unsupported)
