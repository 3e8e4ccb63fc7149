"""Rows of a width that leaves most of a workgroup's threads idle, more of them than a launch has workgroups for with a head to each."""
import pytest
import torch

from paper_2512_24449_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_many_rows_of_an_odd_width():
    heads, dim, n = 3, 258, 7 * 857143                           # 129 pairs: a head to a workgroup; 9.3 GB
    rotary = binding.Rotary(dim)
    some = torch.randn(7, heads, dim, generator=torch.Generator().manual_seed(1)).half().to(DEV)
    few = torch.tensor([0, 1, 2 ** 31 - 1, -7, 1000, 5, 77777], dtype=torch.int32, device=DEV)
    want = rotary.kv_rotary(some, few)
    x = torch.empty(n // 7, 7, heads, dim, dtype=torch.float16, device=DEV)
    x.copy_(some)
    got = rotary.kv_rotary(x.view(n, heads, dim), few.repeat(n // 7), out=x.view(n, heads, dim))
    assert got.data_ptr() == x.data_ptr()
    for part in x.split(100000):
        assert bool((part == want).all())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype, shift", [(torch.float16, 0), (torch.bfloat16, 0), (torch.float32, 0), (torch.bfloat16, 4)])
def test_outputs_larger_than_the_caches(dtype, shift, interleaved):
    """The same values as in parts that caches hold, at any alignment."""
    n, heads, dim = 17001, 32, 128
    rotary = binding.Rotary(dim, 96, interleaved=interleaved)
    flat = torch.randn(n * heads * dim + shift, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(dtype)
    q, p = flat[shift:].view(n, heads, dim), torch.arange(n, dtype=torch.int32, device=DEV) * 3
    got = rotary.kv_rotary(q, p)
    assert got.numel() * got.element_size() >= 2 ** 27
    for a, x, at in zip(got.split(1000), q.split(1000), p.split(1000)):
        assert torch.equal(a, rotary.kv_rotary(x, at))
