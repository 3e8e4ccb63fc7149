"""Sizes and scales at the edge of what the 4-bit paged cache takes: refused on the host, without a launch."""
import ctypes as C

import pytest

from paper_2512_24449_amd import binding
from tests.test_fp4_refusals import ARG, SOME, UNSUPPORTED, Handle, batch


def handle(heads, dim):
    held = Handle(binding.kv_fp4_config_t(heads, heads, dim, 5), SOME, SOME)
    return C.cast(C.pointer(held), C.c_void_p), held


@pytest.mark.parametrize("scale", [2.4e38, -3e38])
def test_scales_that_the_exponential_cannot_take(scale):
    """sm_scale * log2(e) is beyond fp32."""
    c, held = handle(2, 128)
    assert binding.lib().kv_fp4_attention(c, batch(), SOME, 256, 0, 6, scale, 0, 0, SOME, 0, None, None) == ARG


@pytest.mark.parametrize("heads, dim, max_new", [(128, 128, 2 ** 24), (128, 64, 2 ** 25), (1, 128, 2 ** 31 - 1), (1000, 128, 2 ** 31 - 1)])
def test_more_workgroups_than_a_launch_takes(heads, dim, max_new):
    """A launch has fewer than 2^32 threads along an axis, one to 64 channels of a row here."""
    c, held = handle(heads, dim)
    rows = batch(max_new=max_new)
    assert binding.lib().kv_fp4_append(c, rows, SOME, heads * dim, SOME, heads * dim, 0, 6, None) == UNSUPPORTED
    assert binding.lib().kv_fp4_read(c, rows, SOME, SOME, 0, 6, None) == UNSUPPORTED
