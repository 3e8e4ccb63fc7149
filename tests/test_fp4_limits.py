"""Sizes and scales at the edge of what the 4-bit paged cache takes: refused on the host, without a launch."""
import ctypes as C

import pytest

from paper_2512_24449_amd import binding
from tests.test_fp4_refusals import ARG, SOME, Handle, batch


def handle(heads, dim):
    held = Handle(binding.kv_fp4_config_t(heads, heads, dim, 5), SOME, SOME)
    return C.cast(C.pointer(held), C.c_void_p), held


@pytest.mark.parametrize("scale", [2.4e38, -3e38])
def test_scales_that_the_exponential_cannot_take(scale):
    """sm_scale * log2(e) is beyond fp32."""
    c, held = handle(2, 128)
    assert binding.lib().kv_fp4_attention(c, batch(), SOME, 256, 0, 6, scale, 0, 0, SOME, 0, None, None) == ARG
