"""Rotary positions into memory that the call still reads are refused by the library, but for rows turned where they are: no GPU is touched."""
import ctypes as C

import pytest

from paper_2512_24449_amd import binding
from tests.test_fp4_refusals import ARG

MB = 1 << 20
Q, K, OUT, K_OUT, POSITIONS, TURNS = (MB * i for i in range(1, 7))
ROWS, D, HQ, HK = 5, 64, 4, 2


def turn(q=Q, qs=HQ * D, out=OUT, outs=HQ * D, k=K, ks=HK * D, k_out=K_OUT, k_outs=HK * D, rows=ROWS, size=2, positions=POSITIONS, turns=TURNS):
    table = binding.kv_rotary_t(D, D, 0, 1.0, turns)
    kind = binding.KV_TYPE_FP32 if size == 4 else binding.KV_TYPE_FP16
    return binding.lib().kv_rotary(C.byref(table), positions, rows, kind, 0, q, qs, HQ, out, outs, k, ks, HK if k else 0, k_out, k_outs, None)


@pytest.mark.parametrize("size", [2, 4])
def test_dense_rows(size):
    q_bytes, k_bytes = ROWS * HQ * D * size, ROWS * HK * D * size
    for shift in (size, -size, HQ * D * size, q_bytes - size, size - q_bytes):
        assert turn(out=Q + shift, size=size) == ARG and turn(out=Q + shift, k=None, size=size) == ARG
    for shift in (size, -size, HK * D * size, k_bytes - size, size - k_bytes):
        assert turn(k_out=K + shift, size=size) == ARG
    for at in (K, K + k_bytes - size, K - q_bytes + size):
        assert turn(out=at, size=size) == ARG
    for at in (Q, Q + q_bytes - size, Q - k_bytes + size, OUT, OUT + q_bytes - size, OUT - k_bytes + size):
        assert turn(k_out=at, size=size) == ARG
    assert turn(q=K, out=K, size=size) == ARG                    # q where it is, while k is read there
    for what, n in ((POSITIONS, 4 * ROWS), (TURNS, 4 * D)):
        for at in (what, what + n - 4, what - q_bytes + 4):
            assert turn(out=at, size=size) == ARG
        for at in (what, what + n - 4, what - k_bytes + 4):
            assert turn(k_out=at, size=size) == ARG


def test_parts_of_wider_rows():
    wide = (HQ + 2 * HK) * D
    k, v = Q + 2 * HQ * D, Q + 2 * (HQ + HK) * D
    own = dict(q=Q, qs=wide, out=Q, outs=wide, k=k, ks=wide, k_out=k, k_outs=wide)
    for bad in (dict(out=Q + 2), dict(out=Q - 2 * HK * D - 2), dict(k_out=v - 2), dict(k_out=k - 2), dict(out=k, k_out=K_OUT), dict(k_out=Q),
                dict(outs=wide + 8), dict(k_outs=wide - 8), dict(out=Q + 2 * wide, rows=2), dict(out=OUT, outs=HQ * D, k_out=OUT + 2 * HQ * D, k_outs=wide)):
        assert turn(**dict(own, **bad)) == ARG, bad
    for bad in (dict(outs=wide), dict(outs=HQ * D + 8, rows=2)):
        assert turn(**dict(dict(q=Q, qs=HQ * D, out=Q, k=None), **bad)) == ARG, bad
