"""Calls around a cache's budget whose outputs lie where the call still reads are refused by the library: no GPU is touched."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2512_24449_amd import binding, build
from tests.test_fp4_refusals import ARG, batch, cache  # noqa: F401 (fixture)

HERE = os.path.dirname(os.path.abspath(__file__))
MB = 1 << 20
LENS, ROWS, FIRST, TABLE, Q, LSE, PAST, MASS, BUDGETS, KEPT, N_KEPT, MASS_OUT, TO_TABLE = (MB * i for i in range(1, 14))
# of the fixture's cache (2 kv-heads, 4 query heads of 128) and a batch of 2 sequences of 4 pages
TOKENS, KEEP = 256, 10
SIZE = {LENS: 8, ROWS: 8, FIRST: 8, TABLE: 32, Q: 5 * 1200 + 1024, LSE: 6 * 4 * 4, PAST: 2 * 2 * TOKENS * 4, MASS: 2 * 2 * TOKENS * 4, BUDGETS: 8,
        KEPT: 2 * 2 * KEEP * 4, N_KEPT: 8, MASS_OUT: 2 * 2 * 9 * 4, TO_TABLE: 32}


def whole():
    return batch(lens=LENS, new_rows=ROWS, first_row=FIRST, page_table=TABLE)


def weights(c, past=PAST, mass=MASS):
    return binding.lib().kv_fp4_weights(c, whole(), Q, 600, 0, 6, 1.0, 0, 0, LSE, past, mass, TOKENS, None)


def select(c, mass=MASS, budgets=BUDGETS, kept=KEPT, n_kept=N_KEPT):
    return binding.lib().kv_fp4_select(c, whole(), mass, TOKENS, KEEP, budgets, 0, 0, kept, n_kept, None)


def compact(c, mass=MASS, mass_out=MASS_OUT):
    to = batch(lens=N_KEPT, new_rows=N_KEPT, page_table=TO_TABLE)
    return binding.lib().kv_fp4_compact(c, whole(), to, KEPT, KEEP, N_KEPT, mass, TOKENS, mass_out, 9, None)


def on(read, written):
    """Addresses of the output `written` that reach `read`'s first or last value."""
    return (read, read + SIZE[read] - 4, read - SIZE[written] + 4)


@pytest.mark.parametrize("read", [LENS, BUDGETS, MASS])
def test_selection(cache, read):  # noqa: F811
    for at in on(read, KEPT):
        assert select(cache, kept=at) == ARG
    for at in on(read, N_KEPT):
        assert select(cache, n_kept=at) == ARG


def test_selection_into_one_place(cache):  # noqa: F811
    for at in on(KEPT, N_KEPT):
        assert select(cache, n_kept=at) == ARG


@pytest.mark.parametrize("read", [LENS, TABLE, MASS, KEPT, N_KEPT, TO_TABLE])
def test_compaction(cache, read):  # noqa: F811
    for at in on(read, MASS_OUT):
        assert compact(cache, mass_out=at) == ARG


@pytest.mark.parametrize("read", [LENS, ROWS, FIRST, TABLE, Q, LSE])
def test_weights(cache, read):  # noqa: F811
    for past in (None, PAST):
        for at in on(read, MASS):
            assert weights(cache, past, at) == ARG


def test_weights_beside_past(cache):  # noqa: F811
    for shift in (4, -4, SIZE[MASS] - 4, 4 - SIZE[MASS]):        # (past itself is what the call is for)
        assert weights(cache, PAST, PAST + shift) == ARG


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("overlap") / "overlap_check.so")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", "-I", build.CSRC, "-o", lib,
                           os.path.join(HERE, "overlap_check.cpp")])
    L = C.CDLL(lib)
    L.rows_overlap.argtypes = [C.c_uint64, C.c_int64, C.c_int64, C.c_int64] * 2
    L.rows_overlap.restype = C.c_int
    return L.rows_overlap


def test_rows_against_every_byte(check):
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(30000):
        a, b = ((rng.randint(0, 60), rng.randint(0, 6), rng.choice([0, 1, 1, 2, 3, 5, 9]), w) for w in (rng.randint(1, 8), rng.randint(1, 8)))
        a, b = ((at, w, w + gap, n) for at, gap, n, w in (a, b))
        if rng.random() < 0.5:
            b = (b[0], min(b[1], a[2]), a[2], b[3])              # the same stride
        bytes_of = lambda at, w, stride, n: {at + i * stride + j for i in range(n) for j in range(w)}
        want = bool(bytes_of(*a) & bytes_of(*b))
        assert check(1000 + a[0], *a[1:], 1000 + b[0], *b[1:]) == want == check(1000 + b[0], *b[1:], 1000 + a[0], *a[1:]), (a, b)
        seen[want] += 1
    assert min(seen) > 5000


def test_rows_without_an_address_and_of_any_size(check):
    most = 2 ** 63 - 1
    assert not check(0, 8, 8, 5, 4, 8, 8, 5) and not check(0, 8, 8, 5, 0, 8, 8, 5)
    assert not check(100, most, most, 0, 50, most, most, most) and not check(2 ** 63, 4, 4, 1, 64, 4, 2 ** 30, 2 ** 32)
    assert check(2 ** 47, 4, 4, 1, 64, most, most, most) and check(2 ** 46 + 64, 4, 4, 1, 64, 4, 2 ** 30, 2 ** 32)
    assert not check(2 ** 46 + 68, 4, 4, 1, 64, 4, 2 ** 30, 2 ** 32)
    # parts of one projection, as many rows as a prompt has
    for n in (1, 8192, 10 ** 9):
        assert not check(4096, 8192, 12288, n, 4096 + 8192, 2048, 12288, n)
        assert check(4096, 8192, 12288, n, 4096 + 8190, 2048, 12288, n)
        assert bool(check(4096 + 12280, 16, 12288, n, 4096, 2, 12288, n)) == (n > 1)
