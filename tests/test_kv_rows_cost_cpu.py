"""How the schedule of the attention of many rows counts its work, without a GPU: all that a call may ask for stays within 32 bits,
and every tile counts for more than what it counts for besides its steps."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2606_17059_gb300 as g

HERE = os.path.dirname(os.path.abspath(__file__))
SET = 2  # kRowsSet


@pytest.fixture(scope="module")
def total(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("cost") / "librows.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", g._build.CSRC, os.path.join(HERE, "host", "rows_cost.cpp"), "-o", lib], check=True)
    f = ctypes.CDLL(lib).rows_total

    def of(pos, members, n_heads, heads, dim, max_tokens, window=0, prefixes=False):
        group = n_heads // heads
        # As the host does: tiles of whole tokens where up to 32 query heads meet, and windows that hide nothing left out.
        for tile_rows in ({128 // group * group, 128} if group <= 32 else {128}):
            pos, members = (np.ascontiguousarray(x, np.int32) for x in (pos, members))
            got, least = ctypes.c_uint64(), ctypes.c_int64()
            same = f(ctypes.c_int64(len(pos)), pos.ctypes.data_as(ctypes.c_void_p), members.ctypes.data_as(ctypes.c_void_p), n_heads, heads,
                     1 if dim > 128 else 2, tile_rows, 6 if dim > 128 else 7, ctypes.c_int64(max_tokens), 0 if window >= max_tokens else window,
                     int(prefixes), ctypes.byref(got), ctypes.byref(least))
            assert same and got.value < 2 ** 32, (got.value / 2 ** 32, tile_rows)
            assert least.value > SET
    return of


@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("n_heads,heads", [(16384, 1), (16384, 16), (8192, 1), (4096, 1), (513, 1), (512, 1), (300, 1), (64, 8), (22, 1), (26, 1), (1, 1), (1024, 1024)])
@pytest.mark.parametrize("cached", [0, 100000, 2 ** 31 - 2 ** 25])
def test_the_largest_calls(total, dim, n_heads, heads, cached):
    """One prompt, or many of one token, of as many rows as a call takes; windows from one token to all."""
    tokens = min(2 ** 29 // n_heads, 2 ** 25 - 1)
    n = min(tokens, 2 ** 20)
    for window in (0, 1, 100, 5000, 10 ** 6, 2 ** 30, 2 ** 31 - 1):
        for most in (cached + tokens, 2 ** 31 - 1):
            total([cached], [tokens], n_heads, heads, dim, most, window)
    # (many: their sum, from a few of them)
    total(np.full(n, cached), np.full(n, 1), n_heads, heads, dim, cached + 1)
    total([cached + 1], [tokens], n_heads, heads, dim, cached + 1, prefixes=True)


def test_calls_of_every_size(total):
    rng = np.random.default_rng(0)
    for _ in range(400):
        heads = int(2 ** rng.uniform(0, 6))
        n_heads = heads * int(2 ** rng.uniform(0, min(14, 13.9 - np.log2(heads))))
        tokens = int(2 ** rng.uniform(0, np.log2(2 ** 29 / n_heads)))
        n = int(2 ** rng.uniform(0, min(12, np.log2(tokens) + 1e-9)))
        cuts = np.sort(rng.integers(0, tokens + 1, n - 1))
        members = np.diff(np.concatenate([[0], cuts, [tokens]]))
        room = 2 ** 31 - 1 - int(members.max())
        pos = (2 ** rng.uniform(0, np.log2(room), n)).astype(np.int64) - 1
        most = int((pos + members).max())
        for dim in (64, 256):
            total(pos, members, n_heads, heads, dim, most, int(2 ** rng.uniform(0, 31)) if rng.integers(2) else 0)
