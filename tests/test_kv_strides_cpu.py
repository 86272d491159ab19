"""Whether rows of two strided arrays share a value, as the host finds it, against the values themselves."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2606_17059_gb300 as g

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("strides") / "libstrides.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", g._build.CSRC, os.path.join(HERE, "host", "strides.cpp"), "-o", lib], check=True)
    f = ctypes.CDLL(lib).meet
    f.argtypes = [ctypes.c_int64] * 9
    return lambda *a: bool(f(*(int(x) for x in a)))


def values(at, row, head, heads, n, dim):
    return set((at + np.arange(n)[:, None, None] * row + np.arange(heads)[:, None] * head + np.arange(dim)).ravel().tolist())


def test_small_arrays(meet):
    rng = np.random.default_rng(0)
    both = [0, 0]
    for _ in range(30000):
        n, dim, apart, row, head, ha, hb = (int(rng.integers(*x)) for x in ((1, 6), (1, 5), (-120, 121), (-30, 31), (-8, 9), (1, 5), (1, 5)))
        row2, head2 = (row, int(rng.integers(-30, 31)))[int(rng.integers(4) == 0)], (head, int(rng.integers(-8, 9)))[int(rng.integers(2))]
        want = bool(values(0, row, head, ha, n, dim) & values(apart, row2, head2, hb, n, dim))
        got = meet(apart, row, head, ha, row2, head2, hb, n, dim)
        assert got == want or (got and n > 1 and row != row2), (apart, row, head, ha, row2, head2, hb, n, dim)
        both[want] += 1
    assert min(both) > 3000


def test_arrays_as_they_are_used(meet):
    """Queries, keys and values side by side in a token's row; head by head; in buffers of their own; broadcast."""
    hq, hkv, d, n = 64, 8, 128, 2 ** 31 - 1
    row = (hq + 2 * hkv) * d
    assert not meet(hq * d, row, d, hq, row, d, hkv, n, d) and not meet(-hq * d, row, d, hkv, row, d, hq, n, d)
    assert meet(hq * d - 1, row, d, hq, row, d, hkv, n, d) and meet(8, row, d, hq, row, d, hq, n, d)
    assert not meet(hq * n * d, d, n * d, hq, d, n * d, hkv, n, d)
    assert meet(hq * n * d - 1, d, n * d, hq, d, n * d, hkv, n, d)
    assert not meet(2 ** 45, hq * d, d, hq, hq * d, d, hq, n, d)
    assert meet(0, 0, 0, hq, hq * d, d, hq, 5, d) and not meet(5 * hq * d, 0, 0, hq, hq * d, d, hq, 5, d)
    # interleaved heads: query heads between the keys'
    assert not meet(d, 3 * d * hkv, 3 * d, hkv, 3 * d * hkv, 3 * d, hkv, 1000, d) and meet(d + 1, 3 * d * hkv, 3 * d, hkv, 3 * d * hkv, d, 2 * hkv, 1000, d)
