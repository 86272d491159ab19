"""The cache's host code without a GPU, over a fake CUDA runtime (host/): what the calls refuse before anything is launched, and a
kernel that cannot be launched."""
import ctypes
import os
import subprocess

import pytest

import paper_2606_17059_gb300 as g

HERE = os.path.dirname(os.path.abspath(__file__))
CUDA = os.path.dirname(os.path.dirname(g._build.NVCC)) if os.sep in g._build.NVCC else "/usr/local/cuda"
INVALID_DEVICE_FUNCTION, OUT_OF_MEMORY = 98, 2


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host") / "libkv.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", os.path.join(CUDA, "include"), "-I", g._build.CSRC, "-I",
                    g._build.INCLUDE, "-o", so, os.path.join(g._build.CSRC, "kv_cache.cpp"), os.path.join(HERE, "host", "fake_kv.cpp")], check=True)
    lib = ctypes.CDLL(so)
    lib.p2p_kv_last_error.restype = ctypes.c_char_p
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.p2p_kv_attend.argtypes = [vp, i32, i32, vp, vp, i64, i64, i32, i32, f32, i32, vp, i64, i64, vp]
    lib.p2p_kv_attend_prompt.argtypes = [vp, i32, i32, vp, vp, i64, vp, i64, i64, i32, i32, f32, i32, vp, i64, i64, vp]
    lib.p2p_kv_attend_shared.argtypes = [vp, i32, i32, vp, i32, vp, i64, vp, i64, i64, i32, i32, f32, i32, vp, i64, i64, vp, vp]
    lib.p2p_kv_write_rotated.argtypes = [vp, i32, i32, vp, vp, i64, ctypes.POINTER(g.KvRotation), vp, i64, i64, i32, vp, vp, i64, i64, i32, vp, i64, i64]
    lib.p2p_kv_set_patience.argtypes = [vp, i64]
    return lib


def create(lib, **changes):
    a = dict(type=g.P2P_KV_BF16, n_layers=2, n_pages=8, page_tokens=4, n_heads=2, head_dim=16, n_seqs=3, max_pages=5, layer_stride=8 * 4 * 2 * 16,
             page_stride=4 * 2 * 16, token_stride=2 * 16, head_stride=16, k=4096, v=1 << 20, table=4096, length=4096, refs=4096)
    a.update(changes)
    layout, h = g.KvLayout(**a), ctypes.c_void_p()
    return lib.p2p_kv_create(ctypes.byref(layout), ctypes.byref(h)), h


def calls(lib, h):
    """attend, attend_prompt and attend_shared of two rows with 4 heads."""
    q, out = 1 << 21, 1 << 22
    return (lib.p2p_kv_attend(h, 0, 2, None, q, 64, 16, g.P2P_KV_BF16, 4, 0.25, 0, out, 64, 16, None),
            lib.p2p_kv_attend_prompt(h, 0, 1, None, 4096, 2, q, 64, 16, g.P2P_KV_BF16, 4, 0.25, 0, out, 64, 16, None),
            lib.p2p_kv_attend_shared(h, 0, 2, None, 1, 4096, 0, q, 64, 16, g.P2P_KV_BF16, 4, 0.25, 0, out, 64, 16, None, 1 << 23))


def test_a_kernel_that_cannot_be_launched(lib):
    """It is the calls that need it that are refused, not the cache; other errors are the creation's."""
    rc, h = create(lib)
    assert rc == g.P2P_OK and calls(lib, h) == (0, 0, 0)
    lib.p2p_kv_destroy(h)
    lib.fake_rows_fail(INVALID_DEVICE_FUNCTION)
    rc, h = create(lib)
    assert rc == g.P2P_OK
    before = lib.fake_launches()
    assert calls(lib, h) == (0, g.P2P_E_CUDA, g.P2P_E_CUDA) and b"registers" in lib.p2p_kv_last_error(h)
    assert lib.fake_launches() == before + 1
    lib.p2p_kv_destroy(h)
    lib.fake_rows_fail(OUT_OF_MEMORY)
    assert create(lib)[0] == g.P2P_E_NOMEM
    lib.fake_rows_fail(0)


def test_rotated_queries_over_other_rows(lib):
    rc, h = create(lib)
    assert rc == g.P2P_OK
    r = g.KvRotation(0, 0, 1.0, 1e-6, None, None, None)
    base, row = 1 << 21, (6 + 2 + 2) * 16     # tokens of 6 query heads, then 2 of keys and of values, 16 each

    def write(out, out_row=row, out_head=16, q=base, n=50):
        return lib.p2p_kv_write_rotated(h, 0, 1, 4096, 4096, n, ctypes.byref(r), q, row, 16, 6, base + 2 * 96, base + 2 * 128, row, 16, g.P2P_KV_BF16, out, out_row, out_head)

    before = lib.fake_launches()
    fine = [write(base), write(base + 2 * 50 * row, 96), write(base - 2 * 6 * 16 * 50, 96), write(1 << 30, 96)]
    assert fine == [0] * 4 and lib.fake_launches() == before + 4
    for bad in ((base + 16,), (base + 2 * row,), (base + 2 * 16,), (base + 2 * 96,), (base + 2 * 128,), (base, 96), (base - 2 * 96 * 10, 96), (base + 2 * 50 * row - 2, 96)):
        assert write(*bad) == g.P2P_E_INVAL and b"overlap" in lib.p2p_kv_last_error(h), bad
    assert lib.fake_launches() == before + 4
    assert write(base, 1, n=1) == 0   # (one token: its distance to the next is of no use)
    lib.p2p_kv_destroy(h)


def test_patience(lib):
    rc, h = create(lib)
    assert rc == g.P2P_OK and lib.p2p_kv_set_patience(h, -1) == 0 and lib.p2p_kv_set_patience(h, 1 << 40) == 0
    assert lib.p2p_kv_set_patience(h, 0) == g.P2P_E_INVAL and lib.p2p_kv_set_patience(h, -2 ** 63) == g.P2P_E_INVAL and lib.p2p_kv_set_patience(None, 1) == g.P2P_E_INVAL
    lib.p2p_kv_destroy(h)
