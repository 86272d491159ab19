"""The paged key-value cache without a GPU: layouts that are refused before anything touches the device, and the model that
the GPU tests compare with, on cases worked out by hand."""
import ctypes

import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
import kv_model as km  # noqa: E402


def layout(**changes):
    a = dict(type=g.P2P_KV_BF16, n_layers=2, n_pages=8, page_tokens=4, n_heads=2, head_dim=16, n_seqs=3, max_pages=5,
             layer_stride=8 * 4 * 2 * 16, page_stride=4 * 2 * 16, token_stride=2 * 16, head_stride=16, k=4096, v=1 << 20,
             table=4096, length=4096, refs=4096, k_scale=None, v_scale=None)
    a.update(changes)
    return g.KvLayout(**a)


@pytest.mark.parametrize("changes", [
    dict(type=3), dict(type=-1), dict(n_layers=0), dict(n_pages=0), dict(n_pages=(1 << 30) + 1), dict(page_tokens=0),
    dict(page_tokens=4097), dict(n_heads=0), dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(n_seqs=0),
    dict(n_seqs=(1 << 20) + 1), dict(max_pages=0), dict(max_pages=1 << 29), dict(k=None), dict(table=None), dict(length=None),
    dict(refs=None), dict(k=4104), dict(v=4098), dict(k_scale=4096), dict(type=g.P2P_KV_E4M3),
    dict(type=g.P2P_KV_E4M3, k_scale=4096, v_scale=4096, head_dim=24, head_stride=24),
    dict(head_stride=8), dict(token_stride=16), dict(page_stride=64), dict(layer_stride=0), dict(layer_stride=-1024),
    dict(head_stride=20, token_stride=40), dict(layer_stride=1 << 45),
    dict(head_stride=32, token_stride=32),
])
def test_layouts_that_are_refused(changes):
    h = ctypes.c_void_p()
    with pytest.raises(g.P2PError) as e:
        g.p2p_kv_create(layout(**changes))
    assert e.value.code == g.P2P_E_INVAL and g.p2p_kv_last_error()
    lib = g._load()
    assert lib.p2p_kv_create(None, ctypes.byref(h)) == g.P2P_E_INVAL and h.value is None


def test_calls_without_a_handle():
    lib = g._load()
    out = (ctypes.c_int64 * 4)()
    for rc in (lib.p2p_kv_set_stream(None, None), lib.p2p_kv_sync(None), lib.p2p_kv_stats(None, ctypes.byref(out)),
               lib.p2p_kv_extend(None, 1, None, None), lib.p2p_kv_trim(None, 1, None, None), lib.p2p_kv_fork(None, 1, None, None, None),
               lib.p2p_kv_compact(None), lib.p2p_kv_write(None, 0, 1, 1, None, None, 1, None, None, 0, 0, 0, 0),
               lib.p2p_kv_attend(None, 0, 1, None, None, 0, 0, 0, 1, 1.0, 0, None, 0, 0, None)):
        assert rc == g.P2P_E_INVAL
    assert g.p2p_kv_launch_count(None) == 0
    g.p2p_kv_destroy(None)


def test_cache_refuses_tensors_that_do_not_fit():
    k = torch.zeros((1, 4, 2, 1, 16), dtype=torch.bfloat16)
    t, n, r = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for args in ((k, k, t, n, r), (k.float(), k.float(), t, n, r), (k, k[:, :3], t, n, r), (k, k, t, n[:1], r), (k, k, t, n, r[:2]),
                 (k, k, t.long(), n, r), (k, k, t, n, r, torch.zeros(1, 2))):
        with pytest.raises(ValueError):  # (the first for want of a GPU tensor)
            g.KvCache(*args)


def test_the_model():
    k = torch.arange(6 * 2, dtype=torch.float32).view(1, 6, 2, 1, 1)
    m = km.Model(k, -k, torch.zeros((3, 3)).int(), torch.zeros(3).int(), torch.zeros(6).int())
    m.extend([1], [3])
    assert m.pages(1) == [0, 1] and m.refs.tolist() == [1, 1, 0, 0, 0, 0]
    m.fork([1], [0], [3])
    assert m.refs.tolist() == [2, 2, 0, 0, 0, 0]
    m.extend([0, 1], [1, 2])        # both leave the shared page; the second takes one more
    assert m.pages(0) == [0, 2] and m.pages(1) == [0, 3, 4] and m.refs.tolist() == [2, 0, 1, 1, 1, 0]
    assert m.k[0, 2, :, 0, 0].tolist() == [2.0, 5.0]
    m.trim([0], [0])
    assert m.refs.tolist() == [1, 0, 0, 1, 1, 0]
    m.compact()
    assert m.pages(1) == [0, 1, 2] and m.refs.tolist() == [1, 1, 1, 0, 0, 0] and m.k[0, 1, :, 0, 0].tolist() == [2.0, 7.0]


def test_the_model_rounds_to_eight_bits_as_torch_does():
    x = np.random.default_rng(0).standard_normal(20000) * np.exp(np.random.default_rng(1).uniform(-9, 6, 20000))
    x = x.astype(np.float32)
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(km.e4m3(x), want)
