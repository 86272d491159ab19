"""Layers and windows that 32 bits do not hold are what they say, not what is left of them."""
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from test_gpu_kv_attend import make, query
    from test_gpu_kv_pages import i32, i64, rows


def test_windows():
    c = make([100, 700, 5], 2, 64, 16, "bf16")
    q = query(3, 4, 64, torch.bfloat16)
    want, want_lse = c.attend(0, q)
    for window in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 63, 10 ** 30):    # (of 2^32 + 5, 32 bits are a window of 5)
        out, lse = c.attend(0, q, window=window)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    for window in (-1, -2 ** 31, -2 ** 32 + 5, -10 ** 30):
        with pytest.raises(g.P2PError) as e:
            c.attend(0, q, window=window)
        assert e.value.code == g.P2P_E_INVAL
    c.sync()


def test_layers():
    c = make([100, 700, 5], 2, 64, 16, "bf16", layers=2)
    q = query(3, 4, 64, torch.bfloat16)
    k, v = rows(c, 1, layers=1)
    for layer in (2, 2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 32, -1, 10 ** 30):
        for call in (lambda: c.attend(layer, q), lambda: c.write(layer, i32([0]), i64([0, 1]), k, v)):
            with pytest.raises(g.P2PError) as e:
                call()
            assert e.value.code == g.P2P_E_INVAL
    c.sync()
