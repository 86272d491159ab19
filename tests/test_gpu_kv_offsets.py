"""Offsets of prompts that do not hold together: an error, and no row is written, whatever work they would have named."""
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from test_gpu_kv_attend import make, query
    from test_gpu_kv_shared import i32


def refused(c, q, offsets, seq=None):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    c.attend_prompt(0, q, torch.tensor(offsets, device="cuda"), seq=seq, out=out, lse=lse)
    with pytest.raises(g.P2PError) as e:
        c.sync()
    assert e.value.code == g.P2P_E_DEVICE and "offsets" in str(e.value)
    assert bool((out == 7).all()) and bool((lse == 7).all())


@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("offsets", [[0, 20, 10, 30], [0, 20, 31, 30], [-1, 20, 25, 30], [30, 20, 10, 0], [0, 10, 20, 31]])
def test_nothing_is_written(dim, offsets):
    c = make([100, 50, 70], 2, dim, 16, "bf16")
    q = query(30, 4, dim, torch.bfloat16)
    refused(c, q, offsets)
    # ... and the call after it works.
    got = c.attend_prompt(0, q, torch.tensor([0, 10, 20, 30], device="cuda"))
    c.sync()
    assert bool(torch.isfinite(got[0]).all())


def test_the_same_rows_again_and_again():
    """Ascending pairs that name the same rows thousands of times, over a sequence of a million tokens: 2^32 steps and more."""
    k = torch.zeros((1, 1, 64, 8, 64), device="cuda").bfloat16()
    c = g.KvCache(k, k.clone(), torch.zeros((1, 15625), dtype=torch.int32, device="cuda"), i32([1000000]), i32([1]))
    refused(c, query(512, 64, 64, torch.bfloat16), [0, 512] * 4096, torch.zeros(8191, dtype=torch.int32, device="cuda"))


def test_many_offsets():
    """A pair that descends far behind the first ones, where another warp looks at it."""
    n = 5000
    c = make([40], 1, 64, 16, "bf16")
    q = query(n, 2, 64, torch.bfloat16)
    offsets = list(range(n + 1))
    offsets[4321], offsets[4322] = offsets[4322], offsets[4321]
    refused(c, q, offsets, torch.zeros(n, dtype=torch.int32, device="cuda"))
