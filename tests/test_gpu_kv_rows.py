"""Where the attention's results go: rows that share memory are refused, all others are written."""
import random

import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from test_gpu_kv_attend import make, query

DIM = 16


def test_rows_that_overlap():
    """Any strides, against the set of all places."""
    rng = random.Random(3)
    seen = {False: 0, True: 0}
    c = make([5, 0, 40, 17, 3], 1, DIM, 16, "bf16")
    for turn in range(300):
        n, heads = rng.randint(1, 5), rng.randint(1, 6)
        row, head = (rng.choice([0, 1, DIM - 1, DIM, DIM + 1, 2 * DIM, 3 * DIM, heads * DIM, n * DIM, rng.randint(0, 120)]) for _ in "rh")
        places = [i * row + h * head + x for i in range(n) for h in range(heads) for x in range(DIM)]
        overlap = len(set(places)) < len(places)
        seen[overlap] += 1
        q = query(n, heads, DIM, torch.bfloat16, seed=turn)
        room = torch.full((max(places) + 9,), 7.0, device="cuda", dtype=torch.bfloat16)
        out = room.as_strided((n, heads, DIM), (row, head, 1))
        if overlap:
            with pytest.raises(g.P2PError) as e:
                c.attend(0, q, out=out)
            assert e.value.code == g.P2P_E_INVAL
            assert bool((room == 7).all())
        else:
            c.attend(0, q, out=out)
            assert torch.equal(out, c.attend(0, q)[0])
            room[torch.tensor(places, device="cuda")] = 7.0
            assert bool((room == 7).all())
    c.sync()
    assert min(seen.values()) > 60


def test_large_strides():
    c = make([5, 40], 2, DIM, 16, "bf16")
    q = query(2, 4, DIM, torch.bfloat16)
    out = torch.empty((2, 4, DIM), device="cuda", dtype=torch.bfloat16)
    call = lambda row, head, n=2, heads=4: g.p2p_kv_attend(  # noqa: E731
        c.handle, 0, n, None, q.data_ptr(), 4 * DIM, DIM, g.P2P_KV_BF16, heads, 0.25, 0, out.data_ptr(), row, head, None)
    for strides in ((-2 ** 63, -DIM + 1), (0, DIM), (2 ** 62, 2 ** 62), (2 ** 62, -2 ** 62)):
        with pytest.raises(g.P2PError) as e:
            call(*strides)
        assert e.value.code == g.P2P_E_INVAL
    call(0, DIM, n=1)    # (of one row its distance does not matter)
    c.sync()
    assert torch.equal(out[0], c.attend(0, q)[0][0])
