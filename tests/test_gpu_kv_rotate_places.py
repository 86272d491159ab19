"""Where write_rotated may put its queries: over q itself, beside it in the same buffer, elsewhere; not over others' rows."""
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from test_gpu_kv_attend import make
    from test_gpu_kv_shared import i32

HQ, HKV, DIM, N = 6, 2, 64, 200


def parts(room):
    return room.split([HQ, HKV, HKV], 1)


def test_places():
    c = make([N], HKV, DIM, 16, "bf16")
    rope = g.Rope(DIM)
    seq, o = i32([0]), torch.tensor([0, N], device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(0)
    room = torch.randn((N, HQ + 2 * HKV, DIM), device="cuda", generator=gen).bfloat16()
    q, k, v = parts(room.clone())
    want = c.write_rotated(0, seq, o, q, k, v, rope)
    keys = c.k.clone()
    # over q itself, with keys and values beside it
    q, k, v = parts(room.clone())
    assert c.write_rotated(0, seq, o, q, k, v, rope, out=q).data_ptr() == q.data_ptr()
    assert torch.equal(q, want) and torch.equal(k, room[:, HQ:HQ + HKV]) and torch.equal(c.k.view(torch.int16), keys.view(torch.int16))
    # beside it, in the same rows and behind them
    wide = torch.zeros((N, 2 * HQ + 2 * HKV, DIM), device="cuda").bfloat16()
    wide[:, :HQ + 2 * HKV] = room
    q, k, v, out = wide.split([HQ, HKV, HKV, HQ], 1)
    c.write_rotated(0, seq, o, q, k, v, rope, out=out)
    assert torch.equal(out, want)
    flat = torch.cat([room.flatten(), torch.zeros(N * HQ * DIM, device="cuda").bfloat16()])
    q, k, v = parts(flat[:room.numel()].view(room.shape))
    out = flat[room.numel():].view(N, HQ, DIM)
    c.write_rotated(0, seq, o, q, k, v, rope, out=out)
    assert torch.equal(out, want)
    c.sync()
    # not where others' rows would be written over
    flat = torch.zeros(room.numel() + 4 * HQ * DIM, device="cuda").bfloat16()
    q, k, v = parts(flat[:room.numel()].view(room.shape))
    row = (HQ + 2 * HKV) * DIM
    for at, strides in ((8, (row, DIM, 1)), (row, (row, DIM, 1)), (DIM, (row, DIM, 1)), (0, (HQ * DIM, DIM, 1)), (HQ * DIM, (row, DIM, 1)),
                        (4 * DIM, (row, DIM, 1)), (HQ * DIM, (HQ * DIM, DIM, 1))):
        with pytest.raises(g.P2PError) as e:
            c.write_rotated(0, seq, o, q, k, v, rope, out=flat.as_strided((N, HQ, DIM), strides, at))
        assert e.value.code == g.P2P_E_INVAL and "overlap" in str(e.value)
    assert bool((flat == 0).all())
    c.sync()
