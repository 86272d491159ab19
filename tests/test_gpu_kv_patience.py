"""Waits of the attention of many rows that run out, as nothing ends them: the kernel ends by itself, the call's error says so, and the next call works."""
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from test_gpu_kv_attend import make, query
    from test_gpu_kv_shared import groups_of, shared_cache

PATIENCE = 4 * 10 ** 9


def gives_up(c, call):
    want = call()
    c.sync()
    g.p2p_kv_set_patience(c.handle, -10 ** 6)
    for _ in range(3):
        call()
        with pytest.raises(g.P2PError) as e:
            c.sync()
        assert e.value.code == g.P2P_E_DEVICE and "gave up" in str(e.value)
    g.p2p_kv_set_patience(c.handle, PATIENCE)
    for _ in range(2):
        got = call()
        c.sync()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind,hq,hkv,dim,page", [("bf16", 14, 2, 64, 16), ("f16", 8, 8, 128, 16), ("e4m3", 16, 2, 128, 32), ("e4m3", 16, 2, 128, 1), ("bf16", 6, 2, 256, 16),
                                                  ("f16", 71, 1, 80, 7), ("e4m3", 6, 2, 256, 100)])
def test_prompts(kind, hq, hkv, dim, page):
    cached, new = [0, 5000, 100], [300, 700, 40]
    c = make([a + b for a, b in zip(cached, new)], hkv, dim, page, kind)
    q = query(sum(new), hq, dim, torch.float16 if kind == "f16" else torch.bfloat16)
    o = torch.tensor([0, 300, 1000, 1040], device="cuda")
    gives_up(c, lambda: c.attend_prompt(0, q, o))


def test_shared():
    c = shared_cache([3000], [list(range(40))], 2, 64, 16, "bf16")
    q = query(40, 14, 64, torch.bfloat16)
    gives_up(c, lambda: c.attend_shared(0, q, groups_of([40]), least=0))


def test_refusals():
    c = make([10], 1, 64, 16, "bf16")
    with pytest.raises(g.P2PError):
        g.p2p_kv_set_patience(c.handle, 0)
    with pytest.raises(g.P2PError):
        g.p2p_kv_set_patience(None, 1)


def test_work_that_takes_longer():
    """NaN values over thousands of tokens that only some rows see take milliseconds to be given to them: that is no wait that ran out."""
    groups = 16
    c = shared_cache([6016] * groups, [[0, 2500, 5000]] * groups, 8, 64, 16, "bf16")
    for i in range(0, 3 * groups, 3):
        c.v[:, c.table[i, 1000 // 16:6016 // 16].long()] = torch.nan
    q = query(3 * groups, 16, 64, torch.bfloat16)
    want = c.attend(0, q, window=5000)
    g.p2p_kv_set_patience(c.handle, 10 ** 6)
    out, lse = c.attend_shared(0, q, groups_of([3] * groups), window=5000, least=0)
    c.sync()
    g.p2p_kv_set_patience(c.handle, PATIENCE)
    assert bool(torch.isnan(out.view(groups, 3, 16, 64)[:, :2]).all()) and torch.equal(torch.isnan(out), torch.isnan(want[0]))
    fine = ~torch.isnan(out)
    assert bool(fine.any()) and torch.allclose(out[fine].float(), want[0][fine].float(), atol=2.0 ** -7, rtol=2.0 ** -7) and torch.allclose(lse, want[1], atol=1e-4)
