"""The last tokens of the longest sequences that a table can hold: their steps end past what 32 bits hold."""
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    import kv_rows_model as rm
    from test_gpu_kv_attend import query
    from test_gpu_kv_shared import i32


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("f16", 128), ("e4m3", 64), ("bf16", 256)])
def test_values_that_not_all_rows_see(kind, dim):
    """Infinite and NaN values among the last tokens go into the rows that see them, and into no other."""
    if torch.cuda.mem_get_info()[0] < 2 << 30:
        pytest.skip("no room")
    n, new, window, pages = 2 ** 31 - 64, 200, 500, 16
    k, v = km.pool(1, pages, 64, 1, dim, kind, "lnht", 0)
    for back, d in ((10, 3), (150, 5), (199, 0)):
        at = (0, (1024 - back) // 64, (1024 - back) % 64, 0, d)
        if kind == "e4m3":
            v.view(torch.uint8)[at] = 0x7F
        else:
            v[at] = torch.nan if d == 5 else torch.inf
    scale = [torch.full((1, 1), 0.02, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
    table = torch.full((1, n // 64), -1, dtype=torch.int32, device="cuda")
    table[0, -pages:] = torch.arange(pages, device="cuda")
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    long = g.KvCache(k, v, table, i32([n]), refs, *scale)
    short = g.KvCache(k, v, torch.arange(pages, dtype=torch.int32, device="cuda")[None].clone(), i32([1024]), refs, *scale)
    q = query(new, 3, dim, torch.float16 if kind == "f16" else torch.bfloat16, size=0.5)
    o = torch.tensor([0, new], device="cuda")
    out, lse = long.attend_prompt(0, q, o, window=window)
    long.sync()
    want, want_lse, spread, reach = rm.prompt(short, 0, q, o, dim ** -0.5, None, window)
    fine = torch.isfinite(want)
    assert bool(fine.any()) and not bool(fine.all())
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(out[torch.isinf(want)].double(), want[torch.isinf(want)])
    off, off_lse = km.bounds(spread, reach, dim, kind, "f16" if kind == "f16" else "bf16")
    assert bool(((out.double() - want).abs() <= off)[fine].all()) and bool(((lse.double() - want_lse).abs() <= off_lse).all())
