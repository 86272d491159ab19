"""Attention of prompts with thousands of query heads a kv head: every row is written, at the largest sizes that a call takes."""
import pytest


torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    from test_gpu_kv_attend import make


@pytest.mark.parametrize("heads,tokens,dim", [(16384, 23168, 8), (16384, 300, 136), (8192, 5000, 64), (600, 9000, 64), (513, 2500, 200)])
def test_every_row(heads, tokens, dim):
    size = heads * tokens * dim * 4 + heads * tokens * 4
    if torch.cuda.mem_get_info()[0] < 1.2 * size + (4 << 30):
        pytest.skip("no room")
    c = make([tokens], 1, dim, 64, "bf16")
    q, out = torch.empty((tokens, heads, dim), device="cuda", dtype=torch.bfloat16), torch.full((tokens, heads, dim), torch.nan, device="cuda", dtype=torch.bfloat16)
    q.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    lse = torch.full((tokens, heads), torch.nan, device="cuda")
    c.attend_prompt(0, q, torch.tensor([0, tokens], device="cuda"), out=out, lse=lse)
    c.sync()
    for x in (out, lse):
        for part in x.split(1024):
            assert bool(torch.isfinite(part).all())
    rows = torch.cat([torch.arange(0, tokens, max(1, tokens // 13)), torch.tensor([1, tokens - 1])])
    some = torch.tensor([0, 1, 127, 128, 255, 256, heads // 2, heads - 1], device="cuda").clamp(max=heads - 1)
    whole = c.length.clone()
    for t in rows.tolist():
        c.length.fill_(t + 1)
        want, want_lse, spread, reach = km.attend(c, 0, q[t:t + 1, some].contiguous(), dim ** -0.5)
        off, off_lse = km.bounds(spread, reach, dim, "bf16", "bf16")
        assert bool(((out[t:t + 1, some].double() - want).abs() <= off).all()) and bool(((lse[t:t + 1, some].double() - want_lse).abs() <= off_lse).all())
    c.length.copy_(whole)
    del q, out, lse
    torch.cuda.empty_cache()
