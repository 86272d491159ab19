"""Scales that are not numbers, or next to nothing, in the calls that take many rows together: as in attend, and in 64 bits."""
import pytest


torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    from test_gpu_kv_attend import make, query
    from test_gpu_kv_shared import groups_of, shared_cache


def both(own, hkv, dim, kind, change, scale):
    """The rows of a group by attend, by attend_shared and, as prompts of one token, by attend_prompt."""
    c = shared_cache([640], [own], hkv, dim, 16, kind)
    change(c)
    q = query(len(own), 6, dim, torch.float16 if kind == "f16" else torch.bfloat16)
    o = torch.arange(len(own) + 1, device="cuda")
    got = [c.attend(0, q, scale), c.attend_shared(0, q, groups_of([len(own)]), scale, least=0), c.attend_prompt(0, q, o, scale)]
    c.sync()
    return got


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 256])
def test_a_scale_that_is_not_a_number(kind, dim):
    for out, lse in both([1, 40, 300], 2, dim, kind, lambda c: None, torch.nan):
        assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_a_scale_of_keys_that_is_not_a_number(dim):
    """Of one kv head: its query heads are NaN, the others are not touched."""
    def change(c):
        c.k_scale[0, 1] = torch.nan
    for out, lse in both([1, 40, 300], 2, dim, "e4m3", change, None):
        assert bool(torch.isnan(out[:, 3:]).all()) and bool(torch.isnan(lse[:, 3:]).all())
        assert bool(torch.isfinite(out[:, :3]).all()) and bool(torch.isfinite(lse[:, :3]).all())


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45, 1e-38, 2.0 ** -123, -2.0 ** -121])
def test_scales_next_to_nothing(scale):
    """Sums of products near the end of 32 bits times a scale at the other end: no more than they are."""
    def change(c):
        c.k.copy_((c.k.float() * 1e18).bfloat16())
    c = make([500, 300], 1, 64, 16, "bf16")
    change(c)
    q = (query(40, 3, 64, torch.bfloat16).float() * 1e17).bfloat16()
    o = torch.tensor([0, 20, 40], device="cuda")
    out, lse = c.attend_prompt(0, q, o, scale)
    c.sync()
    whole = c.length.clone()
    for t in (0, 7, 19):
        c.length.copy_(whole - 19 + t)
        want, want_lse, spread, reach = km.attend(c, 0, q[[t, 20 + t]].contiguous(), scale)
        off, off_lse = km.bounds(spread, reach, 64, "bf16", "bf16")
        assert bool(((out[[t, 20 + t]].double() - want).abs() <= off).all())
        assert bool(((lse[[t, 20 + t]].double() - want_lse).abs() <= off_lse).all())
