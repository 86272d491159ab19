"""Rows of which some or all logits are -infinity (a key that overflowed): the calls agree on them, and with the same in 64 bits."""
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    from test_gpu_kv_attend import make, query
    from test_gpu_kv_shared import groups_of, i32, shared_cache

TYPE = {"bf16": torch.bfloat16, "f16": torch.float16}


def sink(c, s, tokens):
    """Logits of these tokens of sequence s become -infinity for queries whose first value is above 0."""
    page = c.k.shape[2]
    for t in tokens:
        c.k[:, int(c.table[s, t // page]), t % page, :, 0] = -torch.inf


def rising(n, hq, dim, kind):
    q = query(n, hq, dim, TYPE[kind])
    q[..., 0] = q[..., 0].abs() + 0.5
    return q


def near(got, want, spread, reach, dim, kind):
    off, off_lse = km.bounds(spread, reach, dim, kind, kind)
    assert bool(((got[0].double() - want[0]).abs() <= off).all()) and bool(((got[1].double() - want[1]).abs() <= off_lse).all())


SHAPES = [("f16", 14, 2, 64), ("bf16", 8, 8, 128), ("f16", 24, 2, 96), ("f16", 16, 1, 256), ("bf16", 6, 2, 64)]


@pytest.mark.parametrize("kind,hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("prefix", [640, 30000])
def test_own_tokens_without_a_finite_logit(kind, hq, hkv, dim, prefix):
    """What a row holds beyond its group's prefix counts for nothing: the prefix alone comes out."""
    own = [1, 1, 5, 16, 0, 40, 300]
    c = shared_cache([prefix], [own], hkv, dim, 16, kind)
    for s in (0, 2, 3, 5, 6):
        sink(c, s, range(prefix, prefix + own[s]))
    q = rising(len(own), hq, dim, kind)
    got = c.attend_shared(0, q, groups_of([len(own)]), least=0)
    c.sync()
    whole = c.length.clone()
    c.length[[0, 2, 3, 5, 6]] = prefix
    want, want_lse, spread, reach = km.attend(c, 0, q, dim ** -0.5)
    c.length.copy_(whole)
    near(got, (want, want_lse), spread, reach, dim, kind)


@pytest.mark.parametrize("kind,hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("prefix", [640, 20000])
def test_a_prefix_without_a_finite_logit(kind, hq, hkv, dim, prefix):
    own = [7] * 5
    c = shared_cache([prefix], [own], hkv, dim, 16, kind)
    held = prefix // 16 * 16
    sink(c, 0, range(held))
    q = rising(5, hq, dim, kind)
    got = c.attend_shared(0, q, groups_of([5]), least=0)
    c.sync()
    want, want_lse, spread, reach = km.attend(c, 0, q, dim ** -0.5, window=7 + prefix - held)
    near(got, (want, want_lse), spread, reach, dim, kind)


@pytest.mark.parametrize("kind,hq,hkv,dim", SHAPES)
def test_rows_without_a_finite_logit(kind, hq, hkv, dim):
    """Tokens there are, but no weights among them: NaN and -infinity, as from attend, and rows beside them are not touched."""
    own = [3, 30, 0, 3, 3]
    c = shared_cache([640, 640], [own[:3], own[3:]], hkv, dim, 16, kind)
    for s in (0, 1):
        sink(c, s, range(640 + own[s]))
    q = rising(5, hq, dim, kind)
    for out, lse in (c.attend(0, q), c.attend_shared(0, q, groups_of([3, 2]), least=0)):
        c.sync()
        assert bool(torch.isnan(out[:3]).all()) and bool((lse[:3] == -torch.inf).all())
        assert bool(torch.isfinite(out[3:]).all()) and bool(torch.isfinite(lse[3:]).all())


@pytest.mark.parametrize("kind,hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("cached", [0, 900, 20000])
def test_prompts_without_a_finite_logit(kind, hq, hkv, dim, cached):
    """Rows of prompts that see no finite logit, whole or split over the GPU: as from attend."""
    c = make([cached + 5, cached + 5], hkv, dim, 16, kind)
    sink(c, 0, range(cached + 3))
    q = rising(10, hq, dim, kind)
    out, lse = c.attend_prompt(0, q, torch.tensor([0, 5, 10], device="cuda"))
    c.sync()
    assert bool(torch.isnan(out[:3]).all()) and bool((lse[:3] == -torch.inf).all())
    assert bool(torch.isfinite(out[3:]).all()) and bool(torch.isfinite(lse[3:]).all())
    for t in range(5):
        c.length.copy_(i32([cached + 1 + t] * 2))
        a, la = c.attend(0, q[[t, 5 + t]].contiguous())
        c.sync()
        assert torch.equal(torch.isnan(a), torch.isnan(out[[t, 5 + t]])) and torch.equal(torch.isneginf(la), torch.isneginf(lse[[t, 5 + t]]))
